// The balance loss of a router and its gradient.
//
//   loss_g = E / (k n^2) sum_e c[e] M[e],   z_g = 1/n sum_t lse(z_t)^2
//
// over the n live tokens of segment g (a sequence of the batch): c counts how often an expert was chosen,
// M sums its probability over the tokens.  The logits are read once, and once more by the gradient:
//
//   dz = p (G - sum p G) [sigmoid: times 1 - sigmoid(z)] + dz_g 2 lse / n softmax(z),   G = dloss_g E / (k n^2) c
//
// Probabilities and all sums are in 32 bits; a sum goes over a lane's tokens, a block's warps, then the blocks, so that a mass of 4 million
// tokens adds 900 terms, 8 and 600 one after the other: off by 1500 * 2^-24 of itself at the very worst (65536 x 64: 9e-8 measured, 8.4e-8
// with sums in 64 bits), where 64 bits would take two more registers a value and the packed instructions.
//
// Of 65536 x 64 f32 logits the loss takes 11.5 us and the gradient 7.9 (memory alone: 2.6 and 5.1): instructions, the chain of loads at a
// block's start, and for the loss a second launch.
#include <algorithm>

#include "tuna_ops.cuh"
#include "tuna_route.cuh"

namespace tuna_ops {
namespace {

constexpr int kThreads = 256, kSumThreads = 1024;

struct BalanceArgs {
  const void *logits;
  const int32_t *ids;
  const int64_t *offsets;  // segments + 1, or nullptr: one segment of all tokens
  int64_t tokens, ld, ldd;
  int experts, k, scoring, segments;
  int64_t chunk;  // tokens of a block
  // a block's part of a segment, [block + segment]: both only rise along the tokens, so no two parts meet
  float2 *part;        // [slots][experts]: sum of probabilities; choices (as an int)
  float2 *part_token;  // [slots]: sum of lse^2; live tokens (as an int)
  float *loss, *z, *mass;
  int64_t *counts, *live;
  const float *dloss, *dz;
  void *dlogits;
};

__device__ __forceinline__ int64_t bound_of(const BalanceArgs &a, int g) {
  return a.offsets ? min(max(a.offsets[g], (int64_t)0), a.tokens) : g ? a.tokens : 0;
}
// The last segment that begins at t or before it (empty ones before it are passed over), -1 if none does; its bounds.  The whole
// warp looks at 32 segments at a time.
__device__ __forceinline__ int segment_of(const BalanceArgs &a, int64_t t, int64_t &begin, int64_t &end) {
  begin = 0, end = a.tokens;
  if (!a.offsets) return 0;
  const int lane = threadIdx.x & 31;
  int base = 0;
  for (int step = a.segments > 1024 ? 1024 : a.segments > 32 ? 32 : 1; step; step >>= 5) {
    const int g = base + lane * step;
    const int64_t at = bound_of(a, min(g, a.segments));
    const uint32_t before = __ballot_sync(~0u, g < a.segments && at <= t);
    if (!before) {
      end = bound_of(a, 0);
      return -1;
    }
    const int last = 31 - __clz(before);
    base += last * step;
    begin = __shfl_sync(~0u, at, last), end = __shfl_sync(~0u, at, min(last + 1, 31));
    if (last == 31 && step == 1) end = bound_of(a, base + 1);
  }
  return base;
}

template <int LPT>
__device__ __forceinline__ float group_max(float v) {
#pragma unroll
  for (int d = 1; d < LPT; d <<= 1) v = fmaxf(v, __shfl_xor_sync(~0u, v, d));
  return v;
}
template <int LPT>
__device__ __forceinline__ float group_sum(float v) {
#pragma unroll
  for (int d = 1; d < LPT; d <<= 1) v += __shfl_xor_sync(~0u, v, d);
  return v;
}

// A lane's logits of a token, VPL of them from `first` on; those behind the last are -inf.
template <int VPL, typename T>
struct Logits {
  Eight<T> w[VPL / 8];
  int left;
  __device__ __forceinline__ void load(const BalanceArgs &a, int64_t t, int first, bool there) {
    left = there ? a.experts - first : 0;
    const T *p = reinterpret_cast<const T *>(a.logits) + (there ? t : 0) * a.ld + first;
#pragma unroll
    for (int i = 0; i < VPL / 8; ++i) w[i].load_any(p + 8 * i, left - 8 * i);
  }
  __device__ __forceinline__ void values(float (&z)[VPL]) const {
#pragma unroll
    for (int i = 0; i < VPL / 8; ++i) w[i].values(z + 8 * i);
    if (left < VPL) {
#pragma unroll
      for (int i = 0; i < VPL; ++i)
        if (i >= left) z[i] = -INFINITY;
    }
  }
};

// A token's probabilities from its logits.  p = x by; with sigmoids also the softmax, s by_s, and the complements 1 - sigmoid, rest
// (both where they are wanted).  lse is the logarithm of the softmax's sum.  A masked logit (-inf, NaN) has no probability; a token
// without any other is not live.
//
// Per value and exponential: a multiply-add and the power of two, 2^(z log2 e - top log2 e).  The rounding of top log2 e is
// common to the token and cancels while |top| <= 2^16; 2^-20 remains (the exponent's own rounding, at most 2^-23 |z - top|, counts
// where a probability is over e^-8).  Tokens for which that does not do are looked at again with more care: NaN, +inf, larger
// logits, and with sigmoids no logit over 0, where the shares might be 0 / 0.
template <int LPT, int VPL, bool SIGMOID>
struct Token {
  static constexpr int kMore = SIGMOID ? VPL : 2;
  float x[VPL], s[kMore], rest[kMore];
  float by, by_s, lse;
  bool live, endless;
  __device__ __forceinline__ void of(const float (&z)[VPL], bool want_soft, bool want_rest) {
    float top = z[0];
#pragma unroll
    for (int i = 1; i < VPL; ++i) top = fmaxf(top, z[i]);
    top = group_max<LPT>(top);
    live = top != -INFINITY, endless = false;
    float sum = 0.0f;
    if (!SIGMOID || want_soft) {
      const float shift = live ? -top * kLog2E : 0.0f;
      uint64_t all = 0;
#pragma unroll
      for (int i = 0; i < VPL; i += 2) {
        float a, b;
        unpair(fma2(pair(z[i], z[i + 1]), pair(kLog2E, kLog2E), pair(shift, shift)), a, b);
        a = exp2_fast(a), b = exp2_fast(b);
        if constexpr (SIGMOID) s[i] = a, s[i + 1] = b;
        else x[i] = a, x[i + 1] = b;
        all = add2(all, pair(a, b));
      }
      float a, b;
      unpair(all, a, b);
      sum = group_sum<LPT>(a + b);
      by_s = by = live ? reciprocal_fast(sum) : 0.0f, lse = live ? top + __logf(sum) : 0.0f;
    }
    bool careful = !(sum < INFINITY) || (live && fabsf(top) > 65536.0f);  // (the lanes of a row of NaN may find no largest logit)
    if constexpr (SIGMOID) {
      uint64_t all = 0;
#pragma unroll
      for (int i = 0; i < VPL; i += 2) {
        float a, b, c, d;
        unpair(mul2(pair(z[i], z[i + 1]), pair(-kLog2E, -kLog2E)), a, b);
        a = exp2_fast(fminf(a, 127.0f)), b = exp2_fast(fminf(b, 127.0f));  // (finite; the reciprocal of 2^127 is taken for 0)
        unpair(add2(pair(a, b), pair(1.0f, 1.0f)), c, d);
        x[i] = reciprocal_fast(c), x[i + 1] = reciprocal_fast(d);
        if (want_rest) unpair(mul2(pair(a, b), pair(x[i], x[i + 1])), rest[i], rest[i + 1]);
        all = add2(all, pair(x[i], x[i + 1]));
      }
      float a, b;
      unpair(all, a, b);
      sum = group_sum<LPT>(a + b);
      by = live ? reciprocal_fast(sum) : 0.0f;
      careful |= !(sum < INFINITY) || (live && !(top >= 0.0f));
    }
    if (__any_sync(~0u, careful)) again(z, careful);  // (the warp goes together; what a token gets does not depend on its neighbours)
  }
  __device__ __forceinline__ void again(const float (&given)[VPL], bool careful) {
    float z[VPL], top = -INFINITY;
#pragma unroll
    for (int i = 0; i < VPL; ++i) z[i] = logit_of(given[i]), top = fmaxf(top, z[i]);
    top = group_max<LPT>(top);
    const bool some = top != -INFINITY, infinite = top == INFINITY;  // those that hold +inf share the softmax
    const float base = some && !infinite ? top : 0.0f;
    float soft[VPL], sum = 0.0f;
#pragma unroll
    for (int i = 0; i < VPL; ++i) soft[i] = infinite ? (z[i] == INFINITY ? 1.0f : 0.0f) : exp2_fast((z[i] - base) * kLog2E), sum += soft[i];
    sum = group_sum<LPT>(sum);
    if (careful) {
      live = some, endless = infinite;
      by_s = by = some ? reciprocal_fast(sum) : 0.0f, lse = some ? top + __logf(sum) : 0.0f;
#pragma unroll
      for (int i = 0; i < VPL; ++i) {
        if constexpr (SIGMOID) s[i] = soft[i];
        else x[i] = soft[i];
      }
    }
    if constexpr (SIGMOID) {
      // sigmoid(z) e^-m = e^(min(z, 0) - m) / (1 + e^-|z|) with m = min(top, 0); the first factor is the softmax's where no logit is over 0
      sum = 0.0f;
#pragma unroll
      for (int i = 0; i < VPL; ++i) {
        const float e = exp2_fast(-fabsf(z[i]) * kLog2E), one = reciprocal_fast(1.0f + e);
        const bool up = z[i] >= 0.0f;
        const float v = z[i] == -INFINITY ? 0.0f : (top < 0.0f ? soft[i] : up ? 1.0f : e) * one;
        sum += v;
        if (careful) x[i] = v, rest[i] = up ? e * one : one;
      }
      sum = group_sum<LPT>(sum);
      if (careful) by = some ? reciprocal_fast(sum) : 0.0f;
    }
  }
};

// Sums over a warp or, by way of `part`, over a block.
template <typename T>
__device__ __forceinline__ T warp_sum(T v) {
#pragma unroll
  for (int d = 16; d; d >>= 1) v += __shfl_xor_sync(~0u, v, d);
  return v;
}
// loss and z of a segment, by the first lane of a warp
__device__ __forceinline__ void leave_loss(const BalanceArgs &a, int g, float product, float squares, uint32_t n) {
  if ((threadIdx.x & 31) != 0) return;
  // (E / k / n / n in this order: n^2 may have 62 bits)
  a.loss[g] = n ? product * ((float)a.experts / a.k) / n / n : 0.0f;
  if (a.z) a.z[g] = n ? squares / n : 0.0f;
  a.live[g] = n;
}

// A block's tokens.  The steps do not mind the segments: what a step's tokens bring is added to the segments that they are in, and
// a segment's sums leave at its end.  So the first logits are asked for before the segment is known.  ALONE: there is no other
// block, and what it finds is the answer.
constexpr int kIdsHeld = 2048;  // of a block's choices, in shared memory; more are read when they are counted
template <int LPT, int VPL, bool ALONE, bool SIGMOID, typename T>
__global__ void __launch_bounds__(kThreads) tuna_balance_kernel(BalanceArgs a) {
  extern __shared__ __align__(16) char smem[];
  float *mass = (float *)smem;                             // [warps][experts]
  int *count = (int *)(mass + kThreads / 32 * a.experts);  // [experts]
  __shared__ int held[kIdsHeld];
  __shared__ float warp_squares[kThreads / 32];
  __shared__ int warp_live[kThreads / 32];
  __shared__ float products[kThreads / 32];
  wait_previous();
  allow_next();
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, sub = threadIdx.x % LPT;
  constexpr int kStep = kThreads / LPT;
  const int64_t b0 = blockIdx.x * a.chunk, b1 = min(b0 + a.chunk, a.tokens);
  Logits<VPL, T> next;
  int64_t t = b0 + threadIdx.x / LPT;
  next.load(a, t, sub * VPL, t < b1);
  const bool hold = (b1 - b0) * a.k <= kIdsHeld;
  if (hold)
    for (int i = threadIdx.x; i < (int)(b1 - b0) * a.k; i += kThreads)
      asm volatile("cp.async.ca.shared.global [%0], [%1], 4;" ::"r"(smem_u32(held + i)), "l"(a.ids + b0 * a.k + i) : "memory");
  for (int e = threadIdx.x; e < a.experts; e += kThreads) count[e] = 0;
  int64_t begin, end;
  int g = segment_of(a, b0, begin, end);
  if (ALONE || g < 0) g = 0, begin = bound_of(a, 0), end = bound_of(a, 1);
  float sum[VPL], squares = 0.0f;
  int live = 0;
#pragma unroll
  for (int i = 0; i < VPL; ++i) sum[i] = 0.0f;
  // what this block has of segment g; the sums begin anew
  auto leave = [&] {
    const int64_t t0 = max(begin, b0), t1 = min(end, b1);
    if (!ALONE && t0 >= t1) return;
    asm volatile("cp.async.wait_all;" ::: "memory");
    __syncthreads();  // the choices are there, and the counts are zero
    for (int64_t i = t0 * a.k + threadIdx.x; i < t1 * a.k; i += kThreads) {
      const int id = hold ? held[i - b0 * a.k] : a.ids[i];
      if (id >= 0 && id < a.experts) atomicAdd(count + id, 1);
    }
#pragma unroll
    for (int d = LPT; d < 32; d <<= 1)
#pragma unroll
      for (int i = 0; i < VPL; ++i) sum[i] += __shfl_xor_sync(~0u, sum[i], d);
    squares = warp_sum(squares), live = warp_sum(live);
    if (lane < LPT) {
#pragma unroll
      for (int i = 0; i < VPL; ++i)
        if (sub * VPL + i < a.experts) mass[warp * a.experts + sub * VPL + i] = sum[i];
    }
    if (lane == 0) warp_squares[warp] = squares, warp_live[warp] = live;
    __syncthreads();
    float product = 0.0f;
    const int64_t slot = (int64_t)blockIdx.x + g;
    for (int e = threadIdx.x; e < a.experts; e += kThreads) {
      float m = 0.0f;
#pragma unroll
      for (int w = 0; w < kThreads / 32; ++w) m += mass[w * a.experts + e];
      if (ALONE) {
        a.mass[(int64_t)g * a.experts + e] = m, a.counts[(int64_t)g * a.experts + e] = count[e];
        product = fmaf(m, count[e], product);
      } else {
        a.part[slot * a.experts + e] = make_float2(m, __int_as_float(count[e]));
      }
      count[e] = 0;
    }
    squares = lane < kThreads / 32 ? warp_squares[lane] : 0.0f, live = lane < kThreads / 32 ? warp_live[lane] : 0;
    if (ALONE) {
      product = warp_sum(product);
      if (lane == 0) products[warp] = product;
      __syncthreads();
    }
    if (warp == 0) {
      squares = warp_sum(squares), live = warp_sum(live);
      if (ALONE) leave_loss(a, g, warp_sum(lane < kThreads / 32 ? products[lane] : 0.0f), squares, live);
      else if (lane == 0) a.part_token[slot] = make_float2(squares, __int_as_float(live));
    }
    __syncthreads();
    squares = 0.0f, live = 0;
#pragma unroll
    for (int i = 0; i < VPL; ++i) sum[i] = 0.0f;
  };
  for (int64_t tb = b0; tb < b1; tb += kStep, t += kStep) {  // (uniform: the shuffles need whole warps)
    float z[VPL];
    next.values(z);
    next.load(a, t + kStep, sub * VPL, t + kStep < b1);  // on its way during this one
    Token<LPT, VPL, SIGMOID> token;
    token.of(z, a.z != nullptr, false);
    const int64_t stop = min(tb + kStep, b1);
    while (g < a.segments && begin < stop) {
      if (t >= begin && t < min(end, stop) && token.live) {
#pragma unroll
        for (int i = 0; i < VPL; i += 2) unpair(fma2(pair(token.x[i], token.x[i + 1]), pair(token.by, token.by), pair(sum[i], sum[i + 1])), sum[i], sum[i + 1]);
        if (sub == 0) {
          ++live;
          if (a.z) squares = fmaf(token.lse, token.lse, squares);
        }
      }
      if (end > stop) break;
      leave();
      if (++g < a.segments) begin = end, end = max(begin, bound_of(a, g + 1));
    }
  }
  for (; g < a.segments; ++g) {  // the segment that goes on behind this block; ALONE: those without tokens behind it too
    leave();
    if (!ALONE) break;
    if (g + 1 < a.segments) begin = end, end = max(begin, bound_of(a, g + 2));
  }
  asm volatile("cp.async.wait_all;" ::: "memory");  // (a block whose tokens are nobody's has not waited for its choices yet)
}

// A block a segment: the parts of the blocks that met it, every 2nd (or 16th, 32nd ...) of them by one row of threads, then the
// rows in order.
__global__ void __launch_bounds__(kSumThreads) tuna_balance_sum_kernel(BalanceArgs a) {
  __shared__ float2 sums[kSumThreads];
  __shared__ float2 tokens[kSumThreads / 32];
  __shared__ float products[kSumThreads / 32];
  wait_previous();
  allow_next();
  const int g = blockIdx.x, lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const int64_t begin = bound_of(a, g), end = bound_of(a, g + 1);
  const int64_t s0 = begin / a.chunk + g, s1 = end > begin ? (end - 1) / a.chunk + g + 1 : s0;
  const int lanes = (a.experts + 31) / 32 * 32, rows = kSumThreads / lanes;  // (512 experts: 2 rows)
  const int row = threadIdx.x / lanes, e = threadIdx.x - row * lanes;
  float m = 0.0f, q = 0.0f;
  uint32_t c = 0, n = 0;  // (2^31 at most)
  if (row < rows && e < a.experts) {
#pragma unroll 8
    for (int64_t s = s0 + row; s < s1; s += rows) {
      const float2 v = a.part[s * a.experts + e];
      m += v.x, c += __float_as_int(v.y);
    }
  }
  for (int64_t s = s0 + threadIdx.x; s < s1; s += kSumThreads) {
    const float2 v = a.part_token[s];
    q += v.x, n += __float_as_int(v.y);
  }
  sums[threadIdx.x] = make_float2(m, __int_as_float(c));
  q = warp_sum(q), n = warp_sum(n);
  if (lane == 0) tokens[warp] = make_float2(q, __int_as_float(n));
  __syncthreads();
  float product = 0.0f;
  if (threadIdx.x < a.experts) {
    m = 0.0f, c = 0;
#pragma unroll 4
    for (int r = 0; r < rows; ++r) {
      const float2 v = sums[r * lanes + threadIdx.x];
      m += v.x, c += __float_as_int(v.y);
    }
    a.mass[(int64_t)g * a.experts + threadIdx.x] = m, a.counts[(int64_t)g * a.experts + threadIdx.x] = c;
    product = m * (float)c;
  }
  product = warp_sum(product);
  if (lane == 0) products[warp] = product;
  __syncthreads();
  if (warp == 0) leave_loss(a, g, warp_sum(products[lane]), warp_sum(tokens[lane].x), warp_sum((uint32_t)__float_as_int(tokens[lane].y)));
}

// A cluster a segment, a block its share of the experts: the parts of the blocks that met the segment, every 16th (or 32nd, 64th ...)
// of them by one row of threads, then the rows in order.  The first block joins the shares of the loss.
__global__ void __launch_bounds__(kSumThreads) tuna_balance_sum_wide_kernel(BalanceArgs a) {
  __shared__ float2 sums[kSumThreads];
  __shared__ float2 tokens[kSumThreads / 32];
  __shared__ float products[kSumThreads / 32];
  __shared__ __align__(16) float share[4];
  wait_previous();
  allow_next();
  const int blocks = (int)cluster_size(), rank = (int)cluster_rank();
  const int g = blockIdx.x / blocks, lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const int64_t begin = bound_of(a, g), end = bound_of(a, g + 1);
  const int64_t s0 = begin / a.chunk + g, s1 = end > begin ? (end - 1) / a.chunk + g + 1 : s0;
  const int mine = (a.experts + blocks - 1) / blocks, e0 = rank * mine, count = max(0, min(mine, a.experts - e0));
  int lanes = 4;
  while (lanes < mine) lanes *= 2;  // (512 at most)
  const int rows = kSumThreads / lanes, row = threadIdx.x / lanes, e = threadIdx.x & (lanes - 1);
  float m = 0.0f, q = 0.0f;
  uint32_t c = 0, n = 0;  // (2^31 at most)
  if (e < count) {
#pragma unroll 8
    for (int64_t s = s0 + row; s < s1; s += rows) {
      const float2 v = a.part[s * a.experts + e0 + e];
      m += v.x, c += __float_as_int(v.y);
    }
  }
  if (rank == 0)
    for (int64_t s = s0 + threadIdx.x; s < s1; s += kSumThreads) {
      const float2 v = a.part_token[s];
      q += v.x, n += __float_as_int(v.y);
    }
  sums[threadIdx.x] = make_float2(m, __int_as_float(c));
  q = warp_sum(q), n = warp_sum(n);
  if (lane == 0) tokens[warp] = make_float2(q, __int_as_float(n));
  __syncthreads();
  float product = 0.0f;
  if (threadIdx.x < count) {
    m = 0.0f, c = 0;
#pragma unroll 8
    for (int r = 0; r < rows; ++r) {
      const float2 v = sums[r * lanes + threadIdx.x];
      m += v.x, c += __float_as_int(v.y);
    }
    a.mass[(int64_t)g * a.experts + e0 + threadIdx.x] = m, a.counts[(int64_t)g * a.experts + e0 + threadIdx.x] = c;
    product = m * (float)c;
  }
  product = warp_sum(product);
  if (lane == 0) products[warp] = product;
  __syncthreads();
  if (warp == 0) product = warp_sum(lane < kSumThreads / 32 ? products[lane] : 0.0f);
  if (threadIdx.x == 0) share[0] = product;
  cluster_meet();
  if (rank == 0 && warp == 0) {
    product = lane < blocks ? load_from_block(smem_u32(share), lane).x : 0.0f;
    const float2 v = lane < kSumThreads / 32 ? tokens[lane] : make_float2(0.0f, 0.0f);
    leave_loss(a, g, warp_sum(product), warp_sum(v.x), warp_sum((uint32_t)__float_as_int(v.y)));
  }
  cluster_meet();  // no block leaves while its share is read
}

// (Four blocks a multiprocessor, at a few spilled registers with sigmoids: 20011 x 160 14.9 us, with two 17.7.)
template <int LPT, int VPL, bool SIGMOID, typename T>
__global__ void __launch_bounds__(kThreads, VPL > 8 ? 2 : 4) tuna_balance_grad_kernel(BalanceArgs a) {
  wait_previous();
  allow_next();
  const int sub = threadIdx.x % LPT;
  constexpr int kStep = kThreads / LPT;
  const int64_t b0 = blockIdx.x * a.chunk, b1 = min(b0 + a.chunk, a.tokens);
  Logits<VPL, T> next;
  int64_t t = b0 + threadIdx.x / LPT;
  next.load(a, t, sub * VPL, t < b1);
  float pull[VPL] = {}, pull_z = 0.0f;  // G, and dz 2 / n
  int64_t begin, end;
  int g = segment_of(a, b0, begin, end), known = -1;
  for (int64_t tb = b0; tb < b1; tb += kStep, t += kStep) {
    float z[VPL];
    next.values(z);
    next.load(a, t + kStep, sub * VPL, t + kStep < b1);  // on its way during this one
    while (t >= end && g < a.segments) ++g, end = g < a.segments ? bound_of(a, g + 1) : INT64_MAX;
    const bool inside = t < b1 && g >= 0 && g < a.segments;
    if (inside && g != known) {
      const int64_t n = a.live[g];
      int64_t c[VPL];
#pragma unroll
      for (int i = 0; i < VPL; ++i) c[i] = sub * VPL + i < a.experts ? a.counts[(int64_t)g * a.experts + sub * VPL + i] : 0;
      const float over = n > 0 ? 1.0f / (float)n : 0.0f, by = a.dloss[g] * ((float)a.experts / a.k) * over * over;
      pull_z = a.dz ? a.dz[g] * 2.0f * over : 0.0f;
#pragma unroll
      for (int i = 0; i < VPL; ++i) pull[i] = by * (float)c[i];
      known = g;
    }
    Token<LPT, VPL, SIGMOID> token;
    token.of(z, a.dz != nullptr, true);
    const bool part = inside && token.live;
    const float by = part ? token.by : 0.0f;
    uint64_t dots = 0;
#pragma unroll
    for (int i = 0; i < VPL; i += 2) dots = fma2(pair(token.x[i], token.x[i + 1]), pair(pull[i], pull[i + 1]), dots);
    float dot, other;
    unpair(dots, dot, other);
    dot = group_sum<LPT>(dot + other) * by;
    // (a token that holds +inf has an infinite z whatever moves: it gets no part of its gradient)
    const float of_z = part && pull_z != 0.0f && !token.endless ? pull_z * token.lse : 0.0f;
    // Where a gradient of the segment is not finite, neither is dot (0 times it is NaN): what has no probability, and who is nobody's, gets
    // zeros all the same.  (A sigmoid that is 0 has no part of the softmax either.)
    uint32_t none = 0;
    if (!(fabsf(of_z - dot) < INFINITY)) {
#pragma unroll
      for (int i = 0; i < VPL; ++i) none |= (uint32_t)(!part || token.x[i] == 0.0f) << i;
    }
    float d[VPL];
#pragma unroll
    for (int i = 0; i < VPL; i += 2) {
      const uint64_t p = mul2(pair(token.x[i], token.x[i + 1]), pair(by, by));
      if constexpr (SIGMOID) {
        uint64_t v = mul2(mul2(p, pair(token.rest[i], token.rest[i + 1])), add2(pair(pull[i], pull[i + 1]), pair(-dot, -dot)));
        if (a.dz) v = fma2(pair(token.s[i], token.s[i + 1]), pair(of_z * token.by_s, of_z * token.by_s), v);
        unpair(v, d[i], d[i + 1]);
      } else {
        unpair(mul2(p, add2(pair(pull[i], pull[i + 1]), pair(of_z - dot, of_z - dot))), d[i], d[i + 1]);
      }
    }
    if (none) {
#pragma unroll
      for (int i = 0; i < VPL; ++i)
        if (none >> i & 1) d[i] = 0.0f;
    }
    if (t < b1) {
      T *out = reinterpret_cast<T *>(a.dlogits) + t * a.ldd + sub * VPL;
#pragma unroll
      for (int i = 0; i < VPL; i += 8) store_any(out + i, reinterpret_cast<const float(&)[8]>(d[i]), a.experts - sub * VPL - i);
    }
  }
}

// ---- host --------------------------------------------------------------------------------

// Lanes a token and values a lane: the fewest lanes that hold the experts at 8 values each.
template <typename F>
int by_experts(int experts, F f) {
  if (experts <= 8) return f.template operator()<1, 8>();
  if (experts <= 32) return f.template operator()<4, 8>();
  if (experts <= 64) return f.template operator()<8, 8>();
  if (experts <= 128) return f.template operator()<16, 8>();
  if (experts <= 256) return f.template operator()<32, 8>();
  return f.template operator()<32, 16>();
}
struct Rows {  // tokens that a block takes at a time
  template <int LPT, int VPL>
  int operator()() { return kThreads / LPT; }
};

// Tokens of a block: one step where that leaves four blocks a multiprocessor or fewer, as many as keep it at that otherwise; all of
// them where one block is done with them before a second launch would be (a segment's end costs it 1.5 us).  (65536 x 64 with
// gradient, inputs from memory: four blocks a multiprocessor 20.8 us, six 24.3, two 24.6; 20011 x 160 40.3, 41.6, 41.0.)
constexpr int kAloneSegments = 8;
int64_t chunk_of(int64_t tokens, int experts, int segments) {
  const int64_t step = by_experts(experts, Rows{}), steps = ceil_div(tokens, step);
  return std::max<int64_t>(1, steps <= 4 && segments <= kAloneSegments ? steps : ceil_div(steps, 4 * sm_count())) * step;
}
bool alone(const BalanceArgs &a) { return a.tokens <= a.chunk && a.segments <= kAloneSegments; }

template <typename T>
struct BalanceLaunch {
  const BalanceArgs &a;
  cudaStream_t st;
  template <int LPT, int VPL>
  int operator()() {
    const size_t smem = (size_t)(kThreads / 32 + 1) * a.experts * 4;
    const int64_t blocks = ceil_div(a.tokens, a.chunk);
    const bool sigmoid = a.scoring == TUNA_MOE_SIGMOID;
    if (alone(a)) return launch(sigmoid ? tuna_balance_kernel<LPT, VPL, true, true, T> : tuna_balance_kernel<LPT, VPL, true, false, T>, dim3(1), kThreads, smem, st, false, a);
    if (const int rc = launch(sigmoid ? tuna_balance_kernel<LPT, VPL, false, true, T> : tuna_balance_kernel<LPT, VPL, false, false, T>, dim3((unsigned)blocks), kThreads, smem, st, false, a))
      return rc;
    // Eight blocks a segment where it has many parts of many experts.  (Eight and one, us, the blocks' kernel with it: one segment of 8192 x 256 12.4
    // and 18.7, four of 16384 x 256 18.4 and 23.1; one of 8192 x 64 8.3 and 8.5; eight of 65536 x 64 13.3 and 11.6.)
    if (blocks / a.segments * a.experts > 16384) return launch_cluster(tuna_balance_sum_wide_kernel, dim3((unsigned)(a.segments * 8)), 8, kSumThreads, 0, st, false, a);
    return launch(tuna_balance_sum_kernel, dim3((unsigned)a.segments), kSumThreads, 0, st, false, a);
  }
};
template <typename T>
struct BalanceGradLaunch {
  const BalanceArgs &a;
  cudaStream_t st;
  template <int LPT, int VPL>
  int operator()() {
    return launch(a.scoring == TUNA_MOE_SIGMOID ? tuna_balance_grad_kernel<LPT, VPL, true, T> : tuna_balance_grad_kernel<LPT, VPL, false, T>,
                  dim3((unsigned)ceil_div(a.tokens, a.chunk)), kThreads, 0, st, false, a);
  }
};

size_t dtype_size(int dtype) { return dtype == TUNA_DTYPE_F32 ? 4 : dtype == TUNA_DTYPE_BF16 ? 2 : 0; }

int check_balance(int64_t tokens, int experts, int k, int segments) {
  if (tokens < 0 || experts < 1 || k < 1 || segments < 1) return TUNA_ERR_INVALID_ARG;
  if (experts > TUNA_MOE_MAX_EXPERTS || k > TUNA_MOE_MAX_K || tokens > ((int64_t)1 << 31) / k || segments > TUNA_MOE_MAX_SEGMENTS) return TUNA_ERR_RANGE;
  return TUNA_OK;
}
void carve(Carve &c, BalanceArgs &a) {
  const int64_t slots = ceil_div(a.tokens, a.chunk) + a.segments;
  a.part = c.take<float2>(slots * a.experts);
  a.part_token = c.take<float2>(slots);
}

}  // namespace
}  // namespace tuna_ops

using namespace tuna_ops;

extern "C" {

int tuna_moe_balance_workspace_bytes(int64_t tokens, int experts, int segments, size_t *bytes) {
  if (!bytes) return TUNA_ERR_INVALID_ARG;
  if (const int rc = check_balance(tokens, experts, 1, segments)) return rc;
  *bytes = 0;
  BalanceArgs a = {};
  a.tokens = tokens, a.experts = experts, a.segments = segments, a.chunk = chunk_of(tokens, experts, segments);
  if (alone(a)) return TUNA_OK;
  Carve c(nullptr);
  carve(c, a);
  *bytes = c.used;
  return TUNA_OK;
}

int tuna_moe_balance(const void *logits, int dtype, int64_t tokens, int experts, int64_t ld, const int32_t *ids, int k, int scoring, int segments,
                     const int64_t *offsets, float *loss, float *z, int64_t *counts, float *mass, int64_t *live, void *workspace,
                     size_t workspace_bytes, void *stream) {
  if (const int rc = check_balance(tokens, experts, k, segments)) return rc;
  const size_t size = dtype_size(dtype);
  if (!size || (scoring != TUNA_MOE_SOFTMAX && scoring != TUNA_MOE_SIGMOID) || ld < experts || (segments > 1 && !offsets)) return TUNA_ERR_INVALID_ARG;
  if (!loss || !counts || !mass || !live || !aligned(loss, 4) || !aligned(z, 4) || !aligned(counts, 8) || !aligned(mass, 4) || !aligned(live, 8) ||
      !aligned(offsets, 8))
    return TUNA_ERR_INVALID_ARG;
  cudaStream_t st = (cudaStream_t)stream;
  if (tokens == 0) {
    const size_t n = (size_t)segments * experts;
    int rc = note_cuda(cudaMemsetAsync(loss, 0, (size_t)segments * 4, st));
    if (!rc && z) rc = note_cuda(cudaMemsetAsync(z, 0, (size_t)segments * 4, st));
    if (!rc) rc = note_cuda(cudaMemsetAsync(live, 0, (size_t)segments * 8, st));
    if (!rc) rc = note_cuda(cudaMemsetAsync(counts, 0, n * 8, st));
    return rc ? rc : note_cuda(cudaMemsetAsync(mass, 0, n * 4, st));
  }
  if (!logits || !ids || !aligned(logits, size) || !aligned(ids, 4)) return TUNA_ERR_INVALID_ARG;
  BalanceArgs a = {};
  a.logits = logits, a.ids = ids, a.offsets = offsets, a.tokens = tokens, a.ld = ld, a.experts = experts, a.k = k, a.scoring = scoring;
  a.segments = segments, a.chunk = chunk_of(tokens, experts, segments);
  a.loss = loss, a.z = z, a.counts = counts, a.mass = mass, a.live = live;
  if (!alone(a)) {
    Carve c(workspace);
    carve(c, a);
    if (!workspace || !aligned(workspace, 256) || workspace_bytes < c.used) return TUNA_ERR_WORKSPACE;
  }
  return dtype == TUNA_DTYPE_F32 ? by_experts(experts, BalanceLaunch<float>{a, st}) : by_experts(experts, BalanceLaunch<__nv_bfloat16>{a, st});
}

int tuna_moe_balance_backward(const void *logits, int dtype, int64_t tokens, int experts, int64_t ld, int k, int scoring, int segments,
                              const int64_t *offsets, const int64_t *counts, const int64_t *live, const float *dloss, const float *dz, void *dlogits,
                              int64_t ldd, void *stream) {
  if (const int rc = check_balance(tokens, experts, k, segments)) return rc;
  const size_t size = dtype_size(dtype);
  if (!size || (scoring != TUNA_MOE_SOFTMAX && scoring != TUNA_MOE_SIGMOID) || ld < experts || ldd < experts || (segments > 1 && !offsets))
    return TUNA_ERR_INVALID_ARG;
  if (tokens == 0) return TUNA_OK;
  if (!logits || !counts || !live || !dloss || !dlogits || !aligned(logits, size) || !aligned(dlogits, size) || !aligned(counts, 8) || !aligned(live, 8) ||
      !aligned(dloss, 4) || !aligned(dz, 4) || !aligned(offsets, 8))
    return TUNA_ERR_INVALID_ARG;
  BalanceArgs a = {};
  a.logits = logits, a.offsets = offsets, a.tokens = tokens, a.ld = ld, a.ldd = ldd, a.experts = experts, a.k = k, a.scoring = scoring;
  a.segments = segments, a.chunk = chunk_of(tokens, experts, segments);
  a.counts = (int64_t *)counts, a.live = (int64_t *)live, a.dloss = dloss, a.dz = dz, a.dlogits = dlogits;
  cudaStream_t st = (cudaStream_t)stream;
  return dtype == TUNA_DTYPE_F32 ? by_experts(experts, BalanceGradLaunch<float>{a, st}) : by_experts(experts, BalanceGradLaunch<__nv_bfloat16>{a, st});
}

}  // extern "C"
