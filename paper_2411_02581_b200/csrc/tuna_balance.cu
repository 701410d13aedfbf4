// The balance loss of a router and its gradient.
//
//   loss_g = E / (k n^2) sum_e c[e] M[e],   z_g = 1/n sum_t lse(z_t)^2
//
// over the n live tokens of segment g (a sequence of the batch): c counts how often an expert was chosen,
// M sums its probability over the tokens.  The logits are read once, and once more by the gradient:
//
//   dz = p (G - sum p G) [sigmoid: times 1 - sigmoid(z)] + dz_g 2 lse / n softmax(z),   G = dloss_g E / (k n^2) c
//
// Bound by memory, and for small batches by two launches.
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
// The last segment that begins at t or before it (empty ones before it are passed over), -1 if none does.
__device__ __forceinline__ int segment_of(const BalanceArgs &a, int64_t t) {
  int low = -1, high = a.segments;
  while (high - low > 1) {
    const int g = (low + high) >> 1;
    if (bound_of(a, g) <= t) low = g;
    else high = g;
  }
  return low;
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

// A lane's logits of a token, VPL of them from `first` on; a masked one (NaN, or behind the last) is -inf.
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
#pragma unroll
    for (int i = 0; i < VPL; ++i) z[i] = i < left ? logit_of(z[i]) : -INFINITY;
  }
};

// A token's probabilities from its logits: the softmax, the logarithm of its sum, and with sigmoids their shares (in p) and
// the complements 1 - sigmoid (in rest).  A masked logit has none; a token without any other is not live.
// (__expf is within 2 + 1.2 |x| units of 2^-24, which is 2^-19 where a probability is over e^-25.)
template <int LPT, int VPL>
struct Token {
  float soft[VPL], p[VPL], rest[VPL];
  float lse;
  bool live;
  __device__ __forceinline__ void of(const float (&z)[VPL], int scoring, bool want_soft) {
    float top = -INFINITY;
#pragma unroll
    for (int i = 0; i < VPL; ++i) top = fmaxf(top, z[i]);
    top = group_max<LPT>(top);
    live = top != -INFINITY;
    const bool endless = top == INFINITY;  // those that hold +inf share the softmax
    const float base = live && !endless ? top : 0.0f;
    float sum = 0.0f;
#pragma unroll
    for (int i = 0; i < VPL; ++i) {
      soft[i] = __expf(z[i] - base);
      if (endless) soft[i] = z[i] == INFINITY ? 1.0f : 0.0f;
      sum += soft[i];
    }
    if (want_soft || scoring == TUNA_MOE_SOFTMAX) {
      sum = group_sum<LPT>(sum);
      const float by = live ? __fdividef(1.0f, sum) : 0.0f;
      if (scoring == TUNA_MOE_SOFTMAX) {
#pragma unroll
        for (int i = 0; i < VPL; ++i) p[i] = soft[i] = soft[i] * by;
        lse = live ? top + __logf(sum) : 0.0f;
        return;
      }
      lse = live ? top + __logf(sum) : 0.0f;
      shares(z, top, by);
    } else {
      shares(z, top, 0.0f);
    }
  }
  // sigmoid(z) e^-m = e^(min(z, 0) - m) / (1 + e^-|z|) with m = min(top, 0): no share of very negative logits is 0 / 0.
  // The first exponential is 1 or the second one where some logit is not negative, and the softmax's where none is.
  __device__ __forceinline__ void shares(const float (&z)[VPL], float top, float by_soft) {
    float sum = 0.0f;
#pragma unroll
    for (int i = 0; i < VPL; ++i) {
      const float e = __expf(-fabsf(z[i])), one = __fdividef(1.0f, 1.0f + e);
      const bool up = z[i] >= 0.0f;
      p[i] = (top < 0.0f ? soft[i] : up ? 1.0f : e) * one;
      rest[i] = up ? e * one : one;
      soft[i] *= by_soft;
      sum += p[i];
    }
    sum = group_sum<LPT>(sum);
    const float by = live ? __fdividef(1.0f, sum) : 0.0f;
#pragma unroll
    for (int i = 0; i < VPL; ++i) p[i] *= by;
  }
};

// loss and z of a segment by a whole block, whose threads bring the products of their experts
template <int THREADS>
__device__ __forceinline__ void finish(const BalanceArgs &a, int g, double product, double squares, int64_t n) {
  __shared__ double sum[THREADS / 32];
#pragma unroll
  for (int d = 16; d; d >>= 1) product += __shfl_xor_sync(~0u, product, d);
  __syncthreads();
  if (threadIdx.x % 32 == 0) sum[threadIdx.x / 32] = product;
  __syncthreads();
  if (threadIdx.x == 0) {
    double all = 0.0;
    for (int w = 0; w < THREADS / 32; ++w) all += sum[w];
    a.loss[g] = n ? (float)(all * a.experts / ((double)a.k * n * n)) : 0.0f;
    if (a.z) a.z[g] = n ? (float)(squares / n) : 0.0f;
    a.live[g] = n;
  }
}

// A block's tokens, segment by segment.  ALONE: there is no other block, and what it finds is the answer.
template <int LPT, int VPL, bool ALONE, typename T>
__global__ void __launch_bounds__(kThreads) tuna_balance_kernel(BalanceArgs a) {
  extern __shared__ __align__(16) char smem[];
  float *mass = (float *)smem;                    // [warps][experts]
  int *count = (int *)(mass + kThreads / 32 * a.experts);  // [experts]
  __shared__ float warp_squares[kThreads / 32];
  __shared__ int warp_live[kThreads / 32];
  wait_previous();
  allow_next();
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, sub = threadIdx.x % LPT;
  constexpr int kStep = kThreads / LPT;
  const int64_t b0 = blockIdx.x * a.chunk, b1 = min(b0 + a.chunk, a.tokens);
  const int first = ALONE ? 0 : max(segment_of(a, b0), 0);
  for (int g = first; g < a.segments; ++g) {
    const int64_t begin = bound_of(a, g), t0 = max(begin, b0), t1 = min(bound_of(a, g + 1), b1);
    if (!ALONE && begin >= b1) break;
    if (!ALONE && t0 >= t1) continue;
    for (int e = threadIdx.x; e < a.experts; e += kThreads) count[e] = 0;
    float sum[VPL], squares = 0.0f;
    int live = 0;
#pragma unroll
    for (int i = 0; i < VPL; ++i) sum[i] = 0.0f;
    __syncthreads();
    for (int64_t i = t0 * a.k + threadIdx.x; i < t1 * a.k; i += kThreads) {
      const int id = a.ids[i];
      if (id >= 0 && id < a.experts) atomicAdd(count + id, 1);
    }
    Logits<VPL, T> next;
    int64_t t = t0 + threadIdx.x / LPT;
    next.load(a, t, sub * VPL, t < t1);
    for (int64_t tb = t0; tb < t1; tb += kStep, t += kStep) {  // (uniform: the shuffles need whole warps)
      float z[VPL];
      next.values(z);
      next.load(a, t + kStep, sub * VPL, t + kStep < t1);  // on its way during this one
      Token<LPT, VPL> token;
      token.of(z, a.scoring, a.z != nullptr);
#pragma unroll
      for (int i = 0; i < VPL; ++i) sum[i] += token.p[i];
      if (token.live && sub == 0) {
        ++live;
        if (a.z) squares = fmaf(token.lse, token.lse, squares);
      }
    }
#pragma unroll
    for (int d = LPT; d < 32; d <<= 1)
#pragma unroll
      for (int i = 0; i < VPL; ++i) sum[i] += __shfl_xor_sync(~0u, sum[i], d);
#pragma unroll
    for (int d = LPT; d < 32; d <<= 1) squares += __shfl_xor_sync(~0u, squares, d), live += __shfl_xor_sync(~0u, live, d);
    if (lane < LPT) {
#pragma unroll
      for (int i = 0; i < VPL; ++i)
        if (sub * VPL + i < a.experts) mass[warp * a.experts + sub * VPL + i] = sum[i];
    }
    if (lane == 0) warp_squares[warp] = squares, warp_live[warp] = live;
    __syncthreads();
    float all_squares = 0.0f;
    int all_live = 0;
#pragma unroll
    for (int w = 0; w < kThreads / 32; ++w) all_squares += warp_squares[w], all_live += warp_live[w];
    double product = 0.0;
    const int64_t slot = (int64_t)blockIdx.x + g;
    for (int e = threadIdx.x; e < a.experts; e += kThreads) {
      float m = 0.0f;
#pragma unroll
      for (int w = 0; w < kThreads / 32; ++w) m += mass[w * a.experts + e];
      if (ALONE) {
        a.mass[(int64_t)g * a.experts + e] = m, a.counts[(int64_t)g * a.experts + e] = count[e];
        product += (double)m * count[e];
      } else {
        a.part[slot * a.experts + e] = make_float2(m, __int_as_float(count[e]));
      }
    }
    if (ALONE) finish<kThreads>(a, g, product, all_squares, all_live);
    else if (threadIdx.x == 0) a.part_token[slot] = make_float2(all_squares, __int_as_float(all_live));
    __syncthreads();
  }
}

// A block a segment: the parts of the blocks that met it, every 8th (or 16th, 32nd ...) of them by one row of threads, then the
// rows in order.
__global__ void __launch_bounds__(kSumThreads) tuna_balance_sum_kernel(BalanceArgs a) {
  __shared__ float mass[kSumThreads];
  __shared__ int count[kSumThreads];
  __shared__ double squares[kSumThreads / 32];
  __shared__ int live[kSumThreads / 32];
  wait_previous();
  allow_next();
  const int g = blockIdx.x;
  const int64_t begin = bound_of(a, g), end = bound_of(a, g + 1);
  const int64_t s0 = begin / a.chunk + g, s1 = end > begin ? (end - 1) / a.chunk + g + 1 : s0;
  const int lanes = a.experts <= 32 ? 32 : (a.experts + 31) / 32 * 32, rows = kSumThreads / lanes;  // (512 experts: 2 rows)
  const int e = threadIdx.x % lanes, row = threadIdx.x / lanes;
  float m = 0.0f;
  int c = 0;
  if (row < rows && e < a.experts) {
#pragma unroll 4
    for (int64_t s = s0 + row; s < s1; s += rows) {
      const float2 v = a.part[s * a.experts + e];
      m += v.x, c += __float_as_int(v.y);
    }
  }
  mass[threadIdx.x] = m, count[threadIdx.x] = c;
  double q = 0.0;
  int n = 0;
  for (int64_t s = s0 + threadIdx.x; s < s1; s += kSumThreads) {
    const float2 v = a.part_token[s];
    q += v.x, n += __float_as_int(v.y);
  }
#pragma unroll
  for (int d = 16; d; d >>= 1) q += __shfl_xor_sync(~0u, q, d), n += __shfl_xor_sync(~0u, n, d);
  if (threadIdx.x % 32 == 0) squares[threadIdx.x / 32] = q, live[threadIdx.x / 32] = n;
  __syncthreads();
  double product = 0.0;
  if (threadIdx.x < a.experts) {
    int64_t all = 0;
    m = 0.0f;
    for (int r = 0; r < rows; ++r) m += mass[r * lanes + threadIdx.x], all += count[r * lanes + threadIdx.x];
    a.mass[(int64_t)g * a.experts + threadIdx.x] = m, a.counts[(int64_t)g * a.experts + threadIdx.x] = all;
    product = (double)m * all;
  }
  double all_squares = 0.0;
  int64_t all_live = 0;
  if (threadIdx.x == 0)
    for (int w = 0; w < kSumThreads / 32; ++w) all_squares += squares[w], all_live += live[w];
  finish<kSumThreads>(a, g, product, all_squares, all_live);
}

template <int LPT, int VPL, typename T>
__global__ void __launch_bounds__(kThreads) tuna_balance_grad_kernel(BalanceArgs a) {
  wait_previous();
  allow_next();
  const int sub = threadIdx.x % LPT;
  constexpr int kStep = kThreads / LPT;
  const int64_t b0 = blockIdx.x * a.chunk, b1 = min(b0 + a.chunk, a.tokens);
  float pull[VPL], pull_z = 0.0f;  // G, and dz 2 / n
  int g = segment_of(a, b0), known = -1;
  int64_t end = g >= 0 ? bound_of(a, g + 1) : bound_of(a, 0);
  Logits<VPL, T> next;
  int64_t t = b0 + threadIdx.x / LPT;
  next.load(a, t, sub * VPL, t < b1);
  for (int64_t tb = b0; tb < b1; tb += kStep, t += kStep) {
    float z[VPL];
    next.values(z);
    next.load(a, t + kStep, sub * VPL, t + kStep < b1);  // on its way during this one
    while (t >= end && g < a.segments) ++g, end = g < a.segments ? bound_of(a, g + 1) : INT64_MAX;
    const bool inside = t < b1 && g >= 0 && g < a.segments;
    if (inside && g != known) {
      const int64_t n = a.live[g];
      const float by = n > 0 ? (float)((double)a.dloss[g] * a.experts / ((double)a.k * n * n)) : 0.0f;
      pull_z = a.dz && n > 0 ? a.dz[g] * 2.0f / (float)n : 0.0f;
#pragma unroll
      for (int i = 0; i < VPL; ++i) pull[i] = sub * VPL + i < a.experts ? by * (float)a.counts[(int64_t)g * a.experts + sub * VPL + i] : 0.0f;
      known = g;
    }
    Token<LPT, VPL> token;
    token.of(z, a.scoring, a.dz != nullptr);
    float dot = 0.0f;
#pragma unroll
    for (int i = 0; i < VPL; ++i) dot = fmaf(token.p[i], inside ? pull[i] : 0.0f, dot);
    dot = group_sum<LPT>(dot);
    float d[VPL];
#pragma unroll
    for (int i = 0; i < VPL; ++i) {
      float v = token.p[i] * (pull[i] - dot);
      if (a.scoring == TUNA_MOE_SIGMOID) v *= token.rest[i];
      if (pull_z != 0.0f && token.soft[i] != 0.0f) v = fmaf(pull_z * token.lse, token.soft[i], v);
      d[i] = inside && token.live && z[i] != -INFINITY ? v : 0.0f;
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
// them where one block is done with them before a second launch would be.
int64_t chunk_of(int64_t tokens, int experts) {
  const int64_t step = by_experts(experts, Rows{}), steps = ceil_div(tokens, step);
  return std::max<int64_t>(1, steps <= 4 ? steps : ceil_div(steps, 592)) * step;
}

template <typename T>
struct BalanceLaunch {
  const BalanceArgs &a;
  cudaStream_t st;
  template <int LPT, int VPL>
  int operator()() {
    const size_t smem = (size_t)(kThreads / 32 + 1) * a.experts * 4;
    const int64_t blocks = ceil_div(a.tokens, a.chunk);
    if (blocks == 1) return launch(tuna_balance_kernel<LPT, VPL, true, T>, dim3(1), kThreads, smem, st, false, a);
    if (const int rc = launch(tuna_balance_kernel<LPT, VPL, false, T>, dim3((unsigned)blocks), kThreads, smem, st, false, a)) return rc;
    return launch(tuna_balance_sum_kernel, dim3((unsigned)a.segments), kSumThreads, 0, st, false, a);
  }
};
template <typename T>
struct BalanceGradLaunch {
  const BalanceArgs &a;
  cudaStream_t st;
  template <int LPT, int VPL>
  int operator()() {
    return launch(tuna_balance_grad_kernel<LPT, VPL, T>, dim3((unsigned)ceil_div(a.tokens, a.chunk)), kThreads, 0, st, false, a);
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
  a.tokens = tokens, a.experts = experts, a.segments = segments, a.chunk = chunk_of(tokens, experts);
  if (tokens <= a.chunk) return TUNA_OK;
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
  if (!loss || !counts || !mass || !live) return TUNA_ERR_INVALID_ARG;
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
  a.segments = segments, a.chunk = chunk_of(tokens, experts);
  a.loss = loss, a.z = z, a.counts = counts, a.mass = mass, a.live = live;
  if (tokens > a.chunk) {
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
  if (!logits || !counts || !live || !dloss || !dlogits || !aligned(logits, size) || !aligned(dlogits, size)) return TUNA_ERR_INVALID_ARG;
  BalanceArgs a = {};
  a.logits = logits, a.offsets = offsets, a.tokens = tokens, a.ld = ld, a.ldd = ldd, a.experts = experts, a.k = k, a.scoring = scoring;
  a.segments = segments, a.chunk = chunk_of(tokens, experts);
  a.counts = (int64_t *)counts, a.live = (int64_t *)live, a.dloss = dloss, a.dz = dz, a.dlogits = dlogits;
  cudaStream_t st = (cudaStream_t)stream;
  return dtype == TUNA_DTYPE_F32 ? by_experts(experts, BalanceGradLaunch<float>{a, st}) : by_experts(experts, BalanceGradLaunch<__nv_bfloat16>{a, st});
}

}  // extern "C"
