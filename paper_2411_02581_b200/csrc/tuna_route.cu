// Router of a mixture-of-experts layer: the k best experts of every token with their
// weights, the rows' order by expert (the gather map and count matrix that a token
// dispatch takes), the weighted sum that undoes it, and the gradients of both.
//
// All of it is bound by memory, and for a decode step by latency: the logits are read
// once, everything else is a few bytes a token.
#include <algorithm>
#include <mutex>

#include "tuna_fp8.h"
#include "tuna_ops.cuh"
#include "tuna_route.cuh"

namespace tuna_ops {

static __device__ int g_gave_up;  // raised by a kernel whose bounded wait ran out

static thread_local int t_cuda_error = 0;

int note_cuda(cudaError_t e) {
  if (e == cudaSuccess) return TUNA_OK;
  t_cuda_error = (int)e;
  return TUNA_ERR_CUDA;
}

int sm_count() {
  static std::mutex m;
  static int count[64] = {};
  int dev = 0;
  if (cudaGetDevice(&dev) != cudaSuccess || dev < 0 || dev >= 64) return 148;
  std::lock_guard<std::mutex> lock(m);
  if (!count[dev] && cudaDeviceGetAttribute(&count[dev], cudaDevAttrMultiProcessorCount, dev) != cudaSuccess) return 148;
  return count[dev];
}

int *error_word() {
  static std::mutex m;
  static int *at[64] = {};
  int dev = -1;
  if (note_cuda(cudaGetDevice(&dev)) || dev < 0 || dev >= 64) return nullptr;
  std::lock_guard<std::mutex> lock(m);
  if (!at[dev]) {
    void *p = nullptr;
    if (note_cuda(cudaGetSymbolAddress(&p, g_gave_up))) return nullptr;
    at[dev] = (int *)p;
  }
  return at[dev];
}

namespace {

constexpr int kTopThreads = 256;

struct RouteArgs {
  const void *logits;
  int64_t tokens, ld;
  int experts, k, scoring, renormalize, vec;
  float scale;
  int32_t *ids;
  float *weights;
};

// ---- the rows' order ---------------------------------------------------------------------
//
// A stable counting sort of the T k choices by (rank, expert).  The tokens of a rank are cut
// into chunks; `hist` holds how often each chunk chose each expert.  A block of the order
// kernel sums the columns of `hist` itself (they come from L2), so that no scan kernel and no
// third launch is needed, then ranks its own entries: peers of a warp by match, warps by a
// small table in shared memory.

struct OrderArgs {
  const int32_t *ids;
  int64_t tokens;        // in all
  int64_t rank_tokens;   // of one rank
  int experts, k, ranks;
  int chunk;             // tokens a chunk
  int64_t rank_chunks;   // chunks of one rank
  int group;             // chunks that one block of the order kernel takes
  int64_t rank_groups;   // blocks of one rank
  uint16_t *hist;        // [ranks * rank_chunks][experts]
  int64_t *counts, *offsets, *rows, *pos;
};

// The small router has more threads, for its choice.
constexpr int kOrderThreads = 256, kSmallThreads = 1024;

// Shared memory of the order step: base[experts] (64 bits), then the warps' tables, then the
// column sums (64-bit pairs would be wasteful: entries of one call stay below 2^31).
__host__ __device__ inline size_t order_smem(int experts, int threads) {
  return (size_t)experts * 8 + (size_t)(threads / 32) * experts * 4 + (size_t)experts * 8 + 256;
}

template <int THREADS>
__device__ __forceinline__ void place_entries(const OrderArgs &o, char *smem, int64_t first_entry, int64_t last_entry) {
  // base[e]: the row of the first of this block's entries that chose e
  int64_t *base = (int64_t *)smem;
  uint32_t *table = (uint32_t *)(smem + (size_t)o.experts * 16);
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int64_t n = last_entry - first_entry;
  const int64_t per = (n + (THREADS / 32) - 1) / (THREADS / 32);
  const int64_t a = first_entry + min(n, warp * per), b = first_entry + min(n, (warp + 1) * per);
  uint32_t *mine = table + (size_t)warp * o.experts;
  for (int e = threadIdx.x; e < (THREADS / 32) * o.experts; e += THREADS) table[e] = 0;
  // A warp's entries, kHeld rounds of 32 at a time: loaded together, and once where they are no more.
  constexpr int kHeld = 8;
  int held[kHeld];
  auto fetch = [&](int64_t from) {
#pragma unroll
    for (int r = 0; r < kHeld; ++r) {
      const int64_t i = from + r * 32 + lane;
      const int id = i < b ? o.ids[i] : -1;
      held[r] = id >= 0 && id < o.experts ? id : -1;
    }
  };
  fetch(a);
  __syncthreads();
  for (int64_t i = a; i < b; i += kHeld * 32) {
    if (i > a) fetch(i);
#pragma unroll
    for (int r = 0; r < kHeld; ++r) {
      if (i + r * 32 >= b) break;
      const uint32_t peers = __match_any_sync(~0u, held[r]);
      if (held[r] >= 0 && lane == __ffs(peers) - 1) mine[held[r]] += __popc(peers);
      __syncwarp();
    }
  }
  __syncthreads();
  for (int e = threadIdx.x; e < o.experts; e += THREADS) {
    uint32_t sum = 0;
#pragma unroll 8
    for (int w = 0; w < (THREADS / 32); ++w) {
      const uint32_t c = table[(size_t)w * o.experts + e];
      table[(size_t)w * o.experts + e] = sum;
      sum += c;
    }
  }
  __syncthreads();
  if (b - a > kHeld * 32) fetch(a);
  for (int64_t i = a; i < b; i += kHeld * 32) {
    if (i > a) fetch(i);
#pragma unroll
    for (int r = 0; r < kHeld; ++r) {
      const int64_t entry = i + r * 32 + lane;
      if (i + r * 32 >= b) break;
      const int id = held[r];
      const uint32_t peers = __match_any_sync(~0u, id);
      if (id >= 0) {
        const int64_t at = base[id] + mine[id] + __popc(peers & ((1u << lane) - 1));
        o.pos[entry] = at;
        o.rows[at] = (uint32_t)entry / (uint32_t)o.k;  // (entries of one call stay below 2^31)
      } else if (entry < b) {
        o.pos[entry] = -1;
      }
      __syncwarp();
      if (id >= 0 && lane == __ffs(peers) - 1) mine[id] += __popc(peers);
      __syncwarp();
    }
  }
}

// Exclusive scan of v over the block's threads; *total receives the sum.
__device__ __forceinline__ int64_t block_scan(int64_t v, int64_t *total) {
  __shared__ int64_t part[33];
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  int64_t x = v;
#pragma unroll
  for (int d = 1; d < 32; d <<= 1) {
    const int64_t y = __shfl_up_sync(~0u, x, d);
    if (lane >= d) x += y;
  }
  __syncthreads();
  if (lane == 31) part[warp] = x;
  __syncthreads();
  if (warp == 0) {
    int64_t p = lane < (int)(blockDim.x >> 5) ? part[lane] : 0;
#pragma unroll
    for (int d = 1; d < 32; d <<= 1) {
      const int64_t y = __shfl_up_sync(~0u, p, d);
      if (lane >= d) p += y;
    }
    part[lane + 1] = p;
    if (lane == 0) part[0] = 0;
  }
  __syncthreads();
  const int64_t r = x - v + part[warp];
  *total = part[32];
  __syncthreads();
  return r;
}

// Block (rank, group).  Sums the columns of hist: of all earlier ranks (rows before this
// rank), of this rank (for the scan over experts) and of this rank's earlier chunks.
__global__ void __launch_bounds__(kOrderThreads) tuna_order_kernel(OrderArgs o) {
  extern __shared__ __align__(16) char smem[];
  wait_previous();
  allow_next();
  const int E = o.experts;
  const int rank = (int)blockIdx.x / (int)o.rank_groups;
  const int64_t group = (int)blockIdx.x - rank * (int)o.rank_groups;
  int64_t *base = (int64_t *)smem;
  int *total = (int *)(smem + (size_t)E * 8);  // of this rank, per expert
  int *before = total + E;                     // of this rank's earlier chunks
  for (int e = threadIdx.x; e < 2 * E; e += kOrderThreads) total[e] = 0;
  __syncthreads();
  const int64_t chunks = o.rank_chunks, mine = group * o.group;
  // threads take (a row of hist, an expert) with the expert along the lanes
  const int lanes = E >= kOrderThreads ? kOrderThreads : E;  // (more experts than threads: several rounds)
  const int stripes = kOrderThreads / lanes;
  const int stripe = threadIdx.x / lanes;
  // entries of earlier ranks: all of hist before this rank's part, eight at a time (hist is aligned)
  int64_t earlier = 0;
  {
    const int64_t before = rank * chunks * E;
    const uint4 *h = reinterpret_cast<const uint4 *>(o.hist);
#pragma unroll 8
    for (int64_t i = threadIdx.x; i < before / 8; i += kOrderThreads) {
      const uint4 v = h[i];
      earlier += (v.x & 0xffffu) + (v.x >> 16) + (v.y & 0xffffu) + (v.y >> 16) + (v.z & 0xffffu) + (v.z >> 16) + (v.w & 0xffffu) + (v.w >> 16);
    }
    for (int64_t i = before / 8 * 8 + threadIdx.x; i < before; i += kOrderThreads) earlier += o.hist[i];
  }
  for (int e = threadIdx.x % lanes; e < E && stripe < stripes; e += lanes) {
    int t = 0, p = 0;
    const uint16_t *h = o.hist + rank * chunks * E + e;
#pragma unroll 8
    for (int64_t c = stripe; c < chunks; c += stripes) {
      const int v = h[c * E];
      t += v;
      p += c < mine ? v : 0;
    }
    if (t) atomicAdd(total + e, t);
    if (p) atomicAdd(before + e, p);
  }
  int64_t rows_before;
  block_scan(earlier, &rows_before);  // (its barriers also cover the sums above)
  // scan over the experts, kOrderThreads at a time
  for (int e0 = 0; e0 < E; e0 += kOrderThreads) {
    const int e = e0 + threadIdx.x;
    const int64_t t = e < E ? total[e] : 0;
    int64_t sum;
    const int64_t x = block_scan(t, &sum) + rows_before;
    if (e < E) {
      base[e] = x + before[e];
      if (group == 0) {
        if (o.counts) o.counts[(int64_t)rank * E + e] = t;
        if (o.offsets) {
          o.offsets[(int64_t)rank * E + e] = x;
          if (rank == o.ranks - 1 && e == E - 1) o.offsets[(int64_t)o.ranks * E] = x + t;
        }
      }
    }
    rows_before += sum;
  }
  __syncthreads();
  const int64_t t0 = rank * o.rank_tokens + mine * o.chunk;
  const int64_t t1 = min((int64_t)(rank + 1) * o.rank_tokens, t0 + (int64_t)o.group * o.chunk);
  place_entries<kOrderThreads>(o, smem, t0 * o.k, t1 * o.k);
  // rows that no entry fills (masked choices): -1, written by the last rank's blocks, which know the sum
  if (rank == o.ranks - 1)
    for (int64_t j = rows_before + group * kOrderThreads + threadIdx.x; j < o.tokens * o.k; j += o.rank_groups * kOrderThreads) o.rows[j] = -1;
}

// How often a chunk chose each expert, from ids in memory (a block a chunk).
__global__ void __launch_bounds__(256) tuna_order_hist_kernel(OrderArgs o) {
  extern __shared__ int count[];
  wait_previous();
  allow_next();
  for (int e = threadIdx.x; e < o.experts; e += 256) count[e] = 0;
  __syncthreads();
  const int rank = (int)blockIdx.x / (int)o.rank_chunks, c = (int)blockIdx.x - rank * (int)o.rank_chunks;
  const int64_t t0 = rank * o.rank_tokens + (int64_t)c * o.chunk, t1 = min((rank + 1) * o.rank_tokens, t0 + o.chunk);
  for (int64_t i = t0 * o.k + threadIdx.x; i < t1 * o.k; i += 256) {
    const int id = o.ids[i];
    if (id >= 0 && id < o.experts) atomicAdd(count + id, 1);
  }
  __syncthreads();
  for (int e = threadIdx.x; e < o.experts; e += 256) o.hist[(int64_t)blockIdx.x * o.experts + e] = (uint16_t)count[e];
}

// The choice for a chunk of tokens (a block a chunk) and its column of hist.
template <int LPT, int VPL, typename T>
__global__ void __launch_bounds__(kTopThreads) tuna_route_kernel(RouteArgs a, OrderArgs o) {
  extern __shared__ int count[];
  for (int e = threadIdx.x; e < a.experts; e += kTopThreads) count[e] = 0;
  wait_previous();
  allow_next();
  const int rank = (int)blockIdx.x / (int)o.rank_chunks, c = (int)blockIdx.x - rank * (int)o.rank_chunks;
  const int64_t t0 = rank * o.rank_tokens + (int64_t)c * o.chunk, t1 = min((rank + 1) * o.rank_tokens, t0 + o.chunk);
  const int lane = threadIdx.x % LPT;
  constexpr int kStep = kTopThreads / LPT;
  auto fetch = [&](int64_t t, float (&z)[VPL]) {
    if (t < t1) {
      load_logits(reinterpret_cast<const T *>(a.logits) + t * a.ld, lane * VPL, a.experts, a.vec, z);
    } else {
#pragma unroll
      for (int i = 0; i < VPL; ++i) z[i] = -INFINITY;
    }
  };
  float next[VPL];
  int64_t t = t0 + threadIdx.x / LPT;
  fetch(t, next);
  __syncthreads();
  for (int64_t tb = t0; tb < t1; tb += kStep, t += kStep) {  // (uniform: the shuffles need whole warps)
    float z[VPL];
#pragma unroll
    for (int i = 0; i < VPL; ++i) z[i] = next[i];
    fetch(t + kStep, next);  // the next token's logits are on their way during this one's choice
    int id;
    float w;
    choose<LPT>(z, lane, a.k, a.scoring, a.renormalize, a.scale, id, w);
    if (t < t1 && lane < a.k) {
      a.ids[t * a.k + lane] = id;
      a.weights[t * a.k + lane] = w;
      if (id >= 0) atomicAdd(count + id, 1);
    }
  }
  __syncthreads();
  for (int e = threadIdx.x; e < a.experts; e += kTopThreads) o.hist[(int64_t)blockIdx.x * a.experts + e] = (uint16_t)count[e];
}

// A few tokens of one rank: choice and order in one block and one launch.
template <int LPT, int VPL, typename T>
__global__ void __launch_bounds__(kSmallThreads) tuna_route_small_kernel(RouteArgs a, OrderArgs o) {
  extern __shared__ __align__(16) char smem[];
  int64_t *base = (int64_t *)smem;
  int *count = (int *)(smem + (size_t)a.experts * 8);
  for (int e = threadIdx.x; e < a.experts; e += kSmallThreads) count[e] = 0;
  wait_previous();
  allow_next();
  __syncthreads();
  const int lane = threadIdx.x % LPT;
  for (int64_t tb = 0; tb < a.tokens; tb += kSmallThreads / LPT) {
    const int64_t t = tb + threadIdx.x / LPT;
    float z[VPL];
    if (t < a.tokens) {
      load_logits(reinterpret_cast<const T *>(a.logits) + t * a.ld, lane * VPL, a.experts, a.vec, z);
    } else {
#pragma unroll
      for (int i = 0; i < VPL; ++i) z[i] = -INFINITY;
    }
    int id;
    float w;
    choose<LPT>(z, lane, a.k, a.scoring, a.renormalize, a.scale, id, w);
    if (t < a.tokens && lane < a.k) {
      a.ids[t * a.k + lane] = id;
      a.weights[t * a.k + lane] = w;
      if (id >= 0) atomicAdd(count + id, 1);
    }
  }
  __syncthreads();
  const int e = threadIdx.x;  // (experts <= TUNA_MOE_MAX_EXPERTS < kSmallThreads)
  const int64_t c = e < a.experts ? count[e] : 0;
  int64_t sum;
  const int64_t x = block_scan(c, &sum);
  if (e < a.experts) {
    base[e] = x;
    if (o.counts) o.counts[e] = c;
    if (o.offsets) {
      o.offsets[e] = x;
      if (e == a.experts - 1) o.offsets[a.experts] = sum;
    }
  }
  place_entries<kSmallThreads>(o, smem, 0, a.tokens * a.k);
  for (int64_t j = sum + threadIdx.x; j < a.tokens * a.k; j += kSmallThreads) o.rows[j] = -1;
}

// The order of a few choices of one rank in one block and one launch.
__global__ void __launch_bounds__(kSmallThreads) tuna_order_small_kernel(OrderArgs o) {
  extern __shared__ __align__(16) char smem[];
  int64_t *base = (int64_t *)smem;
  int *count = (int *)(smem + (size_t)o.experts * 8);
  for (int e = threadIdx.x; e < o.experts; e += kSmallThreads) count[e] = 0;
  wait_previous();
  allow_next();
  __syncthreads();
  const int64_t n = o.tokens * o.k;
  for (int64_t i = threadIdx.x; i < n; i += kSmallThreads) {
    const int id = o.ids[i];
    if (id >= 0 && id < o.experts) atomicAdd(count + id, 1);
  }
  __syncthreads();
  const int e = threadIdx.x;  // (experts <= TUNA_MOE_MAX_EXPERTS < kSmallThreads)
  const int64_t c = e < o.experts ? count[e] : 0;
  int64_t sum;
  const int64_t x = block_scan(c, &sum);
  if (e < o.experts) {
    base[e] = x;
    if (o.counts) o.counts[e] = c;
    if (o.offsets) {
      o.offsets[e] = x;
      if (e == o.experts - 1) o.offsets[o.experts] = sum;
    }
  }
  place_entries<kSmallThreads>(o, smem, 0, n);
  for (int64_t j = sum + threadIdx.x; j < n; j += kSmallThreads) o.rows[j] = -1;
}

// Gradient of the weights with respect to the logits; the probabilities are computed anew
// from the logits (one read of them) instead of being kept by the forward pass.
//   softmax            dz_e = p_e (g_e - sum_s g_s p_s)          g: dw at the chosen, 0 elsewhere
//   ... renormalised   dz_s = w_s (g_s - sum_s g_s w_s)          over the chosen alone
//   sigmoid            dz_s = g_s p_s (1 - p_s)
//   ... renormalised   dz_s = (g_s - sum_s g_s w_s) / sum p * p_s (1 - p_s)
struct RouteGradArgs {
  const void *logits;
  int64_t tokens, ld, ldd;
  int experts, k, scoring, renormalize, vec;
  float scale;
  const int32_t *ids;
  const float *dweights;
  void *dlogits;
};
template <int LPT, int VPL, typename T>
__global__ void __launch_bounds__(kTopThreads) tuna_route_grad_kernel(RouteGradArgs a) {
  wait_previous();
  allow_next();
  const int lane = threadIdx.x % LPT;
  const int64_t t = (int64_t)blockIdx.x * (kTopThreads / LPT) + threadIdx.x / LPT;
  const bool there = t < a.tokens;
  float z[VPL], d[VPL];
  int id = -1;
  float g = 0.0f;
  if (there && lane < a.k) id = __ldg(a.ids + t * a.k + lane), g = __ldg(a.dweights + t * a.k + lane) * a.scale;
  if (there) {
    load_logits(reinterpret_cast<const T *>(a.logits) + t * a.ld, lane * VPL, a.experts, a.vec, z);
  } else {
#pragma unroll
    for (int i = 0; i < VPL; ++i) z[i] = -INFINITY;
  }
  if (id < 0 || id >= a.experts) id = -1, g = 0.0f;
  // the chosen logit of this lane's slot, anew from memory: it is there already
  const float mine = id < 0 ? -INFINITY : logit_of(to_f32(__ldg(reinterpret_cast<const T *>(a.logits) + t * a.ld + id)));
  const bool soft = a.scoring == TUNA_MOE_SOFTMAX;
  float top = -INFINITY;
#pragma unroll
  for (int i = 0; i < VPL; ++i) top = fmaxf(top, z[i]), d[i] = 0.0f;
#pragma unroll
  for (int s = 1; s < LPT; s <<= 1) top = fmaxf(top, __shfl_xor_sync(~0u, top, s));
  float p = mine == -INFINITY ? 0.0f : soft ? exp_of(mine, top) : sigmoid_of(mine);
  float sum = p;
  if (soft && !a.renormalize) {
    sum = 0.0f;
#pragma unroll
    for (int i = 0; i < VPL; ++i) d[i] = z[i] == -INFINITY ? 0.0f : exp_of(z[i], top), sum += d[i];
  }
#pragma unroll
  for (int s = 1; s < LPT; s <<= 1) sum += __shfl_xor_sync(~0u, sum, s);
  const float over = sum > 0.0f ? 1.0f / sum : 0.0f;
  const float w = soft || a.renormalize ? p * over : p;
  float gw = g * w;
#pragma unroll
  for (int s = 1; s < LPT; s <<= 1) gw += __shfl_xor_sync(~0u, gw, s);
  float mine_d;  // this lane's slot's share
  if (soft)
    mine_d = a.renormalize ? w * (g - gw) : w * g;
  else
    mine_d = (a.renormalize ? (g - gw) * over : g) * p * (1.0f - p);
  if (soft && !a.renormalize) {
#pragma unroll
    for (int i = 0; i < VPL; ++i) d[i] *= -over * gw;
  }
  for (int s = 0; s < a.k; ++s) {
    const int at = __shfl_sync(~0u, id, s, LPT) - lane * VPL;
    const float v = __shfl_sync(~0u, mine_d, s, LPT);
#pragma unroll
    for (int i = 0; i < VPL; ++i) d[i] += at == i ? v : 0.0f;
  }
  if (!there) return;
  T *out = reinterpret_cast<T *>(a.dlogits) + t * a.ldd + lane * VPL;
  if (a.vec && (lane + 1) * VPL <= a.experts) {
    store_row(out, d);
  } else {
#pragma unroll
    for (int i = 0; i < VPL; ++i)
      if (lane * VPL + i < a.experts) out[i] = from_f32<T>(d[i]);
  }
}

// ---- combine -----------------------------------------------------------------------------
//
// out[t] = sum_s w[t,s] y[pos[t,s]], summed in slot order in 32 bits.  Bound by the bytes of
// y and out: a thread takes 8 columns of a token, 16-byte loads of bf16.
struct CombineArgs {
  const void *y, *dout;
  const float *weights;
  const int64_t *pos;
  void *out, *dy;
  float *dweights;
  int64_t rows, tokens, ldy, ldo, lddy;
  int dim, k, vec;
};
template <typename TY, typename TO>
__global__ void __launch_bounds__(256) tuna_combine_kernel(CombineArgs a) {
  wait_previous();
  allow_next();
  // a block takes 2048 columns of a token
  const int c = (int)(blockIdx.y * 256 + threadIdx.x) * 8;
  if (c >= a.dim) return;
  for (int64_t t = blockIdx.x; t < a.tokens; t += gridDim.x) {
    float acc[8] = {};
    for (int s = 0; s < a.k; s += 2) {  // two rows in flight
      Eight<TY> y[2];
      float w[2];
      bool there[2];
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        const int64_t r = s + i < a.k ? __ldg(a.pos + t * a.k + s + i) : -1;
        there[i] = r >= 0 && r < a.rows;
        if (there[i]) {
          w[i] = __ldg(a.weights + t * a.k + s + i);
          y[i].load(reinterpret_cast<const TY *>(a.y) + r * a.ldy + c, a.vec, a.dim - c);
        }
      }
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        if (!there[i]) continue;
        float v[8];
        y[i].values(v);
#pragma unroll
        for (int j = 0; j < 8; ++j) acc[j] = fmaf(w[i], v[j], acc[j]);
      }
    }
    TO *out = reinterpret_cast<TO *>(a.out) + t * a.ldo + c;
    if (a.vec) {
      store_row(out, acc);
    } else {
#pragma unroll
      for (int j = 0; j < 8; ++j)
        if (c + j < a.dim) out[j] = from_f32<TO>(acc[j]);
    }
  }
}

// dy[pos[t,s]] = w[t,s] dout[t];  dw[t,s] = <dout[t], y[pos[t,s]]>.  A block a token; the
// row of dout is read once a slot (from L1 after the first), rows of y once.
template <typename TY, typename TO>
__global__ void __launch_bounds__(256) tuna_combine_grad_kernel(CombineArgs a) {
  __shared__ float part[8];
  wait_previous();
  allow_next();
  for (int64_t t = blockIdx.x; t < a.tokens; t += gridDim.x) {
    const TO *g = reinterpret_cast<const TO *>(a.dout) + t * a.ldo;
    for (int s = 0; s < a.k; ++s) {
      const int64_t r = a.pos[t * a.k + s];
      const bool there = r >= 0 && r < a.rows;
      float dot = 0.0f;
      if (there) {
        const float w = a.weights[t * a.k + s];
        const TY *y = reinterpret_cast<const TY *>(a.y) + r * a.ldy;
        TY *dy = reinterpret_cast<TY *>(a.dy) + r * a.lddy;
        for (int c = threadIdx.x * 8; c < a.dim; c += 2048) {
          float gv[8], yv[8];
          if (a.vec) {
            load_row(g + c, gv);
            load_row(y + c, yv);
          } else {
#pragma unroll
            for (int j = 0; j < 8; ++j) {
              gv[j] = c + j < a.dim ? to_f32(g[c + j]) : 0.0f;
              yv[j] = c + j < a.dim ? to_f32(y[c + j]) : 0.0f;
            }
          }
#pragma unroll
          for (int j = 0; j < 8; ++j) dot = fmaf(gv[j], yv[j], dot), gv[j] *= w;
          if (a.vec) {
            store_row(dy + c, gv);
          } else {
#pragma unroll
            for (int j = 0; j < 8; ++j)
              if (c + j < a.dim) dy[c + j] = from_f32<TY>(gv[j]);
          }
        }
      }
#pragma unroll
      for (int d = 16; d; d >>= 1) dot += __shfl_xor_sync(~0u, dot, d);
      __syncthreads();
      if (threadIdx.x % 32 == 0) part[threadIdx.x / 32] = dot;
      __syncthreads();
      if (threadIdx.x == 0) {
        float sum = 0.0f;
        for (int i = 0; i < 8; ++i) sum += part[i];
        a.dweights[t * a.k + s] = there ? sum : 0.0f;
      }
    }
  }
}

// ---- host --------------------------------------------------------------------------------

// Chunks of 32 to 128 tokens (more where there were thousands of them), the smallest that leave two
// blocks a multiprocessor or fewer: a warp chooses for its tokens one after the other (1024 tokens, 256
// experts, 8 slots: 56.4 us in chunks of 128, 16.6 in chunks of 32).  The blocks of the order
// kernel take as many chunks as keep their number near one a multiprocessor, or four, since each of them
// reads the whole table of counts.  (tokens > 0: there is nothing to cut otherwise.)
void plan_order(OrderArgs &o, int64_t tokens, int experts, int k, int ranks) {
  o.tokens = tokens, o.experts = experts, o.k = k, o.ranks = ranks;
  o.rank_tokens = tokens / ranks;
  int64_t chunk = 32;
  while (ceil_div(tokens, chunk) > (chunk < 128 ? 296 : 2048)) chunk *= 2;
  while (chunk * k > 65535) chunk /= 2;  // 16 bits hold a chunk's count of one expert
  o.chunk = (int)chunk;
  o.rank_chunks = ceil_div(o.rank_tokens, chunk);
  // Smaller groups where a rank's table of counts, which every block sums, is little beside a chunk's entries.
  // (Blocks for 592 and for 148: 65536 tokens, 64 experts, 2 slots, 8 ranks 22.8 and 26.9 us; 128 experts, 8
  // slots 63 and 87.  One rank, 16384 tokens, 64 experts, 2 slots 19.5 and 18.4; 256 experts, 8 slots 73 and 66.)
  const bool little = o.rank_chunks * experts <= 64 * chunk * k;
  o.group = (int)ceil_div(o.rank_chunks * ranks, little ? 592 : 148);
  o.rank_groups = ceil_div(o.rank_chunks, o.group);
}

int check_order(int64_t tokens, int experts, int k, int ranks) {
  if (tokens < 0 || experts < 1 || k < 1 || ranks < 1 || tokens % ranks != 0 || k > experts) return TUNA_ERR_INVALID_ARG;
  if (experts > TUNA_MOE_MAX_EXPERTS || k > kMaxK || tokens > ((int64_t)1 << 31) / k || ranks > TUNA_MOE_MAX_RANKS) return TUNA_ERR_RANGE;
  return TUNA_OK;
}

// counts and offsets of a call without tokens
int zero_order(const OrderArgs &o, int ranks, int experts, cudaStream_t st) {
  const size_t n = (size_t)ranks * experts;
  if (o.counts)
    if (const int rc = note_cuda(cudaMemsetAsync(o.counts, 0, n * 8, st))) return rc;
  if (o.offsets)
    if (const int rc = note_cuda(cudaMemsetAsync(o.offsets, 0, (n + 1) * 8, st))) return rc;
  return TUNA_OK;
}

int launch_order(const OrderArgs &o, cudaStream_t st) {
  static bool set[64] = {};
  if (const int rc = allow_smem(tuna_order_kernel, order_smem(TUNA_MOE_MAX_EXPERTS, kOrderThreads), set)) return rc;
  return launch(tuna_order_kernel, dim3((unsigned)(o.rank_groups * o.ranks)), kOrderThreads, order_smem(o.experts, kOrderThreads), st, false, o);
}

// Lanes a token and values a lane: the fewest lanes that hold the experts at 8 values each
// (one 16-byte load of bf16) and the slots at one a lane.  (With twice the lanes the choice among 64
// experts for 65536 tokens, 2 slots, took 48.7 us instead of 30.2 with its order, among 128, 8 slots, 186 instead of 107.)
template <typename F>
int by_width(int experts, int k, F f) {
  if (experts <= 64 && k <= 8) return f.template operator()<8, 8>();
  if (experts <= 128 && k <= 16) return f.template operator()<16, 8>();
  if (experts <= 256) return f.template operator()<32, 8>();
  return f.template operator()<32, 16>();
}
template <typename T>
struct RouteLaunch {
  const RouteArgs &a;
  const OrderArgs &o;
  cudaStream_t st;
  template <int LPT, int VPL>
  int operator()() {
    return launch(tuna_route_kernel<LPT, VPL, T>, dim3((unsigned)(o.rank_chunks * o.ranks)), kTopThreads, (size_t)a.experts * 4, st, false, a, o);
  }
};
template <typename T>
struct SmallLaunch {
  const RouteArgs &a;
  const OrderArgs &o;
  cudaStream_t st;
  template <int LPT, int VPL>
  int operator()() {
    static bool set[64] = {};
    if (const int rc = allow_smem(tuna_route_small_kernel<LPT, VPL, T>, order_smem(TUNA_MOE_MAX_EXPERTS, kSmallThreads), set)) return rc;
    return launch(tuna_route_small_kernel<LPT, VPL, T>, dim3(1), kSmallThreads, order_smem(a.experts, kSmallThreads), st, false, a, o);
  }
};
template <typename T>
struct GradLaunch {
  const RouteGradArgs &a;
  cudaStream_t st;
  template <int LPT, int VPL>
  int operator()() {
    return launch(tuna_route_grad_kernel<LPT, VPL, T>, dim3((unsigned)ceil_div(a.tokens, kTopThreads / LPT)), kTopThreads, 0, st, false, a);
  }
};

// Tokens that one block chooses for and orders in two rounds; it is then done before a second launch
// would be.  Three rounds are not.  (64 experts, 2 slots: 256 tokens 10.2 us against 15.0, 512 tokens
// 15.4 against 14.9; 256 experts, 8 slots: 64 tokens 14.2 against 16.5, 128 tokens 24.4 against 16.6.)
struct Lanes {
  template <int LPT, int VPL>
  int operator()() { return LPT; }
};
int64_t small_tokens(int experts, int k) { return 2 * kSmallThreads / by_width(experts, k, Lanes{}); }

// Choices that one block orders before two launches would be done.  (One block and two launches, us: 1 token, 64 experts, 2 slots 3.4 and 4.5;
// 64 tokens 3.9 and 4.7; 64 tokens, 512 experts, 8 slots 4.8 and 6.7; 128 tokens, 64 experts, 8 slots 5.7 and 5.2; 1024 tokens, 2 slots 7.7 and 5.2.)
constexpr int64_t kSmallEntries = 512;

size_t dtype_size(int dtype) { return dtype == TUNA_DTYPE_F32 ? 4 : dtype == TUNA_DTYPE_BF16 ? 2 : 0; }

}  // namespace

// The table of counts.
static size_t order_bytes(int64_t tokens, int experts, int k, int ranks) {
  if (tokens == 0) return 0;
  OrderArgs o = {};
  plan_order(o, tokens, experts, k, ranks);
  return (size_t)o.rank_chunks * ranks * experts * 2;
}

}  // namespace tuna_ops

using namespace tuna_ops;

extern "C" {

int tuna_moe_order_workspace_bytes(int64_t tokens, int experts, int k, int ranks, size_t *bytes) {
  if (!bytes) return TUNA_ERR_INVALID_ARG;
  if (const int rc = check_order(tokens, experts, k, ranks)) return rc;
  *bytes = (order_bytes(tokens, experts, k, ranks) + 255) / 256 * 256;
  return TUNA_OK;
}

int tuna_moe_route_workspace_bytes(int64_t tokens, int experts, int k, int ranks, size_t *bytes) {
  if (const int rc = tuna_moe_order_workspace_bytes(tokens, experts, k, ranks, bytes)) return rc;
  if (ranks == 1 && tokens <= small_tokens(experts, k)) *bytes = 0;
  return TUNA_OK;
}

int tuna_moe_order(const int32_t *ids, int64_t tokens, int experts, int k, int ranks, int64_t *counts, int64_t *offsets,
                   int64_t *rows, int64_t *pos, void *workspace, size_t workspace_bytes, void *stream) {
  if (const int rc = check_order(tokens, experts, k, ranks)) return rc;
  cudaStream_t st = (cudaStream_t)stream;
  OrderArgs o = {};
  o.counts = counts, o.offsets = offsets, o.rows = rows, o.pos = pos, o.ids = ids;
  if (tokens == 0) return zero_order(o, ranks, experts, st);
  if (!ids || !rows || !pos) return TUNA_ERR_INVALID_ARG;
  plan_order(o, tokens, experts, k, ranks);
  if (!workspace || !aligned(workspace, 256) || workspace_bytes < order_bytes(tokens, experts, k, ranks)) return TUNA_ERR_WORKSPACE;
  o.hist = (uint16_t *)workspace;
  if (ranks == 1 && tokens * k <= kSmallEntries) {
    static bool set[64] = {};
    if (const int rc = allow_smem(tuna_order_small_kernel, order_smem(TUNA_MOE_MAX_EXPERTS, kSmallThreads), set)) return rc;
    return launch(tuna_order_small_kernel, dim3(1), kSmallThreads, order_smem(experts, kSmallThreads), st, false, o);
  }
  if (const int rc = launch(tuna_order_hist_kernel, dim3((unsigned)(o.rank_chunks * ranks)), 256, (size_t)experts * 4, st, false, o)) return rc;
  return launch_order(o, st);
}

int tuna_moe_route(const void *logits, int dtype, int64_t tokens, int experts, int64_t ld, int k, int ranks, int scoring,
                   int renormalize, float scale, int32_t *ids, float *weights, int64_t *counts, int64_t *offsets, int64_t *rows,
                   int64_t *pos, void *workspace, size_t workspace_bytes, void *stream) {
  if (const int rc = check_order(tokens, experts, k, ranks)) return rc;
  if (!dtype_size(dtype) || (scoring != TUNA_MOE_SOFTMAX && scoring != TUNA_MOE_SIGMOID) || ld < experts) return TUNA_ERR_INVALID_ARG;
  cudaStream_t st = (cudaStream_t)stream;
  OrderArgs o = {};
  o.counts = counts, o.offsets = offsets, o.rows = rows, o.pos = pos, o.ids = ids;
  if (tokens == 0) return zero_order(o, ranks, experts, st);
  if (!logits || !ids || !weights || !rows || !pos || !aligned(logits, dtype_size(dtype))) return TUNA_ERR_INVALID_ARG;
  plan_order(o, tokens, experts, k, ranks);
  const bool small = ranks == 1 && tokens <= small_tokens(experts, k);
  if (!small && (!workspace || !aligned(workspace, 256) || workspace_bytes < order_bytes(tokens, experts, k, ranks))) return TUNA_ERR_WORKSPACE;
  o.hist = (uint16_t *)workspace;
  RouteArgs a = {};
  a.logits = logits, a.tokens = tokens, a.ld = ld, a.experts = experts, a.k = k;
  a.scoring = scoring, a.renormalize = renormalize != 0, a.scale = scale, a.ids = ids, a.weights = weights;
  a.vec = aligned(logits, 16) && ld * dtype_size(dtype) % 16 == 0;
  if (small)
    return dtype == TUNA_DTYPE_F32 ? by_width(experts, k, SmallLaunch<float>{a, o, st}) : by_width(experts, k, SmallLaunch<__nv_bfloat16>{a, o, st});
  const int rc = dtype == TUNA_DTYPE_F32 ? by_width(experts, k, RouteLaunch<float>{a, o, st})
                                         : by_width(experts, k, RouteLaunch<__nv_bfloat16>{a, o, st});
  return rc ? rc : launch_order(o, st);
}

int tuna_moe_route_backward(const void *logits, int dtype, int64_t tokens, int experts, int64_t ld, int k, int scoring,
                            int renormalize, float scale, const int32_t *ids, const float *dweights, void *dlogits, int64_t ldd,
                            void *stream) {
  if (const int rc = check_order(tokens, experts, k, 1)) return rc;
  if (!dtype_size(dtype) || (scoring != TUNA_MOE_SOFTMAX && scoring != TUNA_MOE_SIGMOID) || ld < experts || ldd < experts) return TUNA_ERR_INVALID_ARG;
  if (tokens == 0) return TUNA_OK;
  if (!logits || !ids || !dweights || !dlogits) return TUNA_ERR_INVALID_ARG;
  const size_t size = dtype_size(dtype);
  if (!aligned(logits, size) || !aligned(dlogits, size)) return TUNA_ERR_INVALID_ARG;
  RouteGradArgs a = {};
  a.logits = logits, a.tokens = tokens, a.ld = ld, a.ldd = ldd, a.experts = experts, a.k = k, a.scoring = scoring;
  a.renormalize = renormalize != 0, a.scale = scale, a.ids = ids, a.dweights = dweights, a.dlogits = dlogits;
  a.vec = aligned(logits, 16) && aligned(dlogits, 16) && ld * size % 16 == 0 && ldd * size % 16 == 0;
  return dtype == TUNA_DTYPE_F32 ? by_width(experts, k, GradLaunch<float>{a, (cudaStream_t)stream})
                                 : by_width(experts, k, GradLaunch<__nv_bfloat16>{a, (cudaStream_t)stream});
}

static int check_combine(CombineArgs &a, int y_dtype, int out_dtype) {
  const size_t sy = dtype_size(y_dtype), so = dtype_size(out_dtype);
  if (!sy || !so || a.rows < 0 || a.tokens < 0 || a.dim < 0 || a.k < 1 || a.ldy < a.dim || a.ldo < a.dim) return TUNA_ERR_INVALID_ARG;
  if (a.dim > kMaxDim || a.k > kMaxK || a.tokens > ((int64_t)1 << 31) / a.k) return TUNA_ERR_RANGE;
  if (a.tokens == 0 || a.dim == 0) return TUNA_OK;
  if (!a.weights || !a.pos || (a.rows > 0 && !a.y)) return TUNA_ERR_INVALID_ARG;
  return TUNA_OK;
}

int tuna_moe_combine(const void *y, int y_dtype, int64_t rows, int dim, int64_t ldy, const float *weights, const int64_t *pos,
                     int64_t tokens, int k, void *out, int out_dtype, int64_t ldo, void *stream) {
  CombineArgs a = {};
  a.y = y, a.weights = weights, a.pos = pos, a.out = out, a.rows = rows, a.tokens = tokens, a.ldy = ldy, a.ldo = ldo, a.dim = dim, a.k = k;
  if (const int rc = check_combine(a, y_dtype, out_dtype)) return rc;
  if (tokens == 0 || dim == 0) return TUNA_OK;
  const size_t sy = dtype_size(y_dtype), so = dtype_size(out_dtype);
  if (!out || !aligned(y, sy) || !aligned(out, so)) return TUNA_ERR_INVALID_ARG;
  a.vec = dim % 8 == 0 && aligned(y, 16) && aligned(out, 16) && ldy * sy % 16 == 0 && ldo * so % 16 == 0;
  const dim3 grid((unsigned)std::min<int64_t>(tokens, 1 << 20), (unsigned)ceil_div(dim, 2048));
  cudaStream_t st = (cudaStream_t)stream;
  if (y_dtype == TUNA_DTYPE_F32)
    return out_dtype == TUNA_DTYPE_F32 ? launch(tuna_combine_kernel<float, float>, grid, 256, 0, st, false, a)
                                       : launch(tuna_combine_kernel<float, __nv_bfloat16>, grid, 256, 0, st, false, a);
  return out_dtype == TUNA_DTYPE_F32 ? launch(tuna_combine_kernel<__nv_bfloat16, float>, grid, 256, 0, st, false, a)
                                     : launch(tuna_combine_kernel<__nv_bfloat16, __nv_bfloat16>, grid, 256, 0, st, false, a);
}

int tuna_moe_combine_backward(const void *dout, int out_dtype, int64_t lddo, const void *y, int y_dtype, int64_t rows, int dim,
                              int64_t ldy, const float *weights, const int64_t *pos, int64_t tokens, int k, void *dy, int64_t lddy,
                              float *dweights, void *stream) {
  CombineArgs a = {};
  a.y = y, a.dout = dout, a.weights = weights, a.pos = pos, a.dy = dy, a.dweights = dweights;
  a.rows = rows, a.tokens = tokens, a.ldy = ldy, a.ldo = lddo, a.lddy = lddy, a.dim = dim, a.k = k;
  if (lddy < dim) return TUNA_ERR_INVALID_ARG;
  if (const int rc = check_combine(a, y_dtype, out_dtype)) return rc;
  if (tokens == 0) return TUNA_OK;
  if (dim == 0) return dweights ? note_cuda(cudaMemsetAsync(dweights, 0, (size_t)tokens * k * 4, (cudaStream_t)stream)) : TUNA_ERR_INVALID_ARG;  // empty sums
  const size_t sy = dtype_size(y_dtype), so = dtype_size(out_dtype);
  if (!dout || !dweights || (rows > 0 && !dy) || !aligned(y, sy) || !aligned(dy, sy) || !aligned(dout, so)) return TUNA_ERR_INVALID_ARG;
  a.vec = dim % 8 == 0 && aligned(y, 16) && aligned(dy, 16) && aligned(dout, 16) && ldy * sy % 16 == 0 && lddy * sy % 16 == 0 && lddo * so % 16 == 0;
  const dim3 grid((unsigned)std::min<int64_t>(tokens, (int64_t)sm_count() * 16));
  cudaStream_t st = (cudaStream_t)stream;
  if (y_dtype == TUNA_DTYPE_F32)
    return out_dtype == TUNA_DTYPE_F32 ? launch(tuna_combine_grad_kernel<float, float>, grid, 256, 0, st, false, a)
                                       : launch(tuna_combine_grad_kernel<float, __nv_bfloat16>, grid, 256, 0, st, false, a);
  return out_dtype == TUNA_DTYPE_F32 ? launch(tuna_combine_grad_kernel<__nv_bfloat16, float>, grid, 256, 0, st, false, a)
                                     : launch(tuna_combine_grad_kernel<__nv_bfloat16, __nv_bfloat16>, grid, 256, 0, st, false, a);
}

int tuna_ops_device_status(int *gave_up) {
  if (!gave_up) return TUNA_ERR_INVALID_ARG;
  int *word = error_word();
  if (!word) return TUNA_ERR_CUDA;
  if (const int rc = note_cuda(cudaDeviceSynchronize())) return rc;
  if (const int rc = note_cuda(cudaMemcpy(gave_up, word, sizeof(int), cudaMemcpyDeviceToHost))) return rc;
  return *gave_up ? note_cuda(cudaMemset(word, 0, sizeof(int))) : TUNA_OK;  // the next report is of later calls
}

int tuna_ops_cuda_error(void) { return t_cuda_error; }

}  // extern "C"
