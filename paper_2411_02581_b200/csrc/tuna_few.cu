// A whole mixture-of-experts layer for a few tokens, in one kernel:
//
//   logits = x Wr^T; the k best experts of every token and their weights w;
//   h = silu(x Wg^T) * (x Wu^T) and y = h Wd^T for every (token, expert) chosen;
//   out = sum over the chosen of w y
//
// For so few tokens the layer is bound by reading the chosen experts' weights once (3 D I
// values an expert), so everything else has to stay out of that stream's way.  A block a
// multiprocessor (cooperative launch: the phases are separated by barriers across the grid)
// brings 128 weight rows x 256 bytes at a time into a ring of four stages, 128 KB in flight; the
// tensor cores take them from there as the 128-row operand, with the tokens of one expert as the
// columns of the other one.  The weights are never touched by a thread.  (With stages of half the size
// the thread that issues the steps could not keep up: 840 cycles for 16 KB, and 700 are the memory's
// pace.)  The first form of this
// kernel multiplied with m16n8k16 steps out of registers; widening 8-bit weights to 16 bits and
// adding up the warps' partial sums left it at a quarter of the memory rate (64 tokens: 887 us).
//
// A unit of work is 128 rows x a segment of the contracted axis; segments make enough units for
// all blocks when a token or two meet few experts, and their sums meet in memory: 32-bit partial
// sums of gate and up, which the threads that lay out h add up (SwiGLU is applied there), and of
// y, which the last phase adds up with the tokens' weights.  Nothing is summed in an order that
// depends on timing.
//
// bf16 weights meet x and h in bf16.  h is rounded to it once (2^-9 of each value, as a two-kernel layer would
// store it), because the tensor cores multiply both operands in one type and in 32 bits at half the rate or less.
// 8-bit weights meet two 8-bit pieces of each token value, x = s (p + q / 16) with s a power of
// two for each 128 values, the largest of which lies in [2^7, 2^8) s.  p keeps 4 significant bits and q the
// next 4 while the value is at least 2^-6 s: 8 bits, all that x has and what bf16 would keep of h, down to 2^-13 of
// the block's largest value.  Below, the step of q is fixed, and the error at most 2^-14 s, 2^-21 of the largest.  The pieces are columns of their
// own; a block of 128 is one accumulation, which four warps multiply by the weights' scale.
#include <algorithm>
#include <cmath>
#include <type_traits>

#include "tuna_ops.cuh"
#include "tuna_route.cuh"

namespace tuna_ops {
namespace {

constexpr int kThreads = 512, kWarps = 16;
constexpr int kMaxTokens = TUNA_MOE_FEW_MAX_TOKENS;
constexpr int kStages = 4, kBlockBytes = 128 * 128, kStageBytes = 2 * kBlockBytes;  // a stage: two blocks of 128 rows x 128 bytes
constexpr int kTile = 16;                 // tokens of a group: more of one expert form another group
constexpr int kBufs = 4, kBufCols = 64;   // accumulators in tensor memory: two of 32 columns (8-bit), or one
constexpr int kOperand = 32 * 1024;       // token operand of a segment (two of them)
constexpr int kSplit = kWarps * 64;       // columns of x that a block takes in the router phase
constexpr int kMaxDimFew = 8192;
constexpr int kLoaders = 8;               // warps that lay out the token operands

struct FewArgs {
  const __nv_bfloat16 *x, *router;
  const float *s13, *s2;
  __nv_bfloat16 *out;
  int32_t *ids_out;
  float *weights_out;
  int64_t ldx, ldo;
  int tokens, experts, k, hidden, inter, scoring, renormalize;
  float scale;
  int segment[2], segments[2];  // of either product: 128-byte blocks of a row, and how many segments
  // workspace
  unsigned long long *barrier;  // arrivals of all calls: zero before the first one
  float *part;         // [splits][tokens][experts] logits of a split
  int32_t *ids;        // [tokens * k]
  float *weights;      // [tokens * k]
  float *up;           // [segments][tokens * k][2 inter]
  float *y;            // [segments][tokens * k][hidden]
  int *error;
};

struct Group {
  int16_t expert, first, count;
};
constexpr int kMaxEntries = kMaxTokens * kMaxK;
constexpr int kMaxGroups = TUNA_MOE_MAX_EXPERTS + kMaxEntries / kTile;

// What stays in shared memory through both products.
struct Lists {
  uint64_t full[kStages], empty[kStages], done[kBufs], freed[kBufs], laid[2], used[2], drained;
  alignas(16) float piece_scale[2][8][kTile];  // s of the token operand: operand, block, token
  int16_t entry[kMaxEntries];         // token * k + slot, by expert
  Group group[kMaxGroups];
  int groups, given_up, met;  // met: meetings that the block has arrived at
  uint32_t tmem;
};
// What is needed only until the lists are made: lies where the stages are later.
struct Choice {
  int16_t id[kMaxEntries];
  int16_t begin[TUNA_MOE_MAX_EXPERTS + 1];
  int count[TUNA_MOE_MAX_EXPERTS];
};

constexpr size_t kFewSmem = 1024 + (size_t)kStages * kStageBytes + 2 * kOperand + sizeof(Lists);
static_assert(kFewSmem <= 227 * 1024, "shared memory of a block");
static_assert(kWarps * (kMaxTokens / 8) * 32 * 16 <= kStages * kStageBytes && sizeof(Choice) <= kStages * kStageBytes, "what lies where the stages are later");

__device__ __forceinline__ void mma_bf16(float (&c)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
  asm("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
      : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3]) : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}

// All blocks of the grid meet: one thread arrives for its block (after a barrier of the block), any
// thread may wait.  The counter only grows, by the grid's size at each meeting, so that an arrival is one
// addition and a wait one load (with a generation word that the last block advances, one token took 34 us
// instead of 30).  64 bits never wrap.  A block adds kMeetings to it in every call, also one that gave up a wait:
// the count is then a multiple of the grid's size after every call, and the next one finds its base.
constexpr int kMeetings = 3;
__device__ __forceinline__ unsigned long long meeting_base(const unsigned long long *bar) {
  // read before this block's first arrival: the count is then short of the next multiple
  unsigned long long v;
  asm volatile("ld.relaxed.gpu.global.u64 %0, [%1];" : "=l"(v) : "l"(bar) : "memory");
  return v - v % gridDim.x;
}
__device__ __forceinline__ void grid_arrive(unsigned long long *bar, unsigned long long times = 1) {
  asm volatile("red.release.gpu.global.add.u64 [%0], %1;" ::"l"(bar), "l"(times) : "memory");
}
__device__ bool grid_wait(const unsigned long long *bar, unsigned long long target, volatile int *given_up) {
  const long long t0 = clock64();
  for (;;) {
    unsigned long long v;
    asm volatile("ld.acquire.gpu.global.u64 %0, [%1];" : "=l"(v) : "l"(bar) : "memory");
    if (v >= target) return true;
    if (*given_up || clock64() - t0 > kWaitCycles) {
      *given_up = 1;
      return false;
    }
  }
}
__device__ bool grid_meet(unsigned long long *bar, unsigned long long target, int *given_up) {
  __syncthreads();
  if (threadIdx.x == 0) grid_arrive(bar), grid_wait(bar, target, given_up);
  __syncthreads();
  return !*(volatile int *)given_up;
}

// One of the two products as a block sees it.
struct Product {
  int tiles, segments, segment, blocks;  // row tiles; segments; blocks of a segment, of a row
  int unit0, unit1;                      // this block's units, row tiles fastest, then segments, then groups
};
// A walk over a block's units.  Every role steps through its own; divisions are done once, at the start.
struct Unit {
  int left;               // units from here on
  int g, s, m, blocks;    // group, segment, row tile; blocks of the segment
  __device__ __forceinline__ Unit(const Product &p) {
    left = p.unit1 - p.unit0;
    const int q = p.unit0 / p.tiles;
    m = p.unit0 - q * p.tiles;
    g = q / p.segments;
    s = q - g * p.segments;
    blocks = min(p.segment, p.blocks - s * p.segment);
  }
  __device__ __forceinline__ void turn(const Product &p) {  // to the next segment or group
    m = 0;
    if (++s == p.segments) s = 0, ++g;
    blocks = min(p.segment, p.blocks - s * p.segment);
  }
  __device__ __forceinline__ void step(const Product &p) {
    --left;
    if (++m == p.tiles) turn(p);
  }
  __device__ __forceinline__ bool last(const Product &p) const { return left == 1 || m + 1 == p.tiles; }  // of its group and segment
};

// Position of a 16-byte piece in a swizzled operand of rows of 128 bytes.
__device__ __forceinline__ uint32_t swizzled(int row, int piece) { return (uint32_t)((row >> 3) * 1024 + (row & 7) * 128 + ((piece ^ (row & 7)) * 16)); }

__device__ __forceinline__ float2 e4m3_values(uint32_t two) {
  uint32_t h;
  asm("cvt.rn.f16x2.e4m3x2 %0, %1;" : "=r"(h) : "h"((uint16_t)two));
  __half2 v = *reinterpret_cast<__half2 *>(&h);
  return __half22float2(v);
}

template <bool FP8>
__global__ void __launch_bounds__(kThreads, 1)
    tuna_few_kernel(const __grid_constant__ CUtensorMap map13, const __grid_constant__ CUtensorMap map2, const FewArgs a) {
  extern __shared__ char smem_raw[];
  char *smem = smem_raw + ((1024 - (smem_u32(smem_raw) & 1023)) & 1023);
  const uint32_t ring = smem_u32(smem), operands = ring + kStages * kStageBytes;
  Lists &l = *(Lists *)(smem + kStages * kStageBytes + 2 * kOperand);
  const int tid = threadIdx.x, warp = __shfl_sync(~0u, tid >> 5, 0), lane = tid & 31, row_in = lane >> 2, quad = lane & 3;
  const int T = a.tokens, E = a.experts, K = a.k, D = a.hidden, I = a.inter, n = T * K;
  const int splits = (D + kSplit - 1) / kSplit;
  if (tid == 0) {
    l.given_up = 0, l.met = 1;
    for (int i = 0; i < kStages; ++i) mbar_init(smem_u32(l.full + i), 1), mbar_init(smem_u32(l.empty + i), 1);
    for (int i = 0; i < kBufs; ++i) mbar_init(smem_u32(l.done + i), 1), mbar_init(smem_u32(l.freed + i), 4);
    for (int i = 0; i < 2; ++i) mbar_init(smem_u32(l.laid + i), kLoaders), mbar_init(smem_u32(l.used + i), 5);
    mbar_init(smem_u32(&l.drained), 1);
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  }
  if (warp == 2) tmem_alloc(smem_u32(&l.tmem), kBufs * kBufCols);
  const unsigned long long base = meeting_base(a.barrier);

  // ---- logits: a block takes 16 experts and 1024 columns, a warp 64 of them
  {
    const int units = (E + 15) / 16 * splits, nt = (T + 7) / 8;
    float4 *sums = (float4 *)smem;  // [token tile][warp][lane]
    for (int u = blockIdx.x; u < units; u += gridDim.x) {
      const int m = u / splits, split = u - m * splits;
      const int col = split * kSplit + warp * 64 + quad * 8, e0 = m * 16 + row_in, e1 = e0 + 8;
      const uint4 none = make_uint4(0, 0, 0, 0);
      uint4 w0[2], w1[2];
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        const bool in = col + h * 32 < D;
        w0[h] = in && e0 < E ? __ldg((const uint4 *)(a.router + (int64_t)e0 * D + col + h * 32)) : none;
        w1[h] = in && e1 < E ? __ldg((const uint4 *)(a.router + (int64_t)e1 * D + col + h * 32)) : none;
      }
#pragma unroll 4
      for (int j = 0; j < nt; ++j) {
        const int t = j * 8 + row_in;
        float c[4] = {};
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          const uint4 v = col + h * 32 < D && t < T ? __ldg((const uint4 *)(a.x + t * a.ldx + col + h * 32)) : none;
          mma_bf16(c, w0[h].x, w1[h].x, w0[h].y, w1[h].y, v.x, v.y);
          mma_bf16(c, w0[h].z, w1[h].z, w0[h].w, w1[h].w, v.z, v.w);
        }
        sums[(j * kWarps + warp) * 32 + lane] = make_float4(c[0], c[1], c[2], c[3]);
      }
      __syncthreads();
      for (int j = warp; j < nt; j += kWarps) {
        float4 s = make_float4(0, 0, 0, 0);
#pragma unroll
        for (int w = 0; w < kWarps; ++w) {
          const float4 v = sums[(j * kWarps + w) * 32 + lane];
          s.x += v.x, s.y += v.y, s.z += v.z, s.w += v.w;
        }
        const float r[4] = {s.x, s.y, s.z, s.w};
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const int t = j * 8 + quad * 2 + (i & 1), e = m * 16 + row_in + (i >> 1) * 8;
          if (t < T && e < E) a.part[((int64_t)split * T + t) * E + e] = r[i];
        }
      }
      __syncthreads();
    }
  }
  bool fine = grid_meet(a.barrier, base + gridDim.x, &l.given_up);

  if (fine) {
    // ---- the choice, by every block for itself; the fewer experts, the more tokens a warp takes
    Choice &c = *(Choice *)smem;
    auto take = [&](auto lanes, auto values) {
      constexpr int LPT = decltype(lanes)::value, VPL = decltype(values)::value;
      const int in = lane % LPT;
      for (int t0 = warp * (32 / LPT); t0 < T; t0 += kWarps * (32 / LPT)) {
        const int t = t0 + lane / LPT;
        float z[VPL];
#pragma unroll
        for (int i = 0; i < VPL; ++i) z[i] = t < T && in * VPL + i < E ? 0.0f : -INFINITY;
        if (t < T) {
          const float *part = a.part + (int64_t)t * E + in * VPL;
#pragma unroll 8
          for (int q = 0; q < splits; ++q) {
#pragma unroll
            for (int i = 0; i < VPL; ++i)
              if (in * VPL + i < E) z[i] += __ldcg(part + (int64_t)q * T * E + i);
          }
        }
#pragma unroll
        for (int i = 0; i < VPL; ++i) z[i] = logit_of(z[i]);
        int id;
        float w;
        choose<LPT>(z, in, K, a.scoring, a.renormalize, a.scale, id, w);
        if (t < T && in < K) {
          c.id[t * K + in] = (int16_t)id;
          if (blockIdx.x == 0) {
            a.ids[t * K + in] = id, a.weights[t * K + in] = w;
            if (a.ids_out) a.ids_out[t * K + in] = id;
            if (a.weights_out) a.weights_out[t * K + in] = w;
          }
        }
      }
    };
    using std::integral_constant;
    if (E <= 64 && K <= 8)
      take(integral_constant<int, 8>(), integral_constant<int, 8>());
    else if (E <= 256)
      take(integral_constant<int, 32>(), integral_constant<int, 8>());
    else
      take(integral_constant<int, 32>(), integral_constant<int, 16>());
    for (int e = tid; e < E; e += kThreads) c.count[e] = 0;
    __syncthreads();
    for (int i = tid; i < n; i += kThreads)
      if (c.id[i] >= 0) atomicAdd(&c.count[c.id[i]], 1);
    __syncthreads();
    if (warp == 0) {
      // first entry of each expert, and the groups
      int entries = 0, groups = 0;
      for (int e0 = 0; e0 < E; e0 += 32) {
        const int v = e0 + lane < E ? c.count[e0 + lane] : 0, g = (v + kTile - 1) / kTile;
        int xc = v, xg = g;
#pragma unroll
        for (int d = 1; d < 32; d <<= 1) {
          const int yc = __shfl_up_sync(~0u, xc, d), yg = __shfl_up_sync(~0u, xg, d);
          if (lane >= d) xc += yc, xg += yg;
        }
        if (e0 + lane < E) {
          c.begin[e0 + lane] = (int16_t)(entries + xc - v);
          for (int i = 0; i < g; ++i)
            l.group[groups + xg - g + i] = {(int16_t)(e0 + lane), (int16_t)(entries + xc - v + i * kTile), (int16_t)min(kTile, v - i * kTile)};
        }
        entries += __shfl_sync(~0u, xc, 31), groups += __shfl_sync(~0u, xg, 31);
      }
      if (lane == 0) l.groups = groups;
      __syncwarp();
      for (int i0 = 0; i0 < n; i0 += 32) {
        const int id = i0 + lane < n ? c.id[i0 + lane] : -1;
        const uint32_t peers = __match_any_sync(~0u, id);
        const int at = id >= 0 ? c.begin[id] : 0;
        __syncwarp();
        if (id >= 0) {
          l.entry[at + __popc(peers & ((1u << lane) - 1))] = (int16_t)(i0 + lane);
          if (lane == __ffs(peers) - 1) c.begin[id] = (int16_t)(at + __popc(peers));
        }
        __syncwarp();
      }
    }
    asm volatile("fence.proxy.async.shared::cta;" ::: "memory");  // the copies overwrite what was written here
    tc_fence_before();
    __syncthreads();
    tc_fence_after();

    // ---- the two products
    const int groups = l.groups;
    const uint32_t tmem = __shfl_sync(~0u, l.tmem, 0);
    constexpr int kBlock = FP8 ? 128 : 64;  // columns of a block
    int stage = 0, stage_phase = 0, buf = 0, buf_phase = 0, op = 0, op_phase = 0;
    bool ok = true;
#pragma unroll 1
    for (int phase = 0; phase < 2; ++phase) {
      const bool up = phase == 0;
      const int cols = up ? D : I, rows = up ? 2 * I : D;
      Product p;
      p.tiles = (rows + 127) / 128, p.blocks = (cols + kBlock - 1) / kBlock, p.segment = a.segment[phase], p.segments = a.segments[phase];
      // (at most 640 groups x 8 segments x 128 tiles: the products below fit 32 bits)
      const uint32_t units = (uint32_t)groups * p.segments * p.tiles;
      p.unit0 = (int)(units * blockIdx.x / gridDim.x), p.unit1 = (int)(units * (blockIdx.x + 1) / gridDim.x);
      if (warp == 0) {
        // -- weights
        if (lane == 0) {
          const CUtensorMap *map = up ? &map13 : &map2;
          for (Unit w(p); ok && w.left > 0; w.step(p)) {
            const int expert = l.group[w.g].expert;
            for (int b = 0; b < w.blocks; b += 2) {
              if (!(ok = mbar_wait(smem_u32(l.empty + stage), stage_phase ^ 1, &l.given_up))) break;
              const uint32_t bar = smem_u32(l.full + stage), to = ring + stage * kStageBytes;
              const int col = (w.s * p.segment + b) * kBlock;
              const bool both = b + 1 < w.blocks;
              mbar_expect(bar, both ? kStageBytes : kBlockBytes);
              tma_load_3d(to, map, col, w.m * 128, expert, bar);
              if (both) tma_load_3d(to + kBlockBytes, map, col + kBlock, w.m * 128, expert, bar);
              if (++stage == kStages) stage = 0, stage_phase ^= 1;
            }
          }
        }
      } else if (warp == 1) {
        // -- tensor cores (the whole warp walks, one lane issues)
        {
          bool held = false;  // the group's and segment's operand is at hand
          for (Unit w(p); ok && w.left > 0; w.step(p)) {
            if (!held && !(ok = __all_sync(~0u, mbar_wait(smem_u32(l.laid + op), op_phase, &l.given_up)))) break;
            held = !w.last(p);
            const int N = FP8 && l.group[w.g].count > 8 ? 32 : 16;
            const uint32_t idesc = (1u << 4) | (FP8 ? 0u : (1u << 7) | (1u << 10)) | ((uint32_t)(N >> 3) << 17) | ((uint32_t)(128 >> 4) << 24);
            for (int b = 0; b < w.blocks; b += 2) {
              if (!(ok = __all_sync(~0u, mbar_wait(smem_u32(l.full + stage), stage_phase, &l.given_up)))) break;
              if (FP8 || b == 0)
                if (!(ok = __all_sync(~0u, mbar_wait(smem_u32(l.freed + buf), buf_phase ^ 1, &l.given_up)))) break;
              tc_fence_after();
              const uint64_t da = tc_desc(ring + stage * kStageBytes), db = tc_desc(operands + op * kOperand + b * N * 128);
              const uint32_t d = tmem + buf * kBufCols;
              const bool out = FP8 || b + 2 >= w.blocks;  // the accumulator is complete
              if (elect_one()) {
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                  if (h && b + 1 >= w.blocks) break;
#pragma unroll
                  for (int i = 0; i < 4; ++i) {
                    const uint64_t ha = da + h * (kBlockBytes >> 4) + 2 * i, hb = db + h * (N * 128 >> 4) + 2 * i;
                    if (FP8)
                      tc_mma_fp8(d + h * 32, ha, hb, idesc, i > 0);
                    else
                      tc_mma_bf16(d, ha, hb, idesc, b > 0 || h > 0 || i > 0);
                  }
                }
                tc_commit(smem_u32(l.empty + stage));
                if (out) tc_commit(smem_u32(l.done + buf));
              }
              __syncwarp();
              if (++stage == kStages) stage = 0, stage_phase ^= 1;
              if (out && ++buf == kBufs) buf = 0, buf_phase ^= 1;
            }
            if (ok && !held) {
              if (elect_one()) tc_commit(smem_u32(l.used + op));
              __syncwarp();
              if (++op == 2) op = 0, op_phase ^= 1;
            }
          }
        }
      } else if (warp >= 4 && warp < 8) {
        // -- sums: a thread has one weight row, a register for each token
        const int mine = (warp & 3) * 32 + lane;
        const uint32_t from = tmem + ((uint32_t)((warp & 3) * 32) << 16);
        float *to = up ? a.up : a.y;
        const int block_rows = up ? 2 * ((I + 127) / 128) : (D + 127) / 128;
        // the scales of a unit's blocks for this row
        auto fetch = [&](const Unit &w, float (&ws)[8]) {
          if (!FP8 || w.left <= 0) return;
          const int r = min(w.m * 128 + mine, rows - 1);
          const int br = up && r >= I ? (I + 127) / 128 + (r - I) / 128 : r / 128;
          const float *s = (up ? a.s13 : a.s2) + ((int64_t)l.group[w.g].expert * block_rows + br) * p.blocks + w.s * p.segment;
#pragma unroll
          for (int b = 0; b < 8; ++b) ws[b] = __ldg(s + min(b, w.blocks - 1));
        };
        float next[8];
        Unit ahead(p);
        fetch(ahead, next);
        for (Unit w(p); ok && w.left > 0; w.step(p)) {
          const int first = l.group[w.g].first, count = l.group[w.g].count;
          float ws[8], acc[kTile];
#pragma unroll
          for (int b = 0; b < 8; ++b) ws[b] = next[b];
#pragma unroll
          for (int i = 0; i < kTile; ++i) acc[i] = 0.0f;
          ahead.step(p);
          fetch(ahead, next);
          if constexpr (FP8) {
#pragma unroll
            for (int b = 0; b < 8; b += 2) {
              if (b >= w.blocks) break;
              ok = __all_sync(~0u, mbar_wait(smem_u32(l.done + buf), buf_phase, &l.given_up));
              if (!ok) break;
              tc_fence_after();
              // below 9 tokens, the pieces p and q of a block are 8 columns each, else 16
              uint32_t v[2][32];
              if (count > 8) {
                tmem_load(from + buf * kBufCols, v[0]);
                tmem_load(from + buf * kBufCols + 32, v[1]);
              } else {
                tmem_load(from + buf * kBufCols, reinterpret_cast<uint32_t(&)[16]>(v[0]));
                tmem_load(from + buf * kBufCols + 32, reinterpret_cast<uint32_t(&)[16]>(v[1]));
              }
              tmem_wait(v[0]);
              tmem_wait(v[1]);
              tc_fence_before();
              __syncwarp();
              if (lane == 0) mbar_arrive(smem_u32(l.freed + buf));
#pragma unroll
              for (int h = 0; h < 2; ++h) {
                if (b + h >= w.blocks) break;
                const float4 *xs = (const float4 *)l.piece_scale[op][b + h];
                if (count > 8) {
#pragma unroll
                  for (int i = 0; i < 16; i += 4) {
                    const float4 s = xs[i / 4];
                    const float f[4] = {s.x, s.y, s.z, s.w};
#pragma unroll
                    for (int j = 0; j < 4; ++j)
                      acc[i + j] = fmaf(fmaf(__uint_as_float(v[h][16 + i + j]), 0.0625f, __uint_as_float(v[h][i + j])), ws[b + h] * f[j], acc[i + j]);
                  }
                } else {
#pragma unroll
                  for (int i = 0; i < 8; i += 4) {
                    const float4 s = xs[i / 4];
                    const float f[4] = {s.x, s.y, s.z, s.w};
#pragma unroll
                    for (int j = 0; j < 4; ++j)
                      acc[i + j] = fmaf(fmaf(__uint_as_float(v[h][8 + i + j]), 0.0625f, __uint_as_float(v[h][i + j])), ws[b + h] * f[j], acc[i + j]);
                  }
                }
              }
              if (++buf == kBufs) buf = 0, buf_phase ^= 1;
            }
          } else {
            ok = __all_sync(~0u, mbar_wait(smem_u32(l.done + buf), buf_phase, &l.given_up));
            if (ok) {
              tc_fence_after();
              uint32_t v[16];
              tmem_load(from + buf * kBufCols, v);
              tmem_wait(v);
              tc_fence_before();
              __syncwarp();
              if (lane == 0) mbar_arrive(smem_u32(l.freed + buf));
#pragma unroll
              for (int i = 0; i < kTile; ++i) acc[i] = __uint_as_float(v[i]);
              if (++buf == kBufs) buf = 0, buf_phase ^= 1;
            }
          }
          if (!ok) break;
          const int r = w.m * 128 + mine;
          if (r < rows) {
#pragma unroll
            for (int i = 0; i < kTile; ++i)
              if (i < count) to[((int64_t)w.s * n + l.entry[first + i]) * rows + r] = acc[i];
          }
          if (w.last(p)) {
            __syncwarp();
            if (lane == 0) mbar_arrive(smem_u32(l.used + op));
            if (++op == 2) op = 0, op_phase ^= 1;
          }
        }
      } else if (warp >= kWarps - kLoaders && p.unit0 < p.unit1) {
        // -- the tokens' operands, a (group, segment) ahead of the tensor cores
        if (!up) ok = __all_sync(~0u, lane != 0 || grid_wait(a.barrier, base + 2ull * gridDim.x, &l.given_up));  // every block's sums are there
        const int i0 = tid - (kWarps - kLoaders) * 32;
        for (Unit w(p); ok && w.left > 0; w.left -= p.tiles - w.m, w.turn(p)) {
          const int first = l.group[w.g].first, count = l.group[w.g].count, N = FP8 && count > 8 ? 32 : 16;
          ok = __all_sync(~0u, mbar_wait(smem_u32(l.used + op), op_phase ^ 1, &l.given_up));
          if (!ok) break;
          // A warp takes 128 columns of a token at a time, a lane four of them, several such pieces in flight.
          // The loads of a piece are issued together: one after the other, the four segments' sums of a
          // nine-token group took 80000 cycles to lay out, and the grid waited for that block.
          const int spans = (w.blocks * kBlock + 127) / 128, pieces = spans * count;
          struct Piece {
            int t, span;
            float v[4];
          };
          auto aim = [&](Piece &x, int i) {  // the piece's place; its columns (cols is a multiple of 16: all four or none)
            x.span = i / count, x.t = i - x.span * count;
            return w.s * p.segment * kBlock + x.span * 128 + lane * 4;
          };
          auto load_x = [&](int i) {
            Piece x;
            const int col = aim(x, i);
            if (i >= pieces || col >= cols) return make_uint2(0, 0);
            return __ldg((const uint2 *)(a.x + (l.entry[first + x.t] / K) * a.ldx + col));
          };
          auto load_h = [&](Piece &x, int i) {
            const int col = aim(x, i);
#pragma unroll
            for (int j = 0; j < 4; ++j) x.v[j] = 0.0f;
            if (i >= pieces || col >= cols) return;
            float u[4] = {0.0f, 0.0f, 0.0f, 0.0f};
            const float *g0 = a.up + (int64_t)l.entry[first + x.t] * 2 * I + col;
            const int64_t step = (int64_t)n * 2 * I;
            const float4 zero = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
            for (int s0 = 0; s0 < a.segments[0]; s0 += 4) {
              float4 gs[4], us[4];
#pragma unroll
              for (int s = 0; s < 4; ++s) {
                const bool there = s0 + s < a.segments[0];
                gs[s] = there ? __ldcg((const float4 *)(g0 + (s0 + s) * step)) : zero;
                us[s] = there ? __ldcg((const float4 *)(g0 + (s0 + s) * step + I)) : zero;
              }
#pragma unroll
              for (int s = 0; s < 4; ++s) {
                x.v[0] += gs[s].x, x.v[1] += gs[s].y, x.v[2] += gs[s].z, x.v[3] += gs[s].w;
                u[0] += us[s].x, u[1] += us[s].y, u[2] += us[s].z, u[3] += us[s].w;
              }
            }
#pragma unroll
            for (int j = 0; j < 4; ++j) x.v[j] = __fdividef(x.v[j], 1.0f + __expf(-x.v[j])) * u[j];  // (2^-21: h keeps 8 bits)
          };
          auto lay = [&](const Piece &x) {
            if constexpr (FP8) {
              uint32_t top = max(max(abs_bits(x.v[0]), abs_bits(x.v[1])), max(abs_bits(x.v[2]), abs_bits(x.v[3])));
              top = __reduce_max_sync(~0u, top);
              // s takes the block's largest value to [2^7, 2^8), whatever it is (exponents 1 to 254 leave e in 20 to 247);
              // a block that is not finite is lost to NaN
              const int e = min(max((int)(top >> 23), 27) - 7, 247);
              const float s = top >= 0x7f800000u ? __uint_as_float(0x7fc00000u) : __uint_as_float((uint32_t)e << 23);
              const float by = __uint_as_float((uint32_t)(254 - e) << 23);
              uint32_t h2[2], l2[2];
#pragma unroll
              for (int j = 0; j < 2; ++j) {
                const float f = x.v[2 * j] * by, g = x.v[2 * j + 1] * by;
                h2[j] = e4m3_pair(f, g);
                const float2 have = e4m3_values(h2[j]);
                l2[j] = e4m3_pair((f - have.x) * 16.0f, (g - have.y) * 16.0f);
              }
              const uint32_t to = operands + op * kOperand + x.span * N * 128 + (lane & 3) * 4;
              asm volatile("st.shared.b32 [%0], %1;" ::"r"(to + swizzled(x.t, lane >> 2)), "r"(h2[0] | (h2[1] << 16)) : "memory");
              asm volatile("st.shared.b32 [%0], %1;" ::"r"(to + swizzled(N / 2 + x.t, lane >> 2)), "r"(l2[0] | (l2[1] << 16)) : "memory");
              if (lane == 0) l.piece_scale[op][x.span][x.t] = s;
            } else {
              // (two blocks of 64; the second may lie behind the segment, where its place is unused)
              const int b = x.span * 2 + (lane >> 4);
              if (b < w.blocks)
                asm volatile("st.shared.v2.b32 [%0], {%1, %2};" ::"r"(operands + op * kOperand + b * N * 128 + swizzled(x.t, (lane & 15) >> 1) + (lane & 1) * 8),
                             "r"(pack_bf16(x.v[0], x.v[1])), "r"(pack_bf16(x.v[2], x.v[3]))
                             : "memory");
            }
          };
          if (up) {
            constexpr int kFlight = 6;
            for (int i = i0 >> 5; i < pieces; i += kFlight * kLoaders) {
              uint2 r[kFlight];
#pragma unroll
              for (int f = 0; f < kFlight; ++f) r[f] = load_x(i + f * kLoaders);
#pragma unroll
              for (int f = 0; f < kFlight; ++f) {
                if (i + f * kLoaders >= pieces) break;
                Piece x;
                aim(x, i + f * kLoaders);
                x.v[0] = __uint_as_float(r[f].x << 16), x.v[1] = __uint_as_float(r[f].x & 0xffff0000u);
                x.v[2] = __uint_as_float(r[f].y << 16), x.v[3] = __uint_as_float(r[f].y & 0xffff0000u);
                lay(x);
              }
            }
          } else {
            for (int i = i0 >> 5; i < pieces; i += 2 * kLoaders) {
              Piece x, y;
              load_h(x, i);
              load_h(y, i + kLoaders);
              lay(x);
              if (i + kLoaders < pieces) lay(y);
            }
          }
          asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
          __syncwarp();
          if (lane == 0) mbar_arrive(smem_u32(l.laid + op));
          if (++op == 2) op = 0, op_phase ^= 1;
        }
      }
      __syncwarp();
      __syncthreads();
      if (*(volatile int *)&l.given_up) {
        // Whichever warp it was: nothing may land in shared memory after the block has gone, so the last copies are
        // waited for (oldest first), and no step may be under way when tensor memory is freed.
        int never = 0;
        if (tid == 0) {
          for (int i = 0; i < kStages; ++i)
            mbar_wait(smem_u32(l.full + (stage + i) % kStages), stage_phase ^ (stage + i < kStages ? 1 : 0), &never);
        } else if (warp == 1) {
          if (elect_one()) tc_commit(smem_u32(&l.drained));
          __syncwarp();
          mbar_wait(smem_u32(&l.drained), 0, &never);
        }
        break;
      }
      if (up) {
        // the next product's weights are on their way while the blocks' sums meet
        if (tid == 0) grid_arrive(a.barrier), l.met = 2;
      }
    }
    // (a block without units has not waited for the second meeting: it must not arrive at the third before)
    if (tid == 0 && !l.given_up) grid_wait(a.barrier, base + 2ull * gridDim.x, &l.given_up);
    __syncthreads();
    if (tid == 0 && !l.given_up) l.met = kMeetings;
    fine = !*(volatile int *)&l.given_up && grid_meet(a.barrier, base + 3ull * gridDim.x, &l.given_up);
  }

  // ---- the weighted sum, slots and segments in order
  if (fine) {
    const int four = D / 4;
    for (int i = blockIdx.x * kThreads + tid; i < T * four; i += gridDim.x * kThreads) {
      const int t = i / four, d = (i - t * four) * 4;
      float4 sum = make_float4(0, 0, 0, 0);
      for (int q = 0; q < K; ++q) {
        if (__ldcg(a.ids + t * K + q) < 0) continue;
        const float w = __ldcg(a.weights + t * K + q);
        float4 y = make_float4(0, 0, 0, 0);
#pragma unroll 4
        for (int s = 0; s < a.segments[1]; ++s) {
          const float4 v = __ldcg((const float4 *)(a.y + ((int64_t)s * n + t * K + q) * D + d));
          y.x += v.x, y.y += v.y, y.z += v.z, y.w += v.w;
        }
        sum.x = fmaf(w, y.x, sum.x), sum.y = fmaf(w, y.y, sum.y), sum.z = fmaf(w, y.z, sum.z), sum.w = fmaf(w, y.w, sum.w);
      }
      __nv_bfloat16 *out = a.out + t * a.ldo + d;
      const float r[4] = {sum.x, sum.y, sum.z, sum.w};
#pragma unroll
      for (int j = 0; j < 4; ++j) out[j] = __float2bfloat16_rn(r[j]);
    }
  }
  __syncthreads();
  if (warp == 2) tmem_free(l.tmem, kBufs * kBufCols);
  if (tid == 0) {
    if (*(volatile int *)&l.given_up) *a.error = 1;
    if (l.met < kMeetings) grid_arrive(a.barrier, kMeetings - l.met);
  }
}

// Blocks of a segment: as long as possible (fewer partial sums; 1024 columns fill the operand's memory), while
// some five units a block are expected, which share out evenly enough; and cut for that to four segments at
// most, since what lays out h adds them all up.  (8192 columns are eight segments of the longest.)  Measured in us, shorter and longer: one token of 64 experts, 8-bit, 39 and 35;
// 33 tokens x 6 of 16 narrow experts 65 and 70; 64 tokens x 2 of 64 experts 260 and 248.
void plan_segments(int tokens, int k, int experts, int64_t rows, int64_t cols, int block, int &segment, int &segments) {
  const double chosen = experts * (1.0 - std::pow(1.0 - 1.0 / experts, (double)tokens * k));  // by evenly spread choices
  const double units = std::max<double>(k, chosen) * (double)ceil_div(rows, 128);
  const int64_t blocks = ceil_div(cols, block);
  int64_t s = 1024 / block;
  while (s * block > 128 && units * (double)ceil_div(blocks, s) < 5.0 * sm_count() && ceil_div(blocks, s / 2) <= 4) s /= 2;
  segment = (int)s, segments = (int)ceil_div(blocks, s);
}

size_t carve_few(Carve &c, FewArgs &a, int tokens, int experts, int k, int hidden, int inter, bool fp8) {
  const int64_t n = (int64_t)tokens * k, splits = ceil_div(hidden, kSplit);
  plan_segments(tokens, k, experts, 2 * (int64_t)inter, hidden, fp8 ? 128 : 64, a.segment[0], a.segments[0]);
  plan_segments(tokens, k, experts, hidden, inter, fp8 ? 128 : 64, a.segment[1], a.segments[1]);
  a.barrier = c.take<unsigned long long>(1);
  const size_t zeroed = c.used;
  a.part = c.take<float>(splits * tokens * experts);
  a.ids = c.take<int32_t>(n);
  a.weights = c.take<float>(n);
  a.up = c.take<float>(n * a.segments[0] * 2 * inter);
  a.y = c.take<float>(n * a.segments[1] * hidden);
  return zeroed;
}

int check_few(int tokens, int experts, int k, int hidden, int inter) {
  if (tokens < 0 || experts < 1 || k < 1 || k > experts || hidden < 1 || inter < 1 || hidden % 16 || inter % 16) return TUNA_ERR_INVALID_ARG;
  if (tokens > kMaxTokens || experts > TUNA_MOE_MAX_EXPERTS || k > kMaxK || hidden > kMaxDimFew || inter > kMaxDimFew) return TUNA_ERR_RANGE;
  return TUNA_OK;
}

template <bool FP8>
int launch_few(const FewArgs &a, const void *w13, const void *w2, cudaStream_t st) {
  CUtensorMap m13, m2;
  if (const int rc = make_map(&m13, 3, w13, a.hidden, 2 * (int64_t)a.inter, a.experts, a.hidden, 128, !FP8)) return rc;
  if (const int rc = make_map(&m2, 3, w2, a.inter, a.hidden, a.experts, a.inter, 128, !FP8)) return rc;
  static bool set[64] = {};
  if (const int rc = allow_smem(tuna_few_kernel<FP8>, kFewSmem, set)) return rc;
  return launch(tuna_few_kernel<FP8>, dim3((unsigned)sm_count()), kThreads, kFewSmem, st, true, m13, m2, a);
}

}  // namespace
}  // namespace tuna_ops

using namespace tuna_ops;

extern "C" {

int tuna_moe_few_workspace_bytes(int tokens, int experts, int k, int hidden, int inter, size_t *bytes, size_t *zeroed) {
  if (!bytes || !zeroed) return TUNA_ERR_INVALID_ARG;
  if (const int rc = check_few(tokens, experts, k, hidden, inter)) return rc;
  *bytes = 0;
  for (const bool fp8 : {false, true}) {
    Carve c(nullptr);
    FewArgs a = {};
    *zeroed = carve_few(c, a, tokens, experts, k, hidden, inter, fp8);
    *bytes = std::max(*bytes, c.used);
  }
  return TUNA_OK;
}

int tuna_moe_few(const void *x, int64_t ldx, int tokens, const void *router, int experts, int k, int scoring, int renormalize, float scale,
                 int hidden, int inter, int weight_dtype, const void *w13, const float *s13, const void *w2, const float *s2, void *out,
                 int64_t ldo, int32_t *ids, float *weights, void *workspace, size_t workspace_bytes, void *stream) {
  if (const int rc = check_few(tokens, experts, k, hidden, inter)) return rc;
  const bool fp8 = weight_dtype == TUNA_DTYPE_E4M3;
  if ((!fp8 && weight_dtype != TUNA_DTYPE_BF16) || (scoring != TUNA_MOE_SOFTMAX && scoring != TUNA_MOE_SIGMOID)) return TUNA_ERR_INVALID_ARG;
  if (ldx < hidden || ldo < hidden || ldx % 8) return TUNA_ERR_INVALID_ARG;
  if (tokens == 0) return TUNA_OK;
  if (!x || !router || !w13 || !w2 || !out || (fp8 && (!s13 || !s2))) return TUNA_ERR_INVALID_ARG;
  if (!aligned(x, 16) || !aligned(router, 16) || !aligned(w13, 16) || !aligned(w2, 16) || !aligned(out, 2)) return TUNA_ERR_INVALID_ARG;
  Carve c(workspace);
  FewArgs a = {};
  carve_few(c, a, tokens, experts, k, hidden, inter, fp8);
  if (!workspace || !aligned(workspace, 256) || workspace_bytes < c.used) return TUNA_ERR_WORKSPACE;
  a.x = (const __nv_bfloat16 *)x, a.router = (const __nv_bfloat16 *)router, a.s13 = s13, a.s2 = s2;
  a.out = (__nv_bfloat16 *)out, a.ids_out = ids, a.weights_out = weights, a.ldx = ldx, a.ldo = ldo;
  a.tokens = tokens, a.experts = experts, a.k = k, a.hidden = hidden, a.inter = inter;
  a.scoring = scoring, a.renormalize = renormalize != 0, a.scale = scale;
  a.error = error_word();
  if (!a.error) return TUNA_ERR_CUDA;
  cudaStream_t st = (cudaStream_t)stream;
  return fp8 ? launch_few<true>(a, w13, w2, st) : launch_few<false>(a, w13, w2, st);
}

}  // extern "C"
