// A whole mixture-of-experts layer for a few tokens, in one kernel:
//
//   logits = x Wr^T; the k best experts of every token and their weights w;
//   h = silu(x Wg^T) * (x Wu^T) and y = h Wd^T for every (token, expert) chosen;
//   out = sum over the chosen of w y
//
// For so few tokens the layer is bound by reading the chosen experts' weights once (3 D I
// values an expert).  A block a multiprocessor (cooperative launch: the three phases are
// separated by barriers across the grid) streams them through a ring in shared memory that
// every thread fills for itself with 16-byte asynchronous copies, some 140 KB in flight a
// block.  No thread reads another's part of the ring, so it needs no barriers, and it runs on
// across units and, since the next phase's weights are known, across the second grid barrier.
//
// A unit is 16 weight rows: 8 gate and the 8 up rows of the same places (so that SwiGLU joins
// two values of one thread), or 16 rows of Wd.  The 16 warps split the contracted axis in
// segments of 64 bytes, multiply on the tensor cores (m16n8k16: weight rows x tokens) with the
// tokens' values held in registers from unit to unit, and one warp adds up the 16 partial sums.
// Which of a segment's values form which step of the contraction is immaterial as long as both
// operands agree, so a thread's 16 bytes of a row are used as they come.
//
// bf16 weights meet x and h in bf16 (h rounded once, as a two-kernel layer would store it).
// 8-bit weights are exact in f16, one conversion instruction for two values; x and h then are
// f16 too, after a division by a power of two of the row's largest magnitude: 11 bits, more
// than bf16 holds.  Sums, logits and probabilities are in 32 bits.
#include <type_traits>

#include "tuna_ops.cuh"
#include "tuna_route.cuh"

namespace tuna_ops {
namespace {

constexpr int kThreads = 512, kWarps = 16;
constexpr int kMaxTokens = TUNA_MOE_FEW_MAX_TOKENS;
constexpr int kRing = 10;                 // segments of a thread in the ring (2 rows x 16 bytes each)
constexpr int kSplit = kWarps * 32;       // columns of x that a block takes in the router phase
constexpr int kMaxDimFew = 8192;

struct FewArgs {
  const __nv_bfloat16 *x, *router;
  const void *w13, *w2;
  const float *s13, *s2;
  __nv_bfloat16 *out;
  int32_t *ids_out;
  float *weights_out;
  int64_t ldx, ldo;
  int tokens, experts, k, hidden, inter, scoring, renormalize;
  float scale;
  // workspace
  unsigned *barrier;   // count, generation: zero before the first call, left so
  unsigned *arrived;   // per 16 output columns: units that are done
  float *part;         // [splits][tokens][experts] logits of a split
  uint32_t *x_amax;    // [splits][tokens]
  uint32_t *h_amax;    // [tokens * k]
  float *h;            // [tokens * k][inter]
  float *y;            // [tokens * k][hidden]
  int *error;
};

// Tokens of one expert that are multiplied together; more of them form another group.
struct Group {
  int16_t expert, first, count;
};

struct Lists {
  float weight[kMaxTokens * kMaxK];
  int16_t id[kMaxTokens * kMaxK];
  int16_t entry[kMaxTokens * kMaxK];  // token * k + slot, by expert
  Group group[kMaxTokens * kMaxK];
  int16_t begin[TUNA_MOE_MAX_EXPERTS + 1];
  int count[TUNA_MOE_MAX_EXPERTS];
  float x_scale[kMaxTokens];          // the power of two that x was divided by
  int groups;
  int given_up, done_tile;
};

constexpr size_t kRingBytes = (size_t)kRing * 2 * kThreads * 16;
constexpr size_t kPartBytes = (size_t)2 * kWarps * 2 * 32 * 16;  // two units, warps, token tiles, lanes
constexpr size_t kFewSmem = kRingBytes + kPartBytes + sizeof(Lists);
static_assert(kFewSmem <= 227 * 1024, "shared memory of a block");
static_assert(kWarps * (kMaxTokens / 8) * 32 * 16 <= kRingBytes, "the router's partial sums fit the ring");

__device__ __forceinline__ void copy16(uint32_t dst, const void *src, bool there) {
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst), "l"(src), "r"(there ? 16 : 0) : "memory");
}
__device__ __forceinline__ uint4 lds16(uint32_t addr) {
  uint4 v;
  asm volatile("ld.shared.v4.u32 {%0, %1, %2, %3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "r"(addr) : "memory");
  return v;
}
__device__ __forceinline__ void mma_bf16(float (&c)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
  asm("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
      : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3]) : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}
__device__ __forceinline__ void mma_f16(float (&c)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
  asm("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
      : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3]) : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}
__device__ __forceinline__ uint32_t pack_f16(float lo, float hi) {
  uint32_t r;
  asm("cvt.rn.f16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
  return r;
}
// four e4m3 values to two pairs of f16 (exact)
__device__ __forceinline__ void widen(uint32_t w, uint32_t &lo, uint32_t &hi) {
  asm("{\n .reg .b16 a, b;\n mov.b32 {a, b}, %2;\n cvt.rn.f16x2.e4m3x2 %0, a;\n cvt.rn.f16x2.e4m3x2 %1, b;\n}" : "=r"(lo), "=r"(hi) : "r"(w));
}

// All blocks of the grid meet; false after about two seconds.  `bar`: arrivals, generation.
__device__ bool grid_meet(unsigned *bar, int *given_up) {
  __syncthreads();
  if (threadIdx.x == 0) {
    volatile unsigned *generation = bar + 1;
    const unsigned g = *generation;
    __threadfence();
    if (atomicAdd(bar, 1u) == gridDim.x - 1) {
      bar[0] = 0;
      __threadfence();
      atomicAdd(bar + 1, 1u);
    } else {
      const long long t0 = clock64();
      while (*generation == g) {
        if (clock64() - t0 > kWaitCycles) {
          *given_up = 1;
          break;
        }
      }
    }
    __threadfence();
  }
  __syncthreads();
  return !*(volatile int *)given_up;
}

// The power of two that takes a row's largest magnitude to [2^14, 2^15): f16 keeps 11 bits of
// everything within 2^-28 of it.  Rows of zeros, or that are not finite, are left as they are.
__device__ __forceinline__ float f16_scale(uint32_t amax) {
  if (amax == 0 || amax >= 0x7f800000u) return 1.0f;
  const int e = max((int)(amax >> 23) - 14, 1);
  return __uint_as_float((uint32_t)min(e, 253) << 23);
}
__device__ __forceinline__ float inverse_scale(float s) { return __uint_as_float((uint32_t)(254 - (int)(__float_as_uint(s) >> 23)) << 23); }

// One phase's stream of units.  Rows of `row_bytes`; the tile of a unit starts `tile_rows` rows
// on; the second half of its rows lies `second` rows behind the first.
struct Stream {
  const char *base;
  const float *scales;
  int64_t matrix_rows;   // rows of one expert's matrix (gate and up together)
  int row_bytes, tile_rows, tiles, second, second_block, blocks;  // blocks: 128-blocks of a row
  int block_rows;        // scale rows of one expert
  int per_warp;          // segments a warp and unit
  int unit0, unit1;      // this block's units
};

// MAXC: segments a warp holds of a row, at most; NT: token tiles of a group.
template <bool FP8, int MAXC, int NT>
struct Layer {
  static constexpr int kPer = FP8 ? 8 : 4;  // registers of one segment's token values
  uint32_t b[NT][MAXC][kPer];
  // the stream's feeding end
  const char *p0, *p1;
  int fu, fj, slot;

  __device__ __forceinline__ void point(const Stream &s, const Lists &l, int u) {
    const int lane = threadIdx.x & 31, g = u / s.tiles, tile = u - g * s.tiles;
    const int64_t row = (int64_t)l.group[g].expert * s.matrix_rows + tile * s.tile_rows + (lane >> 2);
    p0 = s.base + row * s.row_bytes + (lane & 3) * 16;
    p1 = p0 + (int64_t)s.second * s.row_bytes;
  }
  // One more segment on its way (or an empty group of copies, which keeps the count).
  __device__ __forceinline__ void feed(const Stream &s, const Lists &l, uint32_t ring) {
    if (fu < s.unit1) {
      const int at = ((threadIdx.x >> 5) + kWarps * fj) * 64;
      const bool there = at + (int)(threadIdx.x & 3) * 16 < s.row_bytes;
      const uint32_t to = ring + ((uint32_t)(slot * 2) * kThreads + threadIdx.x) * 16;
      copy16(to, there ? p0 + at : s.base, there);
      copy16(to + kThreads * 16, there ? p1 + at : s.base, there);
      if (++fj == s.per_warp) {
        fj = 0;
        if (++fu < s.unit1) point(s, l, fu);
      }
    }
    copy_commit();
    if (++slot == kRing) slot = 0;
  }
  __device__ __forceinline__ void start(const Stream &s, const Lists &l, uint32_t ring) {
    fu = s.unit0, fj = 0;
    if (fu < s.unit1) point(s, l, fu);
    for (int i = 0; i < kRing - 1; ++i) feed(s, l, ring);
  }
};

template <bool FP8, int MAXC, int NT>
__global__ void __launch_bounds__(kThreads, 1) tuna_few_kernel(FewArgs a) {
  extern __shared__ __align__(16) char smem[];
  const uint32_t ring = smem_u32(smem);
  float4 *part = (float4 *)(smem + kRingBytes);
  Lists &l = *(Lists *)(smem + kRingBytes + kPartBytes);
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31, row_in = lane >> 2, quad = lane & 3;
  const int T = a.tokens, E = a.experts, K = a.k, D = a.hidden, I = a.inter;
  const int splits = (D + kSplit - 1) / kSplit;
  if (tid == 0) l.given_up = 0;
  if (tid < kMaxTokens) l.count[tid] = 0;  // (the router phase's largest |x| of each token)
  __syncthreads();

  // ---- logits: a block takes 16 experts and 512 columns, a warp 32 of them
  {
    if (FP8 && blockIdx.x == 0)
      for (int i = tid; i < T * K; i += kThreads) a.h_amax[i] = 0;
    const int units = (E + 15) / 16 * splits, nt = (T + 7) / 8;
    float4 *sums = (float4 *)smem;  // [token tile][warp][lane]
    for (int u = blockIdx.x; u < units; u += gridDim.x) {
      const int m = u / splits, split = u - m * splits;
      const int col = split * kSplit + warp * 32 + quad * 8;
      uint4 w0 = make_uint4(0, 0, 0, 0), w1 = w0;
      if (col < D) {
        const int e0 = m * 16 + row_in, e1 = e0 + 8;
        if (e0 < E) w0 = __ldg((const uint4 *)(a.router + (int64_t)e0 * D + col));
        if (e1 < E) w1 = __ldg((const uint4 *)(a.router + (int64_t)e1 * D + col));
      }
      for (int j = 0; j < nt; ++j) {
        const int t = j * 8 + row_in;
        uint4 v = make_uint4(0, 0, 0, 0);
        if (col < D && t < T) v = __ldg((const uint4 *)(a.x + t * a.ldx + col));
        float c[4] = {};
        mma_bf16(c, w0.x, w1.x, w0.y, w1.y, v.x, v.y);
        mma_bf16(c, w0.z, w1.z, w0.w, w1.w, v.z, v.w);
        sums[(j * kWarps + warp) * 32 + lane] = make_float4(c[0], c[1], c[2], c[3]);
        if (FP8 && m == 0) {
          const uint32_t q[4] = {v.x, v.y, v.z, v.w};
          uint32_t top = 0;
#pragma unroll
          for (int i = 0; i < 4; ++i) top = max(top, max((q[i] << 16) & 0x7fffffffu, q[i] & 0x7fff0000u));
          top = max(top, __shfl_xor_sync(~0u, top, 1));
          top = max(top, __shfl_xor_sync(~0u, top, 2));
          if (quad == 0 && t < T) atomicMax((unsigned *)&l.count[t], top);
        }
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
      if (FP8 && m == 0 && tid < T) a.x_amax[split * T + tid] = (uint32_t)l.count[tid], l.count[tid] = 0;
      __syncthreads();
    }
  }
  if (!grid_meet(a.barrier, &l.given_up)) {
    if (tid == 0) *a.error = 1;
    return;
  }

  // ---- the choice, by every block for itself: a warp a token
  for (int t = warp; t < T; t += kWarps) {
    int id;
    float w;
    auto take = [&](auto vpl) {
      constexpr int VPL = decltype(vpl)::value;
      float z[VPL];
#pragma unroll
      for (int i = 0; i < VPL; ++i) {
        const int e = lane * VPL + i;
        float s = -INFINITY;
        if (e < E) {
          s = 0.0f;
          for (int q = 0; q < splits; ++q) s += __ldcg(a.part + ((int64_t)q * T + t) * E + e);
          s = logit_of(s);
        }
        z[i] = s;
      }
      choose<32>(z, lane, K, a.scoring, a.renormalize, a.scale, id, w);
    };
    if (E <= 64)
      take(std::integral_constant<int, 2>());
    else if (E <= 256)
      take(std::integral_constant<int, 8>());
    else
      take(std::integral_constant<int, 16>());
    if (lane < K) {
      l.id[t * K + lane] = (int16_t)id, l.weight[t * K + lane] = w;
      if (blockIdx.x == 0) {
        if (a.ids_out) a.ids_out[t * K + lane] = id;
        if (a.weights_out) a.weights_out[t * K + lane] = w;
      }
    }
    if (FP8) {
      uint32_t top = lane < splits ? __ldcg(a.x_amax + lane * T + t) : 0;
#pragma unroll
      for (int d = 16; d; d >>= 1) top = max(top, __shfl_xor_sync(~0u, top, d));
      if (lane == 0) l.x_scale[t] = f16_scale(top);
    }
  }
  for (int e = tid; e < E; e += kThreads) l.count[e] = 0;
  __syncthreads();
  const int n = T * K;
  for (int i = tid; i < n; i += kThreads)
    if (l.id[i] >= 0) atomicAdd(&l.count[l.id[i]], 1);
  __syncthreads();
  constexpr int kGroup = NT * 8;
  if (warp == 0) {
    // first entry of each expert, and the groups
    int entries = 0, groups = 0;
    for (int e0 = 0; e0 < E; e0 += 32) {
      const int c = e0 + lane < E ? l.count[e0 + lane] : 0, g = (c + kGroup - 1) / kGroup;
      int xc = c, xg = g;
#pragma unroll
      for (int d = 1; d < 32; d <<= 1) {
        const int yc = __shfl_up_sync(~0u, xc, d), yg = __shfl_up_sync(~0u, xg, d);
        if (lane >= d) xc += yc, xg += yg;
      }
      if (e0 + lane < E) {
        l.begin[e0 + lane] = (int16_t)(entries + xc - c);
        for (int i = 0; i < g; ++i)
          l.group[groups + xg - g + i] = {(int16_t)(e0 + lane), (int16_t)(entries + xc - c + i * kGroup), (int16_t)min(kGroup, c - i * kGroup)};
      }
      entries += __shfl_sync(~0u, xc, 31), groups += __shfl_sync(~0u, xg, 31);
    }
    if (lane == 0) l.groups = groups;
    __syncwarp();
    for (int i0 = 0; i0 < n; i0 += 32) {
      const int id = i0 + lane < n ? l.id[i0 + lane] : -1;
      const uint32_t peers = __match_any_sync(~0u, id);
      const int at = id >= 0 ? l.begin[id] : 0;
      __syncwarp();
      if (id >= 0) {
        l.entry[at + __popc(peers & ((1u << lane) - 1))] = (int16_t)(i0 + lane);
        if (lane == __ffs(peers) - 1) l.begin[id] = (int16_t)(at + __popc(peers));
      }
      __syncwarp();
    }
  }
  __syncthreads();
  const int groups = l.groups;

  // ---- the two products
  Layer<FP8, MAXC, NT> f;
  f.slot = 0;
  int read = 0;  // the ring's reading end
  constexpr int kSize = FP8 ? 1 : 2;
#pragma unroll 1
  for (int phase = 0; phase < 2; ++phase) {
    const bool up = phase == 0;
    const int cols = up ? D : I;
    Stream s;
    s.base = (const char *)(up ? a.w13 : a.w2), s.scales = up ? a.s13 : a.s2;
    s.row_bytes = cols * kSize, s.tile_rows = up ? 8 : 16, s.tiles = up ? I / 8 : D / 16;
    s.second = up ? I : 8, s.matrix_rows = up ? 2 * I : D;
    s.blocks = (cols + 127) / 128, s.block_rows = up ? 2 * ((I + 127) / 128) : (D + 127) / 128, s.second_block = up ? (I + 127) / 128 : 0;
    s.per_warp = (s.row_bytes + 64 * kWarps - 1) / (64 * kWarps);
    const int64_t units = (int64_t)groups * s.tiles;
    s.unit0 = (int)(units * blockIdx.x / gridDim.x), s.unit1 = (int)(units * (blockIdx.x + 1) / gridDim.x);
    f.slot = read;
    f.start(s, l, ring);
    if (!up && !grid_meet(a.barrier, &l.given_up)) {  // h of every block is there
      copy_wait<0>();
      if (tid == 0) *a.error = 1;
      return;
    }
    // this lane's scale of the unit: segment lane / 2 of this warp, first or second rows
    auto scale_of = [&](int u) -> float {
      const int j = lane >> 1;
      const int at = (warp + kWarps * j) * 64;
      if (!FP8 || u >= s.unit1 || j >= s.per_warp || at >= s.row_bytes) return 0.0f;
      const int g = u / s.tiles, tile = u - g * s.tiles;
      const int64_t r = (int64_t)l.group[g].expert * s.block_rows + tile * s.tile_rows / 128 + (lane & 1) * s.second_block;
      return __ldg(s.scales + r * s.blocks + at / 128);
    };
    float next_scale = scale_of(s.unit0);
    int held = -1;  // the group whose token values are in registers
    for (int u = s.unit0; u < s.unit1; ++u) {
      const int g = u / s.tiles, tile = u - g * s.tiles;
      const int expert_first = l.group[g].first, count = l.group[g].count;
      if (g != held) {
        held = g;
#pragma unroll
        for (int t8 = 0; t8 < NT; ++t8) {
          const int i = t8 * 8 + row_in;
          const int entry = i < count ? l.entry[expert_first + i] : -1;
          const int token = entry / K;
          float down = 1.0f;
          if (FP8 && entry >= 0) down = inverse_scale(up ? l.x_scale[token] : f16_scale(__ldcg(a.h_amax + entry)));
#pragma unroll
          for (int j = 0; j < MAXC; ++j) {
            const int at = ((warp + kWarps * j) * 64 + quad * 16) / kSize;  // first column of this thread's 16 bytes
            const bool there = entry >= 0 && j < s.per_warp && at < cols;
#pragma unroll
            for (int q = 0; q < Layer<FP8, MAXC, NT>::kPer / 4; ++q) {
              // 8 columns: four pairs
              uint32_t w[4] = {0, 0, 0, 0};
              if (there) {
                float v[8];
                if (up) {
                  const uint4 r = __ldg((const uint4 *)(a.x + token * a.ldx + at + q * 8));
                  if (!FP8) {
                    w[0] = r.x, w[1] = r.y, w[2] = r.z, w[3] = r.w;
                  } else {
                    const uint32_t k4[4] = {r.x, r.y, r.z, r.w};
#pragma unroll
                    for (int i2 = 0; i2 < 4; ++i2)
                      w[i2] = pack_f16(__uint_as_float(k4[i2] << 16) * down, __uint_as_float(k4[i2] & 0xffff0000u) * down);
                  }
                } else {
                  const float4 *h = (const float4 *)(a.h + (int64_t)entry * I + at + q * 8);
                  const float4 h0 = __ldcg(h), h1 = __ldcg(h + 1);
                  v[0] = h0.x, v[1] = h0.y, v[2] = h0.z, v[3] = h0.w, v[4] = h1.x, v[5] = h1.y, v[6] = h1.z, v[7] = h1.w;
#pragma unroll
                  for (int i2 = 0; i2 < 4; ++i2)
                    w[i2] = FP8 ? pack_f16(v[2 * i2] * down, v[2 * i2 + 1] * down) : pack_bf16(v[2 * i2], v[2 * i2 + 1]);
                }
              }
#pragma unroll
              for (int i2 = 0; i2 < 4; ++i2) f.b[t8][j][q * 4 + i2] = w[i2];
            }
          }
        }
      }
      const float unit_scale = next_scale;
      next_scale = scale_of(u + 1);
      const bool two = NT > 1 && count > 8;
      float c[NT][4];
#pragma unroll
      for (int t8 = 0; t8 < NT; ++t8) c[t8][0] = c[t8][1] = c[t8][2] = c[t8][3] = 0.0f;
#pragma unroll
      for (int j = 0; j < MAXC; ++j) {
        if (j < s.per_warp) {
          copy_wait<kRing - 2>();
          const uint32_t at = ring + ((uint32_t)(read * 2) * kThreads + tid) * 16;
          const uint4 r0 = lds16(at), r1 = lds16(at + kThreads * 16);
          if (++read == kRing) read = 0;
          f.feed(s, l, ring);
          const uint32_t k0[4] = {r0.x, r0.y, r0.z, r0.w}, k1[4] = {r1.x, r1.y, r1.z, r1.w};
          if constexpr (FP8) {
            const float s0 = __shfl_sync(~0u, unit_scale, 2 * j), s1 = __shfl_sync(~0u, unit_scale, 2 * j + 1);
            uint32_t A0[8], A1[8];
#pragma unroll
            for (int i = 0; i < 4; ++i) widen(k0[i], A0[2 * i], A0[2 * i + 1]), widen(k1[i], A1[2 * i], A1[2 * i + 1]);
#pragma unroll
            for (int t8 = 0; t8 < NT; ++t8) {
              if (t8 == 0 || two) {
                float p[4] = {};
#pragma unroll
                for (int i = 0; i < 4; ++i)
                  mma_f16(p, A0[2 * i], A1[2 * i], A0[2 * i + 1], A1[2 * i + 1], f.b[t8][j][2 * i], f.b[t8][j][2 * i + 1]);
                c[t8][0] = fmaf(p[0], s0, c[t8][0]), c[t8][1] = fmaf(p[1], s0, c[t8][1]);
                c[t8][2] = fmaf(p[2], s1, c[t8][2]), c[t8][3] = fmaf(p[3], s1, c[t8][3]);
              }
            }
          } else {
#pragma unroll
            for (int t8 = 0; t8 < NT; ++t8) {
              if (t8 == 0 || two) {
#pragma unroll
                for (int i = 0; i < 2; ++i)
                  mma_bf16(c[t8], k0[2 * i], k1[2 * i], k0[2 * i + 1], k1[2 * i + 1], f.b[t8][j][2 * i], f.b[t8][j][2 * i + 1]);
              }
            }
          }
        }
      }
      float4 *mine = part + (u & 1) * (kWarps * 2 * 32);
#pragma unroll
      for (int t8 = 0; t8 < NT; ++t8) mine[(t8 * kWarps + warp) * 32 + lane] = make_float4(c[t8][0], c[t8][1], c[t8][2], c[t8][3]);
      __syncthreads();
      if (warp != (u & (kWarps - 1))) continue;
      // one warp adds up; the others are at the next unit, which writes the other half of `part`
#pragma unroll
      for (int t8 = 0; t8 < NT; ++t8) {
        if (t8 && !two) continue;
        float4 v = make_float4(0, 0, 0, 0);
#pragma unroll
        for (int w = 0; w < kWarps; ++w) {
          const float4 q = mine[(t8 * kWarps + w) * 32 + lane];
          v.x += q.x, v.y += q.y, v.z += q.z, v.w += q.w;
        }
#pragma unroll
        for (int i = 0; i < 2; ++i) {
          const int at = t8 * 8 + quad * 2 + i;
          const int entry = at < count ? l.entry[expert_first + at] : -1;
          float lo = i ? v.y : v.x, hi = i ? v.w : v.z;
          if (up) {
            if (FP8) {
              const float by = entry >= 0 ? l.x_scale[entry / K] : 0.0f;
              lo *= by, hi *= by;
            }
            const float h = lo / (1.0f + expf(-lo)) * hi;
            if (entry >= 0) a.h[(int64_t)entry * I + tile * 8 + row_in] = h;
            if (FP8) {
              uint32_t top = entry >= 0 ? abs_bits(h) : 0;
              top = max(top, __shfl_xor_sync(~0u, top, 4));
              top = max(top, __shfl_xor_sync(~0u, top, 8));
              top = max(top, __shfl_xor_sync(~0u, top, 16));
              if (row_in == 0 && entry >= 0) atomicMax(a.h_amax + entry, top);
            }
          } else if (entry >= 0) {
            const float by = FP8 ? f16_scale(__ldcg(a.h_amax + entry)) : 1.0f;
            float *y = a.y + (int64_t)entry * D + tile * 16 + row_in;
            y[0] = lo * by, y[8] = hi * by;
          }
        }
      }
      if (!up) {
        // the group that completes these 16 columns sums the tokens' slots, in slot order
        __threadfence();
        __syncwarp();
        unsigned before = 0;
        if (lane == 0) before = atomicAdd(a.arrived + tile, 1u);
        before = __shfl_sync(~0u, before, 0);
        if (before == (unsigned)groups - 1) {
          __threadfence();
          if (lane == 0) a.arrived[tile] = 0;
          const int d = tile * 16 + (lane & 15);
          for (int t = lane >> 4; t < T; t += 2) {
            float sum = 0.0f;
            for (int q = 0; q < K; ++q) {
              const int i = t * K + q;
              if (l.id[i] >= 0) sum = fmaf(l.weight[i], __ldcg(a.y + (int64_t)i * D + d), sum);
            }
            a.out[t * a.ldo + d] = __float2bfloat16_rn(sum);
          }
        }
      }
    }
    __syncthreads();
  }
  copy_wait<0>();
  // a choice that is empty for every token: nothing is summed
  if (groups == 0)
    for (int i = blockIdx.x * kThreads + tid; i < T * D; i += gridDim.x * kThreads) a.out[i / D * a.ldo + i % D] = __float2bfloat16_rn(0.0f);
}

struct FewSpace {
  size_t zeroed;  // bytes at the front that must be zero before the first call
};
FewSpace carve_few(Carve &c, FewArgs &a, int tokens, int experts, int k, int hidden, int inter) {
  FewSpace w = {};
  const int64_t n = (int64_t)tokens * k, splits = ceil_div(hidden, kSplit);
  a.barrier = c.take<unsigned>(2);
  a.arrived = c.take<unsigned>(kMaxDimFew / 16);
  w.zeroed = c.used;
  a.part = c.take<float>(splits * tokens * experts);
  a.x_amax = c.take<uint32_t>(splits * tokens);
  a.h_amax = c.take<uint32_t>(n);
  a.h = c.take<float>(n * inter);
  a.y = c.take<float>(n * hidden);
  return w;
}

int check_few(int tokens, int experts, int k, int hidden, int inter) {
  if (tokens < 0 || experts < 1 || k < 1 || k > experts || hidden < 1 || inter < 1 || hidden % 16 || inter % 16) return TUNA_ERR_INVALID_ARG;
  if (tokens > kMaxTokens || experts > TUNA_MOE_MAX_EXPERTS || k > kMaxK || hidden > kMaxDimFew || inter > kMaxDimFew) return TUNA_ERR_RANGE;
  return TUNA_OK;
}

template <bool FP8, int MAXC, int NT>
int launch_few(const FewArgs &a, cudaStream_t st) {
  static bool set[64] = {};
  auto kernel = tuna_few_kernel<FP8, MAXC, NT>;
  if (const int rc = allow_smem(kernel, kFewSmem, set)) return rc;
  return launch(kernel, dim3((unsigned)sm_count()), kThreads, kFewSmem, st, true, a);
}

}  // namespace
}  // namespace tuna_ops

using namespace tuna_ops;

extern "C" {

int tuna_moe_few_workspace_bytes(int tokens, int experts, int k, int hidden, int inter, size_t *bytes, size_t *zeroed) {
  if (!bytes || !zeroed) return TUNA_ERR_INVALID_ARG;
  if (const int rc = check_few(tokens, experts, k, hidden, inter)) return rc;
  Carve c(nullptr);
  FewArgs a = {};
  *zeroed = carve_few(c, a, tokens, experts, k, hidden, inter).zeroed;
  *bytes = c.used;
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
  carve_few(c, a, tokens, experts, k, hidden, inter);
  if (!workspace || !aligned(workspace, 256) || workspace_bytes < c.used) return TUNA_ERR_WORKSPACE;
  a.x = (const __nv_bfloat16 *)x, a.router = (const __nv_bfloat16 *)router, a.w13 = w13, a.w2 = w2, a.s13 = s13, a.s2 = s2;
  a.out = (__nv_bfloat16 *)out, a.ids_out = ids, a.weights_out = weights, a.ldx = ldx, a.ldo = ldo;
  a.tokens = tokens, a.experts = experts, a.k = k, a.hidden = hidden, a.inter = inter;
  a.scoring = scoring, a.renormalize = renormalize != 0, a.scale = scale;
  a.error = error_word();
  if (!a.error) return TUNA_ERR_CUDA;
  cudaStream_t st = (cudaStream_t)stream;
  // Token values a thread holds: rows up to 4096 columns leave registers for two token tiles.
  const bool wide = hidden > 4096 || inter > 4096;
  if (fp8) return wide ? launch_few<true, 8, 1>(a, st) : launch_few<true, 4, 2>(a, st);
  return wide ? launch_few<false, 16, 1>(a, st) : launch_few<false, 8, 2>(a, st);
}

}  // extern "C"
