// Matrices in 4-bit floating point with a power of two for every 32 values along the contracted axis (microscaling: e2m1
// values, e8m0 scales), and their products, dense and grouped by expert.
//
//   y[m,n] = sum_b 2^(ea[m,b] + eb[n,b]) sum_{k in block b} a[m,k] b[n,k]
//
// The tensor cores apply the scales themselves, so a product accumulates in tensor memory from the first step to the last.
#include <algorithm>

#include "tuna_fp4.h"
#include "tuna_ops.cuh"

namespace tuna_ops {
namespace {

// ---- values --------------------------------------------------------------------------------

// The scale's byte: the exponent of the block's largest magnitude less that of the largest 4-bit value (6 = 1.5 * 2^2), 2^-127
// at least; 255, which stands for NaN, where the block holds a NaN or an infinity.
__device__ __forceinline__ uint32_t fp4_scale(uint32_t amax_bits) {
  const int e = amax_bits >> 23;
  return e == 255 ? 255u : (uint32_t)max(e - 2, 0);
}
__device__ __forceinline__ float fp4_power(uint32_t byte) {  // 2^(byte - 127)
  return __uint_as_float(byte == 255 ? 0x7fc00000u : byte ? byte << 23 : 0x00400000u);
}
__device__ __forceinline__ float fp4_inverse(uint32_t byte) { return __uint_as_float((254u - min(byte, 253u)) << 23); }  // 2^(127 - byte)
// Eight values, already over their scale, to 4 bits each, the first lowest; halves to even, at most 6.
__device__ __forceinline__ uint32_t fp4_eight(const float *v) {
  uint32_t r;
  asm("{\n .reg .b8 a, b, c, d;\n"
      " cvt.rn.satfinite.e2m1x2.f32 a, %2, %1;\n cvt.rn.satfinite.e2m1x2.f32 b, %4, %3;\n"
      " cvt.rn.satfinite.e2m1x2.f32 c, %6, %5;\n cvt.rn.satfinite.e2m1x2.f32 d, %8, %7;\n"
      " mov.b32 %0, {a, b, c, d};\n}"
      : "=r"(r) : "f"(v[0]), "f"(v[1]), "f"(v[2]), "f"(v[3]), "f"(v[4]), "f"(v[5]), "f"(v[6]), "f"(v[7]));
  return r;
}
__device__ __forceinline__ void fp4_values(uint32_t q, float (&v)[8]) {
  uint32_t h[4];
  asm("{\n .reg .b8 a, b, c, d;\n mov.b32 {a, b, c, d}, %4;\n"
      " cvt.rn.f16x2.e2m1x2 %0, a;\n cvt.rn.f16x2.e2m1x2 %1, b;\n cvt.rn.f16x2.e2m1x2 %2, c;\n cvt.rn.f16x2.e2m1x2 %3, d;\n}"
      : "=r"(h[0]), "=r"(h[1]), "=r"(h[2]), "=r"(h[3]) : "r"(q));
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const float2 f = __half22float2(*reinterpret_cast<const __half2 *>(&h[i]));
    v[2 * i] = f.x, v[2 * i + 1] = f.y;
  }
}

// The largest magnitude of values: an infinity or a NaN, if there is one.
__device__ __forceinline__ float top_of(float a, float b, float c) {
  float r;
  asm("max.NaN.abs.f32 %0, %1, %2, %3;" : "=f"(r) : "f"(a), "f"(b), "f"(c));
  return r;
}
// silu(g) * u of two values.  1 / (1 + 2^(-g log2 e)): the exponent's rounding makes it off by |g| 2^-23, the rest by 2^-21; from g = -88 down
// it is 0.  (Six instructions a value: with expf and a division the results of a tile took longer than its steps.  An h that is so near to
// the middle of two 4-bit values may become the other one, as it may by the order of the sums that g and u are: one in some 2^16 of them.)
__device__ __forceinline__ uint64_t swiglu2(float g0, float g1, float u0, float u1) {
  const uint64_t g = pair(g0, g1);
  float a, b, c, d;
  unpair(mul2(g, pair(-kLog2E, -kLog2E)), a, b);
  unpair(add2(pair(exp2_fast(a), exp2_fast(b)), pair(1.0f, 1.0f)), a, b);
  c = reciprocal_fast(a), d = reciprocal_fast(b);
  return mul2(mul2(g, pair(c, d)), pair(u0, u1));
}

// ---- quantisation --------------------------------------------------------------------------
//
// Bound by memory: two bytes (bf16) read and 17/32 written a value.  A warp takes 256 columns of four rows that are 32
// apart, 8 columns a lane, so that a lane loads 16 bytes of bf16 a row, and the four rows' scales of four blocks are 16 bytes in a
// row.  A block of threads takes eight such sets of rows, a quarter of a tile, and `strips` times 256 columns of them.  Rows on
// 16-byte boundaries come by asynchronous copies, several strips ahead, to a place of the warp's own in shared memory (so that
// no warp waits for another); others by loads of what width they allow, one strip ahead.  8192 x 4096: bf16 12.3 us (7.0 TB/s: some of it stays in
// the cache), f32 25.6 us (5.9 TB/s).
template <typename T>
__host__ __device__ constexpr int ahead() { return sizeof(T) == 2 ? 3 : 2; }  // strips on their way and under way: 48 and 64 KB a block of threads
struct Quant4Args {
  const void *x;
  int64_t rows, ldx, ldq, in_rows;
  int cols, runs, strips;
  const int64_t *gather;
  const int64_t *offsets;  // of groups; nullptr: none
  int groups;
  uint8_t *q, *scale;
};

// The rows of tile slot `slot`: [row, end), none if row >= end.  Every lane of a warp comes here.
__device__ __forceinline__ void slot_rows(const int64_t *offsets, int groups, int64_t rows, int64_t slot, int64_t &row, int64_t &end) {
  if (!offsets) {
    row = slot * 128, end = min(row + 128, rows);
    return;
  }
  const int lane = threadIdx.x & 31;
  auto cut = [&](int g) { return min(max(offsets[g], (int64_t)0), rows); };
  // the last group whose tiles begin at the slot or before it: among every 32nd group (there are 1024 at most), then among 32
  int g = lane * 32;
  const uint32_t coarse = __ballot_sync(~0u, g < groups && cut(min(g, groups - 1)) / 128 + g <= slot);
  row = 0, end = 0;
  if (!(coarse & 1)) return;
  const int base = (31 - __clz(coarse)) * 32;
  g = base + lane;
  const uint32_t fine = __ballot_sync(~0u, g < groups && cut(min(g, groups - 1)) / 128 + g <= slot);
  if (!(fine & 1)) return;
  g = base + 31 - __clz(fine);
  const int64_t begin = cut(g);
  row = begin + (slot - begin / 128 - g) * 128, end = min(row + 128, cut(g + 1));
}

// A lane's eight values of four rows: their 4-bit words, and in lane 4 j + i of the sixteen of a run the scales of row i.
template <typename T>
__device__ __forceinline__ void quantize_four(const Eight<T> (&x)[4], uint32_t (&q)[4], uint32_t &scales) {
  float v[4][8];
  uint32_t top[2];  // the upper halves of the largest magnitudes (their exponents are all that counts), two rows a word
#pragma unroll
  for (int i = 0; i < 4; i += 2) {
    float t[2];
#pragma unroll
    for (int j = 0; j < 2; ++j) {
      x[i + j].values(v[i + j]);
      const float(&w)[8] = v[i + j];
      t[j] = top_of(top_of(top_of(top_of(w[0], w[1], w[2]), w[3], w[4]), w[5], w[6]), w[7], 0.0f);
    }
    top[i / 2] = __byte_perm(__float_as_uint(t[0]), __float_as_uint(t[1]), 0x7632) & 0x7fff7fffu;
  }
#pragma unroll
  for (int d = 1; d < 4; d <<= 1)
#pragma unroll
    for (int i = 0; i < 2; ++i) top[i] = __vmaxu2(top[i], __shfl_xor_sync(~0u, top[i], d));
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const uint32_t e = i & 1 ? top[i >> 1] >> 23 : top[i >> 1] >> 7 & 255;
    const float inverse = __uint_as_float(min(256 - e, 254u) << 23);  // that of fp4_scale(e)
    const uint64_t by = pair(inverse, inverse);
#pragma unroll
    for (int j = 0; j < 8; j += 2) unpair(mul2(pair(v[i][j], v[i][j + 1]), by), v[i][j], v[i][j + 1]);
    q[i] = fp4_eight(v[i]);
  }
  const uint32_t own = threadIdx.x & 2 ? top[1] : top[0];
  uint32_t mine = fp4_scale(threadIdx.x & 1 ? own & 0xffff0000u : own << 16) << (threadIdx.x & 12) * 2;
  mine |= __shfl_xor_sync(~0u, mine, 4);
  scales = mine | __shfl_xor_sync(~0u, mine, 8);
}
template <typename T, bool ALIGNED>
__global__ void __launch_bounds__(256) tuna_quantize4_rows_kernel(Quant4Args a) {
  extern __shared__ __align__(16) uint4 ring[];  // [kAhead][4][warps][a row's 256 values]
  constexpr int kAhead = ahead<T>(), kWords = Eight<T>::kWords, kPiece = 8 / kWords;  // (16 bytes)
  wait_previous();
  allow_next();
  const int lane = threadIdx.x & 31, l = (blockIdx.x & 3) * 8 + (threadIdx.x >> 5);
  const int64_t slot = blockIdx.x >> 2;
  int64_t row0, end;
  slot_rows(a.offsets, a.groups, a.rows, slot, row0, end);
  if (row0 + l >= end) return;
  const int rows = (int)min((end - row0 - l + 31) / 32, (int64_t)4);
  int c0 = (int)blockIdx.y * a.strips * 256;                        // first column of the strip
  const int last = min(a.cols, c0 + a.strips * 256);                // end of this block's columns
  const T *from[4];
  uint32_t *to[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const int64_t r = row0 + l + 32 * min(i, rows - 1);  // (a row that is not there: the last one again, which nobody stores)
    const int64_t at = a.gather ? min(max(__ldg(a.gather + r), (int64_t)0), a.in_rows - 1) : r;
    from[i] = reinterpret_cast<const T *>(a.x) + at * a.ldx + c0 + lane * (ALIGNED ? kPiece : 8);
    to[i] = reinterpret_cast<uint32_t *>(a.q + r * a.ldq + c0 / 2) + lane;
  }
  uint32_t *scale = reinterpret_cast<uint32_t *>(a.scale + (slot * a.runs + (c0 >> 7) + (lane >> 4)) * kScaleTile + l * 16) + (lane & 3);
  Eight<T> x[4];
  auto fetch = [&](int ahead, int stage) {  // `ahead`: strips from the present one
    if (!ALIGNED) {
#pragma unroll
      for (int i = 0; i < 4; ++i) x[i].load_any(from[i] + ahead * 256, a.cols - c0 - ahead * 256 - lane * 8);
      return;
    }
    if (c0 + ahead * 256 < last) {
      // (a warp's 32 pieces are next to each other, so that whole sectors are asked for)
      const uint32_t at = smem_u32(ring + (stage * 4 * 8 + (threadIdx.x >> 5)) * 32 * kWords + lane);
#pragma unroll
      for (int w = 0; w < kWords; ++w) {
        const int from_here = a.cols - c0 - ahead * 256 - (w * 32 + lane) * kPiece;
        const int bytes = max(0, min(16, from_here * (int)sizeof(T)));  // (the rest of the 16 is zero)
#pragma unroll
        for (int i = 0; i < 4; ++i)
          asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(at + (i * 8 * 32 * kWords + w * 32) * 16),
                       "l"(from[i] + (bytes ? ahead * 256 + w * 32 * kPiece : -lane * kPiece)), "r"(bytes)
                       : "memory");
      }
    }
    asm volatile("cp.async.commit_group;" ::: "memory");
  };
  if (ALIGNED) {
#pragma unroll
    for (int n = 0; n < kAhead - 1; ++n) fetch(n, n);
  } else {
    fetch(0, 0);
  }
  int stage = 0;
  for (; c0 < last; c0 += 256) {
    if (ALIGNED) {
      if (kWords > 1) __syncwarp();  // (a lane reads what two others brought: all have read the strip whose place is taken)
      fetch(kAhead - 1, stage == 0 ? kAhead - 1 : stage - 1);
      asm volatile("cp.async.wait_group %0;" ::"n"(kAhead - 1) : "memory");
      if (kWords > 1) __syncwarp();
#pragma unroll
      for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int w = 0; w < kWords; ++w) x[i].w[w] = ring[((stage * 4 + i) * 8 + (threadIdx.x >> 5)) * 32 * kWords + lane * kWords + w];
      if (++stage == kAhead) stage = 0;
    }
    uint32_t q[4], scales;
    quantize_four(x, q, scales);
    if (!ALIGNED && c0 + 256 < last) fetch(1, 0);
    if (c0 + lane * 8 < (a.cols + 31) / 32 * 32) {
#pragma unroll
      for (int i = 0; i < 4; ++i)
        if (i < rows) *to[i] = q[i];
    }
    if ((lane & 12) == 0 && (c0 >> 7) + (lane >> 4) < a.runs) *scale = scales;
#pragma unroll
    for (int i = 0; i < 4; ++i) from[i] += 256, to[i] += 32;
    scale += 2 * kScaleTile / 4;
  }
}

// A warp's 256 columns of a row, from c on (a lane's), `have` of which are read: to the row's values and to its place in a tile's scales.
template <typename T>
__device__ __forceinline__ void quantize_piece(const T *row, int have, int c, int cols, uint8_t *q, uint8_t *tile, int at, int runs) {
  const int lane = threadIdx.x & 31, run = c >> 7;
  Eight<T> x;
  x.load_any(row + c, have - c);
  uint32_t amax = Eight<T>::top_bits(x.top(0));
  amax = max(amax, __shfl_xor_sync(~0u, amax, 1));
  amax = max(amax, __shfl_xor_sync(~0u, amax, 2));
  const uint32_t byte = fp4_scale(amax);
  const float by = fp4_inverse(byte);
  float v[8];
  x.values(v);
#pragma unroll
  for (int j = 0; j < 8; ++j) v[j] *= by;
  if (c < (cols + 31) / 32 * 32) *reinterpret_cast<uint32_t *>(q + c / 2) = fp4_eight(v);
  uint32_t word = byte << (lane & 12) * 2;
  word |= __shfl_xor_sync(~0u, word, 4);
  word |= __shfl_xor_sync(~0u, word, 8);
  if ((lane & 15) == 0 && run < runs) *reinterpret_cast<uint32_t *>(tile + run * kScaleTile + (at & 31) * 16 + (at >> 5) * 4) = word;
}

// The same for a few rows an expert, whose tiles would be nearly empty: a block takes 2048 columns of one row, a warp 256 of them.
template <typename T>
__global__ void __launch_bounds__(256) tuna_quantize4_few_kernel(Quant4Args a) {
  wait_previous();
  allow_next();
  const int lane = threadIdx.x & 31, c = ((int)blockIdx.y * 8 + (threadIdx.x >> 5)) * 256 + lane * 8;
  const int64_t r = blockIdx.x;
  // on their way together: where the row comes from, and every 32nd group's first row (there are 1024 groups at most)
  const int64_t from = a.gather ? __ldg(a.gather + r) : r;
  auto cut = [&](int g) { return min(max(a.offsets[g], (int64_t)0), a.rows); };
  const uint32_t coarse = __ballot_sync(~0u, lane * 32 < a.groups && cut(min(lane * 32, a.groups - 1)) <= r);
  if (!(coarse & 1)) return;
  int g = (31 - __clz(coarse)) * 32 + lane;
  const int64_t first = cut(min(g, a.groups));
  const uint32_t fine = __ballot_sync(~0u, g < a.groups && first <= r);
  if (!(fine & 1)) return;
  g += 31 - __clz(fine) - lane;  // the last group that begins at r or before it
  const int64_t begin = __shfl_sync(~0u, first, 31 - __clz(fine));
  if (r >= cut(g + 1)) return;
  const bool there = from >= 0 && from < a.in_rows;
  quantize_piece(reinterpret_cast<const T *>(a.x) + (there ? from : 0) * a.ldx, there ? a.cols : 0, c, a.cols, a.q + r * a.ldq,
                 a.scale + (begin / 128 + g + (r - begin) / 128) * a.runs * kScaleTile, (int)((r - begin) % 128), a.runs);
}

// The same for the choices of a few tokens, which it puts in their experts' order itself: a block counts the choices before its own (of
// lower experts, and earlier ones of the same), which is its row.  The first block also leaves the experts' first rows.
constexpr int kPlaceMost = 128;  // choices: a tile's rows, so that an expert has one tile at most
struct Place4Args {
  Quant4Args quant;
  const int32_t *ids;
  int n, k, experts;
  int64_t *first, *pos;  // experts + 1; n: a choice's row, -1 where there is no such expert
};
__global__ void __launch_bounds__(256) tuna_place_quantize4_kernel(Place4Args a) {
  __shared__ int ids[kPlaceMost];
  wait_previous();
  allow_next();
  const int lane = threadIdx.x & 31, c = ((int)blockIdx.y * 8 + (threadIdx.x >> 5)) * 256 + lane * 8, i = blockIdx.x;
  if (threadIdx.x < a.n) {
    const int id = a.ids[threadIdx.x];
    ids[threadIdx.x] = id >= 0 && id < a.experts ? id : INT32_MAX;
  }
  __syncthreads();
  if (i == 0 && blockIdx.y == 0)
    for (int e = threadIdx.x; e <= a.experts; e += 256) {
      int before = 0;
      for (int j = 0; j < a.n; ++j) before += ids[j] < e;
      a.first[e] = before;
    }
  const int mine = ids[i];
  int begin = 0, rank = 0;
  for (int j = lane; j < a.n; j += 32) begin += ids[j] < mine, rank += j < i && ids[j] == mine;
  begin = __reduce_add_sync(~0u, begin), rank = __reduce_add_sync(~0u, rank);
  if (threadIdx.x == 0 && blockIdx.y == 0) a.pos[i] = mine == INT32_MAX ? -1 : begin + rank;
  if (mine == INT32_MAX) return;
  const Quant4Args &q = a.quant;
  quantize_piece(reinterpret_cast<const __nv_bfloat16 *>(q.x) + (i / a.k) * q.ldx, q.cols, c, q.cols, q.q + (int64_t)(begin + rank) * q.ldq,
                 q.scale + (int64_t)(begin / 128 + mine) * q.runs * kScaleTile, rank, q.runs);
}

// Blocks along the columns, for the turned matrix: a block of threads takes a 128 x 128 tile through shared memory in its
// own type; a thread then has 32 rows, one scale block, of two columns, read as pairs.  The tile's scales are one tile of them.
// 8192 x 4096 of bf16 13.4 us (6.4 TB/s).
template <typename T>
struct Turn {
  static constexpr int kPitch = 128 + 16 / sizeof(T);  // rows stay on 16-byte boundaries, four banks apart
  static constexpr size_t kSmem = 128 * kPitch * sizeof(T);
};
template <typename T>
__global__ void __launch_bounds__(256) tuna_quantize4_columns_kernel(Quant4Args a) {
  extern __shared__ __align__(16) char tile_raw[];
  T *tile = reinterpret_cast<T *>(tile_raw);
  constexpr int kPitch = Turn<T>::kPitch;
  __shared__ __align__(16) uint8_t scales[kScaleTile];
  wait_previous();
  allow_next();
  const int col_tiles = (a.cols + 127) / 128, col_tile = blockIdx.x % col_tiles, run = blockIdx.x / col_tiles;
  const int64_t r0 = (int64_t)run * 128;
  const int c0 = col_tile * 128, tid = threadIdx.x;
  const int mine = tid >> 4, c = (tid & 15) * 8;  // rows mine, mine + 16, ...; columns c .. c + 7
  Eight<T> x[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const int64_t r = r0 + mine + i * 16;
    x[i].load_any(reinterpret_cast<const T *>(a.x) + r * a.ldx + c0 + c, r < a.rows ? a.cols - c0 - c : 0);
  }
#pragma unroll
  for (int i = 0; i < 8; ++i)
#pragma unroll
    for (int q = 0; q < Eight<T>::kWords; ++q) *reinterpret_cast<uint4 *>(tile + (mine + i * 16) * kPitch + c + q * (8 / Eight<T>::kWords)) = x[i].w[q];
  __syncthreads();
  const int quarter = tid >> 6;  // rows quarter * 32 .. of two columns: next to each other in bf16, whose words they share, else 64 apart
  auto column = [&](int e) { return sizeof(T) == 2 ? (tid & 63) * 2 + e : (tid & 63) + 64 * e; };
  uint32_t t[2][sizeof(T) == 2 ? 1 : 32], pairs[sizeof(T) == 2 ? 32 : 1], top[2] = {0, 0};
#pragma unroll
  for (int r = 0; r < 32; ++r) {
    const T *p = tile + (quarter * 32 + r) * kPitch;
    if constexpr (sizeof(T) == 2) {
      pairs[r] = *reinterpret_cast<const uint32_t *>(p + column(0));
      top[0] = __vmaxu2(top[0], pairs[r] & 0x7fff7fffu);
    } else {
#pragma unroll
      for (int e = 0; e < 2; ++e) t[e][r] = __float_as_uint(p[column(e)]), top[e] = max(top[e], t[e][r] & 0x7fffffffu);
    }
  }
  if (sizeof(T) == 2) top[1] = top[0] & 0xffff0000u, top[0] <<= 16;
  __syncthreads();  // the tile has been read: the values go out by way of its place, in whole sectors
  uint4 *out = reinterpret_cast<uint4 *>(tile_raw);  // [128 columns][4 quarters], their pieces turned by column
#pragma unroll
  for (int e = 0; e < 2; ++e) {
    const uint32_t byte = fp4_scale(top[e]);
    const uint64_t by = pair(fp4_inverse(byte), fp4_inverse(byte));
    const int col = column(e);
    scales[(col & 31) * 16 + (col >> 5) * 4 + quarter] = (uint8_t)byte;
    uint32_t q[4];
#pragma unroll
    for (int w = 0; w < 4; ++w) {
      float v[8];
#pragma unroll
      for (int j = 0; j < 8; j += 2) {
        float at[2];
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          const int r = w * 8 + j + h;
          if constexpr (sizeof(T) == 2) at[h] = __uint_as_float(e ? pairs[r] & 0xffff0000u : pairs[r] << 16);
          else at[h] = __uint_as_float(t[e][r]);
        }
        unpair(mul2(pair(at[0], at[1]), by), v[j], v[j + 1]);
      }
      q[w] = fp4_eight(v);
    }
    out[col * 4 + (quarter ^ (col >> 1 & 3))] = make_uint4(q[0], q[1], q[2], q[3]);
  }
  __syncthreads();
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    const int col = i * 64 + (tid >> 2), piece = tid & 3;
    if (c0 + col < a.cols && r0 + piece * 32 < a.rows)
      *reinterpret_cast<uint4 *>(a.q + (int64_t)(c0 + col) * a.ldq + (r0 + piece * 32) / 2) = out[col * 4 + (piece ^ (col >> 1 & 3))];
  }
  if (tid < 32) reinterpret_cast<uint4 *>(a.scale + ((int64_t)col_tile * a.runs + run) * kScaleTile)[tid] = reinterpret_cast<const uint4 *>(scales)[tid];
}

// The values that 4-bit rows stand for, in the quantisation's arrangement: 8192 x 4096 to bf16 14.3 us (6.0 TB/s), to f32 27.7 us.  ALIGNED: words of q, and eight values of the
// result, can be taken whole.
template <typename T, bool ALIGNED>
__global__ void __launch_bounds__(256) tuna_dequantize4_kernel(Quant4Args a, T *out, int64_t ldo) {
  wait_previous();
  allow_next();
  const int lane = threadIdx.x & 31, l = (blockIdx.x & 3) * 8 + (threadIdx.x >> 5);
  const int64_t slot = blockIdx.x >> 2;
  int64_t row0, end;
  slot_rows(a.offsets, a.groups, a.rows, slot, row0, end);
  if (row0 + l >= end) return;
  const int rows = (int)min((end - row0 - l + 31) / 32, (int64_t)4);
  int c = (int)blockIdx.y * a.strips * 256 + lane * 8;
  const int last = min(a.cols, (int)(blockIdx.y + 1) * a.strips * 256);
  const uint8_t *from[4];
  T *to[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const int64_t r = row0 + l + 32 * min(i, rows - 1);  // (a row that is not there: the last one again, written only once)
    from[i] = a.q + r * a.ldq + c / 2, to[i] = out + r * ldo + c;
  }
  const uint4 *scale = reinterpret_cast<const uint4 *>(a.scale + (slot * a.runs + (c >> 7)) * kScaleTile + l * 16);
  for (; c < last; c += 256) {
    const uint4 s = __ldg(scale);
    const uint32_t words[4] = {s.x, s.y, s.z, s.w};
    const bool whole = ALIGNED && c + 8 <= a.cols;
    uint32_t q[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      if (whole || (c + 8 <= a.cols && ((uintptr_t)from[i] & 3) == 0)) {
        q[i] = __ldg(reinterpret_cast<const uint32_t *>(from[i]));
      } else {
        q[i] = 0;
#pragma unroll
        for (int j = 0; j < 4; ++j)
          if (c + 2 * j < a.cols) q[i] |= (uint32_t)from[i][j] << (8 * j);
      }
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      if (i >= rows) break;
      const float by = fp4_power(__byte_perm(words[i], 0, 0x4440 | (lane >> 2 & 3)));
      float v[8];
      fp4_values(q[i], v);
#pragma unroll
      for (int j = 0; j < 8; j += 2) unpair(mul2(pair(v[j], v[j + 1]), pair(by, by)), v[j], v[j + 1]);
      if constexpr (sizeof(T) == 4) {
        if (whole) {
          uint32_t u[8];
#pragma unroll
          for (int j = 0; j < 8; ++j) u[j] = __float_as_uint(v[j]);
          store32(to[i], u);
          continue;
        }
      }
      if (whole) store_row(to[i], v);
      else store_any(to[i], v, a.cols - c);
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) from[i] += 128, to[i] += 256;
    scale += 2 * kScaleTile / 16;
  }
}

// Rows of bytes to rows on 16-byte boundaries: a warp takes 512 bytes of a row, a lane 16 of them in the widest pieces that the source
// allows.  (2001 rows of 1448 bytes for a product that follows: 3 us; a copy by the runtime, between the launches, 8.)
__global__ void __launch_bounds__(256) tuna_align4_kernel(const uint8_t *q, int64_t ldq, int64_t rows, int64_t bytes, uint8_t *out, int64_t ldo) {
  wait_previous();
  allow_next();
  const int64_t pieces = (bytes + 15) / 16, all = rows * pieces;
  for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < all; i += (int64_t)gridDim.x * 256) {
    const int64_t r = i / pieces, b = (i - r * pieces) * 16;
    const uint8_t *from = q + r * ldq + b;
    uint8_t *to = out + r * ldo + b;
    if (b + 16 <= bytes && ((uintptr_t)from & 3) == 0) {
      Eight<__nv_bfloat16> v;
      v.load_any(reinterpret_cast<const __nv_bfloat16 *>(from), 8);
      *reinterpret_cast<uint4 *>(to) = v.w[0];
    } else {
      for (int j = 0; j < 16 && b + j < bytes; ++j) to[j] = from[j];
    }
  }
}

// ---- the product -----------------------------------------------------------------------------
//
// A persistent block takes tiles of 128 x BN.  One lane copies 128 x 256 values of a, BN x 256 of b and the scales of both
// into a ring of stages; one elected lane moves a stage's scales into tensor memory, to columns that belong to the stage,
// and issues its four tensor-core steps; eight warps read a finished accumulator back and store it.
//
// What bounds it: the 1000 W limit.  8192 x 4096 x 4096 takes 55 us in bursts with pauses between them (5000 TFLOP/s) and 61 in long runs
// (4500) at a clock of 1.4 to 1.5 GHz, the tensor pipe busy for 57 to 63 % of the cycles, and that time does not change when b is shared by pairs, when the next tile's steps begin
// before an accumulator has been read out, or when the copies of the scales are left out.  A few rows are bound by memory: 64
// matrices of 4096 x 2048 with 4 rows each 45.3 us, 96 % of the copy rate.  (SwiGLU's tiles were bound by their results: with exact division 511 us for
// the first product of 64 experts of 4096 x 2048 and 16384 uneven rows; now 188 in bursts and 222 in long runs, 156 in bursts with 256 rows each, as
// much as two products of its two halves without it.)
//
// With `swiglu` the 256 columns are 128 rows of the gate matrix and the same 128 of the up matrix, so that a thread reads
// both values of a place from its own row of the accumulator, and 32 of them are one block of the 4-bit result.  Blocks behind the
// last column get the scale 0: b's values are zero there, but its scales may be anything, NaN too, and the next product reads the scales
// to the end of the run (and no values).
struct Tile4Args {
  Product4Args p;
  int stages;   // of k: 256 values each
  int n_tiles;
  int store_tiles;     // bf16 results leave through map_out
  int box_a;           // rows of a that a copy brings
  uint32_t most_rows;  // row tiles, at most: their number times n_tiles, and a step beyond, fits 31 bits
  int *error;
};

constexpr int kOutWarps = 8;
constexpr int kThreads4 = 128 + kOutWarps * 32;
constexpr int kMaxGroups4 = TUNA_MOE_MAX_EXPERTS;

// What the groups' bounds come to: first rows (and the end behind the last one), cut to the operand, and tiles of rows before each.
struct Groups4 {
  int row[kMaxGroups4 + 1], tile[kMaxGroups4 + 1];
};

template <int BN, bool STORES, bool PAIR>
struct Shape4 {
  // what is in flight hides the memory's latency, so the stages take the room that the results on their way out leave
  static constexpr int kStages = PAIR ? (STORES ? 5 : 6) : BN == 256 ? 4 : (STORES ? 5 : 6);
  static constexpr int kRowsB = PAIR ? BN / 2 : BN;            // of b in this block's shared memory
  static constexpr int kOperandBytes = (128 + kRowsB) * 128;
  static constexpr int kScaleBytes = 1024 + BN / 128 * 1024;
  static constexpr int kStageBytes = kOperandBytes + kScaleBytes;
  static constexpr int kAccs = BN == 256 ? 1 : 2;              // accumulators
  static constexpr int kScaleCols = 8 + BN / 128 * 8;          // tensor-memory columns of a stage's scales
  static constexpr int kCols = BN / 2;                         // accumulator columns of a warp of the results
  static constexpr int kSumPitch = BN + 4;  // floats: rows of sums that a cluster joins, on 16-byte boundaries and four banks apart
  static_assert(128 * kSumPitch * 4 <= kStages * kStageBytes);
  static constexpr int kOutCols = BN == 256 && !PAIR ? 32 : 64;    // bf16 results that a warp sends out at a time, of 32 rows
  static constexpr int kOutBytes = STORES ? kOutWarps * 32 * kOutCols * 2 : 0;
  static_assert(kAccs * BN + kStages * kScaleCols <= 512);
  static_assert(kStageBytes % 1024 == 0);
  static constexpr size_t kSmem = 1024 + (size_t)kStages * kStageBytes + kOutBytes + sizeof(Groups4) + 256;
  // One block a multiprocessor: a launch that begins early takes its tensor memory before it waits for the one before it, which must
  // not be without its own then.
  static_assert(kSmem > 116 * 1024 && kSmem <= 227 * 1024);
};

// 512 bytes of scales to 4 columns of tensor memory, once for each quarter of the lanes; of a pair, in both of its blocks
template <bool PAIR>
__device__ __forceinline__ void tc_copy_scales(uint32_t to, uint32_t smem) {
  // rows of 16 bytes, 8 of them 128 bytes apart, no swizzle
  const uint64_t desc = (uint64_t)((smem & 0x3ffff) >> 4) | ((uint64_t)(128 >> 4) << 32) | ((uint64_t)1 << 46);
  if (PAIR) asm volatile("tcgen05.cp.cta_group::2.32x128b.warpx4 [%0], %1;" ::"r"(to), "l"(desc) : "memory");
  else asm volatile("tcgen05.cp.cta_group::1.32x128b.warpx4 [%0], %1;" ::"r"(to), "l"(desc) : "memory");
}
__device__ __forceinline__ float load_one(uint32_t addr, uint32_t rank) {  // from a block of the cluster
  float v;
  asm volatile("{\n .reg .b32 a;\n mapa.shared::cluster.u32 a, %1, %2;\n ld.shared::cluster.f32 %0, [a];\n}" : "=f"(v) : "r"(addr), "r"(rank) : "memory");
  return v;
}
// d[tmem] (+)= A (128 x 64, of a pair 256 x 64) * B^T (N x 64), 4-bit values with a scale for each 32 of them
template <bool PAIR>
__device__ __forceinline__ void tc_mma_fp4(uint32_t d, uint64_t a, uint64_t b, uint32_t idesc, uint32_t sa, uint32_t sb, bool accumulate) {
  if (PAIR)
    asm volatile(
        "{\n .reg .pred p;\n setp.ne.u32 p, %4, 0;\n"
        " tcgen05.mma.cta_group::2.kind::mxf4.block_scale.scale_vec::2X [%0], %1, %2, %3, [%5], [%6], p;\n}" ::"r"(d),
        "l"(a), "l"(b), "r"(idesc), "r"((uint32_t)accumulate), "r"(sa), "r"(sb)
        : "memory");
  else
    asm volatile(
        "{\n .reg .pred p;\n setp.ne.u32 p, %4, 0;\n"
        " tcgen05.mma.cta_group::1.kind::mxf4.block_scale.scale_vec::2X [%0], %1, %2, %3, [%5], [%6], p;\n}" ::"r"(d),
        "l"(a), "l"(b), "r"(idesc), "r"((uint32_t)accumulate), "r"(sa), "r"(sb)
        : "memory");
}
// Arrives, when all steps so far are done, at a barrier of this block, or at the same one in both blocks of a pair.
template <bool PAIR>
__device__ __forceinline__ void tc_commit_to(uint32_t bar) {
  if (PAIR)
    asm volatile("tcgen05.commit.cta_group::2.mbarrier::arrive::one.shared::cluster.multicast::cluster.b64 [%0], %1;" ::"r"(bar), "h"((uint16_t)3) : "memory");
  else
    tc_commit(bar);
}
// Tensor copies into this block's shared memory; of a pair, the bytes are counted by the first block's barrier, which `bar` is in.
template <bool PAIR>
__device__ __forceinline__ void load_2d(uint32_t dst, const CUtensorMap *map, int x, int y, uint32_t bar) {
  if (PAIR)
    asm volatile("cp.async.bulk.tensor.2d.cta_group::2.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3}], [%4];" ::"r"(dst),
                 "l"(map), "r"(x), "r"(y), "r"(bar)
                 : "memory");
  else
    tma_load_2d(dst, map, x, y, bar);
}
template <bool PAIR>
__device__ __forceinline__ void load_3d(uint32_t dst, const CUtensorMap *map, int x, int y, int z, uint32_t bar) {
  if (PAIR)
    asm volatile("cp.async.bulk.tensor.3d.cta_group::2.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3, %4}], [%5];" ::"r"(dst),
                 "l"(map), "r"(x), "r"(y), "r"(z), "r"(bar)
                 : "memory");
  else
    tma_load_3d(dst, map, x, y, z, bar);
}
__device__ __forceinline__ uint32_t in_first_block(uint32_t addr) {  // the same place in the shared memory of the cluster's first block
  uint32_t r;
  asm("mapa.shared::cluster.u32 %0, %1, 0;" : "=r"(r) : "r"(addr));
  return r;
}
// (No memory is handed over with it, only room in tensor memory: a release to the cluster would wait for all that the thread
// has stored, 1600 cycles a tile.)
__device__ __forceinline__ void mbar_arrive_far(uint32_t bar) { asm volatile("mbarrier.arrive.shared::cluster.b64 _, [%0];" ::"r"(bar) : "memory"); }
template <bool PAIR>
__device__ __forceinline__ void tmem_take(uint32_t smem_dst) {
  if (PAIR) {
    asm volatile("tcgen05.alloc.cta_group::2.sync.aligned.shared::cta.b32 [%0], 512;" ::"r"(smem_dst) : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::2.sync.aligned;" ::: "memory");
  } else {
    tmem_alloc(smem_dst, 512);
  }
}
template <bool PAIR>
__device__ __forceinline__ void tmem_give(uint32_t addr) {
  if (PAIR) asm volatile("tcgen05.dealloc.cta_group::2.sync.aligned.b32 %0, 512;" ::"r"(addr) : "memory");
  else tmem_free(addr, 512);
}
// Instruction descriptor: e2m1 operands, e8m0 scales, n columns, m rows; `half`: which two of a word's four scales
__host__ __device__ constexpr uint32_t fp4_idesc(int m, int n, int half) {
  return (1u << 7) | (1u << 10) | (1u << 23) | ((uint32_t)(n >> 3) << 17) | ((uint32_t)(m >> 4) << 24) | ((uint32_t)(half * 2) << 29) | ((uint32_t)(half * 2) << 4);
}

// Tile t of the walk: the group it is in (never walked backwards), its rows and columns.
struct Walk4 {
  int g = 0;
  int row, end;  // first row, end of the group's rows
  int slot;      // tile of the rows' scales
  int n0;
};
template <int ROWS>
__device__ __forceinline__ void walk_to(Walk4 &w, int t, const Tile4Args &a, const Groups4 &at, int bn) {
  if (t >= at.tile[w.g + 1] * a.n_tiles) {  // the last group that begins at t or before it
    int high = a.p.groups;
    while (high - w.g > 1) {
      const int g = (w.g + high) >> 1;
      if (at.tile[g] * a.n_tiles <= t) w.g = g;
      else high = g;
    }
  }
  const uint32_t mt = at.tile[w.g + 1] - at.tile[w.g], local = t - at.tile[w.g] * a.n_tiles;
  const uint32_t n = local / mt, m = local - n * mt;  // rows fastest: blocks that run together share b
  const int begin = at.row[w.g];
  w.row = begin + (int)m * ROWS, w.end = at.row[w.g + 1];
  w.slot = begin / 128 + w.g + (int)m * (ROWS / 128);
  if (ROWS == 256 && cluster_rank()) w.row += 128, ++w.slot;  // this block's half
  w.n0 = n * bn;
}

// With PAIR a cluster of two blocks takes a tile of 256 rows: each has 128 of them and half of b's rows in its shared memory, all
// scales of b, and the results of its own rows in its tensor memory.  The first block's elected lane issues the steps for
// both; the copies of both are counted by its barriers.  A multiprocessor then takes 68 bytes a cycle of its tensor cores' rate in
// copies where a block alone takes 102 (BN = 256), and b's half is read by both.
//
// With SPLIT a cluster of 2 or 4 blocks shares one tile: each adds up a part of k, leaves its sums in its shared memory,
// and adds up the parts of some of the rows from all of them, in order of k.
template <int BN, bool SWIGLU, bool SPLIT, bool PAIR, typename TO>
__global__ void __launch_bounds__(kThreads4, 1)
    tuna_product4_kernel(const __grid_constant__ CUtensorMap map_a, const __grid_constant__ CUtensorMap map_b, const __grid_constant__ CUtensorMap map_sa,
                         const __grid_constant__ CUtensorMap map_sb, const __grid_constant__ CUtensorMap map_out, const Tile4Args a) {
  using S = Shape4<BN, !SWIGLU && !SPLIT && sizeof(TO) == 2, PAIR>;
  static_assert(!PAIR || (BN == 256 && !SPLIT));
  constexpr int kRows = PAIR ? 256 : 128;
  extern __shared__ char smem_raw[];
  char *smem = smem_raw + ((1024 - (smem_u32(smem_raw) & 1023)) & 1023);
  Groups4 &groups = *(Groups4 *)(smem + (size_t)S::kStages * S::kStageBytes + S::kOutBytes);
  uint64_t *bars = (uint64_t *)(&groups + 1);
  volatile int *given_up = (volatile int *)(bars + 2 * S::kStages + 2 * S::kAccs + 1);
  uint32_t *tmem_at = (uint32_t *)(given_up + 1);
  const uint32_t full = smem_u32(bars), empty = full + 8 * S::kStages, done = empty + 8 * S::kStages, freed = done + 8 * S::kAccs, drained = freed + 8 * S::kAccs;
  const int warp = __shfl_sync(~0u, threadIdx.x >> 5, 0), lane = threadIdx.x & 31;

  if (threadIdx.x == 32) {
    for (const CUtensorMap *map : {&map_a, &map_b, &map_sa, &map_sb}) asm volatile("prefetch.tensormap [%0];" ::"l"(map) : "memory");
  }
  if (threadIdx.x == 0) {
    for (int s = 0; s < S::kStages; ++s) mbar_init(full + 8 * s, 1), mbar_init(empty + 8 * s, 1);
    for (int s = 0; s < S::kAccs; ++s) mbar_init(done + 8 * s, 1), mbar_init(freed + 8 * s, PAIR ? 2 * kOutWarps : kOutWarps);
    mbar_init(drained, 1);
    *given_up = 0;
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
  }
  if (warp == 2) tmem_take<PAIR>(smem_u32(tmem_at));
  wait_previous();
  allow_next();
  // All bounds are fetched at once; a warp then sums up the tiles, cut at most_rows, which groups that lie apart never come near.
  for (int g = threadIdx.x; g <= a.p.groups; g += kThreads4) groups.row[g] = (int)(a.p.offsets ? min(max(a.p.offsets[g], (int64_t)0), a.p.m) : g ? a.p.m : 0);
  __syncthreads();
  if (warp == 1) {
    uint32_t sum = 0;
    for (int g0 = 0; g0 < a.p.groups; g0 += 32) {
      const int g = g0 + lane, rows = g < a.p.groups ? groups.row[g + 1] - groups.row[g] : 0;
      const uint32_t mt = rows > 0 ? (uint32_t)((rows + kRows - 1) / kRows) : 0;  // (2^24 at most: 32 of them and most_rows fit 32 bits)
      uint32_t x = mt;
#pragma unroll
      for (int d = 1; d < 32; d <<= 1) {
        const uint32_t y = __shfl_up_sync(~0u, x, d);
        if (lane >= d) x += y;
      }
      if (g < a.p.groups) groups.tile[g] = (int)min(sum + x - mt, a.most_rows);
      sum = min(sum + __shfl_sync(~0u, x, 31), a.most_rows);
    }
    if (lane == 0) groups.tile[a.p.groups] = (int)sum;
  }
  tc_fence_before();
  __syncthreads();
  if constexpr (PAIR) cluster_meet();  // the barriers of both blocks are there
  tc_fence_after();
  const uint32_t tmem = __shfl_sync(~0u, *tmem_at, 0);
  const int tiles = groups.tile[a.p.groups] * a.n_tiles;
  const int parts = SPLIT ? (int)cluster_size() : 1, part = SPLIT ? (int)cluster_rank() : 0;
  const int sharers = PAIR ? 2 : parts, first = (int)blockIdx.x / sharers, step = (int)gridDim.x / sharers;
  const int half_b = PAIR ? (int)cluster_rank() : 0;  // of b, and of the pair
  // this block's part of k
  const int s_first = SPLIT ? (int)((int64_t)a.stages * part / parts) : 0, stages = SPLIT ? (int)((int64_t)a.stages * (part + 1) / parts) - s_first : a.stages;
  constexpr int kTileN = SWIGLU ? BN / 2 : BN;

  if (warp == 0) {
    if (lane == 0) {
      // ---- copies
      int stage = 0, phase = 0;
      int64_t issued = 0;
      const int tiles_n = (a.p.n + 127) / 128;
      Walk4 w;
      bool ok = true;
      for (int t = first; ok && t < tiles; t += step) {
        walk_to<kRows>(w, t, a, groups, kTileN);
        // of a, the boxes that hold rows of the group (at least one, so that every block of a pair brings something); what stands
        // in the others' place ends in rows that nobody stores
        const int boxes = max(1, (min(128, w.end - w.row) + a.box_a - 1) / a.box_a);
        const uint32_t left_out = (128 - boxes * a.box_a) * 128;
        // a pair's first block expects what both bring
        const int other = PAIR ? max(1, (min(128, w.end - w.row - 128) + a.box_a - 1) / a.box_a) : 0;
        const uint32_t expected = S::kStageBytes - left_out + (PAIR ? S::kStageBytes - (128 - other * a.box_a) * 128 : 0);
        for (int s = 0; s < stages; ++s) {
          if (!(ok = mbar_wait(empty + 8 * stage, phase ^ 1, given_up))) break;
          const uint32_t at = smem_u32(smem) + stage * S::kStageBytes, scales = at + S::kOperandBytes;
          const uint32_t bar = PAIR ? in_first_block(full + 8 * stage) : full + 8 * stage;
          if (half_b == 0) mbar_expect(full + 8 * stage, expected);
          const int col = (s_first + s) * 128, run = (s_first + s) * 2;
          for (int q = 0; q < boxes; ++q) load_2d<PAIR>(at + q * a.box_a * 128, &map_a, col, w.row + q * a.box_a, bar);
          load_3d<PAIR>(scales, &map_sa, 0, run, w.slot, bar);
          if (SWIGLU) {
#pragma unroll
            for (int q = 0; q < 2; ++q) {
              if (!PAIR || q == half_b) load_3d<PAIR>(at + 128 * 128 + (PAIR ? 0 : q * 128 * 128), &map_b, col, w.n0, w.g * 2 + q, bar);
              load_3d<PAIR>(scales + 1024 + q * 1024, &map_sb, 0, run, (w.g * 2 + q) * tiles_n + w.n0 / 128, bar);
            }
          } else {
            load_3d<PAIR>(at + 128 * 128, &map_b, col, w.n0 + half_b * 128, w.g, bar);
            load_3d<PAIR>(scales + 1024, &map_sb, 0, run, w.g * tiles_n + w.n0 / 128, bar);
          }
          ++issued;
          if (++stage == S::kStages) stage = 0, phase ^= 1;
        }
      }
      // nothing may land in shared memory after the block has gone, whichever warp gives up: the last copies are waited for
      // (of a pair by its first block, which has the barriers; the other one stays until it comes to the meeting)
      int never = 0;
      for (int64_t i = half_b ? issued : max((int64_t)0, issued - S::kStages); i < issued; ++i)
        mbar_wait(full + 8 * (int)(i % S::kStages), (uint32_t)((i / S::kStages) & 1), &never);
      if (PAIR)  // nor may the first block's steps still report to a block that has gone
        for (int64_t i = max((int64_t)0, issued - S::kStages); i < issued; ++i)
          mbar_wait(empty + 8 * (int)(i % S::kStages), (uint32_t)((i / S::kStages) & 1), given_up);
    }
  } else if (warp == 1 && half_b == 0) {
    // ---- tensor cores: the whole warp goes along, one lane issues
    int stage = 0, phase = 0, acc = 0, acc_phase = 0;
    bool ok = true;
    for (int t = first; ok && t < tiles; t += step) {
      ok = __all_sync(~0u, mbar_wait(freed + 8 * acc, acc_phase ^ 1, given_up));
      for (int s = 0; ok && s < stages; ++s) {
        if (!(ok = __all_sync(~0u, mbar_wait(full + 8 * stage, phase, given_up)))) break;
        tc_fence_after();
        const uint32_t at = smem_u32(smem) + stage * S::kStageBytes, scales = at + S::kOperandBytes;
        const uint64_t da = tc_desc(at), db = tc_desc(at + 128 * 128);
        const uint32_t ta = tmem + S::kAccs * BN + stage * S::kScaleCols, tb = ta + 8;
        if (elect_one()) {
#pragma unroll
          for (int r = 0; r < 2; ++r) {  // runs of 128 along k
            tc_copy_scales<PAIR>(ta + r * 4, scales + r * 512);
#pragma unroll
            for (int q = 0; q < BN / 128; ++q) tc_copy_scales<PAIR>(tb + r * (BN / 32) + q * 4, scales + 1024 + q * 1024 + r * 512);
          }
#pragma unroll
          for (int i = 0; i < 4; ++i)  // 32 bytes along k
            tc_mma_fp4<PAIR>(tmem + acc * BN, da + 2 * i, db + 2 * i, fp4_idesc(kRows, BN, i & 1), ta + (i >> 1) * 4, tb + (i >> 1) * (BN / 32), s > 0 || i > 0);
          tc_commit_to<PAIR>(empty + 8 * stage);
          if (s == stages - 1) tc_commit_to<PAIR>(done + 8 * acc);
        }
        __syncwarp();
        if (++stage == S::kStages) stage = 0, phase ^= 1;
      }
      if (++acc == S::kAccs) acc = 0, acc_phase ^= 1;
    }
    // and no step may be under way when tensor memory is freed
    int never = 0;
    if (elect_one()) {
      if (PAIR) asm volatile("tcgen05.commit.cta_group::2.mbarrier::arrive::one.shared::cluster.b64 [%0];" ::"r"(drained) : "memory");
      else tc_commit(drained);
    }
    __syncwarp();
    mbar_wait(drained, 0, &never);
  } else if (warp >= 4) {
    // ---- results: thread = one row, columns [half * kCols, ...) of the tile
    const int half = (warp - 4) >> 2, row_in = (warp & 3) * 32 + lane;
    const uint32_t from = tmem + ((uint32_t)((warp & 3) * 32) << 16);
    int acc = 0, acc_phase = 0;
    Walk4 w;
    for (int t = first; t < tiles; t += step) {
      walk_to<kRows>(w, t, a, groups, kTileN);
      if (!__all_sync(~0u, mbar_wait(done + 8 * acc, acc_phase, given_up))) break;  // (and the warp is whole for the loads)
      tc_fence_after();
      const uint32_t at = from + acc * BN;
      auto release = [&] {  // everything is in registers: the accumulator may be filled again
        tc_fence_before();
        __syncwarp();
        if (lane == 0) {
          if (PAIR) mbar_arrive_far(in_first_block(freed + 8 * acc));
          else mbar_arrive(freed + 8 * acc);
        }
      };
      const int row = w.row + row_in;
      const bool there = row < w.end;
      if constexpr (SPLIT) {
        // the sums to shared memory, where the stages were: every step that read them is done
        float *red = (float *)smem + row_in * S::kSumPitch + half * S::kCols;
#pragma unroll
        for (int c = 0; c < S::kCols; c += 32) {
          uint32_t v[32];
          tmem_load(at + half * S::kCols + c, v);
          tmem_wait(v);
          if (there) {
#pragma unroll
            for (int i = 0; i < 32; i += 4) *reinterpret_cast<uint4 *>(red + c + i) = make_uint4(v[i], v[i + 1], v[i + 2], v[i + 3]);
          }
        }
        release();
      } else if constexpr (SWIGLU) {
        const int c0 = half * 64;
        uint32_t g[2][32], u[2][32], packed[2][4], bytes = 0;
#pragma unroll
        for (int b = 0; b < 2; ++b) tmem_load(at + c0 + b * 32, g[b]), tmem_load(at + 128 + c0 + b * 32, u[b]);
#pragma unroll
        for (int b = 0; b < 2; ++b) tmem_wait(g[b]), tmem_wait(u[b]);
        release();
#pragma unroll
        for (int b = 0; b < 2; ++b) {
          float h[32], top = 0.0f;
#pragma unroll
          for (int i = 0; i < 32; i += 2) {
            unpair(swiglu2(__uint_as_float(g[b][i]), __uint_as_float(g[b][i + 1]), __uint_as_float(u[b][i]), __uint_as_float(u[b][i + 1])), h[i], h[i + 1]);
            top = top_of(top, h[i], h[i + 1]);
          }
          const uint32_t byte = w.n0 + c0 + b * 32 < a.p.n ? fp4_scale(__float_as_uint(top) & 0x7fffffffu) : 0;  // (n is whole blocks)
          const uint64_t by = pair(fp4_inverse(byte), fp4_inverse(byte));
#pragma unroll
          for (int i = 0; i < 32; i += 2) unpair(mul2(pair(h[i], h[i + 1]), by), h[i], h[i + 1]);
#pragma unroll
          for (int i = 0; i < 4; ++i) packed[b][i] = fp4_eight(h + i * 8);
          bytes |= byte << (8 * b);
        }
        if (there) {
          uint8_t *out = (uint8_t *)a.p.out + (int64_t)row * a.p.ldo + (w.n0 + c0) / 2;  // (the pitch covers whole tiles)
          *reinterpret_cast<uint4 *>(out) = make_uint4(packed[0][0], packed[0][1], packed[0][2], packed[0][3]);
          *reinterpret_cast<uint4 *>(out + 16) = make_uint4(packed[1][0], packed[1][1], packed[1][2], packed[1][3]);
          *reinterpret_cast<uint16_t *>(a.p.hs + ((int64_t)w.slot * a.n_tiles + w.n0 / 128) * kScaleTile + lane * 16 + (warp & 3) * 4 + half * 2) = (uint16_t)bytes;
        }
      } else if constexpr (sizeof(TO) == 2) {
        uint32_t packed[S::kCols / 2];
#pragma unroll
        for (int c = 0; c < S::kCols; c += 32) {
          uint32_t v[32];
          tmem_load(at + half * S::kCols + c, v);
          tmem_wait(v);
#pragma unroll
          for (int i = 0; i < 16; ++i) packed[c / 2 + i] = pack_bf16(__uint_as_float(v[2 * i]), __uint_as_float(v[2 * i + 1]));
        }
        release();
        // kOutCols columns at a time to shared memory, in 16-byte pieces swizzled by row.  32 whole rows leave from there by a
        // tensor copy; rows that a group's end cuts, or that a tensor copy cannot reach (a pitch that is no multiple of 16
        // bytes), leave in whole rows as the warp reads them back.
        constexpr int kRowBytes = S::kOutCols * 2, kPieces = kRowBytes / 16;
        auto place = [](int r, int piece) { return (uint32_t)(r * kRowBytes + (kPieces == 8 ? piece ^ (r & 7) : piece ^ ((r >> 1) & 3)) * 16); };
        const uint32_t to = smem_u32(smem) + S::kStages * S::kStageBytes + (warp - 4) * 32 * kRowBytes;
        const int row0 = row - lane, valid = max(0, min(32, w.end - row0));
#pragma unroll
        for (int c = 0; c < S::kCols; c += S::kOutCols) {
          const int c0 = w.n0 + half * S::kCols + c;
          if (lane == 0) tma_store_read();
          __syncwarp();
#pragma unroll
          for (int i = 0; i < kPieces; ++i)
            asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %4};" ::"r"(to + place(lane, i)), "r"(packed[c / 2 + i * 4]), "r"(packed[c / 2 + i * 4 + 1]),
                         "r"(packed[c / 2 + i * 4 + 2]), "r"(packed[c / 2 + i * 4 + 3])
                         : "memory");
          if (a.store_tiles && valid == 32) {
            asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
            __syncwarp();
            if (lane == 0 && c0 < a.p.n) tma_store_2d(&map_out, c0, row0, to);
          } else {
            __syncwarp();
            __nv_bfloat16 *out = (__nv_bfloat16 *)a.p.out + (int64_t)row0 * a.p.ldo + c0;
            if (a.store_tiles && c0 + S::kOutCols <= a.p.n) {
              for (int i = lane; i < valid * kPieces; i += 32) {
                const int r = i / kPieces, piece = i % kPieces;
                uint4 u;
                asm volatile("ld.shared.v4.b32 {%0, %1, %2, %3}, [%4];" : "=r"(u.x), "=r"(u.y), "=r"(u.z), "=r"(u.w) : "r"(to + place(r, piece)) : "memory");
                *reinterpret_cast<uint4 *>(out + r * a.p.ldo + piece * 8) = u;
              }
            } else {
              const int cols = min(S::kOutCols, a.p.n - c0);
              for (int r = 0; r < valid; ++r)
                for (int j = lane; j < cols; j += 32) {
                  uint16_t u;
                  asm volatile("ld.shared.b16 %0, [%1];" : "=h"(u) : "r"(to + place(r, j >> 3) + (j & 7) * 2) : "memory");
                  reinterpret_cast<uint16_t *>(out)[r * a.p.ldo + j] = u;
                }
            }
          }
          __syncwarp();
        }
      } else {
        // 32-bit results, in whole 32-byte sectors
        float *out = (float *)a.p.out + (int64_t)row * a.p.ldo;
        const bool vec = (((uintptr_t)a.p.out | (uint64_t)a.p.ldo * 4) & 31) == 0;
#pragma unroll
        for (int c = 0; c < S::kCols; c += 32) {
          uint32_t v[32];
          tmem_load(at + half * S::kCols + c, v);
          tmem_wait(v);
          if (c + 32 == S::kCols) release();
          const int c0 = w.n0 + half * S::kCols + c;
          if (!there) continue;
#pragma unroll
          for (int i = 0; i < 32; i += 8) {
            if (vec && c0 + i + 8 <= a.p.n) {
              const uint32_t u[8] = {v[i], v[i + 1], v[i + 2], v[i + 3], v[i + 4], v[i + 5], v[i + 6], v[i + 7]};
              store32(out + c0 + i, u);
            } else {
#pragma unroll
              for (int j = 0; j < 8; ++j)
                if (c0 + i + j < a.p.n) out[c0 + i + j] = __uint_as_float(v[i + j]);
            }
          }
        }
      }
      __syncwarp();
      if (++acc == S::kAccs) acc = 0, acc_phase ^= 1;
    }
    if (S::kOutBytes && lane == 0) tma_store_done();
  }
  __syncwarp();
  if constexpr (SPLIT) {
    cluster_meet();
    if (first < tiles && !*given_up) {
      Walk4 w;
      walk_to<kRows>(w, first, a, groups, kTileN);
      const int rows = min(128, w.end - w.row), mine = (rows - part + parts - 1) / parts;
      if constexpr (SWIGLU) {
        // a warp a row and block of 32: a lane has a gate and an up sum
        for (int i = warp; i < mine * 4; i += kThreads4 / 32) {
          const int r = part + (i >> 2) * parts, c = (i & 3) * 32 + lane;
          const uint32_t at = smem_u32(smem) + (r * S::kSumPitch + c) * 4;
          float g = 0.0f, u = 0.0f;
          for (int q = 0; q < parts; ++q) g += load_one(at, q), u += load_one(at + 128 * 4, q);
          float h, unused;
          unpair(swiglu2(g, g, u, u), h, unused);
          const uint32_t most = __reduce_max_sync(~0u, abs_bits(h)), byte = w.n0 + (i & 3) * 32 < a.p.n ? fp4_scale(most) : 0;
          const float v = h * fp4_inverse(byte);
          // eight neighbours' values to the first of them
          float eight[8];
#pragma unroll
          for (int j = 0; j < 8; ++j) eight[j] = __shfl_down_sync(~0u, v, j);
          if ((lane & 7) == 0) *reinterpret_cast<uint32_t *>((uint8_t *)a.p.out + (int64_t)(w.row + r) * a.p.ldo + (w.n0 + c) / 2) = fp4_eight(eight);
          if (lane == 0)
            a.p.hs[((int64_t)w.slot * a.n_tiles + w.n0 / 128) * kScaleTile + (r & 31) * 16 + (r >> 5) * 4 + (i & 3)] = (uint8_t)byte;
        }
      } else {
        for (int i = threadIdx.x; i < mine * (BN / 4); i += kThreads4) {
          const int r = part + i / (BN / 4) * parts, c = i % (BN / 4) * 4;
          float v[4] = {0.0f, 0.0f, 0.0f, 0.0f};
          for (int q = 0; q < parts; ++q) {
            const float4 x = load_from_block(smem_u32(smem) + (r * S::kSumPitch + c) * 4, q);
            v[0] += x.x, v[1] += x.y, v[2] += x.z, v[3] += x.w;
          }
          TO *out = (TO *)a.p.out + (int64_t)(w.row + r) * a.p.ldo + w.n0 + c;
#pragma unroll
          for (int j = 0; j < 4; ++j)
            if (w.n0 + c + j < a.p.n) out[j] = from_f32<TO>(v[j]);
        }
      }
    }
    cluster_meet();  // no block leaves while its sums are read
  }
  tc_fence_before();
  __syncthreads();
  if constexpr (PAIR) cluster_meet();  // neither block's memory is used by the other one any more
  tc_fence_after();
  if (warp == 2) tmem_give<PAIR>(tmem);
  if (threadIdx.x == 0 && *given_up) *a.error = 1;
}

// ---- host ------------------------------------------------------------------------------------

enum { kAlone, kSplit, kPair };
// Tiles of `rows` rows, at most: every group may have one that is not full, and none more than it has rows.  (Offsets that make
// groups overlap can ask for more; blocks that go on from tile to tile take those too, clusters that take one each do not reach them.)
int64_t row_tiles(const Product4Args &p, int rows) { return p.offsets ? std::min(p.m, ceil_div(p.m, rows) + p.groups - 1) : ceil_div(p.m, rows); }
template <int BN, bool SWIGLU, typename TO, int HOW = kAlone>
int run_tiles4(const Product4Args &p, cudaStream_t st, int parts = 1) {
  constexpr bool SPLIT = HOW == kSplit, PAIR = HOW == kPair;
  constexpr int kRows = PAIR ? 256 : 128;
  using S = Shape4<BN, !SWIGLU && !SPLIT && sizeof(TO) == 2, PAIR>;
  Tile4Args a = {};
  a.p = p;
  const int64_t bytes = ceil_div(p.k, 2), runs = ceil_div(p.k, 128), tiles_n = ceil_div(p.n, 128), matrices = (int64_t)p.groups * (SWIGLU ? 2 : 1);
  a.stages = (int)ceil_div(p.k, 256);
  a.n_tiles = (int)ceil_div(p.n, SWIGLU ? BN / 2 : BN);
  a.most_rows = (INT32_MAX - (1 << 20)) / a.n_tiles;
  a.error = error_word();
  if (!a.error) return TUNA_ERR_CUDA;
  CUtensorMap ma, mb, msa, msb, mo;
  a.box_a = p.offsets ? 32 : 128;
  if (const int rc = make_map(&ma, 2, p.a, bytes, p.m, 1, p.lda, a.box_a)) return rc;
  if (const int rc = make_map(&mb, 3, p.b, bytes, p.n, matrices, p.ldb, SWIGLU ? 128 : S::kRowsB)) return rc;
  if (const int rc = make_scale_map(&msa, p.sa, runs, fp4_slots(p.m, p.offsets ? p.groups : 0), 1)) return rc;
  if (const int rc = make_scale_map(&msb, p.sb, runs, matrices * tiles_n, SWIGLU ? 1 : BN / 128)) return rc;
  mo = ma;
  a.store_tiles = S::kOutBytes && aligned(p.out, 16) && p.ldo % 8 == 0 && p.n % 8 == 0;  // (a tensor copy's rows end on 16 bytes)
  if (a.store_tiles)
    if (const int rc = make_out_map(&mo, p.out, p.n, p.m, p.ldo, S::kOutCols * 2)) return rc;
  static bool set[64] = {};
  auto kernel = tuna_product4_kernel<BN, SWIGLU, SPLIT, PAIR, TO>;
  if (const int rc = allow_smem(kernel, S::kSmem, set)) return rc;
  const int64_t most = row_tiles(p, kRows) * a.n_tiles;
  if (PAIR)
    return launch_cluster(kernel, dim3((unsigned)std::min<int64_t>(most, std::max(sm_count() / 2, 1)) * 2), 2, kThreads4, S::kSmem, st, false, ma, mb, msa, msb, mo, a);
  if (SPLIT) return launch_cluster(kernel, dim3((unsigned)(most * parts)), parts, kThreads4, S::kSmem, st, false, ma, mb, msa, msb, mo, a);
  return launch(kernel, dim3((unsigned)std::min<int64_t>(most, sm_count())), kThreads4, S::kSmem, st, false, ma, mb, msa, msb, mo, a);
}

size_t dtype_size(int dtype) { return dtype == TUNA_DTYPE_F32 ? 4 : dtype == TUNA_DTYPE_BF16 ? 2 : 0; }

}  // namespace

int launch_product4(const Product4Args &p, cudaStream_t st) {
  // Pairs of blocks where they have six rounds of tiles or more, and groups four tiles of rows on average.  (Pairs and blocks alone, us: 8192 x 8192 x
  // 4096 101.6 and 105.7, 8192 x 4096 x 2048 33.1 and 34.2, 16384 x 4096 x 512 28.7 and 29.6; with fewer rounds 4096 x 4096 x 2048 20.4 and 19.8, 3000^3 19.6
  // and 17.7.  64 experts of 4096 x 2048, both products and what is around them, rows of an expert 512: 561 and 524, 1024: 964 and 961, 1536: 1406
  // and 1430.)
  const int64_t pairs = std::max(sm_count() / 2, 1), tiles = ceil_div(p.m, 256) * ceil_div(p.n, p.swiglu ? 128 : 256);
  if (tiles >= 6 * pairs && (!p.offsets || p.m >= 1024 * (int64_t)p.groups)) {
    if (p.swiglu) return run_tiles4<256, true, uint8_t, kPair>(p, st);
    return p.out_f32 ? run_tiles4<256, false, float, kPair>(p, st) : run_tiles4<256, false, __nv_bfloat16, kPair>(p, st);
  }
  const int64_t rows = row_tiles(p, 128), stages = ceil_div(p.k, 256);
  const int64_t wide = rows * ceil_div(p.n, 256), narrow = rows * ceil_div(p.n, 128);
  // Tiles of 256 columns where they take fewer rounds.  (Of 256 and of 128, us: 1024 x 4096 x 4096, one round and two, 10.5 and 16.2; 777 x 2000 x
  // 2896, one of either, 11.7 and 8.9; 1024 x 4736 x 4096, two of either, 16.3 and 16.5; 64 groups of 4096 x 2048 with 16 rows each, 7 and 14: 49 and 53.)
  if (!p.swiglu && ceil_div(wide, sm_count()) < ceil_div(narrow, sm_count()))
    return p.out_f32 ? run_tiles4<256, false, float>(p, st) : run_tiles4<256, false, __nv_bfloat16>(p, st);
  // Few tiles: a cluster shares each, while its blocks find room at once and every one is spared six stages, which pay for the meeting
  // (and every one has some).  (narrow: with SwiGLU too, whose tiles have 128 columns of the result.  One row in fours, twos, alone, us: 4096 x
  // 4096 6.7, 6.6, 8.2; 2048 x 2048 4.6, 5.2, 5.5; 512 x 8192 6.1, 8.2, 13.1; 4096 x 1024 4.6, 4.6, 4.3; 128 rows, 2048 x 1536 6.8, 6.8, 5.3.)
  int parts = 4;
  while (parts > 1 && (narrow * parts > 128 || stages - stages / parts < 6 || stages < 2 * parts)) parts /= 2;
  if (p.swiglu) return parts > 1 ? run_tiles4<256, true, uint8_t, kSplit>(p, st, parts) : run_tiles4<256, true, uint8_t>(p, st);
  if (parts > 1) return p.out_f32 ? run_tiles4<128, false, float, kSplit>(p, st, parts) : run_tiles4<128, false, __nv_bfloat16, kSplit>(p, st, parts);
  return p.out_f32 ? run_tiles4<128, false, float>(p, st) : run_tiles4<128, false, __nv_bfloat16>(p, st);
}

// The grid over quarters of row tiles and strips of 256 columns: as many strips a block as leave `blocks` of them a multiprocessor, so
// that what finds its rows is shared, and what is ahead is on its way (2^24 columns are 2^16 strips, of which a block takes several then).
static dim3 strips_grid(int64_t tiles, int cols, int blocks, int &strips) {
  const int64_t quarters = tiles * 4, all = ceil_div(cols, 256);
  strips = (int)std::max<int64_t>(1, std::min<int64_t>(all, quarters * all / (blocks * sm_count())));
  return dim3((unsigned)quarters, (unsigned)ceil_div(all, strips));
}

template <typename T>
static int run_quantize_rows(Quant4Args a, int64_t tiles, cudaStream_t st) {
  const dim3 grid = strips_grid(tiles, a.cols, 6, a.strips);
  if (!aligned(a.x, 16) || a.ldx * sizeof(T) % 16) return launch(tuna_quantize4_rows_kernel<T, false>, grid, 256, 0, st, false, a);
  static bool set[64] = {};
  constexpr size_t smem = ahead<T>() * 4 * Eight<T>::kWords * 256 * 16;
  if (const int rc = allow_smem(tuna_quantize4_rows_kernel<T, true>, smem, set)) return rc;
  return launch(tuna_quantize4_rows_kernel<T, true>, grid, 256, smem, st, false, a);
}

int launch_quantize4_rows(const void *x, bool f32, int64_t rows, int cols, int64_t ldx, const int64_t *gather, int64_t in_rows, int groups,
                          const int64_t *offsets, void *q, int64_t ldq, uint8_t *scale, cudaStream_t st) {
  Quant4Args a = {};
  a.x = x, a.rows = rows, a.cols = cols, a.ldx = ldx, a.gather = gather, a.in_rows = in_rows, a.groups = groups, a.offsets = offsets;
  a.q = (uint8_t *)q, a.ldq = ldq, a.scale = scale, a.runs = (int)ceil_div(cols, 128);
  // A few rows a group.  (64 groups, 4096 columns of bf16, us: 16 rows a group 5.6 and 13.6 in tiles, 32 rows 10.0 and 14.3, 64 rows 18 and 14.4.)
  if (offsets && rows < 48 * (int64_t)groups) {
    const dim3 grid((unsigned)rows, (unsigned)ceil_div(cols, 2048));
    return f32 ? launch(tuna_quantize4_few_kernel<float>, grid, 256, 0, st, false, a) : launch(tuna_quantize4_few_kernel<__nv_bfloat16>, grid, 256, 0, st, false, a);
  }
  const int64_t tiles = fp4_slots(rows, offsets ? groups : 0);
  return f32 ? run_quantize_rows<float>(a, tiles, st) : run_quantize_rows<__nv_bfloat16>(a, tiles, st);
}

bool places_quantize4(int64_t choices) { return choices <= kPlaceMost; }
int launch_place_quantize4(const void *x, int64_t tokens, int cols, int64_t ldx, const int32_t *ids, int k, int experts, void *q, int64_t ldq,
                           uint8_t *scale, int64_t *first, int64_t *pos, cudaStream_t st) {
  Place4Args a = {};
  a.quant.x = x, a.quant.cols = cols, a.quant.ldx = ldx, a.quant.q = (uint8_t *)q, a.quant.ldq = ldq, a.quant.scale = scale;
  a.quant.runs = (int)ceil_div(cols, 128);
  a.ids = ids, a.n = (int)(tokens * k), a.k = k, a.experts = experts, a.first = first, a.pos = pos;
  return launch(tuna_place_quantize4_kernel, dim3((unsigned)a.n, (unsigned)ceil_div(cols, 2048)), 256, 0, st, false, a);
}

}  // namespace tuna_ops

using namespace tuna_ops;

static int check_groups4(int64_t rows, int cols, int groups, const int64_t *offsets) {
  if (groups < 0 || (groups > 0) != (offsets != nullptr)) return TUNA_ERR_INVALID_ARG;
  if (groups > TUNA_MOE_MAX_EXPERTS || cols > kMaxDim || rows > INT32_MAX - 256) return TUNA_ERR_RANGE;
  return TUNA_OK;
}

extern "C" {

int tuna_fp4_scale_tiles(int64_t rows, int groups, int64_t *tiles) {
  if (!tiles || rows < 0 || groups < 0) return TUNA_ERR_INVALID_ARG;
  *tiles = fp4_slots(rows, groups);
  return TUNA_OK;
}

int tuna_fp4_quantize(const void *x, int dtype, int64_t rows, int cols, int64_t ldx, int layout, int groups, const int64_t *offsets, void *q,
                      int64_t ldq, void *scale, void *stream) {
  const size_t size = dtype_size(dtype);
  if (!size || rows < 0 || cols < 0 || ldx < cols || (layout != TUNA_FP4_ROWS && layout != TUNA_FP4_COLUMNS)) return TUNA_ERR_INVALID_ARG;
  if (layout == TUNA_FP4_COLUMNS && offsets) return TUNA_ERR_INVALID_ARG;
  if (const int rc = check_groups4(rows, cols, groups, offsets)) return rc;
  if (ldq % 16 != 0 || ldq < ceil_div(layout == TUNA_FP4_COLUMNS ? rows : cols, 2)) return TUNA_ERR_INVALID_ARG;
  if (layout == TUNA_FP4_COLUMNS && (rows > kMaxDim || ceil_div(rows, 128) * ceil_div(cols, 128) > INT32_MAX)) return TUNA_ERR_RANGE;
  if (rows == 0 || cols == 0) return TUNA_OK;
  if (!x || !q || !scale || !aligned(x, size) || !aligned(q, 16) || !aligned(scale, 16) || !aligned(offsets, 8)) return TUNA_ERR_INVALID_ARG;
  cudaStream_t st = (cudaStream_t)stream;
  const bool f32 = dtype == TUNA_DTYPE_F32;
  if (layout == TUNA_FP4_ROWS) return launch_quantize4_rows(x, f32, rows, cols, ldx, nullptr, rows, groups, offsets, q, ldq, (uint8_t *)scale, st);
  Quant4Args a = {};
  a.x = x, a.rows = rows, a.cols = cols, a.ldx = ldx, a.q = (uint8_t *)q, a.ldq = ldq, a.scale = (uint8_t *)scale, a.runs = (int)ceil_div(rows, 128);
  const dim3 grid((unsigned)(ceil_div(rows, 128) * ceil_div(cols, 128)));
  static bool set[2][64] = {};
  if (f32) {
    if (const int rc = allow_smem(tuna_quantize4_columns_kernel<float>, Turn<float>::kSmem, set[0])) return rc;
    return launch(tuna_quantize4_columns_kernel<float>, grid, 256, Turn<float>::kSmem, st, false, a);
  }
  if (const int rc = allow_smem(tuna_quantize4_columns_kernel<__nv_bfloat16>, Turn<__nv_bfloat16>::kSmem, set[1])) return rc;
  return launch(tuna_quantize4_columns_kernel<__nv_bfloat16>, grid, 256, Turn<__nv_bfloat16>::kSmem, st, false, a);
}

int tuna_fp4_dequantize(const void *q, int64_t ldq, const void *scale, int64_t rows, int cols, int groups, const int64_t *offsets, void *out,
                        int out_dtype, int64_t ldo, void *stream) {
  const size_t size = dtype_size(out_dtype);
  if (!size || rows < 0 || cols < 0 || ldq < ceil_div(cols, 2) || ldo < cols) return TUNA_ERR_INVALID_ARG;
  if (const int rc = check_groups4(rows, cols, groups, offsets)) return rc;
  if (rows == 0 || cols == 0) return TUNA_OK;
  if (!q || !scale || !out || !aligned(scale, 16) || !aligned(out, size) || !aligned(offsets, 8)) return TUNA_ERR_INVALID_ARG;
  Quant4Args a = {};
  a.rows = rows, a.cols = cols, a.groups = groups, a.offsets = offsets, a.q = (uint8_t *)q, a.ldq = ldq, a.scale = (uint8_t *)scale;
  a.runs = (int)ceil_div(cols, 128);
  const dim3 grid = strips_grid(fp4_slots(rows, groups), cols, 8, a.strips);
  cudaStream_t st = (cudaStream_t)stream;
  const bool whole = aligned(q, 4) && ldq % 4 == 0 && aligned(out, 8 * size) && ldo % 8 == 0;
  if (out_dtype == TUNA_DTYPE_F32)
    return launch(whole ? tuna_dequantize4_kernel<float, true> : tuna_dequantize4_kernel<float, false>, grid, 256, 0, st, false, a, (float *)out, ldo);
  return launch(whole ? tuna_dequantize4_kernel<__nv_bfloat16, true> : tuna_dequantize4_kernel<__nv_bfloat16, false>, grid, 256, 0, st, false, a, (__nv_bfloat16 *)out, ldo);
}

int tuna_fp4_align(const void *q, int64_t ldq, int64_t rows, int64_t bytes, void *out, int64_t ldo, void *stream) {
  if (rows < 0 || bytes < 0 || ldq < bytes || ldo < bytes || ldo % 16) return TUNA_ERR_INVALID_ARG;
  if (rows > INT32_MAX || bytes > kMaxDim) return TUNA_ERR_RANGE;
  if (rows == 0 || bytes == 0) return TUNA_OK;
  if (!q || !out || !aligned(out, 16)) return TUNA_ERR_INVALID_ARG;
  const int64_t blocks = std::min<int64_t>(ceil_div(rows * ceil_div(bytes, 16), 256), 16 * sm_count());
  return launch(tuna_align4_kernel, dim3((unsigned)blocks), 256, 0, (cudaStream_t)stream, false, (const uint8_t *)q, ldq, rows, bytes, (uint8_t *)out, ldo);
}

int tuna_fp4_matmul(const void *a, const void *a_scale, int64_t m, int64_t lda, const void *b, const void *b_scale, int n, int64_t ldb, int k, int groups,
                    const int64_t *offsets, void *out, int out_dtype, int64_t ldo, void *stream) {
  const size_t so = dtype_size(out_dtype);
  if (!so || m < 0 || n < 0 || k < 0 || k % 2 || lda < k / 2 || ldb < k / 2 || ldo < n || lda % 16 || ldb % 16) return TUNA_ERR_INVALID_ARG;
  if (const int rc = check_groups4(m, n, groups, offsets)) return rc;
  if (k > kMaxDim) return TUNA_ERR_RANGE;
  const int matrices = std::max(groups, 1);
  if (matrices * (ceil_div(m, 128) + 1) * ceil_div(n, 128) > INT32_MAX) return TUNA_ERR_RANGE;  // tiles, whatever the offsets hold
  if (m == 0 || n == 0) return TUNA_OK;
  if (!out || !aligned(out, so) || !aligned(offsets, 8)) return TUNA_ERR_INVALID_ARG;
  cudaStream_t st = (cudaStream_t)stream;
  if (k == 0) return launch_empty_sums(out, out_dtype == TUNA_DTYPE_F32, m, n, ldo, groups, offsets, st);
  if (!a || !b || !a_scale || !b_scale || !aligned(a, 16) || !aligned(b, 16) || !aligned(a_scale, 16) || !aligned(b_scale, 16))
    return TUNA_ERR_INVALID_ARG;
  Product4Args p = {};
  p.a = a, p.b = b, p.sa = (const uint8_t *)a_scale, p.sb = (const uint8_t *)b_scale, p.m = m, p.n = n, p.k = k, p.lda = lda, p.ldb = ldb, p.ldo = ldo;
  p.groups = matrices, p.offsets = offsets, p.out = out, p.out_f32 = out_dtype == TUNA_DTYPE_F32;
  return launch_product4(p, st);
}

}  // extern "C"
