// Matrix products in 8-bit floating point with a 32-bit scale for each block of 128
// along the contracted axis, dense and grouped by expert, and the quantisation of their
// operands.
//
//   y[m,n] = sum_b sa[b,m] sb[n or n/128,b] (sum_{k in block b} a[m,k] b[n,k])
//
// The inner sum is one accumulation of the tensor cores (exact products of e4m3 values,
// 32-bit sums); the outer one multiplies by arbitrary 32-bit scales, which the tensor
// cores cannot do, so every block's accumulator goes through registers: see the product
// kernel.
#include <algorithm>
#include <mutex>

#include "tuna_fp8.h"
#include "tuna_ops.cuh"

namespace tuna_ops {
namespace {

// ---- quantisation --------------------------------------------------------------------------
//
// Bound by memory: two bytes (bf16) read and one written a value.  Blocks along the row: 8
// lanes a block of 128 columns, 16 columns a lane (two 16-byte loads of bf16, one 16-byte
// store), so a warp takes 512 columns of a row and the largest magnitude costs three shuffles.
struct QuantArgs {
  const void *x;
  int64_t rows, ldx, ldq, in_rows;
  int cols, vec;
  const int64_t *gather;
  uint8_t *q;
  float *scale;
};
// A block of threads takes 16 rows x 512 columns, a warp two of the rows, whose loads it has in
// flight together.
constexpr int kQuantRows = 16;
template <typename T>
__global__ void __launch_bounds__(256) tuna_quantize_rows_kernel(QuantArgs a) {
  wait_previous();
  allow_next();
  const int lane = threadIdx.x & 31, c = (int)blockIdx.y * 512 + lane * 16;
  const int64_t r0 = (int64_t)blockIdx.x * kQuantRows + (threadIdx.x >> 5) * 2;
  Eight<T> x[2][2];
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    const int64_t r = r0 + i;
    const int64_t from = r >= a.rows ? -1 : a.gather ? __ldg(a.gather + r) : r;
    const bool there = from >= 0 && from < a.in_rows;
    const T *p = reinterpret_cast<const T *>(a.x) + (there ? from : 0) * a.ldx + c;
    x[i][0].load(p, a.vec, there ? a.cols - c : 0), x[i][1].load(p + 8, a.vec, there ? a.cols - c - 8 : 0);
  }
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    const int64_t r = r0 + i;
    uint32_t amax = Eight<T>::top_bits(x[i][1].top(x[i][0].top(0)));
#pragma unroll
    for (int d = 1; d < 8; d <<= 1) amax = max(amax, __shfl_xor_sync(~0u, amax, d));
    if (r >= a.rows || c >= a.cols) continue;
    const float s = fp8_scale(amax);
    float v[16];
    x[i][0].values(v), x[i][1].values(v + 8);
    *reinterpret_cast<uint4 *>(a.q + r * a.ldq + c) = fp8_sixteen(v, divisor(s));
    if (lane % 8 == 0) a.scale[(int64_t)(c / 128) * a.rows + r] = s;
  }
}

// Blocks that span rows: a block of threads takes a 128 x 128 tile, 8 columns of 8 rows a thread.
// As they are (kTiles), the tile never leaves the registers.  Turned (kColumns, kTilesT), it goes
// through shared memory in its own type; a thread then has 32 rows of two columns, read as pairs.
enum { kColumns = 1, kTiles = 2, kTilesT = 3 };
template <typename T>
struct TileShape {
  static constexpr int kPitch = 128 + 16 / sizeof(T);  // rows stay on 16-byte boundaries, four banks apart
  static constexpr size_t kSmem = 128 * kPitch * sizeof(T);
};
template <int MODE, typename T>
__global__ void __launch_bounds__(256) tuna_quantize_tile_kernel(QuantArgs a) {
  extern __shared__ __align__(16) char tile_raw[];
  T *tile = reinterpret_cast<T *>(tile_raw);
  constexpr int kPitch = TileShape<T>::kPitch;
  __shared__ uint32_t part[4][128];
  wait_previous();
  allow_next();
  const int col_tiles = (a.cols + 127) / 128;
  const int64_t r0 = (int64_t)(blockIdx.x / col_tiles) * 128;
  const int c0 = (int)(blockIdx.x % col_tiles) * 128;
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const int mine = tid >> 4, c = (tid & 15) * 8;  // rows mine, mine + 16, ...; columns c .. c + 7
  Eight<T> x[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const int64_t r = r0 + mine + i * 16;
    x[i].load(reinterpret_cast<const T *>(a.x) + r * a.ldx + c0 + c, a.vec, r < a.rows ? a.cols - c0 - c : 0);
  }
  uint32_t amax = 0;
  if (MODE != kColumns) {
#pragma unroll
    for (int i = 0; i < 8; ++i) amax = x[i].top(amax);
    amax = Eight<T>::top_bits(amax);
#pragma unroll
    for (int d = 1; d < 32; d <<= 1) amax = max(amax, __shfl_xor_sync(~0u, amax, d));
    if (lane == 0) part[0][warp] = amax;
  }
  if (MODE != kTiles) {
#pragma unroll
    for (int i = 0; i < 8; ++i)
#pragma unroll
      for (int q = 0; q < Eight<T>::kWords; ++q) *reinterpret_cast<uint4 *>(tile + (mine + i * 16) * kPitch + c + q * (8 / Eight<T>::kWords)) = x[i].w[q];
  }
  __syncthreads();
  if (MODE != kColumns) {
#pragma unroll
    for (int w = 0; w < 8; ++w) amax = max(amax, part[0][w]);
  }
  if (MODE == kTiles) {
    const float s = fp8_scale(amax);
    const Divisor by = divisor(s);
    if (tid == 0) a.scale[(r0 / 128) * col_tiles + c0 / 128] = s;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const int64_t r = r0 + mine + i * 16;
      float v[8];
      x[i].values(v);
      uint32_t w[2];
      fp8_run<8>(v, by, w);
      // (rows are written up to the next multiple of 16 columns, with zeros)
      if (r < a.rows && c0 + c < (a.cols + 15) / 16 * 16) *reinterpret_cast<uint2 *>(a.q + r * a.ldq + c0 + c) = make_uint2(w[0], w[1]);
    }
    return;
  }
  const int two = (tid & 63) * 2, quarter = tid >> 6;  // columns two, two + 1; rows quarter * 32 ..
  float t[2][32];
  uint32_t top[2] = {0, 0};
#pragma unroll
  for (int r = 0; r < 32; ++r) {
    const T *p = tile + (quarter * 32 + r) * kPitch + two;
    if constexpr (sizeof(T) == 2) {
      const uint32_t u = *reinterpret_cast<const uint32_t *>(p);
      t[0][r] = __uint_as_float(u << 16), t[1][r] = __uint_as_float(u & 0xffff0000u);
    } else {
      const float2 u = *reinterpret_cast<const float2 *>(p);
      t[0][r] = u.x, t[1][r] = u.y;
    }
    if (MODE == kColumns) top[0] = max(top[0], abs_bits(t[0][r])), top[1] = max(top[1], abs_bits(t[1][r]));
  }
  if (MODE == kColumns) {
    part[quarter][two] = top[0], part[quarter][two + 1] = top[1];
    __syncthreads();
  }
#pragma unroll
  for (int e = 0; e < 2; ++e) {
    const int64_t out_row = c0 + two + e, out_col = r0 + quarter * 32;
    if (MODE == kColumns) amax = max(max(part[0][two + e], part[1][two + e]), max(part[2][two + e], part[3][two + e]));
    const float s = fp8_scale(amax);
    const Divisor by = divisor(s);
    if (MODE == kColumns) {
      if (quarter == 0 && out_row < a.cols) a.scale[(r0 / 128) * a.cols + out_row] = s;
    } else if (tid == 0 && e == 0) {
      a.scale[(c0 / 128) * ((a.rows + 127) / 128) + r0 / 128] = s;
    }
    if (out_row >= a.cols) continue;
    uint4 *q = reinterpret_cast<uint4 *>(a.q + out_row * a.ldq + out_col);
    if (out_col < a.rows) q[0] = fp8_sixteen(t[e], by);
    if (out_col + 16 < a.rows) q[1] = fp8_sixteen(t[e] + 16, by);
  }
}

// ---- the product -----------------------------------------------------------------------------
//
// A persistent block takes tiles of 128 x BN.  One warp copies 128 x 128 blocks of a and BN x
// 128 blocks of b into a ring of stages; one elected lane issues the four tensor-core steps of a
// block into one of two accumulators in tensor memory; sixteen warps read a finished accumulator
// back, multiply it by sa * sb and add it to the 32-bit sums they keep in registers (64 a
// thread at BN = 256), while the tensor cores fill the other one.  Two more warps fetch the scales,
// two blocks ahead, multiply them and leave one factor a row and 128 columns beside each
// accumulator, and a tile's place with its first one: the promotion warps have no registers for either.
//
// What bounds it is the round of an accumulator: steps and commit 940 cycles, promotion 500 (256 of
// packed multiply-adds at least), 200 back to the issuing lane; two accumulators fill the tensor
// memory, so a block of k takes some 800 cycles, its four steps alone 542 at the nominal rate.
// 8192 x 4096 x 4096: 121 us, 2270 TFLOP/s, in a burst; weight gradients (B_ROWS: a factor for
// every column too) 152.  Eight warps of 128 sums had no registers left to load ahead (30 us more); a
// lane that a branch picks moves every operand to uniform registers (6 us, with B_ROWS 20); scales
// four blocks ahead and 16 columns a read spill (8 us).
//
// With `swiglu` the 256 columns are 4 x (32 gate + 32 up) rows of the two matrices, so that the
// thread that holds a gate value holds its up value, and a tile is exactly one 128-block of the
// result: it leaves as e4m3 with its scale, and the 32-bit product never reaches memory.
struct TileArgs {
  ProductArgs p;
  int blocks;   // of k
  int n_tiles;
  int store_tiles;  // results leave through map_out
  int one_copy;     // SWIGLU: map_b brings gate and up rows together
  uint32_t most_rows;  // row tiles, at most: their number times n_tiles, and a step beyond, fits 31 bits
  int *error;
};

constexpr int kSumWarps = 16;   // promotion: four quarters of the columns x 128 rows
constexpr int kGemmThreads = 128 + kSumWarps * 32;
constexpr int kSumPitch = 132;  // floats: rows of sums that a cluster joins, on 16-byte boundaries and four banks apart
constexpr int kCopyRegs = 64, kSumRegs = 104;  // registers of a thread: copying and issuing warps, promotion
// columns that a promotion thread reads at a time, twice: with 16 the sums, both reads and the loop's own values do not fit
// the registers (8192 x 4096 x 4096: 126.8 us, 121.6 with 8; the experts of 8192 tokens x 2: 648 and 633 us)
constexpr int kRun = 8;
constexpr int kMaxGroups = TUNA_MOE_MAX_EXPERTS;
constexpr int kPlaces = 8;  // the scale warps are four tiles ahead of the slowest promotion warp at most

// STORES: bf16 results, which leave through shared memory
template <int BN, bool STORES>
struct Shape {
  static constexpr int kStages = BN == 256 ? (STORES ? 3 : 4) : (STORES ? 5 : 6);
  static constexpr int kStageBytes = 128 * 128 + BN * 128;
  static constexpr int kCols = BN / 4;  // accumulator columns of a thread
  static constexpr int kRowBytes = BN / 2;  // of bf16 results: a promotion warp's columns
  static constexpr int kOutBytes = STORES ? kSumWarps * 32 * kRowBytes : 0;  // each promotion warp's 32 rows of them, on their way out
  // stages, results, then the factors beside the two accumulators, the rows' largest magnitudes, the groups'
  // tile offsets, barriers and flags
  static constexpr size_t kSmem = 1024 + (size_t)kStages * kStageBytes + kOutBytes + 2 * 384 * 4 + 512 * 4 + (kMaxGroups + 8) * 4 + kPlaces * 16 + 256;
};

// Tile t of the walk: the group it is in (never walked backwards), its rows and columns.
// (32 bits: there are fewer rows than 2^31, and a result of 2^31 tiles does not fit the memory.)
struct Walk {
  int g = 0;
  int row, end;  // first row, end of the group's rows
  int n0;
};
__device__ __forceinline__ void walk_to(Walk &w, int t, const TileArgs &a, const int *tile_base, int bn) {
  while (t >= tile_base[w.g + 1] * a.n_tiles) ++w.g;
  const uint32_t mt = tile_base[w.g + 1] - tile_base[w.g], local = t - tile_base[w.g] * a.n_tiles;
  const uint32_t n = local / mt, m = local - n * mt;  // rows fastest: blocks that run together share b
  int64_t begin = 0, end = a.p.m;
  if (a.p.offsets) begin = max(a.p.offsets[w.g], (int64_t)0), end = min(a.p.offsets[w.g + 1], a.p.m);
  w.row = (int)begin + (int)m * 128, w.end = (int)end;
  w.n0 = n * bn;
}

//
// With SPLIT a cluster of 2 or 4 blocks shares one tile: each adds up a part of k, leaves its sums in
// its shared memory, and adds up the parts of some of the rows from all of them, in order of k.  For few
// rows there are fewer tiles than multiprocessors otherwise.
template <int BN, bool SWIGLU, bool B_ROWS, bool SPLIT, typename TO>
__global__ void __launch_bounds__(kGemmThreads, 1)
    tuna_product_kernel(const __grid_constant__ CUtensorMap map_a, const __grid_constant__ CUtensorMap map_b,
                        const __grid_constant__ CUtensorMap map_out, const TileArgs a) {
  using S = Shape<BN, !SWIGLU && !SPLIT && sizeof(TO) == 2>;
  extern __shared__ char smem_raw[];
  char *smem = smem_raw + ((1024 - (smem_u32(smem_raw) & 1023)) & 1023);
  // beside each accumulator: [2][128] factors of the rows for either half of the columns, or with
  // B_ROWS [128] scales of the rows, then [256] of the columns
  float *factors = (float *)(smem + (size_t)S::kStages * S::kStageBytes + S::kOutBytes);
  uint32_t *row_amax = (uint32_t *)(factors + 2 * 384);  // [4][128]
  int *tile_base = (int *)(row_amax + 512);
  uint64_t *bars = (uint64_t *)(tile_base + kMaxGroups + 8);
  int4 *places = (int4 *)(bars + 2 * S::kStages + 6 - (2 * S::kStages & 1));  // of the tiles: row, end, first column
  volatile int *given_up = (volatile int *)(places + kPlaces);
  volatile int *lost = given_up + 1;  // a warp of the promotion gave up
  uint32_t *tmem_at = (uint32_t *)(given_up + 2);
  const uint32_t full = smem_u32(bars), empty = full + 8 * S::kStages, done = empty + 8 * S::kStages, freed = done + 16, drained = freed + 16;
  const int warp = __shfl_sync(~0u, threadIdx.x >> 5, 0), lane = threadIdx.x & 31;  // (the same in all lanes, which the compiler then knows)

  if (threadIdx.x == 0) {
    for (int s = 0; s < S::kStages; ++s) mbar_init(full + 8 * s, 1), mbar_init(empty + 8 * s, 1);
    for (int s = 0; s < 2; ++s) mbar_init(done + 8 * s, 3), mbar_init(freed + 8 * s, kSumWarps);  // done: the tensor cores and two scale warps
    mbar_init(drained, 1);
    *given_up = 0, *lost = 0;
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
  }
  if (warp == 2) tmem_alloc(smem_u32(tmem_at), 2 * BN);
  wait_previous();
  allow_next();
  // Tiles of rows before each group.  Groups that lie apart never come near most_rows (their results would not fit the
  // memory); offsets that make them overlap may, and are cut there.
  if (warp == 1) {
    uint32_t sum = 0;
    for (int g0 = 0; g0 < a.p.groups; g0 += 32) {
      const int g = g0 + lane;
      int64_t rows = 0;
      auto cut = [&](int64_t row) { return min(max(row, (int64_t)0), a.p.m); };
      if (g < a.p.groups) rows = a.p.offsets ? cut(a.p.offsets[g + 1]) - cut(a.p.offsets[g]) : a.p.m;
      const uint32_t mt = rows > 0 ? (uint32_t)((rows + 127) / 128) : 0;  // (2^24 at most: 32 of them and most_rows fit 32 bits)
      uint32_t x = mt;
#pragma unroll
      for (int d = 1; d < 32; d <<= 1) {
        const uint32_t y = __shfl_up_sync(~0u, x, d);
        if (lane >= d) x += y;
      }
      if (g < a.p.groups) tile_base[g] = (int)min(sum + x - mt, a.most_rows);
      sum = min(sum + __shfl_sync(~0u, x, 31), a.most_rows);
    }
    if (lane == 0) tile_base[a.p.groups] = (int)sum;
  }
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem = __shfl_sync(~0u, *tmem_at, 0);
  const int tiles = tile_base[a.p.groups] * a.n_tiles;
  const int parts = SPLIT ? (int)cluster_size() : 1, part = SPLIT ? (int)cluster_rank() : 0;
  auto first = [&] { return (int)(SPLIT ? blockIdx.x / parts : blockIdx.x); };
  auto step = [&] { return (int)(SPLIT ? gridDim.x / parts : gridDim.x); };
  // this block's part of k
  const int kb_first = SPLIT ? (int)((int64_t)a.blocks * part / parts) : 0, blocks = SPLIT ? (int)((int64_t)a.blocks * (part + 1) / parts) - kb_first : a.blocks;

  if (warp < 4) {
    asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(kCopyRegs));
    if (warp == 0 && lane == 0) {
      // ---- copies
      int stage = 0, phase = 0;
      int64_t issued = 0;
      Walk w;
      bool ok = true;
      for (int t = first(); ok && t < tiles; t += step()) {
        walk_to(w, t, a, tile_base, SWIGLU ? BN / 2 : BN);
        for (int kb = 0; kb < blocks; ++kb) {
          if (!(ok = mbar_wait(empty + 8 * stage, phase ^ 1, given_up))) break;
          const uint32_t at = smem_u32(smem) + stage * S::kStageBytes, bar = full + 8 * stage;
          mbar_expect(bar, S::kStageBytes);
          const int col = (kb_first + kb) * 128;
          tma_load_2d(at, &map_a, col, w.row, bar);
          if (SWIGLU && a.one_copy) {
            tma_load_5d(at + 128 * 128, &map_b, col, 0, 0, w.n0 / 32, w.g, bar);
          } else if (SWIGLU) {
#pragma unroll
            for (int q = 0; q < 8; ++q)
              tma_load_3d(at + 128 * 128 + q * 32 * 128, &map_b, col, w.n0 + (q >> 1) * 32, w.g * 2 + (q & 1), bar);
          } else {
            tma_load_3d(at + 128 * 128, &map_b, col, w.n0, w.g, bar);
          }
          ++issued;
          if (++stage == S::kStages) stage = 0, phase ^= 1;
        }
      }
      // nothing may land in shared memory after the block has gone, whichever warp gives up: the last copies are waited for
      int never = 0;
      for (int64_t i = max((int64_t)0, issued - S::kStages); i < issued; ++i)
        mbar_wait(full + 8 * (int)(i % S::kStages), (uint32_t)((i / S::kStages) & 1), &never);
    } else if (warp == 1) {
      // ---- tensor cores: the whole warp goes along, one lane issues
      constexpr uint32_t idesc = (1u << 4) | ((uint32_t)(BN >> 3) << 17) | ((uint32_t)(128 >> 4) << 24);  // f32 sums of e4m3 products
      int stage = 0, phase = 0, buf = 0, buf_phase = 0;
      bool ok = true;
      for (int t = first(); ok && t < tiles; t += step()) {
        for (int kb = 0; kb < blocks; ++kb) {
          if (!(ok = __all_sync(~0u, mbar_wait(full + 8 * stage, phase, given_up) && mbar_wait(freed + 8 * buf, buf_phase ^ 1, given_up)))) break;
          tc_fence_after();
          const uint32_t at = smem_u32(smem) + stage * S::kStageBytes;
          const uint64_t da = tc_desc(at), db = tc_desc(at + 128 * 128);
          if (elect_one()) {
#pragma unroll
            for (int s = 0; s < 4; ++s) tc_mma_fp8(tmem + buf * BN, da + 2 * s, db + 2 * s, idesc, s > 0);  // 32 bytes along k
            tc_commit(empty + 8 * stage);
            tc_commit(done + 8 * buf);
          }
          __syncwarp();
          if (++stage == S::kStages) stage = 0, phase ^= 1;
          if (++buf == 2) buf = 0, buf_phase ^= 1;
        }
      }
      // and no step may be under way when tensor memory is freed
      int never = 0;
      if (elect_one()) tc_commit(drained);
      __syncwarp();
      mbar_wait(drained, 0, &never);
    } else if (warp >= 2) {
      // ---- scales: a lane has two rows of the tile, and with B_ROWS four columns
      constexpr int kAhead = 2, kVals = B_ROWS ? 6 : 4;
      const int i = threadIdx.x - 64, tiles_n = (a.p.n + 127) / 128;
      int buf = 0, buf_phase = 0;
      bool ok = true;
      Walk w;
      const float *sa0 = nullptr, *sa1 = nullptr, *sb0 = nullptr, *sb1 = nullptr;
      // the blocks that are fetched next: one run of kAhead ahead of those handed out, across tiles too
      int ahead_t = first(), ahead_kb = 0, ahead_place = 0;
      float next[kAhead][kVals];
      auto fetch = [&]() {
        if (ahead_t >= tiles) return;
        if (ahead_kb == 0) {
          walk_to(w, ahead_t, a, tile_base, SWIGLU ? BN / 2 : BN);
          // also for the warps that promote, which have no registers for it: `done` tells them
          if (threadIdx.x == 64) places[ahead_place++ % kPlaces] = make_int4(w.row, w.end, w.n0, 0);
          sa0 = a.p.sa + min(w.row + i, w.end - 1), sa1 = a.p.sa + min(w.row + i + 64, w.end - 1);
          if (SWIGLU) {
            sb0 = a.p.sb + ((int64_t)(w.g * 2) * tiles_n + w.n0 / 128) * a.blocks;
            sb1 = sb0 + (int64_t)tiles_n * a.blocks;
          } else if (!B_ROWS) {
            sb0 = a.p.sb + ((int64_t)w.g * tiles_n + w.n0 / 128) * a.blocks;
            sb1 = w.n0 / 128 + 1 < tiles_n ? sb0 + a.blocks : sb0;
          }
        }
#pragma unroll
        for (int j = 0; j < kAhead; ++j) {
          const int kb = kb_first + min(ahead_kb + j, blocks - 1);
          next[j][0] = __ldg(sa0 + (int64_t)kb * a.p.m), next[j][1] = __ldg(sa1 + (int64_t)kb * a.p.m);
          if (B_ROWS) {
#pragma unroll
            for (int q = 0; q < 4; ++q) next[j][2 + q] = __ldg(a.p.sb + (int64_t)kb * a.p.n + min(w.n0 + i + q * 64, a.p.n - 1));
          } else {
            next[j][2] = __ldg(sb0 + kb), next[j][3] = __ldg(sb1 + kb);
          }
        }
        ahead_kb += kAhead;
        if (ahead_kb >= blocks) ahead_kb = 0, ahead_t += step();
      };
      fetch();
      for (int t = first(); ok && t < tiles; t += step()) {
        for (int kb0 = 0; ok && kb0 < blocks; kb0 += kAhead) {
          float now[kAhead][kVals];
#pragma unroll
          for (int j = 0; j < kAhead; ++j)
#pragma unroll
            for (int q = 0; q < kVals; ++q) now[j][q] = next[j][q];
          fetch();
#pragma unroll
          for (int j = 0; j < kAhead; ++j) {
            if (kb0 + j >= blocks) break;
            ok = __all_sync(~0u, mbar_wait(freed + 8 * buf, buf_phase ^ 1, given_up));
            if (!ok) break;
            float *f = factors + buf * 384 + i;
            if (B_ROWS) {
              f[0] = now[j][0], f[64] = now[j][1];
#pragma unroll
              for (int q = 0; q < 4; ++q) f[128 + q * 64] = now[j][2 + q];
            } else {
              f[0] = now[j][0] * now[j][2], f[64] = now[j][1] * now[j][2];
              f[128] = now[j][0] * now[j][3], f[192] = now[j][1] * now[j][3];
            }
            __syncwarp();
            if (lane == 0) mbar_arrive(done + 8 * buf);
            if (++buf == 2) buf = 0, buf_phase ^= 1;
          }
        }
      }
    }
  } else {
    asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(kSumRegs));
    // ---- promotion and results: thread = one row, columns [quarter * kCols, ...) of the tile
    const int quarter = (warp - 4) >> 2, row_in = (warp & 3) * 32 + lane;
    const uint32_t from = tmem + ((uint32_t)((warp & 3) * 32) << 16) + quarter * S::kCols;
    // its factor: of its row and of its half of the columns (SWIGLU: gate, and up 128 places on)
    const uint32_t factor = smem_u32(factors) + (SWIGLU || B_ROWS ? row_in : (BN == 256 ? quarter >> 1 : 0) * 128 + row_in) * 4;
    int buf = 0, buf_phase = 0;
    bool ok = true;
    int place = 0;
    for (int t = first(); ok && t < tiles; t += step(), ++place) {
      uint64_t acc[S::kCols / 2];
#pragma unroll
      for (int i = 0; i < S::kCols / 2; ++i) acc[i] = 0;
      for (int kb = 0; kb < blocks; ++kb) {
        ok = __all_sync(~0u, mbar_wait(done + 8 * buf, buf_phase, given_up));  // (and the warp is whole for the loads)
        if (!ok) break;
        tc_fence_after();
        uint32_t v[2][kRun];
        tmem_load(from + buf * BN, v[0]);
        float s0, s1 = 0.0f;
        asm volatile("ld.shared.f32 %0, [%1];" : "=f"(s0) : "r"(factor + buf * 384 * 4) : "memory");
        if (SWIGLU) asm volatile("ld.shared.f32 %0, [%1];" : "=f"(s1) : "r"(factor + buf * 384 * 4 + 512) : "memory");
        const uint64_t p0 = pair(s0, s0), p1 = pair(s1, s1);
        const float *cs = factors + buf * 384 + 128 + quarter * S::kCols;
#pragma unroll
        for (int c = 0; c < S::kCols / kRun; ++c) {
          tmem_wait(v[c & 1]);
          if (c + 1 < S::kCols / kRun) {
            tmem_load(from + buf * BN + (c + 1) * kRun, v[(c + 1) & 1]);
          } else if (!B_ROWS) {  // everything is in registers, the factors too: the accumulator may be filled again
            asm volatile("" ::"f"(s0), "f"(s1));
            tc_fence_before();
            __syncwarp();
            if (lane == 0) mbar_arrive(freed + 8 * buf);
          }
          uint32_t(&x)[kRun] = v[c & 1];
#pragma unroll
          for (int i = 0; i < kRun / 2; i += 2) {
            uint64_t f = SWIGLU && c * kRun >= 32 ? p1 : p0, g = f;
            if (B_ROWS) {
              const float4 q = *reinterpret_cast<const float4 *>(cs + c * kRun + i * 2);
              f = mul2(p0, pair(q.x, q.y)), g = mul2(p0, pair(q.z, q.w));
            }
            acc[c * (kRun / 2) + i] = fma2(pair(x[2 * i], x[2 * i + 1]), f, acc[c * (kRun / 2) + i]);
            acc[c * (kRun / 2) + i + 1] = fma2(pair(x[2 * i + 2], x[2 * i + 3]), g, acc[c * (kRun / 2) + i + 1]);
          }
        }
        if (B_ROWS) {  // (the column scales have been read only now)
          tc_fence_before();
          __syncwarp();
          if (lane == 0) mbar_arrive(freed + 8 * buf);
        }
        if (++buf == 2) buf = 0, buf_phase ^= 1;
      }
      const int4 at = places[place % kPlaces];
      const int row = at.x + row_in, end = at.y, n0 = at.z;
      const bool there = row < end;
      if constexpr (SPLIT) {
        // the sums to shared memory, where the stages were: every step that read them is done
        float *red = (float *)smem + row_in * kSumPitch + quarter * S::kCols;
        if (ok && there) {
#pragma unroll
          for (int i = 0; i < S::kCols; i += 4) {
            float4 v;
            unpair(acc[i / 2], v.x, v.y), unpair(acc[i / 2 + 1], v.z, v.w);
            *reinterpret_cast<float4 *>(red + i) = v;
          }
        }
      } else if constexpr (!SWIGLU) {
        if (!ok) break;
        if constexpr (S::kOutBytes != 0) {
          // bf16 results go to shared memory, in 16-byte pieces swizzled by row.  32 whole rows leave from
          // there by a tensor copy, which runs on during the next tile (stored from registers, all blocks
          // at once, they cost 3 us a tile); rows that a group's end cuts, or that a tensor copy cannot
          // reach (a pitch that is no multiple of 16 bytes), leave in whole rows as the warp reads them back.
          constexpr int kPieces = S::kRowBytes / 16;
          auto place = [](int r, int piece) { return (uint32_t)(r * S::kRowBytes + (kPieces == 8 ? piece ^ (r & 7) : piece ^ ((r >> 1) & 3)) * 16); };
          const uint32_t to = smem_u32(smem) + S::kStages * S::kStageBytes + (warp - 4) * 32 * S::kRowBytes;
          const int row0 = row - lane;
          const int valid = max(0, min(32, end - row0)), c0 = n0 + quarter * S::kCols;
          if (lane == 0) tma_store_read();
          __syncwarp();
#pragma unroll
          for (int i = 0; i < kPieces; ++i) {
            float v[8];
#pragma unroll
            for (int j = 0; j < 4; ++j) unpair(acc[i * 4 + j], v[2 * j], v[2 * j + 1]);
            asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %4};" ::"r"(to + place(lane, i)), "r"(pack_bf16(v[0], v[1])),
                         "r"(pack_bf16(v[2], v[3])), "r"(pack_bf16(v[4], v[5])), "r"(pack_bf16(v[6], v[7]))
                         : "memory");
          }
          if (a.store_tiles && valid == 32) {
            asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
            __syncwarp();
            if (lane == 0 && c0 < a.p.n) tma_store_2d(&map_out, c0, row0, to);
          } else {
            __syncwarp();
            __nv_bfloat16 *out = (__nv_bfloat16 *)a.p.out + (int64_t)row0 * a.p.ldo + c0;
            if (a.store_tiles && c0 + S::kCols <= a.p.n) {
              for (int i = lane; i < valid * kPieces; i += 32) {
                const int r = i / kPieces, piece = i % kPieces;
                uint4 u;
                asm volatile("ld.shared.v4.b32 {%0, %1, %2, %3}, [%4];" : "=r"(u.x), "=r"(u.y), "=r"(u.z), "=r"(u.w) : "r"(to + place(r, piece)) : "memory");
                *reinterpret_cast<uint4 *>(out + r * a.p.ldo + piece * 8) = u;
              }
            } else {
              const int cols = min(S::kCols, a.p.n - c0);
              for (int r = 0; r < valid; ++r)
                for (int c = lane; c < cols; c += 32) {
                  uint16_t u;
                  asm volatile("ld.shared.b16 %0, [%1];" : "=h"(u) : "r"(to + place(r, c >> 3) + (c & 7) * 2) : "memory");
                  reinterpret_cast<uint16_t *>(out)[r * a.p.ldo + c] = u;
                }
            }
          }
          __syncwarp();
        } else if (there) {
          // 32-bit results, in whole 32-byte sectors
          static_assert(sizeof(TO) == 4);
          float *out = (float *)a.p.out + (int64_t)row * a.p.ldo;
          const int c0 = n0 + quarter * S::kCols;
          const bool vec = (((uintptr_t)a.p.out | (uint64_t)a.p.ldo * 4) & 31) == 0;
#pragma unroll
          for (int i = 0; i < S::kCols; i += 8) {
            float v[8];
#pragma unroll
            for (int j = 0; j < 4; ++j) unpair(acc[i / 2 + j], v[2 * j], v[2 * j + 1]);
            if (vec && c0 + i + 8 <= a.p.n) {
              uint32_t u[8];
#pragma unroll
              for (int j = 0; j < 8; ++j) u[j] = __float_as_uint(v[j]);
              store32(out + c0 + i, u);
            } else {
#pragma unroll
              for (int j = 0; j < 8; ++j)
                if (c0 + i + j < a.p.n) out[c0 + i + j] = v[j];
            }
          }
        }
      } else {
        if (!ok) *lost = 1;  // told before the barrier that the sixteen warps share: they leave together
        // columns 0..31: gate, 32..63: up of the same 32 places
        float h[32];
        uint32_t amax = 0;
#pragma unroll
        for (int i = 0; i < 16; ++i) {
          float g[2], u[2];
          unpair(acc[i], g[0], g[1]);
          unpair(acc[16 + i], u[0], u[1]);
#pragma unroll
          for (int j = 0; j < 2; ++j) {
            // (2^-20 of the value, which is rounded to 4 significant bits next; with the exact functions 501 tokens
            // x 2 of 64 experts of 2048 x 1408 take 127.8 us in place of 118.2)
            const float x = __fdividef(g[j], 1.0f + __expf(-g[j])) * u[j];
            h[2 * i + j] = x;
            amax = max(amax, abs_bits(x));
          }
        }
        row_amax[quarter * 128 + row_in] = amax;
        asm volatile("bar.sync 1, 512;" ::: "memory");
        if (*lost) break;
#pragma unroll
        for (int q = 0; q < 4; ++q) amax = max(amax, row_amax[q * 128 + row_in]);
        asm volatile("bar.sync 1, 512;" ::: "memory");  // before the next tile's values
        const float s = fp8_scale(amax);
        if (there) {
          if (quarter == 0) a.p.hs[(int64_t)(n0 / 128) * a.p.m + row] = s;
          const Divisor by = divisor(s);
          uint4 *out = (uint4 *)((uint8_t *)a.p.out + (int64_t)row * a.p.ldo + n0 + quarter * 32);  // (the pitch covers whole blocks)
          out[0] = fp8_sixteen(h, by), out[1] = fp8_sixteen(h + 16, by);
        }
      }
      __syncwarp();
    }
    if (S::kOutBytes && lane == 0) tma_store_done();
  }
  __syncwarp();
  if constexpr (SPLIT) {
    cluster_meet();
    if (first() < tiles && !*given_up) {
      Walk w;
      walk_to(w, first(), a, tile_base, BN);
      const int rows = min(128, w.end - w.row);
      for (int i = threadIdx.x; i < (rows - part + parts - 1) / parts * (BN / 4); i += kGemmThreads) {
        const int r = part + i / (BN / 4) * parts, c = i % (BN / 4) * 4;
        float v[4] = {0.0f, 0.0f, 0.0f, 0.0f};
        for (int q = 0; q < parts; ++q) {
          const float4 x = load_from_block(smem_u32(smem) + (r * kSumPitch + c) * 4, q);
          v[0] += x.x, v[1] += x.y, v[2] += x.z, v[3] += x.w;
        }
        TO *out = (TO *)a.p.out + (int64_t)(w.row + r) * a.p.ldo + w.n0 + c;
#pragma unroll
        for (int j = 0; j < 4; ++j)
          if (w.n0 + c + j < a.p.n) out[j] = from_f32<TO>(v[j]);
      }
    }
    cluster_meet();  // no block leaves while its sums are read
  }
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  if (warp == 2) tmem_free(tmem, 2 * BN);
  if (threadIdx.x == 0 && *given_up) *a.error = 1;
}

template <typename T>
__global__ void __launch_bounds__(256) tuna_empty_sums_kernel(T *out, int64_t m, int n, int64_t ldo, const int64_t *offsets) {
  wait_previous();
  allow_next();
  auto cut = [&](int g) { return min(max(offsets[g], (int64_t)0), m); };
  const int64_t end = cut(blockIdx.x + 1);
  for (int64_t r = cut(blockIdx.x) + blockIdx.y; r < end; r += gridDim.y)
    for (int c = threadIdx.x; c < n; c += 256) out[r * ldo + c] = from_f32<T>(0.0f);
}

// ---- host ------------------------------------------------------------------------------------

template <int BN, bool SWIGLU, bool B_ROWS, typename TO, bool SPLIT = false>
int run_tiles(const ProductArgs &p, cudaStream_t st, int parts = 1) {
  using S = Shape<BN, !SWIGLU && !SPLIT && sizeof(TO) == 2>;
  TileArgs a = {};
  a.p = p;
  a.blocks = (int)ceil_div(p.k, 128);
  a.n_tiles = (int)ceil_div(p.n, SWIGLU ? BN / 2 : BN);
  a.most_rows = (INT32_MAX - (1 << 20)) / a.n_tiles;
  a.error = error_word();
  if (!a.error) return TUNA_ERR_CUDA;
  CUtensorMap ma, mb, mo;
  if (const int rc = make_map(&ma, 2, p.a, p.k, p.m, 1, p.lda, 128)) return rc;
  // One copy of 32 KB for a block's gate and up rows, instead of eight of 4 KB (64 experts of 4096 x 2048,
  // 16384 rows, both products and what is around them: 649 us and 658, means of five).  Its 32-row steps
  // must not cross from one matrix into the next.
  a.one_copy = SWIGLU && p.n % 32 == 0;
  if (a.one_copy) {
    if (const int rc = make_gate_up_map(&mb, p.b, p.k, p.n, p.groups, p.ldb)) return rc;
  } else {
    if (const int rc = make_map(&mb, 3, p.b, p.k, p.n, (int64_t)p.groups * (SWIGLU ? 2 : 1), p.ldb, SWIGLU ? 32 : BN)) return rc;
  }
  mo = ma;
  a.store_tiles = S::kOutBytes && !SWIGLU && !p.out_f32 && aligned(p.out, 16) && p.ldo % 8 == 0 && p.n % 8 == 0;  // (a tensor copy's rows end on 16 bytes)
  if (a.store_tiles)
    if (const int rc = make_out_map(&mo, p.out, p.n, p.m, p.ldo, S::kRowBytes)) return rc;
  static bool set[64] = {}, fits = false;
  auto kernel = tuna_product_kernel<BN, SWIGLU, B_ROWS, SPLIT, TO>;
  if (!__atomic_load_n(&fits, __ATOMIC_ACQUIRE)) {
    // the warps' shares of registers (setmaxnreg) come out of what the block is launched with
    cudaFuncAttributes at;
    if (const int rc = note_cuda(cudaFuncGetAttributes(&at, kernel))) return rc;
    if ((at.numRegs + 7) / 8 * 8 * kGemmThreads < 128 * kCopyRegs + kSumWarps * 32 * kSumRegs) return TUNA_ERR_INTERNAL;
    __atomic_store_n(&fits, true, __ATOMIC_RELEASE);
  }
  if (const int rc = allow_smem(kernel, S::kSmem, set)) return rc;
  const int64_t most = (ceil_div(p.m, 128) + (p.offsets ? p.groups : 0)) * a.n_tiles;
  if (SPLIT) return launch_cluster(kernel, dim3((unsigned)(most * parts)), parts, kGemmThreads, S::kSmem, st, false, ma, mb, mo, a);
  return launch(kernel, dim3((unsigned)std::min<int64_t>(most, sm_count())), kGemmThreads, S::kSmem, st, false, ma, mb, mo, a);
}

size_t dtype_size(int dtype) { return dtype == TUNA_DTYPE_F32 ? 4 : dtype == TUNA_DTYPE_BF16 ? 2 : 0; }

template <int MODE, typename T>
int run_quantize_tiles(const QuantArgs &a, cudaStream_t st) {
  static bool set[64] = {};
  const size_t smem = MODE == kTiles ? 0 : TileShape<T>::kSmem;
  if (const int rc = allow_smem(tuna_quantize_tile_kernel<MODE, T>, smem, set)) return rc;
  return launch(tuna_quantize_tile_kernel<MODE, T>, dim3((unsigned)(ceil_div(a.rows, 128) * ceil_div(a.cols, 128))), 256, smem, st, false, a);
}

}  // namespace

using EncodeTiled = CUresult (*)(CUtensorMap *, CUtensorMapDataType, cuuint32_t, void *, const cuuint64_t *, const cuuint64_t *,
                                 const cuuint32_t *, const cuuint32_t *, CUtensorMapInterleave, CUtensorMapSwizzle, CUtensorMapL2promotion,
                                 CUtensorMapFloatOOBfill);
static EncodeTiled encoder() {
  static std::mutex m;
  static EncodeTiled fn = nullptr;
  std::lock_guard<std::mutex> lock(m);
  if (!fn) {
    void *p = nullptr;
    cudaDriverEntryPointQueryResult found;
    if (!note_cuda(cudaGetDriverEntryPointByVersion("cuTensorMapEncodeTiled", &p, 12000, cudaEnableDefault, &found)) &&
        found == cudaDriverEntryPointSuccess)
      fn = (EncodeTiled)p;
  }
  return fn;
}

// An e4m3 operand (or bf16 results): k contiguous, then rows, then matrices; boxes of 128 bytes x `box` rows.
int make_map(CUtensorMap *map, int rank, const void *p, int64_t k, int64_t rows, int64_t matrices, int64_t ld, int box, bool bf16) {
  EncodeTiled f = encoder();
  if (!f) return TUNA_ERR_CUDA;
  const cuuint64_t dims[3] = {(cuuint64_t)k, (cuuint64_t)rows, (cuuint64_t)matrices};
  const int size = bf16 ? 2 : 1;
  const cuuint64_t strides[2] = {(cuuint64_t)(ld * size), (cuuint64_t)(ld * size * rows)};
  const cuuint32_t boxes[3] = {(cuuint32_t)(128 / size), (cuuint32_t)box, 1}, ones[3] = {1, 1, 1};
  const CUresult r = f(map, bf16 ? CU_TENSOR_MAP_DATA_TYPE_BFLOAT16 : CU_TENSOR_MAP_DATA_TYPE_UINT8, (cuuint32_t)rank, const_cast<void *>(p), dims, strides, boxes, ones,
                       CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
                       CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE);
  return r == CUDA_SUCCESS ? TUNA_OK : note_cuda(cudaErrorInvalidValue);
}

int launch_empty_sums(void *out, bool f32, int64_t m, int n, int64_t ldo, int groups, const int64_t *offsets, cudaStream_t st) {
  const size_t size = f32 ? 4 : 2;
  if (!offsets) return note_cuda(cudaMemset2DAsync(out, ldo * size, 0, n * size, m, st));
  const dim3 grid((unsigned)groups, (unsigned)std::min<int64_t>(m, 64));
  if (f32) return launch(tuna_empty_sums_kernel<float>, grid, 256, 0, st, false, (float *)out, m, n, ldo, offsets);
  return launch(tuna_empty_sums_kernel<__nv_bfloat16>, grid, 256, 0, st, false, (__nv_bfloat16 *)out, m, n, ldo, offsets);
}

int make_out_map(CUtensorMap *map, void *p, int64_t cols, int64_t rows, int64_t ld, int row_bytes) {
  EncodeTiled f = encoder();
  if (!f) return TUNA_ERR_CUDA;
  const cuuint64_t dims[2] = {(cuuint64_t)cols, (cuuint64_t)rows};
  const cuuint64_t strides[1] = {(cuuint64_t)(ld * 2)};
  const cuuint32_t boxes[2] = {(cuuint32_t)(row_bytes / 2), 32}, ones[2] = {1, 1};
  const CUresult r = f(map, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 2, p, dims, strides, boxes, ones, CU_TENSOR_MAP_INTERLEAVE_NONE,
                       row_bytes == 128 ? CU_TENSOR_MAP_SWIZZLE_128B : CU_TENSOR_MAP_SWIZZLE_64B, CU_TENSOR_MAP_L2_PROMOTION_NONE,
                       CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE);
  return r == CUDA_SUCCESS ? TUNA_OK : note_cuda(cudaErrorInvalidValue);
}

int make_scale_map(CUtensorMap *map, const void *p, int64_t runs, int64_t tiles, int box) {
  EncodeTiled f = encoder();
  if (!f) return TUNA_ERR_CUDA;
  const cuuint64_t dims[3] = {128, (cuuint64_t)runs, (cuuint64_t)tiles};
  const cuuint64_t strides[2] = {512, (cuuint64_t)(512 * runs)};
  const cuuint32_t boxes[3] = {128, 2, (cuuint32_t)box}, ones[3] = {1, 1, 1};
  const CUresult r = f(map, CU_TENSOR_MAP_DATA_TYPE_UINT32, 3, const_cast<void *>(p), dims, strides, boxes, ones, CU_TENSOR_MAP_INTERLEAVE_NONE,
                       CU_TENSOR_MAP_SWIZZLE_NONE, CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE);
  return r == CUDA_SUCCESS ? TUNA_OK : note_cuda(cudaErrorInvalidValue);
}

int make_gate_up_map(CUtensorMap *map, const void *p, int64_t k, int64_t rows, int64_t groups, int64_t ld) {
  EncodeTiled f = encoder();
  if (!f) return TUNA_ERR_CUDA;
  const cuuint64_t dims[5] = {(cuuint64_t)k, 32, 2, (cuuint64_t)(rows / 32), (cuuint64_t)groups};
  const cuuint64_t strides[4] = {(cuuint64_t)ld, (cuuint64_t)(ld * rows), (cuuint64_t)(ld * 32), (cuuint64_t)(ld * rows * 2)};
  const cuuint32_t boxes[5] = {128, 32, 2, 4, 1}, ones[5] = {1, 1, 1, 1, 1};
  const CUresult r = f(map, CU_TENSOR_MAP_DATA_TYPE_UINT8, 5, const_cast<void *>(p), dims, strides, boxes, ones, CU_TENSOR_MAP_INTERLEAVE_NONE,
                       CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE);
  return r == CUDA_SUCCESS ? TUNA_OK : note_cuda(cudaErrorInvalidValue);
}

int launch_product(const ProductArgs &p, cudaStream_t st) {
  if (p.swiglu) return run_tiles<256, true, false, uint8_t>(p, st);
  const int64_t wide = (ceil_div(p.m, 128) + (p.offsets ? p.groups - 1 : 0)) * ceil_div(p.n, 256);
  if (p.b_rows) {
    if (p.out_f32) return run_tiles<256, false, true, float>(p, st);
    return run_tiles<256, false, true, __nv_bfloat16>(p, st);
  }
  // A round of tiles of 256 columns takes 6 / 5 of the time of one of 128 (the promotion is shared by as
  // many warps), so the rounds decide.  (k = 4096: 1024 x 4096 is 1 round or 2: 20.0 us against 28.2; 512 x
  // 4096 one of either: 18.9 against 16.5; 1024 x 4736 two of either: 32.4 against 28.4; 1280 x 4096 two or three: 32.6 against 37.9.)
  const int64_t narrow = (ceil_div(p.m, 128) + (p.offsets ? p.groups - 1 : 0)) * ceil_div(p.n, 128);
  if (6 * ceil_div(wide, sm_count()) < 5 * ceil_div(narrow, sm_count())) {
    if (p.out_f32) return run_tiles<256, false, false, float>(p, st);
    return run_tiles<256, false, false, __nv_bfloat16>(p, st);
  }
  if (!p.offsets) {
    // Few tiles: a cluster shares each, while its blocks find room at once and every one is spared 12 blocks
    // of k, which pay for the meeting.  (Rows 1 to 128, k = 4096: 10.1 us in fours, 12.1 in twos, 14.3 alone,
    // for 1024 to 4096 columns; clusters of 8 are no faster, and 16 of them are not resident together: 17.8 us.
    // 128 x 2048 x 2048: 8.6 in fours, 9.5 in twos, 9.0 alone.  128 x 4096 x 1024: 8.3 in fours, 6.7 alone.
    // 256 x 4096: 12.9 in twos and 15.5 alone at k = 4096, 9.9 and 9.3 at 2048.)
    const int64_t tiles = ceil_div(p.m, 128) * ceil_div(p.n, 128), blocks = ceil_div(p.k, 128);
    int parts = 4;
    while (parts > 1 && (tiles * parts > 128 || blocks - blocks / parts < 12)) parts /= 2;
    if (parts > 1) {
      if (p.out_f32) return run_tiles<128, false, false, float, true>(p, st, parts);
      return run_tiles<128, false, false, __nv_bfloat16, true>(p, st, parts);
    }
  }
  if (p.out_f32) return run_tiles<128, false, false, float>(p, st);
  return run_tiles<128, false, false, __nv_bfloat16>(p, st);
}

int launch_quantize_rows(const void *x, bool f32, int64_t rows, int cols, int64_t ldx, const int64_t *gather, int64_t in_rows,
                         void *q, int64_t ldq, float *scale, cudaStream_t st) {
  QuantArgs a = {};
  a.x = x, a.rows = rows, a.cols = cols, a.ldx = ldx, a.gather = gather, a.in_rows = in_rows, a.q = (uint8_t *)q, a.ldq = ldq, a.scale = scale;
  a.vec = aligned(x, 16) && ldx * (f32 ? 4 : 2) % 16 == 0;
  const dim3 grid((unsigned)ceil_div(rows, kQuantRows), (unsigned)ceil_div(cols, 512));
  return f32 ? launch(tuna_quantize_rows_kernel<float>, grid, 256, 0, st, false, a)
             : launch(tuna_quantize_rows_kernel<__nv_bfloat16>, grid, 256, 0, st, false, a);
}

}  // namespace tuna_ops

using namespace tuna_ops;

extern "C" {

int tuna_fp8_quantize(const void *x, int dtype, int64_t rows, int cols, int64_t ldx, int layout, void *q, int64_t ldq, float *scale,
                      void *stream) {
  const size_t size = dtype_size(dtype);
  if (!size || rows < 0 || cols < 0 || ldx < cols || layout < TUNA_FP8_ROWS || layout > TUNA_FP8_TILES_T) return TUNA_ERR_INVALID_ARG;
  const bool turned = layout == TUNA_FP8_COLUMNS || layout == TUNA_FP8_TILES_T;
  if (ldq < (turned ? rows : cols) || ldq % 16 != 0) return TUNA_ERR_INVALID_ARG;
  if (cols > kMaxDim || (turned && rows > kMaxDim) || rows > INT32_MAX || ceil_div(rows, 128) * ceil_div(cols, 128) > INT32_MAX) return TUNA_ERR_RANGE;
  if (rows == 0 || cols == 0) return TUNA_OK;
  if (!x || !q || !scale || !aligned(x, size) || !aligned(q, 16) || !aligned(scale, 4)) return TUNA_ERR_INVALID_ARG;
  cudaStream_t st = (cudaStream_t)stream;
  if (layout == TUNA_FP8_ROWS) return launch_quantize_rows(x, dtype == TUNA_DTYPE_F32, rows, cols, ldx, nullptr, rows, q, ldq, scale, st);
  QuantArgs a = {};
  a.x = x, a.rows = rows, a.cols = cols, a.ldx = ldx, a.q = (uint8_t *)q, a.ldq = ldq, a.scale = scale;
  a.vec = aligned(x, 16) && ldx * size % 16 == 0;
  const bool f32 = dtype == TUNA_DTYPE_F32;
  if (layout == TUNA_FP8_COLUMNS)
    return f32 ? run_quantize_tiles<kColumns, float>(a, st) : run_quantize_tiles<kColumns, __nv_bfloat16>(a, st);
  if (layout == TUNA_FP8_TILES) return f32 ? run_quantize_tiles<kTiles, float>(a, st) : run_quantize_tiles<kTiles, __nv_bfloat16>(a, st);
  return f32 ? run_quantize_tiles<kTilesT, float>(a, st) : run_quantize_tiles<kTilesT, __nv_bfloat16>(a, st);
}

int tuna_fp8_matmul(const void *a, const float *a_scale, int64_t m, int64_t lda, const void *b, const float *b_scale, int b_layout, int n,
                    int64_t ldb, int k, int groups, const int64_t *offsets, void *out, int out_dtype, int64_t ldo, void *stream) {
  const size_t so = dtype_size(out_dtype);
  if (!so || m < 0 || n < 0 || k < 0 || groups < 1 || lda < k || ldb < k || ldo < n || lda % 16 || ldb % 16) return TUNA_ERR_INVALID_ARG;
  if (b_layout != TUNA_FP8_TILES && b_layout != TUNA_FP8_ROWS) return TUNA_ERR_INVALID_ARG;
  if ((groups > 1 && !offsets) || (b_layout == TUNA_FP8_ROWS && offsets)) return TUNA_ERR_INVALID_ARG;
  if (groups > TUNA_MOE_MAX_EXPERTS || n > kMaxDim || k > kMaxDim || m > INT32_MAX - 256) return TUNA_ERR_RANGE;
  if (groups * (ceil_div(m, 128) + 1) * ceil_div(n, 128) > INT32_MAX) return TUNA_ERR_RANGE;  // tiles, whatever the offsets hold
  if (m == 0 || n == 0) return TUNA_OK;
  if (!out || !aligned(out, so) || !aligned(offsets, 8)) return TUNA_ERR_INVALID_ARG;
  cudaStream_t st = (cudaStream_t)stream;
  if (k == 0) return launch_empty_sums(out, out_dtype == TUNA_DTYPE_F32, m, n, ldo, groups, offsets, st);
  if (!a || !b || !a_scale || !b_scale || !aligned(a, 16) || !aligned(b, 16) || !aligned(a_scale, 4) || !aligned(b_scale, 4)) return TUNA_ERR_INVALID_ARG;
  ProductArgs p = {};
  p.a = a, p.b = b, p.sa = a_scale, p.sb = b_scale, p.m = m, p.n = n, p.k = k, p.lda = lda, p.ldb = ldb, p.ldo = ldo;
  p.groups = groups, p.offsets = offsets, p.b_rows = b_layout == TUNA_FP8_ROWS, p.out = out, p.out_f32 = out_dtype == TUNA_DTYPE_F32;
  return launch_product(p, st);
}

}  // extern "C"
