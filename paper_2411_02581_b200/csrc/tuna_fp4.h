// 4-bit microscaled operands and their product as the other operators call them (tuna_fp4.cu).
#ifndef TUNA_FP4_H
#define TUNA_FP4_H

#include <cuda_runtime.h>
#include <stdint.h>

namespace tuna_ops {

constexpr int kScaleTile = 512;  // bytes: the scales of 128 rows and 4 blocks of 32 columns, [32][4 rows a step of 32][4 blocks]

// Row tiles of 128 that the scales of `rows` rows in `groups` groups (0: ungrouped) take: group g's begin at
// offsets[g] / 128 + g, which leaves every group whole tiles of its own.
inline int64_t fp4_slots(int64_t rows, int groups) { return groups ? rows / 128 + groups : (rows + 127) / 128; }

// One product y = a b^T.
struct Product4Args {
  const void *a, *b;        // 4-bit values, two a byte, K-major
  const uint8_t *sa, *sb;   // sa [slots of a][runs][512]; sb [groups (x 2 with swiglu)][n tiles][runs][512], runs of 128 along k
  int64_t m;                // rows of a
  int n, k;                 // k: columns that are read, even
  int64_t lda, ldb, ldo;    // pitches: bytes of a and b (the matrices of b are n * ldb apart), elements of out
  int groups;
  const int64_t *offsets;   // device, groups + 1, or nullptr: one group of all rows
  void *out;
  int out_f32;              // 0: bf16
  // gate and up product with SwiGLU: b holds 2 matrices of n rows a group; out: 4-bit rows of pitch ldo bytes (a multiple
  // of 64 that covers n), hs their scales [slots of a][runs of n][512]
  bool swiglu;
  uint8_t *hs;
};
int launch_product4(const Product4Args &p, cudaStream_t st);

// Rows of x (bf16 or f32), optionally taken through `gather` out of in_rows ones, to 4 bits with blocks along the row;
// with offsets (device, groups + 1) the scales lie in the groups' own tiles.
int launch_quantize4_rows(const void *x, bool f32, int64_t rows, int cols, int64_t ldx, const int64_t *gather, int64_t in_rows, int groups,
                          const int64_t *offsets, void *q, int64_t ldq, uint8_t *scale, cudaStream_t st);

// The same for the choices of a few tokens (as many as places_quantize4 allows), bf16, put in their experts' order on the way: `first`
// receives the experts' first rows (experts + 1), `pos` each choice's row, -1 where there is no such expert.
bool places_quantize4(int64_t choices);
int launch_place_quantize4(const void *x, int64_t tokens, int cols, int64_t ldx, const int32_t *ids, int k, int experts, void *q, int64_t ldq,
                           uint8_t *scale, int64_t *first, int64_t *pos, cudaStream_t st);

}  // namespace tuna_ops
#endif
