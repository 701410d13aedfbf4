// The 8-bit products as the other operators call them (tuna_fp8.cu).
#ifndef TUNA_FP8_H
#define TUNA_FP8_H

#include <cuda_runtime.h>
#include <stdint.h>

namespace tuna_ops {

// One product y = a b^T over blocks of 128 along k, a with a scale for each row and block.
struct ProductArgs {
  const void *a, *b;         // e4m3, K-major
  const float *sa, *sb;      // sa [blocks][a_rows]; sb [groups][n tiles][blocks], or [blocks][n] with b_rows
  int64_t m;                 // rows of a (the most that the groups can cover)
  int n, k;
  int64_t lda, ldb, ldo;     // pitches; ldb also separates the matrices of b: group g starts at g * n * ldb
  int groups;                // matrices of b
  const int64_t *offsets;    // device, groups + 1: the rows of each group; nullptr: one group, all rows
  bool b_rows;               // b has a scale for each row and block, like a
  void *out;
  int out_f32;               // 0: bf16
  // gate and up product with SwiGLU: b holds 2 matrices of n rows a group, out is e4m3 with hs [n blocks][m]
  bool swiglu;
  float *hs;
};
int launch_product(const ProductArgs &p, cudaStream_t st);

// Rows of x (bf16 or f32), optionally taken through `gather`, to e4m3 with 1 x 128 blocks; scale [blocks][rows].
int launch_quantize_rows(const void *x, bool f32, int64_t rows, int cols, int64_t ldx, const int64_t *gather, int64_t in_rows,
                         void *q, int64_t ldq, float *scale, cudaStream_t st);

}  // namespace tuna_ops
#endif
