// Shared by the mixture-of-experts operators (tuna_route.cu, tuna_balance.cu, tuna_fp8.cu, tuna_fp4.cu, tuna_moe.cu):
// launch helper, argument checks, small device helpers, and the PTX of barriers,
// tensor copies and the fifth-generation tensor cores.
#ifndef TUNA_OPS_CUH
#define TUNA_OPS_CUH

#include <cuda.h>
#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cuda_fp8.h>
#include <cuda_runtime.h>
#include <stdint.h>

#include "tuna.h"

namespace tuna_ops {

// ---- host ----------------------------------------------------------------------------

constexpr int kMaxDim = 1 << 24;  // columns of an operand, at most: keeps every in-row index in 32 bits

inline bool aligned(const void *p, size_t n) { return ((uintptr_t)p & (n - 1)) == 0; }
inline int64_t ceil_div(int64_t a, int64_t b) { return (a + b - 1) / b; }

// The operators keep no handle, so the CUDA error behind TUNA_ERR_CUDA is kept per thread.
int note_cuda(cudaError_t e);
int sm_count();
int *error_word();  // device address of the flag that a bounded wait raises (nullptr: no device)

// Launches `kernel` so that it may be scheduled while the stream's previous kernel drains: it
// begins with wait_previous().  A cooperative one is launched behind the previous kernel's end, and need not.
// `cluster`: blocks of a cluster.
template <typename... P, typename... A>
inline int launch_cluster(void (*kernel)(P...), dim3 grid, int cluster, int threads, size_t smem, cudaStream_t st, bool cooperative, A... args) {
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = grid;
  cfg.blockDim = dim3(threads);
  cfg.dynamicSmemBytes = smem;
  cfg.stream = st;
  cudaLaunchAttribute at[2];
  if (cooperative) {
    at[0].id = cudaLaunchAttributeCooperative;
    at[0].val.cooperative = 1;
  } else {
    at[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    at[0].val.programmaticStreamSerializationAllowed = 1;
  }
  at[1].id = cudaLaunchAttributeClusterDimension;
  at[1].val.clusterDim.x = cluster, at[1].val.clusterDim.y = 1, at[1].val.clusterDim.z = 1;
  cfg.attrs = at;
  cfg.numAttrs = cluster > 1 ? 2 : 1;
  return note_cuda(cudaLaunchKernelEx(&cfg, kernel, P(args)...));
}
template <typename... P, typename... A>
inline int launch(void (*kernel)(P...), dim3 grid, int threads, size_t smem, cudaStream_t st, bool cooperative, A... args) {
  return launch_cluster(kernel, grid, 1, threads, smem, st, cooperative, args...);
}

// Dynamic shared memory above the default needs the kernel's leave, once a device (`set`: one
// flag a device and kernel; two threads that both find it clear do the same harmless thing).
template <typename K>
inline int allow_smem(K kernel, size_t bytes, bool (&set)[64]) {
  int dev = 0;
  if (const int rc = note_cuda(cudaGetDevice(&dev))) return rc;
  if (dev >= 0 && dev < 64 && __atomic_load_n(&set[dev], __ATOMIC_ACQUIRE)) return TUNA_OK;
  if (const int rc = note_cuda(cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)bytes))) return rc;
  if (dev >= 0 && dev < 64) __atomic_store_n(&set[dev], true, __ATOMIC_RELEASE);
  return TUNA_OK;
}

// Tensor map of a matrix stack: rows of k values (e4m3 bytes, or bf16), k contiguous with pitch ld, then
// rows, then `matrices` back to back; boxes of 128 bytes x `box` rows, swizzled (tuna_fp8.cu).
int make_map(CUtensorMap *map, int rank, const void *p, int64_t k, int64_t rows, int64_t matrices, int64_t ld, int box, bool bf16 = false);

// The same for gate and up matrices that alternate (groups x 2 x rows x k bytes, rows a multiple of 32):
// boxes of 128 bytes x 32 rows x gate, up x 4, so that one copy brings the rows that a tile interleaves.
int make_gate_up_map(CUtensorMap *map, const void *p, int64_t k, int64_t rows, int64_t groups, int64_t ld);

// bf16 results: boxes of `row_bytes` (128 or 64, swizzled alike) x 32 rows.
int make_out_map(CUtensorMap *map, void *p, int64_t cols, int64_t rows, int64_t ld, int row_bytes);

// Scales of 4-bit operands: tiles x runs x 512 bytes; boxes of 512 bytes x 2 runs x `box` tiles (tuna_fp4.cu).
int make_scale_map(CUtensorMap *map, const void *p, int64_t runs, int64_t tiles, int box);

// Zeros for the results of a product whose contracted axis is empty (f32 or bf16, n columns of pitch ldo), in the rows of the
// groups alone (offsets: device, groups + 1, or nullptr: all m rows) (tuna_fp8.cu).
int launch_empty_sums(void *out, bool f32, int64_t m, int n, int64_t ldo, int groups, const int64_t *offsets, cudaStream_t st);

// Carves a caller's workspace into 256-byte aligned pieces; with base == nullptr it only adds up.
struct Carve {
  char *base;
  size_t used = 0;
  explicit Carve(void *p) : base((char *)p) {}
  template <typename T>
  T *take(int64_t n) {
    T *r = base ? (T *)(base + used) : nullptr;
    used += ((size_t)n * sizeof(T) + 255) / 256 * 256;
    return r;
  }
};

#ifdef __CUDACC__
// ---- device --------------------------------------------------------------------------

__device__ __forceinline__ void wait_previous() { asm volatile("griddepcontrol.wait;" ::: "memory"); }
__device__ __forceinline__ void allow_next() { asm volatile("griddepcontrol.launch_dependents;" ::: "memory"); }

__device__ __forceinline__ float to_f32(float v) { return v; }
__device__ __forceinline__ float to_f32(__nv_bfloat16 v) { return __bfloat162float(v); }
template <typename T>
__device__ __forceinline__ T from_f32(float v);
template <>
__device__ __forceinline__ float from_f32<float>(float v) { return v; }
template <>
__device__ __forceinline__ __nv_bfloat16 from_f32<__nv_bfloat16>(float v) { return __float2bfloat16_rn(v); }

__device__ __forceinline__ uint32_t pack_bf16(float lo, float hi) {
  uint32_t r;
  asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
  return r;
}

// N consecutive values as 32-bit floats; `vec` says that the address is on a 16-byte boundary.
template <int N>
__device__ __forceinline__ void load_row(const __nv_bfloat16 *p, float (&v)[N]) {
#pragma unroll
  for (int i = 0; i < N / 8; ++i) {
    const uint4 u = reinterpret_cast<const uint4 *>(p)[i];
    const uint32_t w[4] = {u.x, u.y, u.z, u.w};
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      v[i * 8 + j * 2] = __uint_as_float(w[j] << 16);
      v[i * 8 + j * 2 + 1] = __uint_as_float(w[j] & 0xffff0000u);
    }
  }
}
template <int N>
__device__ __forceinline__ void load_row(const float *p, float (&v)[N]) {
#pragma unroll
  for (int i = 0; i < N / 4; ++i) {
    const float4 u = reinterpret_cast<const float4 *>(p)[i];
    v[i * 4] = u.x, v[i * 4 + 1] = u.y, v[i * 4 + 2] = u.z, v[i * 4 + 3] = u.w;
  }
}
template <int N>
__device__ __forceinline__ void store_row(__nv_bfloat16 *p, const float (&v)[N]) {
#pragma unroll
  for (int i = 0; i < N / 8; ++i)
    reinterpret_cast<uint4 *>(p)[i] = make_uint4(pack_bf16(v[i * 8], v[i * 8 + 1]), pack_bf16(v[i * 8 + 2], v[i * 8 + 3]),
                                                 pack_bf16(v[i * 8 + 4], v[i * 8 + 5]), pack_bf16(v[i * 8 + 6], v[i * 8 + 7]));
}
template <int N>
__device__ __forceinline__ void store_row(float *p, const float (&v)[N]) {
#pragma unroll
  for (int i = 0; i < N / 4; ++i)
    reinterpret_cast<float4 *>(p)[i] = make_float4(v[i * 4], v[i * 4 + 1], v[i * 4 + 2], v[i * 4 + 3]);
}

// 32 bytes to a 32-byte boundary in one instruction: a whole sector for every lane
__device__ __forceinline__ void store32(void *p, const uint32_t (&v)[8]) {
  asm volatile("st.global.v8.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};" ::"l"(p), "r"(v[0]), "r"(v[1]), "r"(v[2]), "r"(v[3]), "r"(v[4]),
               "r"(v[5]), "r"(v[6]), "r"(v[7])
               : "memory");
}

// ---- 8-bit values --------------------------------------------------------------------

// scale = max(amax, 2^-100) / 448 (448 is the largest e4m3 value).  The floor keeps the scale of
// an all-zero block normal, so that 0 / scale is 0.  `amax_bits` is the largest |x| as raw bits:
// as integers a NaN exceeds an infinity exceeds every finite value, so nothing non-finite is
// lost on the way, and a block that holds one gets a NaN scale and products that are NaN.
__device__ __forceinline__ float fp8_scale(uint32_t amax_bits) {
  if (amax_bits >= 0x7f800000u) return __uint_as_float(0x7fc00000u);
  return __fdiv_rn(fmaxf(__uint_as_float(amax_bits), 7.888609052210118e-31f /* 2^-100 */), 448.0f);
}
__device__ __forceinline__ uint32_t abs_bits(float v) { return __float_as_uint(v) & 0x7fffffffu; }
// Division by a block's scale, correctly rounded as the definition has it: many 16-bit inputs sit
// exactly halfway between two 8-bit values, and a product with 1 / s would send them the other way.
// Markstein's theorem (IBM J. Res. Dev. 34, 1990): with y = 1 / s correctly rounded and q within one
// unit of x / s, q + (x - q s) y in fused operations is x / s correctly rounded, unless the fraction of
// s is all ones.  x y is within 1.5 units, one correction brings it within one, the next one ends it:
// five packed operations for two values.  x - q s must not underflow, so very small (and very large,
// and NaN) scales divide.  The quotient is kept with its sign turned (y is -1 / s), which carries the
// sign of a zero through the corrections; the codes' signs are turned back four at a time.
struct Divisor {
  uint64_t y, s2;  // -1 / s, s
  float s;
  bool plain;
};
__device__ __forceinline__ uint64_t pair(uint32_t lo, uint32_t hi) {
  uint64_t r;
  asm("mov.b64 %0, {%1, %2};" : "=l"(r) : "r"(lo), "r"(hi));
  return r;
}
__device__ __forceinline__ uint64_t pair(float lo, float hi) { return pair(__float_as_uint(lo), __float_as_uint(hi)); }
__device__ __forceinline__ void unpair(uint64_t v, float &lo, float &hi) {
  uint32_t a, b;
  asm("mov.b64 {%0, %1}, %2;" : "=r"(a), "=r"(b) : "l"(v));
  lo = __uint_as_float(a), hi = __uint_as_float(b);
}
__device__ __forceinline__ uint64_t fma2(uint64_t a, uint64_t b, uint64_t c) {
  uint64_t r;
  asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r) : "l"(a), "l"(b), "l"(c));
  return r;
}
__device__ __forceinline__ uint64_t mul2(uint64_t a, uint64_t b) {
  uint64_t r;
  asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
  return r;
}
__device__ __forceinline__ uint64_t add2(uint64_t a, uint64_t b) {
  uint64_t r;
  asm("add.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
  return r;
}
// 2^x and 1 / x, within 2^-22 of themselves; results below the smallest normal number are 0.
__device__ __forceinline__ float exp2_fast(float x) {
  float r;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(x));
  return r;
}
__device__ __forceinline__ float reciprocal_fast(float x) {
  float r;
  asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(x));
  return r;
}
constexpr float kLog2E = 1.4426950408889634f;
__device__ __forceinline__ Divisor divisor(float s) {
  Divisor d;
  const uint32_t bits = __float_as_uint(s);
  d.plain = !(s >= 8.271806125530277e-25f /* 2^-80 */ && s <= 1.2676506002282294e30f /* 2^100 */) || (bits & 0x7fffff) == 0x7fffff;
  const float y = -__frcp_rn(s);
  d.s = s, d.y = pair(y, y), d.s2 = pair(s, s);
  return d;
}
__device__ __forceinline__ uint32_t e4m3_pair(float lo, float hi) {
  uint16_t r;
  asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;" : "=h"(r) : "f"(hi), "f"(lo));
  return r;
}
// N (a multiple of 4) values over the scale, to N / 4 words
template <int N>
__device__ __forceinline__ void fp8_run(const float *v, const Divisor &d, uint32_t (&out)[N / 4]) {
  if (d.plain) {
#pragma unroll
    for (int i = 0; i < N; i += 4)
      out[i / 4] = e4m3_pair(__fdiv_rn(v[i], d.s), __fdiv_rn(v[i + 1], d.s)) | (e4m3_pair(__fdiv_rn(v[i + 2], d.s), __fdiv_rn(v[i + 3], d.s)) << 16);
    return;
  }
#pragma unroll
  for (int i = 0; i < N; i += 4) {
    uint32_t half[2];
#pragma unroll
    for (int j = 0; j < 2; ++j) {
      const uint64_t x = pair(v[i + 2 * j], v[i + 2 * j + 1]);
      uint64_t q = mul2(x, d.y);
      q = fma2(fma2(q, d.s2, x), d.y, q);
      q = fma2(fma2(q, d.s2, x), d.y, q);
      float lo, hi;
      unpair(q, lo, hi);
      half[j] = e4m3_pair(lo, hi);
    }
    out[i / 4] = __byte_perm(half[0], half[1], 0x5410) ^ 0x80808080u;
  }
}
__device__ __forceinline__ uint4 fp8_sixteen(const float *v, const Divisor &d) {
  uint32_t w[4];
  fp8_run<16>(v, d, w);
  return make_uint4(w[0], w[1], w[2], w[3]);
}

// Eight consecutive values as they are stored, for loads that are all issued before the first use.
template <typename T>
struct Eight {
  static constexpr int kWords = sizeof(T) / 2;
  uint4 w[kWords];
  __device__ __forceinline__ void load(const T *p, bool vec, int left) {  // `left`: how many of them there are
    if (vec && left >= 8) {
#pragma unroll
      for (int i = 0; i < kWords; ++i) w[i] = __ldg(reinterpret_cast<const uint4 *>(p) + i);
    } else {
      union {
        uint4 u[kWords];
        T t[8];
      } x;
#pragma unroll
      for (int i = 0; i < kWords; ++i) x.u[i] = make_uint4(0, 0, 0, 0);
#pragma unroll
      for (int i = 0; i < 8; ++i)
        if (i < left) x.t[i] = p[i];
#pragma unroll
      for (int i = 0; i < kWords; ++i) w[i] = x.u[i];
    }
  }
  // The same from any address: in the widest pieces that its alignment allows.  (A bf16 row that starts between two
  // words is taken as a half, three words and a half.)
  __device__ __forceinline__ void load_any(const T *p, int left) {
    const uint32_t at = (uint32_t)(uintptr_t)p & 15;
    if (left >= 8 && at == 0) {
#pragma unroll
      for (int i = 0; i < kWords; ++i) w[i] = __ldg(reinterpret_cast<const uint4 *>(p) + i);
    } else if (left >= 8 && (at & 7) == 0) {
#pragma unroll
      for (int i = 0; i < kWords; ++i) {
        const uint2 a = __ldg(reinterpret_cast<const uint2 *>(p) + 2 * i), b = __ldg(reinterpret_cast<const uint2 *>(p) + 2 * i + 1);
        w[i] = make_uint4(a.x, a.y, b.x, b.y);
      }
    } else if (left >= 8 && (at & 3) == 0) {
      const uint32_t *u = reinterpret_cast<const uint32_t *>(p);
#pragma unroll
      for (int i = 0; i < kWords; ++i) w[i] = make_uint4(__ldg(u + 4 * i), __ldg(u + 4 * i + 1), __ldg(u + 4 * i + 2), __ldg(u + 4 * i + 3));
    } else if (left >= 8 && sizeof(T) == 2) {
      const uint16_t *h = reinterpret_cast<const uint16_t *>(p);
      const uint32_t *u = reinterpret_cast<const uint32_t *>(h + 1);
      const uint32_t a = __ldg(h), b = __ldg(u), c = __ldg(u + 1), d = __ldg(u + 2), e = __ldg(h + 7);
      w[0] = make_uint4(a | b << 16, __funnelshift_l(b, c, 16), __funnelshift_l(c, d, 16), d >> 16 | e << 16);
    } else {
      load(p, false, left);
    }
  }
  // the largest magnitude's bits, kept as `T` has them (two 16-bit values in a word for bf16)
  __device__ __forceinline__ uint32_t top(uint32_t so_far) const {
    constexpr uint32_t mask = sizeof(T) == 2 ? 0x7fff7fffu : 0x7fffffffu;
#pragma unroll
    for (int i = 0; i < kWords; ++i) {
      const uint32_t x[4] = {w[i].x, w[i].y, w[i].z, w[i].w};
#pragma unroll
      for (int j = 0; j < 4; ++j) so_far = sizeof(T) == 2 ? __vmaxu2(so_far, x[j] & mask) : max(so_far, x[j] & mask);
    }
    return so_far;
  }
  static __device__ __forceinline__ uint32_t top_bits(uint32_t t) { return sizeof(T) == 2 ? max(t << 16, t & 0xffff0000u) : t; }
  __device__ __forceinline__ void values(float *v) const {
#pragma unroll
    for (int i = 0; i < kWords; ++i) {
      const uint32_t x[4] = {w[i].x, w[i].y, w[i].z, w[i].w};
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        if (sizeof(T) == 2)
          v[2 * j] = __uint_as_float(x[j] << 16), v[2 * j + 1] = __uint_as_float(x[j] & 0xffff0000u);
        else
          v[4 * i + j] = __uint_as_float(x[j]);
      }
    }
  }
};

// Eight consecutive values to any address, `left` of them there are, in the widest pieces that it allows.
__device__ __forceinline__ void store_any(float *p, const float (&v)[8], int left) {
  const uint32_t at = (uint32_t)(uintptr_t)p & 15;
  if (left >= 8 && at == 0) {
    store_row(p, v);
  } else if (left >= 8 && (at & 7) == 0) {
#pragma unroll
    for (int i = 0; i < 4; ++i) reinterpret_cast<float2 *>(p)[i] = make_float2(v[2 * i], v[2 * i + 1]);
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i)
      if (i < left) p[i] = v[i];
  }
}
__device__ __forceinline__ void store_any(__nv_bfloat16 *p, const float (&v)[8], int left) {
  const uint32_t at = (uint32_t)(uintptr_t)p & 15;
  const uint32_t w[4] = {pack_bf16(v[0], v[1]), pack_bf16(v[2], v[3]), pack_bf16(v[4], v[5]), pack_bf16(v[6], v[7])};
  uint16_t *h = reinterpret_cast<uint16_t *>(p);
  if (left >= 8 && at == 0) {
    *reinterpret_cast<uint4 *>(p) = make_uint4(w[0], w[1], w[2], w[3]);
  } else if (left >= 8 && (at & 7) == 0) {
    reinterpret_cast<uint2 *>(p)[0] = make_uint2(w[0], w[1]), reinterpret_cast<uint2 *>(p)[1] = make_uint2(w[2], w[3]);
  } else if (left >= 8 && (at & 3) == 0) {
#pragma unroll
    for (int i = 0; i < 4; ++i) reinterpret_cast<uint32_t *>(p)[i] = w[i];
  } else if (left >= 8) {
    uint32_t *u = reinterpret_cast<uint32_t *>(h + 1);
    h[0] = (uint16_t)w[0], h[7] = (uint16_t)(w[3] >> 16);
#pragma unroll
    for (int i = 0; i < 3; ++i) u[i] = __funnelshift_r(w[i], w[i + 1], 16);
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i)
      if (i < left) h[i] = (uint16_t)(w[i / 2] >> (16 * (i & 1)));
  }
}

// True in one lane of a whole warp.  What a warp issues to the tensor cores is issued so: the
// operands stay in uniform registers, where a branch on the lane would move each of them there.
__device__ __forceinline__ bool elect_one() {
  uint32_t r;
  asm volatile("{\n .reg .pred p;\n elect.sync _|p, 0xffffffff;\n selp.b32 %0, 1, 0, p;\n}" : "=r"(r));
  return r != 0;
}

// ---- clusters ---------------------------------------------------------------------------

__device__ __forceinline__ uint32_t cluster_rank() {
  uint32_t r;
  asm("mov.u32 %0, %%cluster_ctarank;" : "=r"(r));
  return r;
}
__device__ __forceinline__ uint32_t cluster_size() {
  uint32_t r;
  asm("mov.u32 %0, %%cluster_nctarank;" : "=r"(r));
  return r;
}
// All threads of the cluster's blocks meet (every thread comes here, whatever it gave up before).
__device__ __forceinline__ void cluster_meet() {
  asm volatile("barrier.cluster.arrive.release.aligned;\n barrier.cluster.wait.acquire.aligned;" ::: "memory");
}
__device__ __forceinline__ float4 load_from_block(uint32_t addr, uint32_t rank) {
  float4 v;
  asm volatile("{\n .reg .b32 a;\n mapa.shared::cluster.u32 a, %4, %5;\n ld.shared::cluster.v4.f32 {%0, %1, %2, %3}, [a];\n}"
               : "=f"(v.x), "=f"(v.y), "=f"(v.z), "=f"(v.w) : "r"(addr), "r"(rank) : "memory");
  return v;
}

// ---- barriers in shared memory ---------------------------------------------------------

__device__ __forceinline__ uint32_t smem_u32(const void *p) { return (uint32_t)__cvta_generic_to_shared(p); }
__device__ __forceinline__ void mbar_init(uint32_t bar, uint32_t count) {
  asm volatile("mbarrier.init.shared::cta.b64 [%0], %1;" ::"r"(bar), "r"(count) : "memory");
}
__device__ __forceinline__ void mbar_expect(uint32_t bar, uint32_t bytes) {
  asm volatile("mbarrier.arrive.expect_tx.shared::cta.b64 _, [%0], %1;" ::"r"(bar), "r"(bytes) : "memory");
}
__device__ __forceinline__ void mbar_arrive(uint32_t bar) {
  asm volatile("mbarrier.arrive.shared::cta.b64 _, [%0];" ::"r"(bar) : "memory");
}
__device__ __forceinline__ bool mbar_try(uint32_t bar, uint32_t parity) {
  uint32_t ok;
  asm volatile(
      "{\n .reg .pred p;\n mbarrier.try_wait.parity.shared::cta.b64 p, [%1], %2;\n selp.b32 %0, 1, 0, p;\n}"
      : "=r"(ok) : "r"(bar), "r"(parity) : "memory");
  return ok != 0;
}
// A wait that ends: false after about two seconds, or once another warp of the block gave up.
constexpr long long kWaitCycles = 4000000000LL;
__device__ __forceinline__ bool mbar_wait(uint32_t bar, uint32_t parity, volatile int *given_up) {
  if (mbar_try(bar, parity)) return true;
  const long long t0 = clock64();
  while (!mbar_try(bar, parity)) {
    if (*given_up || clock64() - t0 > kWaitCycles) {
      *given_up = 1;
      return false;
    }
  }
  return true;
}

// ---- tensor copies and tensor cores ------------------------------------------------------

__device__ __forceinline__ void tma_load_2d(uint32_t dst, const CUtensorMap *map, int x, int y, uint32_t bar) {
  asm volatile("cp.async.bulk.tensor.2d.shared::cta.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3}], [%4];" ::"r"(dst),
               "l"(map), "r"(x), "r"(y), "r"(bar)
               : "memory");
}
__device__ __forceinline__ void tma_load_3d(uint32_t dst, const CUtensorMap *map, int x, int y, int z, uint32_t bar) {
  asm volatile("cp.async.bulk.tensor.3d.shared::cta.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3, %4}], [%5];" ::"r"(dst),
               "l"(map), "r"(x), "r"(y), "r"(z), "r"(bar)
               : "memory");
}
__device__ __forceinline__ void tma_load_5d(uint32_t dst, const CUtensorMap *map, int x, int y, int z, int u, int v, uint32_t bar) {
  asm volatile("cp.async.bulk.tensor.5d.shared::cta.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3, %4, %5, %6}], [%7];" ::"r"(dst),
               "l"(map), "r"(x), "r"(y), "r"(z), "r"(u), "r"(v), "r"(bar)
               : "memory");
}
__device__ __forceinline__ void tma_store_2d(const CUtensorMap *map, int x, int y, uint32_t src) {
  asm volatile("cp.async.bulk.tensor.2d.global.shared::cta.tile.bulk_group [%0, {%1, %2}], [%3];" ::"l"(map), "r"(x), "r"(y), "r"(src) : "memory");
  asm volatile("cp.async.bulk.commit_group;" ::: "memory");
}
__device__ __forceinline__ void tma_store_read() { asm volatile("cp.async.bulk.wait_group.read 0;" ::: "memory"); }  // the source may be rewritten
__device__ __forceinline__ void tma_store_done() { asm volatile("cp.async.bulk.wait_group 0;" ::: "memory"); }
__device__ __forceinline__ void tmem_alloc(uint32_t smem_dst, uint32_t cols) {
  asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_dst), "r"(cols) : "memory");
  asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
}
__device__ __forceinline__ void tmem_free(uint32_t addr, uint32_t cols) {
  asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(addr), "r"(cols) : "memory");
}
__device__ __forceinline__ void tc_fence_before() { asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void tc_fence_after() { asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void tc_commit(uint32_t bar) {
  asm volatile("tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];" ::"r"(bar) : "memory");
}
// d[tmem] (+)= A (128 x 32) * B^T (N x 32), both e4m3, K-major in shared memory
__device__ __forceinline__ void tc_mma_fp8(uint32_t d, uint64_t a, uint64_t b, uint32_t idesc, bool accumulate) {
  asm volatile(
      "{\n .reg .pred p;\n setp.ne.u32 p, %4, 0;\n"
      " tcgen05.mma.cta_group::1.kind::f8f6f4 [%0], %1, %2, %3, p;\n}" ::"r"(d),
      "l"(a), "l"(b), "r"(idesc), "r"((uint32_t)accumulate)
      : "memory");
}
// the same for bf16 operands (128 x 16)
__device__ __forceinline__ void tc_mma_bf16(uint32_t d, uint64_t a, uint64_t b, uint32_t idesc, bool accumulate) {
  asm volatile(
      "{\n .reg .pred p;\n setp.ne.u32 p, %4, 0;\n"
      " tcgen05.mma.cta_group::1.kind::f16 [%0], %1, %2, %3, p;\n}" ::"r"(d),
      "l"(a), "l"(b), "r"(idesc), "r"((uint32_t)accumulate)
      : "memory");
}
// Operand descriptor: rows of 128 bytes, swizzled in atoms of 8 rows (1024 bytes).
__device__ __forceinline__ uint64_t tc_desc(uint32_t addr) {
  return (uint64_t)((addr & 0x3ffff) >> 4) | ((uint64_t)1 << 16) | ((uint64_t)(1024 >> 4) << 32) | ((uint64_t)1 << 46) | ((uint64_t)2 << 61);
}
// 8, 16 or 32 accumulator columns of the calling warp's 32 lanes
__device__ __forceinline__ void tmem_load(uint32_t addr, uint32_t (&r)[32]) {
  asm volatile(
      "tcgen05.ld.sync.aligned.32x32b.x32.b32 {%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,%16,%17,%18,%19,%20,%21,%22,%23,"
      "%24,%25,%26,%27,%28,%29,%30,%31}, [%32];"
      : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]), "=r"(r[8]), "=r"(r[9]),
        "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15]), "=r"(r[16]), "=r"(r[17]), "=r"(r[18]), "=r"(r[19]),
        "=r"(r[20]), "=r"(r[21]), "=r"(r[22]), "=r"(r[23]), "=r"(r[24]), "=r"(r[25]), "=r"(r[26]), "=r"(r[27]), "=r"(r[28]), "=r"(r[29]),
        "=r"(r[30]), "=r"(r[31])
      : "r"(addr));
}
__device__ __forceinline__ void tmem_load(uint32_t addr, uint32_t (&r)[8]) {
  asm volatile("tcgen05.ld.sync.aligned.32x32b.x8.b32 {%0,%1,%2,%3,%4,%5,%6,%7}, [%8];"
               : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]) : "r"(addr));
}
__device__ __forceinline__ void tmem_load(uint32_t addr, uint32_t (&r)[16]) {
  asm volatile(
      "tcgen05.ld.sync.aligned.32x32b.x16.b32 {%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15}, [%16];"
      : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]), "=r"(r[8]), "=r"(r[9]),
        "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15])
      : "r"(addr));
}
// Completes the loads into `r`; the values are tied to it so that no use moves before it.
template <int N>
__device__ __forceinline__ void tmem_wait(uint32_t (&r)[N]) {
  asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory");
#pragma unroll
  for (int i = 0; i < N; ++i) asm volatile("" : "+r"(r[i]));
}
#endif  // __CUDACC__

}  // namespace tuna_ops
#endif
