// The dense product (switch_moe_linear_*): what its files share.
#pragma once

#include <cmath>

#include "dropout_rng.cuh"

namespace swmoe {

// Of one product D [rows, cols] = sum_k A(row, k) B(k, col) on the tensor cores.  An operand is "k-major" where its
// contraction index is contiguous in memory ([rows][ld] of A, [cols][ld] of B), else stored [k][ld] with rows or columns
// contiguous.
struct DenseOperand {
  const void* p;          // bf16 values, or the three bf16 parts of float32 values, [3][rows of storage][ld]
  long long ld;           // elements
  // float32: where the original values are, for results that have to be formed again; element (i, k) at i * si + k * sk
  const float* f32;
  long long si, sk;
};

struct DenseEpilogue {    // forward pass only
  const float* bias;
  const void* residual;
  void* pre;
  int activation;
  int dropout_blocks;     // ceil(cols / 8)
  DropoutParams dropout;
};

struct DenseProduct {
  int rows, cols, k;
  int f32;                // operands as parts, float32 result
  int splits;             // > 1: `out` is float32 [splits][rows][ld_out], to be added up
  DenseOperand a, b;
  void* out;
  long long ld_out;
  int* status;
  bool clear_status;
};

enum DenseKind { kDenseFwd = 0, kDenseDx = 1, kDenseDw = 2 };   // A, B k-major: yes, no; yes, yes; no, no

// Forward product and dx of few rows: a kernel of their own (linear_rows.cu).
inline bool few_rows(bool f32, long long rows) { return rows <= (f32 ? 16 : 64); }
int launch_dense_rows(DenseKind kind, const DenseProduct& q, const DenseEpilogue& e, cudaStream_t st);
int dense_splits(long long rows, long long cols, long long k);
int launch_dense(DenseKind kind, const DenseProduct& q, const DenseEpilogue& e, cudaStream_t st);

// The float32 operands of the tensor cores: x 2^24 as the exact sum of three bfloat16 values (f32_gemm_sm100.cu).
constexpr float kPartUp = 16777216.f, kPartDown = 1.f / (kPartUp * kPartUp);

// Two float32 in one register pair: packed instructions round each half like the scalar ones and take half the issue slots.
__device__ __forceinline__ uint64_t pair_of(float lo, float hi) {
  uint64_t r;
  asm("mov.b64 %0, {%1, %2};" : "=l"(r) : "f"(lo), "f"(hi));
  return r;
}
__device__ __forceinline__ float2 halves_of(uint64_t v) {
  float2 r;
  asm("mov.b64 {%0, %1}, %2;" : "=f"(r.x), "=f"(r.y) : "l"(v));
  return r;
}
__device__ __forceinline__ uint64_t pair_fma(uint64_t a, uint64_t b, uint64_t c) {
  uint64_t r;
  asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r) : "l"(a), "l"(b), "l"(c));
  return r;
}
__device__ __forceinline__ uint64_t pair_mul(uint64_t a, uint64_t b) {
  uint64_t r;
  asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
  return r;
}
__device__ __forceinline__ uint64_t pair_add(uint64_t a, uint64_t b) {
  uint64_t r;
  asm("add.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
  return r;
}

// GELU and its derivative, two values at a time: gelu_cdf_pdf's approximation (Abramowitz and Stegun 7.1.26, Phi(-|z|) to
// 7.5e-8) with the sign carried by |z| instead of a selection: with h = 1/2 - Phi(-|z|),
//   GELU(z) = z / 2 + |z| h,   GELU'(z) = 1/2 + sign(z) h + z phi(z).
// 9 issue slots and two special functions a value; the special functions (a quarter of the lanes a cycle) bound it.
__device__ __forceinline__ void gelu_h(uint64_t z, uint64_t az, uint64_t* h, uint64_t* e) {
  const float2 x = halves_of(pair_mul(pair_mul(z, pair_of(-0.72134752044448170f, -0.72134752044448170f)), z));
  float2 ex, t;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(ex.x) : "f"(x.x));
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(ex.y) : "f"(x.y));
  constexpr float c = 0.3275911f * 0.70710678118654752f;
  const float2 d = halves_of(pair_fma(az, pair_of(c, c), pair_of(1.f, 1.f)));
  asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(t.x) : "f"(d.x));
  asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(t.y) : "f"(d.y));
  const uint64_t tt = pair_of(t.x, t.y);
  *e = pair_of(ex.x, ex.y);
  constexpr float a5 = -0.5f * 1.061405429f, a4 = 0.5f * 1.453152027f, a3 = -0.5f * 1.421413741f, a2 = 0.5f * 0.284496736f,
                  a1 = -0.5f * 0.254829592f;
  uint64_t poly = pair_fma(pair_of(a5, a5), tt, pair_of(a4, a4));
  poly = pair_fma(poly, tt, pair_of(a3, a3));
  poly = pair_fma(poly, tt, pair_of(a2, a2));
  poly = pair_fma(poly, tt, pair_of(a1, a1));
  *h = pair_fma(pair_mul(poly, tt), *e, pair_of(0.5f, 0.5f));
}
__device__ __forceinline__ void gelu_pair(float* z0, float* z1) {
  const uint64_t z = pair_of(*z0, *z1), az = pair_of(fabsf(*z0), fabsf(*z1));
  uint64_t h, e;
  gelu_h(z, az, &h, &e);
  const float2 r = halves_of(pair_fma(az, h, pair_mul(z, pair_of(0.5f, 0.5f))));
  // (an infinity: +inf / 2 + inf . 1/2 and -inf / 2 + inf . 1/2; the limit of the latter is 0)
  *z0 = *z0 == -INFINITY ? 0.f : r.x;
  *z1 = *z1 == -INFINITY ? 0.f : r.y;
}
__device__ __forceinline__ float2 gelu_grad_pair(float z0, float z1) {
  const uint64_t z = pair_of(z0, z1), az = pair_of(fabsf(z0), fabsf(z1));
  uint64_t h, e;
  gelu_h(z, az, &h, &e);
  const float2 hh = halves_of(h);
  const uint64_t sh = pair_of(copysignf(hh.x, z0), copysignf(hh.y, z1));
  // (z phi(z) underflows to 0 long before z overflows; an infinity is held off it)
  const uint64_t zc = pair_of(fminf(fmaxf(z0, -64.f), 64.f), fminf(fmaxf(z1, -64.f), 64.f));
  const uint64_t cdf = pair_add(sh, pair_of(0.5f, 0.5f));
  float2 g = halves_of(pair_fma(pair_mul(e, pair_of(0.3989422804014327f, 0.3989422804014327f)), zc, cdf));
  if (z0 != z0) g.x = z0;                              // (fminf and fmaxf drop a NaN)
  if (z1 != z1) g.y = z1;
  return g;
}

}  // namespace swmoe
