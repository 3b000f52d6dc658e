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
  int splits, width;      // dense_tiling's choice; splits > 1: `out` is float32 [splits][rows][ld_out], to be added up
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
// Into how many parts the contraction is cut, and the columns of a tile.
struct DenseTiling {
  int splits, width;
};
// Weight and bias gradient of few rows, with dz kept for dx (linear_rows.cu).
struct RowsDw {
  const void* dy; const void* pre; const void* x;
  void* dW; float* dbias; void* dz;
  int M, K, N, act, per_row;
  long long ldx, ldw, ldy, ldn;
  DropoutParams dropout;
  int* status;
};
// Up to where one launch takes less than the pass over dz and the tensor-core product (us: 16 rows, 512 x 2880 14 against 21,
// 40 rows, 576 x 2752 31 and 31, 13 rows, 1008 x 7506 27 and 26).
inline bool rows_dw_pays(long long M, long long K, long long N) { return M * K * N <= 50000000ll; }
int launch_rows_dw(bool f32, const RowsDw& d, cudaStream_t st);
DenseTiling dense_tiling(DenseKind kind, bool f32, long long rows, long long cols, long long k);
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

// GELU and its derivative, two values at a time: with n = max(-|z|, -10),
//   GELU(z) = max(z, 0) + n Phi(n),   GELU'(z) = Phi(n) + n phi(n), or 1 minus that for z > 0.
// Phi(n) = 2^R(n) with a polynomial R of degree 12 fitted to log2 Phi on [-10, 0], so that the tail keeps its relative error:
// float32 evaluation included 7.3e-7 from -2 on, 5.2e-6 from -6 on, 7.5e-5 from -10 on, and 3.6e-8 absolute in n Phi(n).  Below -10
// GELU is the constant -7.6e-23.  A form with an absolute error, P(a) exp(-a^2 / 2), is off by 8% at -5 and needs as many
// instructions; erfc, or a rational form with its reciprocal, needs a second special function a value, whose unit takes a quarter
// of a warp a cycle.  min and max keep a NaN.
__device__ __forceinline__ float max_nan(float a, float b) {
  float r;
  asm("max.NaN.f32 %0, %1, %2;" : "=f"(r) : "f"(a), "f"(b));
  return r;
}
__device__ __forceinline__ uint64_t pair_same(float v) { return pair_of(v, v); }
__device__ __forceinline__ uint64_t pair_exp2(uint64_t v) {
  const float2 x = halves_of(v);
  float2 e;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(e.x) : "f"(x.x));
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(e.y) : "f"(x.y));
  return pair_of(e.x, e.y);
}
__device__ __forceinline__ uint64_t normal_tail(uint64_t n) {          // Phi(n)
  uint64_t r = pair_fma(pair_same(-4.2411133632791476e-11f), n, pair_same(-2.6161950383851718e-09f));
  r = pair_fma(r, n, pair_same(-7.09738188220399e-08f));
  r = pair_fma(r, n, pair_same(-1.1100130450358847e-06f));
  r = pair_fma(r, n, pair_same(-1.0956950063700788e-05f));
  r = pair_fma(r, n, pair_same(-6.879954162286595e-05f));
  r = pair_fma(r, n, pair_same(-0.00023773251450620592f));
  r = pair_fma(r, n, pair_same(0.0001084727919078432f));
  r = pair_fma(r, n, pair_same(0.007098168600350618f));
  r = pair_fma(r, n, pair_same(0.05255275219678879f));
  r = pair_fma(r, n, pair_same(-0.45918235182762146f));
  r = pair_fma(r, n, pair_same(1.1511086225509644f));
  return pair_exp2(pair_fma(r, n, pair_same(-1.f)));
}
__device__ __forceinline__ void gelu_pair(float* z0, float* z1) {
  const uint64_t n = pair_of(max_nan(-fabsf(*z0), -10.f), max_nan(-fabsf(*z1), -10.f));
  const float2 r = halves_of(pair_fma(n, normal_tail(n), pair_of(max_nan(*z0, 0.f), max_nan(*z1, 0.f))));
  *z0 = r.x;
  *z1 = r.y;
}
__device__ __forceinline__ float2 gelu_grad_pair(float z0, float z1) {
  const uint64_t n = pair_of(max_nan(-fabsf(z0), -10.f), max_nan(-fabsf(z1), -10.f));
  // phi(n) = 2^(-n^2 / 2 log2 e - log2 sqrt(2 pi))
  const uint64_t density = pair_exp2(pair_fma(pair_mul(n, n), pair_same(-0.72134752044448170f), pair_same(-1.3257480647361593f)));
  const float2 w = halves_of(pair_fma(n, density, normal_tail(n)));
  return make_float2(z0 > 0.f ? 1.f - w.x : w.x, z1 > 0.f ? 1.f - w.y : w.y);
}

// Everything after the product for eight results of a row: bias, z saved, activation, dropout, residual, store.
template <typename ET>
__device__ __forceinline__ void finish8(const DenseEpilogue& e, const DropoutState& rng, void* out, long long ld, int cols,
                                        long long row, int col, float* x) {
  const int n = min(8, cols - col);
  const long long at = row * ld + col;
  auto put = [&](void* base, const float* v) {
    ET* o = static_cast<ET*>(base) + at;
    if constexpr (sizeof(ET) == 2) {
      if (n == 8) {
        __nv_bfloat162 h[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) h[i] = __floats2bfloat162_rn(v[2 * i], v[2 * i + 1]);
        *reinterpret_cast<uint4*>(o) = *reinterpret_cast<const uint4*>(h);
      } else {
#pragma unroll
        for (int i = 0; i < 8; ++i)
          if (i < n) o[i] = __float2bfloat16(v[i]);
      }
    } else {
      if (n == 8) {
        *reinterpret_cast<float4*>(o) = make_float4(v[0], v[1], v[2], v[3]);
        *reinterpret_cast<float4*>(o + 4) = make_float4(v[4], v[5], v[6], v[7]);
      } else {
#pragma unroll
        for (int i = 0; i < 8; ++i)
          if (i < n) o[i] = v[i];
      }
    }
  };
  if (e.bias != nullptr) {
#pragma unroll
    for (int i = 0; i < 8; ++i) x[i] += i < n ? e.bias[col + i] : 0.f;
  }
  if (e.pre != nullptr) put(e.pre, x);
  if (e.activation == SWITCH_MOE_ACT_RELU) {
#pragma unroll
    for (int i = 0; i < 8; ++i) x[i] = max_nan(x[i], 0.f);
  } else if (e.activation == SWITCH_MOE_ACT_GELU) {
#pragma unroll
    for (int i = 0; i < 8; i += 2) gelu_pair(x + i, x + i + 1);
  }
  if (e.dropout.rng != nullptr)
    dropout8(e.dropout, dropout_bits(e.dropout, rng, (unsigned long long)row * (unsigned)e.dropout_blocks + (unsigned)(col >> 3)), x);
  if (e.residual != nullptr) {
    const ET* r = static_cast<const ET*>(e.residual) + at;
#pragma unroll
    for (int i = 0; i < 8; ++i)
      if (i < n) x[i] += (float)r[i];
  }
  put(out, x);
}

// Eight consecutive elements of a row, the first `n` of them inside; 16-byte aligned.
__device__ __forceinline__ void load8(const float* p, int n, float* f) {
  if (n >= 8) {
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      const float4 v = *reinterpret_cast<const float4*>(p + 4 * i);
      f[4 * i] = v.x; f[4 * i + 1] = v.y; f[4 * i + 2] = v.z; f[4 * i + 3] = v.w;
    }
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i) f[i] = i < n ? p[i] : 0.f;
  }
}
// The same in flight: loaded now, converted when it is needed.
template <typename ET> struct Raw8;
template <> struct Raw8<__nv_bfloat16> {
  uint4 v;
  __device__ __forceinline__ void load(const __nv_bfloat16* p, int n) {
    if (n >= 8) {
      v = *reinterpret_cast<const uint4*>(p);
    } else {
      const uint16_t* q = reinterpret_cast<const uint16_t*>(p);
      uint32_t w[4];
#pragma unroll
      for (int i = 0; i < 4; ++i) w[i] = (2 * i < n ? q[2 * i] : 0u) | (2 * i + 1 < n ? (uint32_t)q[2 * i + 1] << 16 : 0u);
      v = make_uint4(w[0], w[1], w[2], w[3]);
    }
  }
  __device__ __forceinline__ void get(float* f) const {
    const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) { f[2 * i] = __uint_as_float(w[i] << 16); f[2 * i + 1] = __uint_as_float(w[i] & 0xFFFF0000u); }
  }
};
template <> struct Raw8<float> {
  float f8[8];
  __device__ __forceinline__ void load(const float* p, int n) { load8(p, n, f8); }
  __device__ __forceinline__ void get(float* f) const {
#pragma unroll
    for (int i = 0; i < 8; ++i) f[i] = f8[i];
  }
};
__device__ __forceinline__ void store8(__nv_bfloat16* p, int n, const float* f) {
  if (n >= 8) {
    uint4 v;
    __nv_bfloat162* h = reinterpret_cast<__nv_bfloat162*>(&v);
#pragma unroll
    for (int i = 0; i < 4; ++i) h[i] = __floats2bfloat162_rn(f[2 * i], f[2 * i + 1]);
    *reinterpret_cast<uint4*>(p) = v;
  } else {
    for (int i = 0; i < n; ++i) p[i] = __float2bfloat16(f[i]);
  }
}
__device__ __forceinline__ void store8(float* p, int n, const float* f) {
  if (n >= 8) {
#pragma unroll
    for (int i = 0; i < 2; ++i)
      *reinterpret_cast<float4*>(p + 4 * i) = make_float4(f[4 * i], f[4 * i + 1], f[4 * i + 2], f[4 * i + 3]);
  } else {
    for (int i = 0; i < n; ++i) p[i] = f[i];
  }
}
// Eight values of dy become those of dz = dropout(dy) . activation'(z); `block` is their place in the dropout's count.
__device__ __forceinline__ void dz8(int act, const DropoutParams& dropout, const DropoutState& rng, unsigned long long block,
                                    const float* z, float* g) {
  if (dropout.rng != nullptr) dropout8(dropout, dropout_bits(dropout, rng, block), g);
  if (act == SWITCH_MOE_ACT_RELU) {
#pragma unroll
    for (int i = 0; i < 8; ++i) g[i] = z[i] > 0.f ? g[i] : 0.f;
  } else if (act == SWITCH_MOE_ACT_GELU) {
#pragma unroll
    for (int i = 0; i < 8; i += 2) {
      const float2 d = gelu_grad_pair(z[i], z[i + 1]);
      g[i] *= d.x;
      g[i + 1] *= d.y;
    }
  }
}

}  // namespace swmoe
