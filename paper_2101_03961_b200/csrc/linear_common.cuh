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
  bool round_dz;                   // dz is rounded to the activation type before it is multiplied
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
__device__ __forceinline__ uint64_t pair_add(uint64_t a, uint64_t b) {
  uint64_t r;
  asm("add.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
  return r;
}

// GELU and its derivative, two values at a time and without selections: with a = min(|z|, 6), beyond which Phi(-a) and
// a phi(a) are below 4e-8, and q = -Phi(-a),
//   GELU(z) = max(z, 0) + a q,   GELU'(z) = 1/2 + sign(z) (1/2 + q + a phi(a)).
// q = P(a) exp(-a^2 / 2) with a polynomial of degree 10 fitted to -Phi(-a) exp(a^2 / 2) on [0, 6], least in the largest error
// that it makes in q and in a q: 1.5e-7 both, float32 evaluation included (the rational form of gelu_cdf_pdf: 7.5e-8 in q, 4e-7
// in a q).  Packed, a value costs 10 issue slots and one special function; the rational form's reciprocal makes it two of
// those, whose unit takes a quarter of a warp a cycle.  min and max keep a NaN.
__device__ __forceinline__ float min_nan(float a, float b) {
  float r;
  asm("min.NaN.f32 %0, %1, %2;" : "=f"(r) : "f"(a), "f"(b));
  return r;
}
__device__ __forceinline__ float max_nan(float a, float b) {
  float r;
  asm("max.NaN.f32 %0, %1, %2;" : "=f"(r) : "f"(a), "f"(b));
  return r;
}
__device__ __forceinline__ uint64_t pair_same(float v) { return pair_of(v, v); }
// q's factors P(a) and exp(-a^2 / 2).
__device__ __forceinline__ void gelu_tail(uint64_t a, uint64_t* poly, uint64_t* e) {
  const float2 x = halves_of(pair_mul(pair_mul(a, pair_same(-0.72134752044448170f)), a));
  float2 ex;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(ex.x) : "f"(x.x));
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(ex.y) : "f"(x.y));
  *e = pair_of(ex.x, ex.y);
  uint64_t s = pair_fma(pair_same(-1.2713327350866166e-06f), a, pair_same(2.8995684260735288e-05f));
  s = pair_fma(s, a, pair_same(-0.000295169185847044f));
  s = pair_fma(s, a, pair_same(0.0018014268716797233f));
  s = pair_fma(s, a, pair_same(-0.007541901897639036f));
  s = pair_fma(s, a, pair_same(0.02376292459666729f));
  s = pair_fma(s, a, pair_same(-0.06070178374648094f));
  s = pair_fma(s, a, pair_same(0.1323055922985077f));
  s = pair_fma(s, a, pair_same(-0.24986957013607025f));
  s = pair_fma(s, a, pair_same(0.39893248677253723f));
  *poly = pair_fma(s, a, pair_same(-0.49999988079071045f));
}
__device__ __forceinline__ void gelu_pair(float* z0, float* z1) {
  const uint64_t a = pair_of(min_nan(fabsf(*z0), 6.f), min_nan(fabsf(*z1), 6.f));
  uint64_t poly, e;
  gelu_tail(a, &poly, &e);
  const float2 r = halves_of(pair_fma(a, pair_mul(poly, e), pair_of(max_nan(*z0, 0.f), max_nan(*z1, 0.f))));
  *z0 = r.x;
  *z1 = r.y;
}
__device__ __forceinline__ float2 gelu_grad_pair(float z0, float z1) {
  const uint64_t a = pair_of(min_nan(fabsf(z0), 6.f), min_nan(fabsf(z1), 6.f));
  uint64_t poly, e;
  gelu_tail(a, &poly, &e);
  // 1/2 + e (poly + a / sqrt(2 pi))
  const float2 h = halves_of(pair_fma(e, pair_fma(a, pair_same(0.3989422804014327f), poly), pair_same(0.5f)));
  return halves_of(pair_add(pair_of(copysignf(h.x, z0), copysignf(h.y, z1)), pair_same(0.5f)));
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
