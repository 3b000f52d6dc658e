// The dense product (switch_moe_linear_*): what its files share.
#pragma once

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

int dense_splits(long long rows, long long cols, long long k);
int launch_dense(DenseKind kind, const DenseProduct& q, const DenseEpilogue& e, cudaStream_t st);

// The float32 operands of the tensor cores: x 2^24 as the exact sum of three bfloat16 values (f32_gemm_sm100.cu).
constexpr float kPartUp = 16777216.f, kPartDown = 1.f / (kPartUp * kPartUp);

__device__ __forceinline__ float activation_derivative(int act, float z) {
  if (act == SWITCH_MOE_ACT_RELU) return z > 0.f ? 1.f : 0.f;
  if (act == SWITCH_MOE_ACT_GELU) {
    float cdf, pdf;
    gelu_cdf_pdf(z, &cdf, &pdf);
    return fmaf(z, pdf, cdf);
  }
  return 1.f;
}

}  // namespace swmoe
