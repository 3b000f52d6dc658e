// Dropout on its own: y = residual + x keep / (1 - rate), and its backward pass, which is the same without the residual.
// The mask is drawn from each element's place (dropout_rng.cuh) and never stored, so a call reads its inputs and writes
// its output once.  A thread takes eight elements of a row: one call of the generator, 16 bytes of bfloat16 or twice 16 of
// float32 per tensor.
#include "dropout_rng.cuh"

namespace swmoe {
namespace {

constexpr int kThreads = 256;

template <typename ET> struct Eight;
template <> struct Eight<__nv_bfloat16> {
  static __device__ __forceinline__ void load(const __nv_bfloat16* p, float* f) {
    const uint4 v = *reinterpret_cast<const uint4*>(p);
    const __nv_bfloat162* h = reinterpret_cast<const __nv_bfloat162*>(&v);
#pragma unroll
    for (int i = 0; i < 4; ++i) { const float2 t = __bfloat1622float2(h[i]); f[2 * i] = t.x; f[2 * i + 1] = t.y; }
  }
  static __device__ __forceinline__ void store(__nv_bfloat16* p, const float* f) {
    uint4 v;
    __nv_bfloat162* h = reinterpret_cast<__nv_bfloat162*>(&v);
#pragma unroll
    for (int i = 0; i < 4; ++i) h[i] = __floats2bfloat162_rn(f[2 * i], f[2 * i + 1]);
    *reinterpret_cast<uint4*>(p) = v;
  }
};
template <> struct Eight<float> {
  static __device__ __forceinline__ void load(const float* p, float* f) {
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      const float4 v = *reinterpret_cast<const float4*>(p + 4 * i);
      f[4 * i] = v.x; f[4 * i + 1] = v.y; f[4 * i + 2] = v.z; f[4 * i + 3] = v.w;
    }
  }
  static __device__ __forceinline__ void store(float* p, const float* f) {
#pragma unroll
    for (int i = 0; i < 2; ++i)
      *reinterpret_cast<float4*>(p + 4 * i) = make_float4(f[4 * i], f[4 * i + 1], f[4 * i + 2], f[4 * i + 3]);
  }
};
__device__ __forceinline__ float to_f(float v) { return v; }
__device__ __forceinline__ float to_f(__nv_bfloat16 v) { return __bfloat162float(v); }
__device__ __forceinline__ void from_f(float v, float* o) { *o = v; }
__device__ __forceinline__ void from_f(float v, __nv_bfloat16* o) { *o = __float2bfloat16(v); }

// A dropped element of x is 0 whatever it held (infinities and NaN too): the factor selects, it does not multiply.
template <typename ET, bool kRes>
__global__ void __launch_bounds__(kThreads)
dropout_kernel(const ET* x, const ET* res, ET* y, long long blocks, int per_row, int cols, long long ld, DropoutParams d) {
  pdl_launch_dependents();
  pdl_wait();
  const DropoutState s = dropout_state(d);
  const long long step = (long long)gridDim.x * kThreads;
  for (long long b = (long long)blockIdx.x * kThreads + threadIdx.x; b < blocks; b += step) {
    const long long row = blocks <= 0x7fffffffll ? (long long)((unsigned)b / (unsigned)per_row) : b / per_row;
    const int col = (int)(b - row * per_row) * 8;
    const long long at = row * ld + col;
    float v[8], r[8];
    const bool whole = col + 8 <= cols;
    if (whole) {
      Eight<ET>::load(x + at, v);
      if (kRes) Eight<ET>::load(res + at, r);
    } else {
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        v[i] = col + i < cols ? to_f(x[at + i]) : 0.f;
        if (kRes) r[i] = col + i < cols ? to_f(res[at + i]) : 0.f;
      }
    }
    if (d.rng != nullptr) {
      const uint4 bits = dropout_bits(d, s, (unsigned long long)b);
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const float f = dropout_factor(d, bits, i);
        v[i] = f != 0.f ? v[i] * f : 0.f;
      }
    }
    if (kRes) {
#pragma unroll
      for (int i = 0; i < 8; ++i) v[i] += r[i];
    }
    if (whole) {
      Eight<ET>::store(y + at, v);
    } else {
#pragma unroll
      for (int i = 0; i < 8; ++i)
        if (col + i < cols) from_f(v[i], y + at + i);
    }
  }
}

template <typename ET>
int launch(const switch_moe_dropout_config& c, const void* x, const void* res, const uint64_t* rng, void* y, int q,
           cudaStream_t st) {
  const int per_row = (int)(((long long)c.cols + 7) / 8);
  const long long blocks = (long long)c.rows * per_row, ld = c.ld > 0 ? c.ld : c.cols;
  const long long want = (blocks + kThreads - 1) / kThreads, most = (long long)sm_count_or_default() * 8;
  const dim3 grid((unsigned)(want < most ? want : most));
  const DropoutParams d = dropout_params(rng, q, c.site);
  const ET* xt = static_cast<const ET*>(x);
  const ET* rt = static_cast<const ET*>(res);
  if (res != nullptr)
    launch_k(dropout_kernel<ET, true>, grid, dim3(kThreads), 0, st, xt, rt, static_cast<ET*>(y), blocks, per_row, c.cols, ld, d);
  else
    launch_k(dropout_kernel<ET, false>, grid, dim3(kThreads), 0, st, xt, rt, static_cast<ET*>(y), blocks, per_row, c.cols, ld, d);
  return launch_status();
}

int run(const switch_moe_dropout_config* cfg, const void* x, const void* res, const uint64_t* rng, void* y, void* stream) {
  if (cfg == nullptr) return SWITCH_MOE_INVALID_ARGUMENT;
  const switch_moe_dropout_config& c = *cfg;
  if (c.rows < 0 || c.cols <= 0 || c.ld < 0 || (c.ld > 0 && c.ld < c.cols) || c.reserved[0] != 0 || c.reserved[1] != 0)
    return SWITCH_MOE_INVALID_ARGUMENT;
  if (c.dtype != SWITCH_MOE_BF16 && c.dtype != SWITCH_MOE_F32) return SWITCH_MOE_INVALID_ARGUMENT;
  const int q = dropout_threshold(c.rate);
  if (q < 0 || c.site < 0 || c.site > 65535) return SWITCH_MOE_INVALID_ARGUMENT;
  const long long elt = c.dtype == SWITCH_MOE_BF16 ? 2 : 4, ld = c.ld > 0 ? c.ld : c.cols;
  if (c.rows > 1 && ld * elt % 16 != 0) return SWITCH_MOE_UNSUPPORTED_SHAPE;
  if ((long long)c.rows * (((long long)c.cols + 7) / 8) >= 1ll << 48) return SWITCH_MOE_UNSUPPORTED_SHAPE;
  if (c.rows == 0) return SWITCH_MOE_OK;
  if (x == nullptr || y == nullptr || (q > 0 && rng == nullptr)) return SWITCH_MOE_INVALID_ARGUMENT;
  if (!aligned16(x) || !aligned16(y) || !aligned16(res) || (reinterpret_cast<uintptr_t>(rng) & 7u) != 0)
    return SWITCH_MOE_UNSUPPORTED_SHAPE;
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  return c.dtype == SWITCH_MOE_BF16 ? launch<__nv_bfloat16>(c, x, res, rng, y, q, st)
                                    : launch<float>(c, x, res, rng, y, q, st);
}

}  // namespace
}  // namespace swmoe

extern "C" int switch_moe_dropout_fwd(const switch_moe_dropout_config* cfg, const void* x, const void* residual,
                                      const uint64_t* rng, void* y, void* stream) {
  return swmoe::run(cfg, x, residual, rng, y, stream);
}

extern "C" int switch_moe_dropout_bwd(const switch_moe_dropout_config* cfg, const void* dy, const uint64_t* rng, void* dx,
                                      void* stream) {
  return swmoe::run(cfg, dy, nullptr, rng, dx, stream);
}
