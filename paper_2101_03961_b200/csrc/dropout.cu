// Dropout on its own: y = residual + x keep / (1 - rate), and its backward pass, which is the same without the residual.
// The mask is drawn from each element's place (dropout_rng.cuh) and never stored, so a call reads its inputs and writes
// its output once.  A thread takes eight elements of a row: one call of the generator, 16 bytes of bfloat16 or twice 16 of
// float32 per tensor.  32768 x 2048 bfloat16 (ncu): with a residual 64 us, 6.3 TB/s; without one 53, 5.1 TB/s.  There neither the
// bytes (41 us) nor the generator's multiplies (93 cycles of a scheduler per warp and eight elements each, 21 us) bound it alone:
// 0.6 instructions a cycle and scheduler with two loads of 16 bytes in flight a thread.
#include "dropout_rng.cuh"

namespace swmoe {
namespace {

constexpr int kThreads = 256;

// Eight elements in flight: loaded now, converted when they are needed.
template <typename ET> struct Eight;
template <> struct Eight<__nv_bfloat16> {
  uint4 v;
  __device__ __forceinline__ void load(const __nv_bfloat16* p) { v = *reinterpret_cast<const uint4*>(p); }
  __device__ __forceinline__ void load(const __nv_bfloat16* p, int n) {
    const uint16_t* q = reinterpret_cast<const uint16_t*>(p);
    uint32_t w[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) w[i] = (2 * i < n ? q[2 * i] : 0u) | (2 * i + 1 < n ? (uint32_t)q[2 * i + 1] << 16 : 0u);
    v = make_uint4(w[0], w[1], w[2], w[3]);
  }
  __device__ __forceinline__ void get(float* f) const {
    const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) { f[2 * i] = __uint_as_float(w[i] << 16); f[2 * i + 1] = __uint_as_float(w[i] & 0xFFFF0000u); }
  }
  static __device__ __forceinline__ void store(__nv_bfloat16* p, const float* f) {
    uint4 o;
    __nv_bfloat162* h = reinterpret_cast<__nv_bfloat162*>(&o);
#pragma unroll
    for (int i = 0; i < 4; ++i) h[i] = __floats2bfloat162_rn(f[2 * i], f[2 * i + 1]);
    *reinterpret_cast<uint4*>(p) = o;
  }
  static __device__ __forceinline__ void store1(__nv_bfloat16* p, float f) { *p = __float2bfloat16(f); }
};
template <> struct Eight<float> {
  float4 lo, hi;
  __device__ __forceinline__ void load(const float* p) {
    lo = *reinterpret_cast<const float4*>(p);
    hi = *reinterpret_cast<const float4*>(p + 4);
  }
  __device__ __forceinline__ void load(const float* p, int n) {
    float f[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) f[i] = i < n ? p[i] : 0.f;
    lo = make_float4(f[0], f[1], f[2], f[3]);
    hi = make_float4(f[4], f[5], f[6], f[7]);
  }
  __device__ __forceinline__ void get(float* f) const {
    f[0] = lo.x; f[1] = lo.y; f[2] = lo.z; f[3] = lo.w;
    f[4] = hi.x; f[5] = hi.y; f[6] = hi.z; f[7] = hi.w;
  }
  static __device__ __forceinline__ void store(float* p, const float* f) {
    *reinterpret_cast<float4*>(p) = make_float4(f[0], f[1], f[2], f[3]);
    *reinterpret_cast<float4*>(p + 4) = make_float4(f[4], f[5], f[6], f[7]);
  }
  static __device__ __forceinline__ void store1(float* p, float f) { *p = f; }
};

// kDense: rows follow each other without a gap and in whole blocks of eight.  Two blocks of eight per thread are asked for
// before the first is worked on; with one, the loads' latency bounded the kernel.  Five and four blocks an SM; float32 with a
// residual spills 20 bytes for it (rows with gaps 76).
template <typename ET, bool kRes, bool kDense>
__global__ void __launch_bounds__(kThreads, sizeof(ET) == 2 ? 5 : 4)
dropout_kernel(const ET* x, const ET* res, ET* y, long long blocks, int per_row, int cols, long long ld, DropoutParams d) {
  pdl_launch_dependents();
  pdl_wait();
  constexpr int kAhead = 2;
  const DropoutState s = dropout_state(d);
  const long long step = (long long)gridDim.x * kThreads;   // a thread's two are a grid apart: a small call has one, in every block
  for (long long b0 = (long long)blockIdx.x * kThreads + threadIdx.x; b0 < blocks; b0 += kAhead * step) {
    Eight<ET> a[kAhead], r[kAhead];
    long long at[kAhead];
    int n[kAhead];                                    // elements of the block that are in the row
#pragma unroll
    for (int k = 0; k < kAhead; ++k) {
      const long long b = b0 + k * step;
      n[k] = 0;
      if (b >= blocks) continue;
      if (kDense) {
        at[k] = b * 8;
        n[k] = 8;
      } else {
        const long long row = blocks <= 0x7fffffffll ? (long long)((unsigned)b / (unsigned)per_row) : b / per_row;
        const int col = (int)(b - row * per_row) * 8;
        at[k] = row * ld + col;
        n[k] = min(8, cols - col);
      }
      if (n[k] == 8) {
        a[k].load(x + at[k]);
        if (kRes) r[k].load(res + at[k]);
      } else {
        a[k].load(x + at[k], n[k]);
        if (kRes) r[k].load(res + at[k], n[k]);
      }
    }
#pragma unroll
    for (int k = 0; k < kAhead; ++k) {
      const long long b = b0 + k * step;
      if (b >= blocks) break;
      float v[8];
      a[k].get(v);
      if (d.rng != nullptr) dropout8(d, dropout_bits(d, s, (unsigned long long)b), v);
      if (kRes) {
        float add[8];
        r[k].get(add);
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] += add[i];
      }
      if (n[k] == 8) {
        Eight<ET>::store(y + at[k], v);
      } else {
#pragma unroll
        for (int i = 0; i < 8; ++i)
          if (i < n[k]) Eight<ET>::store1(y + at[k] + i, v[i]);
      }
    }
  }
}

template <typename ET>
int launch(const switch_moe_dropout_config& c, const void* x, const void* res, const uint64_t* rng, void* y, int q,
           cudaStream_t st) {
  const int per_row = (int)(((long long)c.cols + 7) / 8);
  const long long blocks = (long long)c.rows * per_row, ld = c.ld > 0 ? c.ld : c.cols;
  const long long want = (blocks + kThreads - 1) / kThreads, most = (long long)sm_count_or_default() * 8;
  const dim3 grid((unsigned)(want < most ? want : most));   // (a small call has a block of eight per thread, a larger one two)
  const DropoutParams d = dropout_params(rng, q, c.site);
  const ET* xt = static_cast<const ET*>(x);
  const ET* rt = static_cast<const ET*>(res);
  const bool dense = ld == c.cols && c.cols % 8 == 0;
  auto go = [&](auto kernel) {
    launch_k(kernel, grid, dim3(kThreads), 0, st, xt, rt, static_cast<ET*>(y), blocks, per_row, c.cols, ld, d);
  };
  if (res != nullptr) dense ? go(dropout_kernel<ET, true, true>) : go(dropout_kernel<ET, true, false>);
  else dense ? go(dropout_kernel<ET, false, true>) : go(dropout_kernel<ET, false, false>);
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
  if (c.rows > kMaxExtent || c.cols > kMaxExtent) return SWITCH_MOE_UNSUPPORTED_SHAPE;
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
