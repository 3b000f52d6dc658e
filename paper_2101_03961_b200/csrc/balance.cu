// The load-balancing loss of any router (Eq. 4-6 over its softmax, Eq. 1) and its gradient.
//
// Forward: L lanes (a power of two up to 32) share a row of logits, a lane holds 16-byte pieces of it (single elements
// where rows are not 16-byte aligned), so that a row is read once, and its softmax, its k largest logits and the running
// sum of its probabilities stay in registers.  A block works on rows of one group and leaves its sums P, its integer counts
// and its number of tokens in the workspace; a second kernel adds the blocks up in a fixed order, 32 experts per block,
// and the last of its blocks to finish adds up the loss.
// Backward: one pass, dlogits = p (g - <p, g>), g_i = d_loss alpha E (counts_i - counts_0) / (k n^2 groups).
// Bound by the logits, read (and written) once, and by the instructions on them (0.6 a cycle and scheduler at two blocks an SM).
// 262144 x 128 float32, two choices, eight groups (ncu): forward 48 + 6 us, and with half of the rows padding 34 where every group
// has as many, 46 where they have 1/9 to 8/9: a group's blocks work on its rows alone, so that the launch lasts as long as the
// group with the most tokens.  Backward, which writes every row, 36 us with two thirds of the rows padding; four blocks an SM
// there cost one layout (float32, four pieces a lane) 16 bytes of spills.
#include <cfloat>
#include <cmath>
#include <type_traits>

#include "dropout_rng.cuh"

namespace swmoe {
namespace {

constexpr int kThreads = 256, kWarps = kThreads / 32;
constexpr int kMaxE = 1024, kMaxK = 16;
constexpr int kFinalExperts = 32;                    // experts per block of the second kernel, of
constexpr int kFinalThreads = 1024, kFinalWarps = kFinalThreads / 32;

struct BalanceShape {
  int T, E, k, G, Tg, blocks;      // blocks per group
  bool alone;                      // one block does everything
  long long ld;
  float alpha;
  int f32;
};

struct BalancePlan {
  size_t ticket, loss_part, tokens, counts, psum, total;
};

int resolve(const switch_moe_balance_config* cfg, BalanceShape* s) {
  if (cfg == nullptr) return SWITCH_MOE_INVALID_ARGUMENT;
  const switch_moe_balance_config& c = *cfg;
  if (c.T < 0 || c.E <= 0 || c.k <= 0 || c.k > c.E || c.groups < 0 || c.ld < 0 || (c.ld > 0 && c.ld < c.E) ||
      c.reserved[0] != 0 || c.reserved[1] != 0)
    return SWITCH_MOE_INVALID_ARGUMENT;
  if (c.dtype != SWITCH_MOE_BF16 && c.dtype != SWITCH_MOE_F32) return SWITCH_MOE_INVALID_ARGUMENT;
  if (!std::isfinite(c.alpha)) return SWITCH_MOE_INVALID_ARGUMENT;
  const int G = c.groups > 0 ? c.groups : 1;
  if (c.T % G != 0) return SWITCH_MOE_INVALID_ARGUMENT;
  if (c.E > kMaxE || c.k > kMaxK || G > 65535 || (long long)c.T * c.k > kMaxExtent) return SWITCH_MOE_UNSUPPORTED_SHAPE;
  s->T = c.T; s->E = c.E; s->k = c.k; s->G = G; s->Tg = c.T / G;
  s->ld = c.ld > 0 ? c.ld : c.E;
  s->alpha = c.alpha; s->f32 = c.dtype == SWITCH_MOE_F32;
  // about two blocks per SM over all groups (what its registers allow at once), each with 8 rows a warp or more
  long long want = ((long long)2 * kChipSms + G - 1) / G, most = (s->Tg + 8 * kWarps - 1) / (8 * kWarps);
  s->blocks = (int)(want < most ? want : most);
  if (s->blocks < 1) s->blocks = 1;
  s->alone = false;                // (decided where the layout is known)
  return SWITCH_MOE_OK;
}

void make_plan(const BalanceShape& s, BalancePlan* p) {
  size_t off = 0;
  auto take = [&](size_t bytes) { size_t o = off; off = (off + bytes + 255) / 256 * 256; return o; };
  const size_t rows = (size_t)s.G * s.blocks;
  p->ticket = take(4);
  p->loss_part = take((size_t)s.G * ((s.E + kFinalExperts - 1) / kFinalExperts) * 4);
  p->tokens = take(rows * 4);
  p->counts = take(rows * s.E * 4);
  p->psum = take(rows * s.E * 4);
  p->total = (off + 1023) / 1024 * 1024;
}

// V consecutive elements
template <typename ET, int V> struct Piece;
template <> struct Piece<float, 4> {
  static __device__ __forceinline__ void load(const float* p, float* f) {
    const float4 v = *reinterpret_cast<const float4*>(p);
    f[0] = v.x; f[1] = v.y; f[2] = v.z; f[3] = v.w;
  }
  static __device__ __forceinline__ void store(float* p, const float* f) {
    *reinterpret_cast<float4*>(p) = make_float4(f[0], f[1], f[2], f[3]);
  }
};
template <> struct Piece<__nv_bfloat16, 8> {
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
template <> struct Piece<float, 1> {
  static __device__ __forceinline__ void load(const float* p, float* f) { *f = *p; }
  static __device__ __forceinline__ void store(float* p, const float* f) { *p = *f; }
};
template <> struct Piece<__nv_bfloat16, 1> {
  static __device__ __forceinline__ void load(const __nv_bfloat16* p, float* f) { *f = __bfloat162float(*p); }
  static __device__ __forceinline__ void store(__nv_bfloat16* p, const float* f) { *p = __float2bfloat16(*f); }
};

// pairs: rows that are not 16-byte aligned, but all start and end on pairs
template <> struct Piece<float, 2> {
  static __device__ __forceinline__ void load(const float* p, float* f) {
    const float2 v = *reinterpret_cast<const float2*>(p);
    f[0] = v.x; f[1] = v.y;
  }
  static __device__ __forceinline__ void store(float* p, const float* f) { *reinterpret_cast<float2*>(p) = make_float2(f[0], f[1]); }
};
template <> struct Piece<__nv_bfloat16, 2> {
  static __device__ __forceinline__ void load(const __nv_bfloat16* p, float* f) {
    const float2 v = __bfloat1622float2(*reinterpret_cast<const __nv_bfloat162*>(p));
    f[0] = v.x; f[1] = v.y;
  }
  static __device__ __forceinline__ void store(__nv_bfloat16* p, const float* f) {
    *reinterpret_cast<__nv_bfloat162*>(p) = __floats2bfloat162_rn(f[0], f[1]);
  }
};

template <typename T>
__device__ __forceinline__ T lane_sum(T v, int L) {
  for (int o = L >> 1; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
  return v;
}
__device__ __forceinline__ float lane_max(float v, int L) {
  for (int o = L >> 1; o > 0; o >>= 1) v = fmaxf(v, __shfl_xor_sync(0xffffffffu, v, o));
  return v;
}
__device__ __forceinline__ int lane_min(int v, int L) {
  for (int o = L >> 1; o > 0; o >>= 1) v = min(v, __shfl_xor_sync(0xffffffffu, v, o));
  return v;
}
__device__ __forceinline__ int lane_or(int v, int L) {
  for (int o = L >> 1; o > 0; o >>= 1) v |= __shfl_xor_sync(0xffffffffu, v, o);
  return v;
}

// A row across L lanes: lane l holds the pieces l, l + L, .. of V elements; -infinity beyond E.
template <typename ET, int V, int NV>
struct Row {
  float x[V * NV];
  __device__ __forceinline__ void load(const ET* row, bool valid, int l, int L, int E) {
#pragma unroll
    for (int j = 0; j < NV; ++j) {
      const int at = (l + j * L) * V;
      if (valid && at < E) Piece<ET, V>::load(row + at, x + j * V);    // (V > 1: E is a multiple of V)
      else {
#pragma unroll
        for (int i = 0; i < V; ++i) x[j * V + i] = -INFINITY;
      }
    }
  }
  // p . scale = the softmax; returns whether the row counts (some logit is not -infinity).  A NaN anywhere, or +infinity, makes the
  // row's probabilities NaN, as in the definition: through the sum, which only a row without a finite maximum does not show.
  __device__ __forceinline__ bool softmax(int L, float* p, float* scale_out, float* max_out) const {
    float m = -INFINITY;
#pragma unroll
    for (int i = 0; i < V * NV; ++i) m = fmaxf(m, x[i]);
    m = lane_max(m, L);
    *max_out = m;
    bool counts = true;
    if (__any_sync(0xffffffffu, m == -INFINITY)) {
      int nan = 0;
#pragma unroll
      for (int i = 0; i < V * NV; ++i) nan |= isnan(x[i]) ? 1 : 0;
      nan = lane_or(nan, L);
      counts = m != -INFINITY || nan != 0;
    }
    // exp(x - m) = 2^((x - m) log2 e): the argument's rounding is 2^-24 of up to 30, the unit's error 2^-22
    float s = 0.f;
#pragma unroll
    for (int i = 0; i < V * NV; ++i) {
      asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(p[i]) : "f"((x[i] - m) * 1.44269504f));
      s += p[i];
    }
    s = lane_sum(s, L);
    *scale_out = 1.f / s;
    return counts;
  }
};

template <typename ET, int V, int NV>
__global__ void __launch_bounds__(kThreads)
balance_rows_kernel(const ET* logits, const int* index, const uint8_t* mask, BalanceShape s, int L, unsigned* ticket,
                    int* tokens_out, int* counts_out, float* psum_out, float* loss) {
  pdl_launch_dependents();
  pdl_wait();
  extern __shared__ int smem[];                       // counts [E], then sums [warps][E]
  float* sums = reinterpret_cast<float*>(smem + s.E);
  __shared__ int warp_tokens[kWarps];
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, l = lane & (L - 1), per_warp = 32 / L;
  for (int e = threadIdx.x; e < s.E; e += kThreads) smem[e] = 0;
  if (blockIdx.x == 0 && blockIdx.y == 0 && threadIdx.x == 0) *ticket = 0;
  __syncthreads();
  const int g = blockIdx.y;
  const long long row0 = (long long)g * s.Tg;
  float acc[V * NV];
#pragma unroll
  for (int i = 0; i < V * NV; ++i) acc[i] = 0.f;
  int n = 0;
  const int stride = (int)gridDim.x * kWarps * per_warp;
  const int first = ((int)blockIdx.x * kWarps + warp) * per_warp;
  // every lane of a warp takes the same number of steps: rows beyond the group's end are rows that do not count
  auto counts = [&](int t) {
    const int at = t + lane / L;
    return at < s.Tg && (mask == nullptr || mask[row0 + at] != 0);
  };
  auto fetch = [&](int t, bool valid, Row<ET, V, NV>& r) {
    r.load(logits + (row0 + (valid ? t + lane / L : 0)) * s.ld, valid, l, L, s.E);
  };
  // The logits of the next step are on their way during this one, and the mask of the one after that.
  Row<ET, V, NV> next;
  bool next_valid = counts(first), after_valid = counts(first + stride);
  fetch(first, next_valid, next);
  for (int t = first; t < s.Tg; t += stride) {
    const Row<ET, V, NV> raw = next;
    const bool valid = next_valid;
    next_valid = after_valid;
    fetch(t + stride, next_valid, next);
    after_valid = counts(t + 2 * stride);
    if (!__any_sync(0xffffffffu, valid)) continue;    // padding, mostly at the ends of sequences
    float m, scale, p[V * NV];
    const bool used = raw.softmax(L, p, &scale, &m) && valid;
    if (used) {
#pragma unroll
      for (int i = 0; i < V * NV; ++i) acc[i] = fmaf(p[i], scale, acc[i]);   // (sums beyond E are never stored)
      n += l == 0;
    }
    auto expert_of = [&](int i) { return (l + (i / V) * L) * V + i % V; };
    if (index != nullptr) {
      if (used)
        for (int c = l; c < s.k; c += L) {
          const int e = index[(row0 + t + lane / L) * s.k + c];
          if ((unsigned)e < (unsigned)s.E) atomicAdd(&smem[e], 1);
        }
      continue;
    }
    // Choices.  The k-th largest distinct logit; with no ties among the k largest the choices are the logits from it on.
    float kth = m;
    for (int c = 1; c < s.k; ++c) {
      float below = -INFINITY;
#pragma unroll
      for (int i = 0; i < V * NV; ++i) below = raw.x[i] < kth ? fmaxf(below, raw.x[i]) : below;
      kth = lane_max(below, L);
    }
    uint32_t chosen = 0;
    const float from = used ? fmaxf(kth, -FLT_MAX) : INFINITY;        // never -infinity; nothing of a row that does not count
#pragma unroll
    for (int i = 0; i < V * NV; ++i) chosen |= raw.x[i] >= from ? 1u << i : 0u;
    if (!used) chosen = 0;
    if (__any_sync(0xffffffffu, lane_sum(__popc(chosen), L) > s.k)) {
      // ties: the largest logit not yet taken, the lowest index among equals, k times
      uint32_t taken = 0;
      for (int c = 0; c < s.k; ++c) {
        float top = -INFINITY;
#pragma unroll
        for (int i = 0; i < V * NV; ++i)
          if (!(taken >> i & 1u)) top = fmaxf(top, raw.x[i]);
        top = lane_max(top, L);
        int best = 0x7fffffff, slot = 0;
#pragma unroll
        for (int i = V * NV - 1; i >= 0; --i)
          if (!(taken >> i & 1u) && raw.x[i] == top) { best = expert_of(i); slot = i; }
        if (lane_min(best, L) == best && top != -INFINITY) taken |= 1u << slot;
      }
      chosen = used ? taken : 0;
    }
    while (chosen != 0) {
      const int i = __ffs(chosen) - 1;
      chosen &= chosen - 1;
      atomicAdd(&smem[expert_of(i)], 1);
    }
  }
  // lanes with the same l of a warp, then the warps in order
  for (int o = L; o < 32; o <<= 1) {
#pragma unroll
    for (int i = 0; i < V * NV; ++i) acc[i] += __shfl_xor_sync(0xffffffffu, acc[i], o);
    n += __shfl_xor_sync(0xffffffffu, n, o);
  }
  if (lane < L) {
#pragma unroll
    for (int i = 0; i < V * NV; ++i) {
      const int e = (l + (i / V) * L) * V + i % V;
      if (e < s.E) sums[warp * s.E + e] = acc[i];
    }
  }
  if (lane == 0) warp_tokens[warp] = n;
  __syncthreads();
  const long long part = (long long)g * gridDim.x + blockIdx.x;
  double term = 0.0;
  for (int e = threadIdx.x; e < s.E; e += kThreads) {
    float p = 0.f;
#pragma unroll
    for (int w = 0; w < kWarps; ++w) p += sums[w * s.E + e];
    counts_out[part * s.E + e] = smem[e];
    if (!s.alone) psum_out[part * s.E + e] = p;
    else term += (double)smem[e] * (double)p;
  }
  int total = 0;
  for (int w = 0; w < kWarps; ++w) total += warp_tokens[w];
  if (threadIdx.x == 0) tokens_out[part] = total;
  if (!s.alone) return;
  // the only block: counts and tokens went to the caller's arrays, and the loss follows from its own sums
  __shared__ double terms[kWarps];
  for (int o = 16; o > 0; o >>= 1) term += __shfl_xor_sync(0xffffffffu, term, o);
  if (lane == 0) terms[warp] = term;
  __syncthreads();
  if (threadIdx.x == 0) {
    term = 0.0;
    for (int w = 0; w < kWarps; ++w) term += terms[w];
    const double n2 = total > 0 ? (double)total * total : 1.0;
    *loss = total > 0 ? (float)((double)s.alpha * s.E * term / (s.k * n2)) : 0.f;
  }
}

// Adds up the blocks of group blockIdx.y for 32 experts: warp w takes the blocks w, w + 32, ..; lane = expert.
__global__ void __launch_bounds__(kFinalThreads)
balance_sum_kernel(const int* tokens_part, const int* counts_part, const float* psum_part, BalanceShape s,
                   unsigned* ticket, float* loss_part, float* loss, int* counts, int* tokens) {
  pdl_launch_dependents();
  pdl_wait();
  __shared__ double p_s[kFinalWarps][32];
  __shared__ int c_s[kFinalWarps][32], n_s[kFinalWarps];
  __shared__ bool last;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, g = blockIdx.y;
  const int e = blockIdx.x * kFinalExperts + lane;
  double p = 0.0;                                     // (a group may have millions of tokens)
  int c = 0, n = 0;
#pragma unroll 4
  for (int b = warp; b < s.blocks; b += kFinalWarps) {
    const long long part = (long long)g * s.blocks + b;
    if (e < s.E) {
      p += (double)psum_part[part * s.E + e];
      c += counts_part[part * s.E + e];
    }
    n += tokens_part[part];
  }
  p_s[warp][lane] = p;
  c_s[warp][lane] = c;
  if (lane == 0) n_s[warp] = n;
  __syncthreads();
  if (warp == 0) {
    p = 0.0; c = 0; n = 0;
    for (int w = 0; w < kFinalWarps; ++w) { p += p_s[w][lane]; c += c_s[w][lane]; n += n_s[w]; }
    if (e < s.E) counts[(long long)g * s.E + e] = c;
    if (blockIdx.x == 0 && lane == 0) tokens[g] = n;
    double term = e < s.E && n > 0 ? (double)c * p : 0.0;
    for (int o = 16; o > 0; o >>= 1) term += __shfl_xor_sync(0xffffffffu, term, o);
    if (lane == 0) {
      const double dn = n > 0 ? (double)n : 1.0;
      loss_part[(long long)g * gridDim.x + blockIdx.x] = (float)((double)s.alpha * s.E * term / (s.k * dn * dn));
      __threadfence();
      last = atomicAdd(ticket, 1u) == gridDim.x * gridDim.y - 1;
    }
  }
  __syncthreads();
  if (!last) return;
  __threadfence();
  // the loss: all parts, in an order that does not depend on which block came last
  const long long parts = (long long)gridDim.x * gridDim.y;
  double sum = 0.0;
  for (long long i = threadIdx.x; i < parts; i += kFinalThreads) sum += (double)__ldcg(loss_part + i);
  for (int o = 16; o > 0; o >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, o);
  __syncthreads();
  if (lane == 0) p_s[warp][0] = sum;
  __syncthreads();
  if (threadIdx.x == 0) {
    sum = 0.0;
    for (int w = 0; w < kFinalWarps; ++w) sum += p_s[w][0];
    *loss = (float)(sum / s.G);
  }
}

template <typename ET, int V, int NV>
__global__ void __launch_bounds__(kThreads, V * NV <= 16 ? 4 : 1)
balance_bwd_kernel(const ET* logits, const uint8_t* mask, const int* counts, const int* tokens, BalanceShape s, int L,
                   float factor, ET* dlogits) {
  pdl_launch_dependents();
  pdl_wait();
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, l = lane & (L - 1), per_warp = 32 / L;
  const int g = blockIdx.y;
  const long long row0 = (long long)g * s.Tg;
  const int n = tokens[g];
  const float up = n > 0 ? factor / ((float)n * (float)n) : 0.f;   // factor = d_loss alpha E / (k groups)
  // p (g - <p, g>) does not change with a constant added to g, as the probabilities sum to one: counted from the first
  // expert's choices, the more even the router, the less cancels (and nothing is left where all are chosen alike).
  const int base = counts[(long long)g * s.E];
  float grad[V * NV];
#pragma unroll
  for (int i = 0; i < V * NV; ++i) {
    const int e = (l + (i / V) * L) * V + i % V;
    grad[i] = e < s.E ? up * (float)(counts[(long long)g * s.E + e] - base) : 0.f;
  }
  const int stride = (int)gridDim.x * kWarps * per_warp;
  const int first = ((int)blockIdx.x * kWarps + warp) * per_warp;
  for (int t = first; t < s.Tg; t += stride) {
    const int at = t + lane / L;
    const bool valid = at < s.Tg && (mask == nullptr || mask[row0 + at] != 0);
    Row<ET, V, NV> r;
    r.load(logits + (row0 + (valid ? at : 0)) * s.ld, valid, l, L, s.E);
    float m, scale = 0.f, dot = 0.f, p[V * NV];
    bool used = false;
    if (__any_sync(0xffffffffu, valid)) {
      used = r.softmax(L, p, &scale, &m) && valid;
#pragma unroll
      for (int i = 0; i < V * NV; ++i) {
        p[i] *= scale;
        dot += p[i] * grad[i];
      }
      dot = lane_sum(dot, L);
    }
    if (at < s.Tg) {
      ET* out = dlogits + (row0 + at) * s.ld;
#pragma unroll
      for (int j = 0; j < NV; ++j) {
        const int p0 = (l + j * L) * V;
        float o[V];
#pragma unroll
        for (int i = 0; i < V; ++i) o[i] = used ? p[j * V + i] * (grad[j * V + i] - dot) : 0.f;
        if (p0 < s.E) Piece<ET, V>::store(out + p0, o);
      }
    }
  }
}

// Calls f with the row layout of a shape: pieces of the most bytes, up to 16, on whose multiples every row starts and ends.
template <typename ET, typename F>
int with_layout(const BalanceShape& s, const void* a, const void* b, F&& f) {
  constexpr int W = 16 / (int)sizeof(ET);
  const uintptr_t at = reinterpret_cast<uintptr_t>(a) | reinterpret_cast<uintptr_t>(b) | (uintptr_t)(s.ld * sizeof(ET)) |
                       (uintptr_t)(s.E * sizeof(ET));
  const int V = at % 16 == 0 ? W : at % (2 * sizeof(ET)) == 0 ? 2 : 1;
  const int pieces = (s.E + V - 1) / V;
  // Few lanes a row, 16 elements each (8 in small pieces), so that the rows of a warp share the steps of its reductions; but
  // at least 64 consecutive bytes.
  int L = 1;
  while (L < 32 && L < pieces && (L * V * (int)sizeof(ET) < 64 || pieces * V > (V == W ? 16 : 8) * L)) L *= 2;
  const int nv = (pieces + L - 1) / L;
  using std::integral_constant;
#define SWMOE_NV(vv, n) \
  if (V == vv && nv <= n) return f(integral_constant<int, vv>{}, integral_constant<int, n>{}, L);
  SWMOE_NV(W, 1) SWMOE_NV(W, 2) SWMOE_NV(W, 4)
  if constexpr (W == 4) { SWMOE_NV(W, 8) }
  SWMOE_NV(2, 1) SWMOE_NV(2, 2) SWMOE_NV(2, 4) SWMOE_NV(2, 16)
  SWMOE_NV(1, 1) SWMOE_NV(1, 2) SWMOE_NV(1, 4) SWMOE_NV(1, 8) SWMOE_NV(1, 32)
#undef SWMOE_NV
  return SWITCH_MOE_UNSUPPORTED_SHAPE;
}

template <typename ET>
int forward(BalanceShape s, const BalancePlan& p, const void* logits, const int32_t* index, const uint8_t* mask,
            float* loss, int32_t* counts, int32_t* tokens, void* ws, cudaStream_t st) {
  unsigned* ticket = ws_ptr<unsigned>(ws, p.ticket);
  int* tp = ws_ptr<int>(ws, p.tokens);
  int* cp = ws_ptr<int>(ws, p.counts);
  float* pp = ws_ptr<float>(ws, p.psum);
  const int rc = with_layout<ET>(s, logits, logits, [&](auto v, auto nv, int L) {
    const size_t smem = (size_t)s.E * 4 * (1 + kWarps);
    // What one block does in four steps of its warps is one block and one launch: the second one takes 2.5 us of host time.
    s.alone = s.G == 1 && s.T <= 4 * kWarps * (32 / L);
    if (s.alone) { s.blocks = 1; tp = tokens; cp = counts; }
    launch_k(balance_rows_kernel<ET, decltype(v)::value, decltype(nv)::value>, dim3(s.blocks, s.G), dim3(kThreads), smem, st,
             static_cast<const ET*>(logits), index, mask, s, L, ticket, tp, cp, pp, loss);
    return launch_status();
  });
  if (rc != SWITCH_MOE_OK || s.alone) return rc;
  launch_k(balance_sum_kernel, dim3((s.E + kFinalExperts - 1) / kFinalExperts, s.G), dim3(kFinalThreads), 0, st,
           static_cast<const int*>(tp), static_cast<const int*>(cp), static_cast<const float*>(pp), s, ticket,
           ws_ptr<float>(ws, p.loss_part), loss, counts, tokens);
  return launch_status();
}

template <typename ET>
int backward(const BalanceShape& s, const void* logits, const uint8_t* mask, const int32_t* counts, const int32_t* tokens,
             float d_loss, void* dlogits, cudaStream_t st) {
  const float factor = (float)((double)d_loss * s.alpha * s.E / ((double)s.k * s.G));
  return with_layout<ET>(s, logits, dlogits, [&](auto v, auto nv, int L) {
    const int rows_per_block = kWarps * (32 / L);
    long long most = ((long long)s.Tg + rows_per_block - 1) / rows_per_block;
    const long long want = ((long long)16 * kChipSms + s.G - 1) / s.G;
    if (most > want) most = want;
    launch_k(balance_bwd_kernel<ET, decltype(v)::value, decltype(nv)::value>, dim3((unsigned)most, s.G), dim3(kThreads), 0, st,
             static_cast<const ET*>(logits), mask, static_cast<const int*>(counts), static_cast<const int*>(tokens), s, L,
             factor, static_cast<ET*>(dlogits));
    return launch_status();
  });
}

}  // namespace
}  // namespace swmoe

using namespace swmoe;

extern "C" int switch_moe_balance_workspace_bytes(const switch_moe_balance_config* cfg, size_t* bytes_out) {
  if (bytes_out == nullptr) return SWITCH_MOE_INVALID_ARGUMENT;
  BalanceShape s;
  const int rc = resolve(cfg, &s);
  if (rc != SWITCH_MOE_OK) return rc;
  BalancePlan p;
  make_plan(s, &p);
  *bytes_out = p.total;
  return SWITCH_MOE_OK;
}

extern "C" int switch_moe_balance_fwd(const switch_moe_balance_config* cfg, const void* logits,
                                      const int32_t* expert_index, const uint8_t* token_mask, float* loss,
                                      int32_t* counts, int32_t* tokens, void* workspace, size_t workspace_bytes,
                                      void* stream) {
  BalanceShape s;
  const int rc = resolve(cfg, &s);
  if (rc != SWITCH_MOE_OK) return rc;
  BalancePlan p;
  make_plan(s, &p);
  if ((logits == nullptr && s.T > 0) || loss == nullptr || counts == nullptr || tokens == nullptr || workspace == nullptr)
    return SWITCH_MOE_INVALID_ARGUMENT;
  if ((reinterpret_cast<uintptr_t>(workspace) & 1023u) != 0 || (reinterpret_cast<uintptr_t>(logits) & (s.f32 ? 3u : 1u)) != 0)
    return SWITCH_MOE_UNSUPPORTED_SHAPE;
  if (workspace_bytes < p.total) return SWITCH_MOE_WORKSPACE_TOO_SMALL;
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  return s.f32 ? forward<float>(s, p, logits, expert_index, token_mask, loss, counts, tokens, workspace, st)
               : forward<__nv_bfloat16>(s, p, logits, expert_index, token_mask, loss, counts, tokens, workspace, st);
}

extern "C" int switch_moe_balance_bwd(const switch_moe_balance_config* cfg, const void* logits, const uint8_t* token_mask,
                                      const int32_t* counts, const int32_t* tokens, float d_loss, void* dlogits,
                                      void* stream) {
  BalanceShape s;
  const int rc = resolve(cfg, &s);
  if (rc != SWITCH_MOE_OK) return rc;
  if (s.T == 0) return SWITCH_MOE_OK;
  if (logits == nullptr || counts == nullptr || tokens == nullptr || dlogits == nullptr) return SWITCH_MOE_INVALID_ARGUMENT;
  if (((reinterpret_cast<uintptr_t>(logits) | reinterpret_cast<uintptr_t>(dlogits)) & (s.f32 ? 3u : 1u)) != 0)
    return SWITCH_MOE_UNSUPPORTED_SHAPE;
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  return s.f32 ? backward<float>(s, logits, token_mask, counts, tokens, d_loss, dlogits, st)
               : backward<__nv_bfloat16>(s, logits, token_mask, counts, tokens, d_loss, dlogits, st);
}
