// Dropout masks from a counter: what switch_moe.h states under "Dropout", for every kernel that applies one.
// Philox4x32-10 (Salmon, Moraes, Dror and Shaw, "Parallel random numbers: as easy as 1, 2, 3", 2011), one call for eight
// elements: 16 bits decide an element, so a rate is a multiple of 1/65536, and the generator's cost per element is a
// quarter of a call with 32 bits each.
#pragma once

#include "switch_common.cuh"

namespace swmoe {

constexpr float kDropoutUnit = 65536.f;
constexpr int kMaxExtent = 1 << 30;     // of a dimension: places in a tile or a step past the last one still fit 32 bits

struct DropoutParams {
  const unsigned long long* rng;   // DEVICE {key, offset}; null: no dropout
  uint32_t threshold;              // q << 16: an element is kept if its 16 bits, in the upper half of a word, reach it
  uint32_t site;                   // << 16
  float scale;                     // 65536 / (65536 - q)
};

// q of a rate in [0, 1), or -1 for a rate that is none.
inline int dropout_threshold(float rate) {
  if (!(rate >= 0.f && rate < 1.f)) return -1;
  const int q = (int)((double)rate * 65536.0 + 0.5);
  return q < 65536 ? q : -1;
}

inline DropoutParams dropout_params(const uint64_t* rng, int q, int site) {
  DropoutParams d{};
  d.rng = q > 0 ? reinterpret_cast<const unsigned long long*>(rng) : nullptr;
  d.threshold = (uint32_t)q << 16;
  d.site = (uint32_t)site << 16;
  d.scale = kDropoutUnit / (kDropoutUnit - (float)q);
  return d;
}

#ifdef __CUDACC__
struct DropoutState {
  uint32_t k0[10], k1[10], o0, o1;                   // the rounds' keys; the counter's upper half
};

__device__ __forceinline__ DropoutState dropout_state(const DropoutParams& d) {
  unsigned long long key = 0, off = 0;
  if (d.rng != nullptr) {
    key = d.rng[0];
    off = d.rng[1];
  }
  DropoutState s;
#pragma unroll
  for (int r = 0; r < 10; ++r) {
    s.k0[r] = (uint32_t)key + (uint32_t)r * 0x9E3779B9u;
    s.k1[r] = (uint32_t)(key >> 32) + (uint32_t)r * 0xBB67AE85u;
  }
  s.o0 = (uint32_t)off;
  s.o1 = (uint32_t)(off >> 32);
  return s;
}

// The 128 bits of eight elements; `block` = row . ceil(columns / 8) + column / 8.
__device__ __forceinline__ uint4 dropout_bits(const DropoutParams& d, const DropoutState& s, unsigned long long block) {
  uint32_t c0 = (uint32_t)block, c1 = (uint32_t)(block >> 32) + d.site, c2 = s.o0, c3 = s.o1;
#pragma unroll
  for (int r = 0; r < 10; ++r) {
    const unsigned long long a = (unsigned long long)c0 * 0xD2511F53u, b = (unsigned long long)c2 * 0xCD9E8D57u;
    c0 = (uint32_t)(b >> 32) ^ c1 ^ s.k0[r];
    c1 = (uint32_t)b;
    c2 = (uint32_t)(a >> 32) ^ c3 ^ s.k1[r];
    c3 = (uint32_t)a;
  }
  return make_uint4(c0, c1, c2, c3);
}

// Eight values after dropout.  A dropped one is 0 whatever it was (an infinity or a NaN too).
__device__ __forceinline__ void dropout8(const DropoutParams& d, const uint4& bits, float* v) {
  const uint32_t w[4] = {bits.x, bits.y, bits.z, bits.w};
#pragma unroll
  for (int i = 0; i < 8; ++i)
    v[i] = ((i & 1) ? w[i >> 1] : w[i >> 1] << 16) >= d.threshold ? v[i] * d.scale : 0.f;
}
#endif

}  // namespace swmoe
