// The products of the dense layer on pairs of SMs (tcgen05 cta_group::2, M = 256): y = x W with bias, activation, dropout
// and residual in its epilogue, dx = dz W^T, dW = x^T dz.
//
// A CTA pair works on tiles of 256 x TN outputs (TN 256, or 192 or 128 where that fills the chip better); each CTA stages its own
// 128 rows of A and half of B's columns per 64-deep block of the contraction by TMA, the leader's MMA warp issues the
// instructions for both, and sixteen epilogue warps of each CTA drain its 128 accumulator lanes (a lane = an output row)
// while the next tile's products run in the other half of tensor memory.  A warp has 32 rows and a quarter of the columns,
// and works on its own: 32 columns at a time from tensor memory through the epilogue into 64-byte-swizzled shared memory,
// and from there by TMA, which also brings the residual into the very buffer that the result leaves from and clips what is
// outside (a store in whole 16-byte pieces: the last columns of a row that does not end on one are written element by
// element).  With GELU the epilogue is bound by latency (32768 x 768 x 2048, z saved: eight warps 169 us, sixteen 120, at 0.5
// instructions a cycle and scheduler), hence sixteen.
//
// Sums of bfloat16 products stay in the tensor pipe over the whole contraction, which truncates each addition to float32: 2^-23
// a step of 16, far below the result's rounding unless thousands of steps cancel.
//
// Float32 operands come as three bfloat16 parts (x 2^24 = h + m + l, exact); of the nine cross products six are formed,
// the others are below 2^-25 of the product.  The tensor pipe adds with truncation, so an accumulator lives for one block
// of 64 steps only (the corrections first, h.h last) and is then added to a float32 sum in registers, round to nearest.
// Results that are not finite are formed again by fused multiply-adds from the float32 operands (operands from 2^104 on
// and sums from 2^80 on end there too).  Its wide tiles hold up to 64 sums a thread and spill 88 (192 columns) to 144 bytes.
//
// Every wait is bounded in time; after one gave up all roles leave.
#include <algorithm>
#include <cmath>

#include "linear_common.cuh"
#include "tc_common.cuh"

namespace swmoe {
using namespace tc;
namespace {

constexpr int kEpiWarps = 16;
constexpr int kThreads = 64 + 32 * kEpiWarps;        // TMA, MMA, epilogue
constexpr int kABlock = 16384;                       // 128 rows x 64 steps of bfloat16
constexpr int kBufferBytes = 32 * 64;                // 32 rows x 64 bytes of output
constexpr int kWarpStage = 2 * kBufferBytes;
constexpr int kStagingBytes = kEpiWarps * kWarpStage;
constexpr int kRingBytes = 163840;
constexpr int kMaxRing = 8;
constexpr int kBiasBytes = kEpiWarps * 32 * 4;
constexpr int kBarBytes = 512;
constexpr int kSmem = kRingBytes + kStagingBytes + kBiasBytes + kBarBytes;
static_assert(kSmem <= 232448, "shared memory of a block");
constexpr uint32_t kPeer = 0xFEFFFFFFu;              // clears the CTA-rank bit of a shared::cluster address
constexpr int kBand = 8;                             // row tiles that are walked together along the columns

enum Mode { kBf16 = 0, kPartial = 1, kF32 = 2 };     // bf16 -> bf16; bf16 -> float32 part sums; float32 parts -> float32

struct DenseParams {
  int rows, cols, k_blocks;
  int m_tiles, n_tiles, splits, k_per_split;
  long long k;
  int activation, dropout_blocks;
  int has_residual, has_pre;
  const float* bias;
  DropoutParams dropout;
  const float* a; long long a_si, a_sk;
  const float* b; long long b_si, b_sk;
  int whole_cols;                                    // columns in whole 16-byte pieces: a TMA store clips at these, the rest
  void* out; void* pre; const void* residual; long long ld_out, split_out; // of a row is written by the threads themselves
  int* status;
  int clear_status;
};

struct DenseMaps {
  CUtensorMap a, b, out, pre, residual;
};

__device__ __forceinline__ uint32_t cta_rank() {
  uint32_t r;
  asm volatile("mov.u32 %0, %%cluster_ctarank;" : "=r"(r));
  return r;
}
__device__ __forceinline__ void cluster_sync() {
  asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory");
  asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory");
}
__device__ __forceinline__ void arrive_at(uint32_t local_bar, uint32_t cta) {
  asm volatile(
      "{\n\t.reg .b32 ra;\n\t"
      "mapa.shared::cluster.u32 ra, %0, %1;\n\t"
      "mbarrier.arrive.shared::cluster.b64 _, [ra];\n\t}" ::"r"(local_bar), "r"(cta) : "memory");
}
__device__ __forceinline__ void store_at(uint32_t local, uint32_t cta, uint32_t v) {
  asm volatile(
      "{\n\t.reg .b32 ra;\n\t"
      "mapa.shared::cluster.u32 ra, %0, %1;\n\t"
      "st.volatile.shared::cluster.u32 [ra], %2;\n\t}" ::"r"(local), "r"(cta), "r"(v) : "memory");
}
__device__ __forceinline__ void load_pair(uint32_t dst, const CUtensorMap* tm, uint32_t leader_bar, int c0, int c1, int c2) {
  asm volatile(
      "cp.async.bulk.tensor.3d.cta_group::2.shared::cluster.global.mbarrier::complete_tx::bytes"
      " [%0], [%1, {%3, %4, %5}], [%2];" ::"r"(dst), "l"(reinterpret_cast<uint64_t>(tm)), "r"(leader_bar), "r"(c0), "r"(c1),
      "r"(c2) : "memory");
}
__device__ __forceinline__ void store_box(const CUtensorMap* tm, uint32_t src, int c0, int c1, int c2) {
  asm volatile("cp.async.bulk.tensor.3d.global.shared::cta.bulk_group [%0, {%2, %3, %4}], [%1];" ::"l"(
                   reinterpret_cast<uint64_t>(tm)), "r"(src), "r"(c0), "r"(c1), "r"(c2) : "memory");
}
__device__ __forceinline__ void commit_pair(uint32_t bar) {
  asm volatile(
      "tcgen05.commit.cta_group::2.mbarrier::arrive::one.shared::cluster.multicast::cluster.b64 [%0], %1;" ::"r"(bar),
      "h"((uint16_t)3) : "memory");
}
__device__ __forceinline__ void mma_pair(uint32_t d, uint64_t a, uint64_t b, uint32_t idesc, uint32_t accumulate) {
  asm volatile(
      "{\n\t.reg .pred p;\n\t"
      "setp.ne.b32 p, %4, 0;\n\t"
      "tcgen05.mma.cta_group::2.kind::f16 [%0], %1, %2, %3, p;\n\t}" ::"r"(d), "l"(a), "l"(b), "r"(idesc), "r"(accumulate)
      : "memory");
}
// Registers pass through so that no use of them moves ahead of the wait.
__device__ __forceinline__ void wait_ld(uint32_t* r) {
  asm volatile("tcgen05.wait::ld.sync.aligned;"
               : "+r"(r[0]), "+r"(r[1]), "+r"(r[2]), "+r"(r[3]), "+r"(r[4]), "+r"(r[5]), "+r"(r[6]), "+r"(r[7]),
                 "+r"(r[8]), "+r"(r[9]), "+r"(r[10]), "+r"(r[11]), "+r"(r[12]), "+r"(r[13]), "+r"(r[14]), "+r"(r[15]),
                 "+r"(r[16]), "+r"(r[17]), "+r"(r[18]), "+r"(r[19]), "+r"(r[20]), "+r"(r[21]), "+r"(r[22]), "+r"(r[23]),
                 "+r"(r[24]), "+r"(r[25]), "+r"(r[26]), "+r"(r[27]), "+r"(r[28]), "+r"(r[29]), "+r"(r[30]), "+r"(r[31])
               :: "memory");
}
__device__ __forceinline__ uint32_t pack2_bf16(float lo, float hi) {
  const __nv_bfloat162 h = __floats2bfloat162_rn(lo, hi);
  return *reinterpret_cast<const uint32_t*>(&h);
}

// The columns of a piece of eight that belong to no whole 16 bytes of the row.
template <bool kOut4>
__device__ __forceinline__ void store_ragged(const DenseParams& p, void* base, long long at, int col, const float* x) {
#pragma unroll
  for (int i = 0; i < 8; ++i)
    if (col + i >= p.whole_cols && col + i < p.cols) {
      if (kOut4) static_cast<float*>(base)[at + i] = x[i];
      else static_cast<__nv_bfloat16*>(base)[at + i] = __float2bfloat16(x[i]);
    }
}

struct Unit {
  int m0, n0, split, kb0, kb1;
};
// Bands of kBand row tiles, walked column by column, so that what runs at one time shares rows of A and columns of B.
__device__ __forceinline__ Unit decode(const DenseParams& p, int id, int TN) {
  Unit u;
  const int tiles = p.m_tiles * p.n_tiles;
  u.split = id / tiles;
  const int t = id - u.split * tiles, per_band = kBand * p.n_tiles, band = t / per_band, r = t - band * per_band;
  const int height = min(kBand, p.m_tiles - band * kBand), n = r / height;
  u.m0 = (band * kBand + r - n * height) * 256;
  u.n0 = n * TN;
  u.kb0 = u.split * p.k_per_split;
  u.kb1 = min(p.k_blocks, u.kb0 + p.k_per_split);
  return u;
}

template <bool kAMn, bool kBMn, int TN, int kMode>
__global__ void __cluster_dims__(2, 1, 1) __launch_bounds__(kThreads, 1)
dense_gemm_kernel(const __grid_constant__ DenseMaps maps, const __grid_constant__ DenseParams p) {
  constexpr bool kFwd = !kAMn && kBMn && kMode != kPartial;  // the only product with an epilogue of its own
  constexpr bool kOut4 = kMode != kBf16;                     // float32 output
  // This CTA's half of B: TN / 2 columns x 64 steps (n-major in boxes of 64 columns, of which TN = 192 uses one and a half)
  constexpr int kBBoxes = (TN / 2 + 63) / 64, kBBytes = kBMn ? kBBoxes * kAtomBytes : TN * 64;
  constexpr int kStage = kABlock + kBBoxes * kAtomBytes;
  constexpr int kStages = kRingBytes / kStage < kMaxRing ? kRingBytes / kStage : kMaxRing;
  constexpr int kParts = kMode == kF32 ? 3 : 1;              // of a block of 64 steps; a stage holds one part of A and of B
  pdl_launch_dependents();
  extern __shared__ __align__(1024) uint8_t gen[];           // (all of an SM's shared memory: no room to align it by hand)
  const uint32_t base = smem_u32(gen);
  float* bias_s = reinterpret_cast<float*>(gen + kRingBytes + kStagingBytes);
  uint8_t* bar_gen = gen + kRingBytes + kStagingBytes + kBiasBytes;
  const uint32_t bars = base + kRingBytes + kStagingBytes + kBiasBytes;
  // full[8] | empty[8] | acc_full[2] | acc_empty[2] | tmem | abort, progress | .. | residual[16 warps x 2]
  const uint32_t full0 = bars, empty0 = bars + 64u, afull0 = bars + 128u, aempty0 = bars + 144u, res0 = bars + 256u;
  volatile uint32_t* tmem_s = reinterpret_cast<volatile uint32_t*>(bar_gen + 160);
  volatile int* abort_flag = reinterpret_cast<volatile int*>(bar_gen + 168);
  const uint32_t progress = bars + 172u;
  const int warp = uniform_warp_id(), lane = threadIdx.x & 31;
  const uint32_t rank = __shfl_sync(0xffffffffu, cta_rank(), 0);
  if (threadIdx.x == 0) {
    for (int s = 0; s < kMaxRing; ++s) { mbar_init(full0 + 8u * s, 1); mbar_init(empty0 + 8u * s, 1); }
    for (int a = 0; a < 2; ++a) { mbar_init(afull0 + 8u * a, 1); mbar_init(aempty0 + 8u * a, 2 * kEpiWarps); }
    for (int a = 0; a < 2 * kEpiWarps; ++a) mbar_init(res0 + 8u * a, 1);
    abort_flag[0] = 0;
    abort_flag[1] = 0;
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
  }
  if (warp == 2) {
    asm volatile("tcgen05.alloc.cta_group::2.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(
                     smem_u32(const_cast<uint32_t*>(tmem_s))), "r"(kTmemCols) : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::2.sync.aligned;" ::: "memory");
  }
  pdl_wait();
  if (p.clear_status && blockIdx.x == 0 && threadIdx.x < kStatusWords) p.status[threadIdx.x] = 0;
  tc_fence_before();
  cluster_sync();
  tc_fence_after();
  const uint32_t tmem = *tmem_s;
  const int n_units = p.m_tiles * p.n_tiles * p.splits, pair = blockIdx.x >> 1, n_pairs = gridDim.x >> 1;
  constexpr bool kProgress = kMode == kF32;                  // redone results take their time

  if (warp == 0) {
    // ------------------------------------------------------------------------------------------ loads (both CTAs)
    uint32_t stage = 0, phase = 0;
    bool ok = true;
    for (int id = pair; id < n_units && ok; id += n_pairs) {
      const Unit u = decode(p, id, TN);
      const int am = u.m0 + 128 * (int)rank, bn = u.n0 + TN / 2 * (int)rank;
#pragma unroll 1
      for (int kb = u.kb0; kb < u.kb1 && ok; ++kb) {
#pragma unroll 1
        for (int part = kParts - 1; part >= 0; --part) {     // low, middle, high
          ok = mbar_wait_warp<kProgress>(empty0 + 8u * stage, phase ^ 1u, abort_flag, p.status, 41);
          if (!ok) break;
          const uint32_t a_dst = base + stage * kStage, b_dst = a_dst + kABlock, fb = full0 + 8u * stage;
          const uint32_t lead = fb & kPeer;                  // both CTAs' bytes count on the leader's barrier
          const int k0 = kb * kBK;
          if (elect_one()) {
            if (rank == 0) mbar_arrive_expect_tx(fb, 2u * (kABlock + kBBytes));
            if (kAMn) {
              load_pair(a_dst, &maps.a, lead, am, k0, part);
              load_pair(a_dst + kAtomBytes, &maps.a, lead, am + 64, k0, part);
            } else {
              load_pair(a_dst, &maps.a, lead, k0, am, part);
            }
            if (kBMn) {
              load_pair(b_dst, &maps.b, lead, bn, k0, part);
              if (kBBoxes > 1) load_pair(b_dst + kAtomBytes, &maps.b, lead, bn + 64, k0, part);
            } else {
              load_pair(b_dst, &maps.b, lead, k0, bn, part);
            }
          }
          if (++stage == kStages) { stage = 0; phase ^= 1u; }
        }
      }
    }
    if (*abort_flag != 0) {
      const long long t0 = clock64();
      while (clock64() - t0 < 4000000ll) __nanosleep(1000);  // let copies in flight land (about 2 ms)
    }
  } else if (warp == 1) {
    // ------------------------------------------------------------------------------------------ products (leader CTA)
    if (rank == 0) {
      constexpr uint32_t idesc = (1u << 4) | (1u << 7) | (1u << 10) | ((uint32_t)kAMn << 15) | ((uint32_t)kBMn << 16) |
                                 ((uint32_t)(TN >> 3) << 17) | ((uint32_t)(256 >> 4) << 24);
      constexpr uint32_t a_step = (kAMn ? kUmmaK * 128u : kUmmaK * 2u) >> 4, b_step = (kBMn ? kUmmaK * 128u : kUmmaK * 2u) >> 4;
      const uint64_t a_desc = make_smem_desc(base, kAMn ? kAtomBytes : 16u, 1024u);
      const uint64_t b_desc = make_smem_desc(base + kABlock, kBMn ? kAtomBytes : 16u, 1024u);
      uint32_t stage = 0, phase = 0, it = 0;
      bool ok = true;
      for (int id = pair; id < n_units && ok; id += n_pairs) {
        const Unit u = decode(p, id, TN);
        uint32_t d = 0;
#pragma unroll 1
        for (int kb = u.kb0; kb < u.kb1 && ok; ++kb) {
          const bool first = kMode == kF32 || kb == u.kb0, done = kMode == kF32 || kb == u.kb1 - 1;
          const uint32_t side = it & 1u;
          if (first) {                                       // this half's previous accumulator has been read out
            ok = mbar_wait_warp<kProgress>(aempty0 + 8u * side, ((it >> 1) & 1u) ^ 1u, abort_flag, p.status, 42);
            if (!ok) break;
            tc_fence_after();
            d = tmem + side * 256u;
          }
          auto desc_at = [&](uint64_t d0, uint32_t s) { return d0 + (uint64_t)(s * (kStage >> 4)); };
          auto multiply = [&](uint32_t sa, uint32_t sb, uint32_t acc) {      // one elected lane
            const uint64_t ad = desc_at(a_desc, sa), bd = desc_at(b_desc, sb);
#pragma unroll
            for (int ks = 0; ks < kBK / kUmmaK; ++ks)
              mma_pair(d, ad + ks * a_step, bd + ks * b_step, idesc, ks > 0 ? 1u : acc);
          };
          auto arrived = [&](uint32_t s, uint32_t ph) {
            ok = ok && mbar_wait_warp<kProgress>(full0 + 8u * s, ph, abort_flag, p.status, 43);
            tc_fence_after();
          };
          if constexpr (kMode != kF32) {
            arrived(stage, phase);
            if (!ok) break;
            if (elect_one()) {
              multiply(stage, stage, first ? 0u : 1u);
              commit_pair(empty0 + 8u * stage);
              if (done) commit_pair(afull0 + 8u * side);
            }
            if (++stage == kStages) { stage = 0; phase ^= 1u; }
          } else {
            // Six of the nine part products; a part is loaded once and released after its last: the low one after half of
            // the block, so that the next block's is there in time.  (Loaded anew for every product, 24 or 32 KB per 256
            // or 512 cycles of the tensor pipe, they took longer: 4001 tokens, 512 x 2048, GELU, a training step 234 us, so 205.)
            uint32_t s[3], ph[3];
#pragma unroll
            for (int i = 0; i < 3; ++i) {
              s[i] = stage; ph[i] = phase;
              if (++stage == kStages) { stage = 0; phase ^= 1u; }
            }
            arrived(s[1], ph[1]);
            if (!ok) break;
            if (elect_one()) multiply(s[1], s[1], 0u);                       // m.m
            arrived(s[0], ph[0]);
            arrived(s[2], ph[2]);
            if (!ok) break;
            if (elect_one()) {
              multiply(s[2], s[0], 1u);                                      // h.l
              multiply(s[0], s[2], 1u);                                      // l.h
              commit_pair(empty0 + 8u * s[0]);
              multiply(s[2], s[1], 1u);                                      // h.m
              multiply(s[1], s[2], 1u);                                      // m.h
              commit_pair(empty0 + 8u * s[1]);
              multiply(s[2], s[2], 1u);                                      // h.h
              commit_pair(empty0 + 8u * s[2]);
              commit_pair(afull0 + 8u * side);
            }
          }
          if (done) ++it;
        }
      }
    }
  } else {
    // ------------------------------------------------------------------------------------------ epilogue (both CTAs)
    const int lg = warp & 3, ew = warp - 2, quarter = ew >> 2;
    uint8_t* stage_g = gen + kRingBytes + ew * kWarpStage;
    const uint32_t stage_s = base + kRingBytes + (uint32_t)(ew * kWarpStage);
    float* bias_w = bias_s + 32 * ew;
    const uint32_t res_bar = res0 + 16u * ew;
    const uint32_t row_off = (uint32_t)lane * 64u, sw = (uint32_t)(lane >> 1) & 3u;
    const bool pre = kFwd && p.has_pre, residual = kFwd && p.has_residual;
    DropoutState rng{};
    if (kFwd) rng = dropout_state(p.dropout);
    uint32_t it = 0, n_block = 0, res_phase = 0;             // res_phase: a bit per buffer
    bool ok = true;
    // Bias, then (once `saved` has been called with z) activation and dropout of 32 columns of this thread's row.  Step after
    // step over all of them, not column after column: a store to shared memory between two columns would keep the second
    // one's loads behind it, and the warps (four a scheduler) wait for their own results often enough.
    auto finish = [&](float* x, long long row, int col, auto&& saved) {
      if constexpr (kFwd) {
        if (p.bias != nullptr) {
#pragma unroll
          for (int i = 0; i < 32; i += 4) {
            const float4 b = *reinterpret_cast<const float4*>(bias_w + i);
            x[i] += b.x; x[i + 1] += b.y; x[i + 2] += b.z; x[i + 3] += b.w;
          }
        }
        if (pre) saved(x);
        if (p.activation == SWITCH_MOE_ACT_RELU) {
#pragma unroll
          for (int i = 0; i < 32; ++i) x[i] = max_nan(x[i], 0.f);
        } else if (p.activation == SWITCH_MOE_ACT_GELU) {
#pragma unroll
          for (int i = 0; i < 32; i += 2) gelu_pair(x + i, x + i + 1);
        }
        if (p.dropout.rng != nullptr) {
          const unsigned long long block = (unsigned long long)row * (unsigned)p.dropout_blocks + (unsigned)(col >> 3);
#pragma unroll
          for (int i = 0; i < 4; ++i) dropout8(p.dropout, dropout_bits(p.dropout, rng, block + i), x + 8 * i);
        }
      }
    };
    // Of a tile's blocks of 32 columns this warp has every fourth: one or two.
    constexpr int kMost = (TN / 32 + 3) / 4;
    const int n_blocks = TN == 192 ? (quarter < 2 ? 2 : 1) : kMost;
    const int row_in = 128 * (int)rank + 32 * lg, col_in = quarter * 32;     // this warp's place in a tile
    // The residual of the block after the one at hand is asked for ahead (unless z takes the other buffer).
    const bool ahead = residual && !pre && !kOut4;
    auto fetch_residual = [&](uint32_t b, int c0, int r0) {  // one lane
      const uint32_t rb = res_bar + (b ? 8u : 0u);
      mbar_arrive_expect_tx(rb, kBufferBytes);
      tma_load_3d(stage_s + b, &maps.residual, rb, c0, r0, 0);
    };
    auto fetch_after = [&](int id, int b, uint32_t buffer) { // that of the next block inside, from block b of unit id on
      for (; id < n_units; id += n_pairs, b = 0) {
        const Unit u = decode(p, id, TN);
        for (; b < n_blocks; ++b)
          if (u.n0 + col_in + 128 * b < p.cols && u.m0 + row_in < p.rows) {
            if (lane == 0) fetch_residual(buffer, u.n0 + col_in + 128 * b, u.m0 + row_in);
            return;
          }
      }
    };
    if (ahead) fetch_after(pair, 0, 0u);
    for (int id = pair; id < n_units && ok; id += n_pairs) {
      const Unit u = decode(p, id, TN);
      const int row0 = u.m0 + row_in, n0 = u.n0 + col_in;
      float bias_r[kMost];                                   // on its way while the accumulator is awaited
#pragma unroll
      for (int b = 0; b < kMost; ++b)
        bias_r[b] = kFwd && p.bias != nullptr && n0 + 128 * b + lane < p.cols ? p.bias[n0 + 128 * b + lane] : 0.f;
      const long long row = row0 + lane;
      const uint32_t taddr0 = tmem + ((uint32_t)(lg * 32) << 16) + quarter * 32;
      float sum[kMode == kF32 ? 32 * kMost : 1];
      if constexpr (kMode == kF32) {                         // blocks of the contraction are added up in registers
#pragma unroll
        for (int i = 0; i < 32 * kMost; ++i) sum[i] = 0.f;
        for (int kb = u.kb0; kb < u.kb1; ++kb, ++it) {
          const uint32_t side = it & 1u;
          ok = mbar_wait_warp<true>(afull0 + 8u * side, (it >> 1) & 1u, abort_flag, p.status, 44);
          if (!ok) break;
          tc_fence_after();
#pragma unroll
          for (int b = 0; b < kMost; ++b) {
            if (b >= n_blocks) break;
            uint32_t v[32];
            tc_ld32(taddr0 + side * 256u + 128u * b, v);
            wait_ld(v);
            if (b == n_blocks - 1) {
              tc_fence_before();
              __syncwarp();
              if (lane == 0) arrive_at(aempty0 + 8u * side, 0);
            }
#pragma unroll
            for (int i = 0; i < 32; ++i) sum[32 * b + i] += __uint_as_float(v[i]);
          }
        }
      } else {
        ok = mbar_wait_warp(afull0 + 8u * (it & 1u), (it >> 1) & 1u, abort_flag, p.status, 44);
        tc_fence_after();
      }
      if (!ok) break;
      // One copy of this loop's code, not one per block: unrolled, it streams through the instruction caches (32768 tokens,
      // 768 x 2048, GELU: 199 us against 169 with eight warps).
#pragma unroll 1
      for (int b = 0; b < n_blocks; ++b) {
        const int col0 = n0 + 128 * b;
        const bool inside = col0 < p.cols && row0 < p.rows;  // the same in the whole warp
        // bf16: a block is one buffer of 64-byte rows; with pre the results use the first and z the second.  Float32: both.
        const uint32_t buf = pre || kOut4 ? 0u : (n_block & 1u) * kBufferBytes;
        uint32_t v[32];
        if constexpr (kMode != kF32) tc_ld32(taddr0 + (it & 1u) * 256u + 128u * b, v);
        auto buffers_read = [&] {                            // this block's (and with `ahead` the next one's) buffers have
          if (pre || kOut4 || ahead) asm volatile("cp.async.bulk.wait_group.read 0;" ::: "memory");   // been read by their
          else asm volatile("cp.async.bulk.wait_group.read 1;" ::: "memory");                         // last stores
        };
        if (inside) {
          if (residual && !kOut4 && lane == 0) {             // (else: when the accumulator is there, below)
            buffers_read();
            if (!ahead) fetch_residual(buf, col0, row0);
          }
          if (ahead) fetch_after(id, b + 1, buf ^ kBufferBytes);
          if (kFwd && p.bias != nullptr) bias_w[lane] = b == 0 ? bias_r[0] : bias_r[kMost - 1];
          __syncwarp();
        }
        if constexpr (kMode != kF32) {
          wait_ld(v);
          if (b == n_blocks - 1) {                           // the accumulator has been read out
            tc_fence_before();
            __syncwarp();
            if (lane == 0) arrive_at(aempty0 + 8u * (it & 1u), 0);
          }
        }
        if (!inside) continue;
        // Without a residual the buffers are not needed before the first value is written: their last stores have all of the
        // block's arithmetic to be read in (16384 tokens, 768 x 2048, bias and z saved: 52 us with the wait up here, 47 with it
        // there; GELU 48 and 42, dropout 49 and 43).
        const bool wait_late = !residual || kOut4;
        auto wait_now = [&] {
          if (wait_late) {
            if (lane == 0) buffers_read();
            __syncwarp();
          }
        };
        if (residual && !kOut4) {
          const uint32_t bit = buf ? 2u : 1u;
          ok = mbar_wait_warp(res_bar + (buf ? 8u : 0u), (res_phase & bit) ? 1u : 0u, abort_flag, p.status, 45);
          res_phase ^= bit;
          if (!ok) break;
        }
        uint8_t* const dst = stage_g + buf + row_off;
        auto piece_at = [&](int j) -> float4* {              // float32: 16-byte piece j (0 .. 7) of the row's 32 columns
          return reinterpret_cast<float4*>(stage_g + (j >> 2) * kBufferBytes + row_off + (((uint32_t)(j & 3) ^ sw) << 4));
        };
        const bool edge = col0 + 32 > p.whole_cols && row < p.rows;     // columns that belong to no whole 16 bytes
        float x[32];
        if constexpr (kMode == kF32) {
          bool finite = true;
#pragma unroll
          for (int i = 0; i < 32; ++i) {
            x[i] = (kMost == 1 || b == 0 ? sum[i] : sum[kMost == 1 ? 0 : 32 + i]) * kPartDown;
            finite = finite && isfinite(x[i]);
          }
          const bool again_here = !finite && row < p.rows;
          if (__any_sync(0xffffffffu, again_here)) {
            if (lane == 0) buffers_read();                   // (they are written now)
            __syncwarp();
          }
          if (again_here) {                                  // formed again, by way of this thread's row of the buffers
#pragma unroll
            for (int j = 0; j < 8; ++j) *piece_at(j) = make_float4(x[4 * j], x[4 * j + 1], x[4 * j + 2], x[4 * j + 3]);
            const float* pa = p.a + row * p.a_si;
            const long long k1 = min(p.k, (long long)u.kb1 * kBK);
#pragma unroll 1
            for (int i = 0; i < 32 && col0 + i < p.cols; ++i) {
              float* at = reinterpret_cast<float*>(piece_at(i >> 2)) + (i & 3);
              if (isfinite(*at)) continue;
              float again = 0.f;
              const float* pb = p.b + (long long)(col0 + i) * p.b_si;
              for (long long k = (long long)u.kb0 * kBK; k < k1; ++k) again = fmaf(pa[k * p.a_sk], pb[k * p.b_sk], again);
              *at = again;
              for (uint32_t cta = 0; cta < 2; ++cta)         // the waiting warps of both CTAs see that work goes on
                store_at(progress, cta, (uint32_t)clock64());
            }
#pragma unroll
            for (int j = 0; j < 8; ++j) {
              const float4 f = *piece_at(j);
              x[4 * j] = f.x; x[4 * j + 1] = f.y; x[4 * j + 2] = f.z; x[4 * j + 3] = f.w;
            }
          }
          __syncwarp();
        } else {
#pragma unroll
          for (int i = 0; i < 32; ++i) x[i] = __uint_as_float(v[i]);
        }
        auto at16 = [&](uint8_t* row_at, int j) { return reinterpret_cast<uint4*>(row_at + (((uint32_t)j ^ sw) << 4)); };
        auto put = [&](uint8_t* row_at, const float* f) {    // bf16: four pieces of 16 bytes; float32: eight, in both buffers
          if constexpr (kOut4) {
#pragma unroll
            for (int j = 0; j < 8; ++j) *piece_at(j) = make_float4(f[4 * j], f[4 * j + 1], f[4 * j + 2], f[4 * j + 3]);
          } else {
#pragma unroll
            for (int j = 0; j < 4; ++j)
              *at16(row_at, j) = make_uint4(pack2_bf16(f[8 * j], f[8 * j + 1]), pack2_bf16(f[8 * j + 2], f[8 * j + 3]),
                                            pack2_bf16(f[8 * j + 4], f[8 * j + 5]), pack2_bf16(f[8 * j + 6], f[8 * j + 7]));
          }
        };
        auto put_edge = [&](void* to, long long at, const float* f) {
#pragma unroll
          for (int j = 0; j < 4; ++j) store_ragged<kOut4>(p, to, at + 8 * j, col0 + 8 * j, f + 8 * j);
        };
        auto send4 = [&](const CUtensorMap* map, int split) {           // float32: both buffers
          if (col0 < p.whole_cols) store_box(map, stage_s, col0, row0, split);
          if (col0 + 16 < p.whole_cols) store_box(map, stage_s + kBufferBytes, col0 + 16, row0, split);
        };
        uint32_t zp[kFwd && !kOut4 ? 16 : 1];                // z, rounded and packed
        finish(x, row, col0, [&](const float* z) {
          if (edge) put_edge(p.pre, row * p.ld_out + col0, z);
          if constexpr (kFwd && !kOut4) {
#pragma unroll
            for (int i = 0; i < 16; ++i) zp[i] = pack2_bf16(z[2 * i], z[2 * i + 1]);
          } else if constexpr (kOut4) {                      // on its way before the results take its place
            wait_now();
            put(stage_g + row_off, z);
            asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
            __syncwarp();
            if (lane == 0) {
              send4(&maps.pre, 0);
              asm volatile("cp.async.bulk.commit_group;" ::: "memory");
            }
          }
        });
        if (kOut4 && pre) {
          if (lane == 0) asm volatile("cp.async.bulk.wait_group.read 0;" ::: "memory");
          __syncwarp();
        }
        if (residual) {
          if constexpr (kOut4) {
            const float* rs = static_cast<const float*>(p.residual) + row * p.ld_out + col0;
            if (row < p.rows) {
#pragma unroll
              for (int i = 0; i < 32; i += 4) {
                if (col0 + i + 4 <= p.cols) {
                  const float4 f = *reinterpret_cast<const float4*>(rs + i);
                  x[i] += f.x; x[i + 1] += f.y; x[i + 2] += f.z; x[i + 3] += f.w;
                } else {
#pragma unroll
                  for (int n = 0; n < 4; ++n)
                    if (col0 + i + n < p.cols) x[i + n] += rs[i + n];
                }
              }
            }
          } else {
            uint4 q[4];
#pragma unroll
            for (int j = 0; j < 4; ++j) q[j] = *at16(dst, j);
#pragma unroll
            for (int j = 0; j < 4; ++j) {
              const uint32_t ww[4] = {q[j].x, q[j].y, q[j].z, q[j].w};
#pragma unroll
              for (int i = 0; i < 4; ++i) {
                x[8 * j + 2 * i] += __uint_as_float(ww[i] << 16);
                x[8 * j + 2 * i + 1] += __uint_as_float(ww[i] & 0xFFFF0000u);
              }
            }
          }
        }
        if (edge) put_edge(p.out, u.split * p.split_out + row * p.ld_out + col0, x);
        if (!(kOut4 && pre)) wait_now();
        if constexpr (kFwd && !kOut4) {
          if (pre) {
#pragma unroll
            for (int j = 0; j < 4; ++j)
              *at16(stage_g + kBufferBytes + row_off, j) = make_uint4(zp[4 * j], zp[4 * j + 1], zp[4 * j + 2], zp[4 * j + 3]);
          }
        }
        put(dst, x);
        asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
        __syncwarp();
        if (lane == 0) {
          if constexpr (kOut4) {
            send4(&maps.out, u.split);
          } else if (col0 < p.whole_cols) {
            store_box(&maps.out, stage_s + buf, col0, row0, u.split);
            if (pre) store_box(&maps.pre, stage_s + kBufferBytes, col0, row0, 0);
          }
          asm volatile("cp.async.bulk.commit_group;" ::: "memory");
        }
        ++n_block;
      }
      if (kMode != kF32) ++it;
    }
    if (lane == 0) asm volatile("cp.async.bulk.wait_group 0;" ::: "memory");
  }

  // ---------------------------------------------------------------------------------------------- teardown
  __syncwarp();
  tc_fence_before();
  cluster_sync();
  if (warp == 2) {
    tc_fence_after();
    asm volatile("tcgen05.dealloc.cta_group::2.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(kTmemCols) : "memory");
  }
}

// Persistent grid: one CTA pair per two SMs, as many as can be resident (kept per device and kernel).
template <typename Kernel>
int dense_grid(Kernel kernel, int* cached, int dev, cudaStream_t st, int* grid_out) {
  int grid = dev >= 0 && dev < 64 ? cached[dev] : 0;
  if (grid == 0) {
    if (cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, kSmem) != cudaSuccess) return SWITCH_MOE_CUDA_ERROR;
    const int sms = sm_count_or_default();
    cudaLaunchConfig_t lc = {};
    lc.gridDim = dim3((unsigned)(sms & ~1));
    lc.blockDim = dim3(kThreads);
    lc.dynamicSmemBytes = kSmem;
    lc.stream = st;
    int clusters = 0;
    if (cudaOccupancyMaxActiveClusters(&clusters, kernel, &lc) != cudaSuccess || clusters < 1) {
      (void)cudaGetLastError();
      clusters = sms / 2;
    }
    grid = 2 * (clusters < sms / 2 ? clusters : sms / 2);
    if (grid < 2) return SWITCH_MOE_CUDA_ERROR;
    if (dev >= 0 && dev < 64) cached[dev] = grid;
  }
  *grid_out = grid;
  return SWITCH_MOE_OK;
}

template <bool kAMn, bool kBMn, int TN, int kMode>
int launch_kernel(const DenseMaps& m, const DenseParams& p, cudaStream_t st) {
  static int cached[64] = {0};
  auto kernel = dense_gemm_kernel<kAMn, kBMn, TN, kMode>;
  int dev = 0, grid = 0;
  if (cudaGetDevice(&dev) != cudaSuccess) return SWITCH_MOE_CUDA_ERROR;
  const int rc = dense_grid(kernel, cached, dev, st, &grid);
  if (rc != SWITCH_MOE_OK) return rc;
  const long long units = (long long)p.m_tiles * p.n_tiles * p.splits;
  if (2 * units < grid) grid = (int)(2 * units);
  launch_k(kernel, dim3(grid), dim3(kThreads), kSmem, st, m, p);
  return launch_status();
}

template <bool kAMn, bool kBMn, int kMode>
int launch_kind(const DenseProduct& q, const DenseEpilogue& e, cudaStream_t st) {
  const int TN = q.width;
  DenseParams p{};
  p.rows = q.rows; p.cols = q.cols; p.k = q.k;
  p.k_blocks = (int)(((long long)q.k + kBK - 1) / kBK);
  const long long m_tiles = ((long long)q.rows + 255) / 256, n_tiles = ((long long)q.cols + TN - 1) / TN;
  if (m_tiles * n_tiles * q.splits > 0x3fffffffll || n_tiles * kBand > 0x3fffffffll) return SWITCH_MOE_UNSUPPORTED_SHAPE;
  p.m_tiles = (int)m_tiles; p.n_tiles = (int)n_tiles; p.splits = q.splits;
  p.k_per_split = (p.k_blocks + q.splits - 1) / q.splits;
  p.activation = e.activation; p.dropout_blocks = e.dropout_blocks; p.dropout = e.dropout; p.bias = e.bias;
  p.has_residual = e.residual != nullptr; p.has_pre = e.pre != nullptr;
  p.a = q.a.f32; p.a_si = q.a.si; p.a_sk = q.a.sk;
  p.b = q.b.f32; p.b_si = q.b.si; p.b_sk = q.b.sk;
  const int unit = kMode == kBf16 ? 8 : 4;
  p.whole_cols = kMode == kPartial ? q.cols : q.cols / unit * unit;     // (part sums: rows padded to whole pieces)
  p.out = q.out; p.pre = e.pre; p.residual = e.residual; p.ld_out = q.ld_out; p.split_out = (long long)q.rows * q.ld_out;
  p.status = q.status; p.clear_status = q.clear_status ? 1 : 0;
  DenseMaps m;
  const int depth = q.f32 ? 3 : 1, elt = kMode == kBf16 ? 2 : 4;
  int rc = kAMn ? make_map_rows(&m.a, q.a.p, 2, depth, q.k, q.rows, q.a.ld, 128, 64) : make_map_rows(&m.a, q.a.p, 2, depth, q.rows, q.k, q.a.ld, 128, 128);
  if (rc == SWITCH_MOE_OK)
    rc = kBMn ? make_map_rows(&m.b, q.b.p, 2, depth, q.k, q.cols, q.b.ld, 128, 64) : make_map_rows(&m.b, q.b.p, 2, depth, q.cols, q.k, q.b.ld, 128, TN / 2);
  const long long stored = kMode == kPartial ? q.ld_out : p.whole_cols > 0 ? p.whole_cols : unit;
  if (rc == SWITCH_MOE_OK) rc = make_map_rows(&m.out, q.out, elt, q.splits, q.rows, stored, q.ld_out, 64, 32);
  m.pre = m.out;
  m.residual = m.out;
  if (rc == SWITCH_MOE_OK && e.pre != nullptr) rc = make_map_rows(&m.pre, e.pre, elt, 1, q.rows, stored, q.ld_out, 64, 32);
  if (rc == SWITCH_MOE_OK && e.residual != nullptr) rc = make_map_rows(&m.residual, e.residual, elt, 1, q.rows, q.cols, q.ld_out, 64, 32);
  if (rc != SWITCH_MOE_OK) return rc;
  if (TN == 256) return launch_kernel<kAMn, kBMn, 256, kMode>(m, p, st);
  return TN == 192 ? launch_kernel<kAMn, kBMn, 192, kMode>(m, p, st) : launch_kernel<kAMn, kBMn, 128, kMode>(m, p, st);
}

}  // namespace

// The tiling whose estimated time is least.  A round of tiles over the CTA pairs takes a time per 64 steps of the contraction
// that falls with the width, but by less than the width does, since A is staged as before (us with 256 / 192 / 128 columns,
// the kernel alone after cold caches, ncu: 32768 tokens, 2048 x 768 forward 75.6 / 75.6 / 103, dx of 768 x 2048, k-major, 75.8 / 72.7 /
// 82.6; 8192 tokens, 768 x 2048 25.9 / 27.2 / 32.5; 1000 tokens 11.9 / 10.7 / 10.7; float32 4001, 512 x 2048 forward 47.6 / 52.7 /
// 45.2, where the rule takes 256, dx 43.0 / 45.2 / 41.2), and one for its epilogue.  Cutting the contraction fills the pairs
// where the output has few tiles, a weight gradient's or that of a few hundred tokens; the parts are written and read once more, by
// one more launch.
DenseTiling dense_tiling(DenseKind kind, bool f32, long long rows, long long cols, long long k) {
  const long long pairs = kChipSms / 2, m = (rows + 255) / 256, blocks = (k + kBK - 1) / kBK;
  const double step_us[3] = {f32 ? 3.0 : 0.40, f32 ? 2.25 : kind == kDenseDx ? 0.32 : 0.35, f32 ? 1.5 : 0.25};
  const double round_us = f32 ? 3.0 : 1.0, join_us = 3.5, part_us = (double)rows * (double)cols * 8.0 / 4e6;   // 4 TB/s
  DenseTiling best{1, 256};
  double best_us = 0;
  // (twice as many units as pairs at most, and coarser steps as parts get many: this runs in every call)
  const long long most = std::min(std::min(32ll, blocks / 4), 2 * pairs / (m * ((cols + 255) / 256)));
  for (int s = 1; s == 1 || s <= most; s += s < 8 ? 1 : s < 16 ? 2 : 8) {
    const long long per = (blocks + s - 1) / s;
    if (s > 1 && (per < 4 || (s - 1) * per >= blocks)) continue;      // (no part without work)
    for (int i = 0; i < 3; ++i) {
      const int w = 256 - 64 * i;
      const long long rounds = (m * ((cols + w - 1) / w) * s + pairs - 1) / pairs;
      const double us = (double)rounds * ((double)per * step_us[i] + round_us) + (s > 1 ? join_us + s * part_us : 0.0);
      if (best_us == 0 || us < best_us) { best = {s, w}; best_us = us; }
    }
  }
  return best;
}

template <bool kAMn, bool kBMn>
int launch_mode(const DenseProduct& q, const DenseEpilogue& e, cudaStream_t st) {
  if (q.f32) return launch_kind<kAMn, kBMn, kF32>(q, e, st);
  return q.splits > 1 ? launch_kind<kAMn, kBMn, kPartial>(q, e, st) : launch_kind<kAMn, kBMn, kBf16>(q, e, st);
}

int launch_dense(DenseKind kind, const DenseProduct& q, const DenseEpilogue& e, cudaStream_t st) {
  if (kind == kDenseFwd) return launch_mode<false, true>(q, e, st);
  return kind == kDenseDx ? launch_mode<false, false>(q, e, st) : launch_mode<true, true>(q, e, st);
}

}  // namespace swmoe
