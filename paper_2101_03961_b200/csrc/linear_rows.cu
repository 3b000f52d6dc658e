// The dense product of few rows (a decoding step): out = x W with the whole epilogue, or dx = dz W^T, up to 64 rows of
// bfloat16 or 16 of float32 (fused multiply-adds: 31 rows, 1792 x 8064 took 101 us here, 50 as bfloat16 parts on the tensor
// cores).  Such a call reads W once and little else, so it is all latency and bandwidth: a tile of the tensor-core kernel
// (256 rows, one CTA pair per 128 columns and all of the contraction) would leave most SMs without work.
//
// Here a block has 64 output columns (32 where that leaves SMs without a block) and a slice of the contraction; the blocks
// of the other slices form a cluster with it.  The groups of eight outputs are dealt out to the cluster's blocks; each block
// writes its sums into the shared memory of the one that finishes them, and after one cluster barrier that one adds them up
// in a fixed order.  64-deep pieces of W and x come in by cp.async, up to kStages at a time.  bfloat16: warp-level MMAs
// (16 columns of W x 8 rows of x x 16 steps: with so few rows a tcgen05 tile would be padding, and the loads bound it in
// either case); float32: fused multiply-adds.
// One token, 768 x 2048, GELU: 6.0 us serialised by ncu for 3.1 MB of weights (the tile kernel 11), 48 rows, 2048 x 768 9.9 (14):
// there 32 sums (8 slices of 4 parts of the steps) meet in each output, added up by 24 threads a block.
#include "linear_common.cuh"

namespace swmoe {
namespace {

constexpr int kThreads = 256;
constexpr int kDepth = 64;                           // steps per stage
constexpr int kMaxSlices = 8;
constexpr int kStages = 6, kStagesF32 = 4;           // ring in shared memory

struct RowsParams {
  const void* x; const void* W;
  long long ldx, ldw, ld_out;
  int M, N;                        // rows, output columns
  long long K;
  int slices, depth_per_slice;     // in stages of kDepth
  int stages;                      // that shared memory holds: all of a slice's, up to a ring of kStages
  DenseEpilogue e;
  void* out;
  int* status;
};

__device__ __forceinline__ uint32_t smem_at(const void* p) { return (uint32_t)__cvta_generic_to_shared(p); }
// 16 bytes of which the first `bytes` are read and the rest are zeros.
__device__ __forceinline__ void copy16(uint32_t dst, const void* src, int bytes) {
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst), "l"(src), "r"(bytes) : "memory");
}
__device__ __forceinline__ void ldm4(uint32_t addr, uint32_t* r) {
  asm volatile("ldmatrix.sync.aligned.m8n8.x4.shared.b16 {%0, %1, %2, %3}, [%4];"
               : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(addr) : "memory");
}
__device__ __forceinline__ void ldm4_trans(uint32_t addr, uint32_t* r) {
  asm volatile("ldmatrix.sync.aligned.m8n8.x4.trans.shared.b16 {%0, %1, %2, %3}, [%4];"
               : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(addr) : "memory");
}
__device__ __forceinline__ void mma16816(float* d, const uint32_t* a, uint32_t b0, uint32_t b1) {
  asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
               : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3]) : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}
__device__ __forceinline__ void cluster_arrive() { asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory"); }
__device__ __forceinline__ void cluster_wait() { asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory"); }
__device__ __forceinline__ void push(uint32_t local, uint32_t cta, float v) {
  asm volatile("{\n\t.reg .b32 ra;\n\tmapa.shared::cluster.u32 ra, %0, %1;\n\tst.shared::cluster.f32 [ra], %2;\n\t}" ::"r"(local),
               "r"(cta), "f"(v) : "memory");
}

// Where a block keeps what the others push: [source][group of its own][8], a source being a slice and a part of a block's steps.
// A row has kRowGroups = columns / 8 groups of eight.
struct Sums {
  uint32_t base;
  int groups, slices;                                 // groups per block
  __device__ __forceinline__ Sums(const RowsParams& p, int row_groups, uint32_t at)
      : base(at), groups((row_groups * p.M + p.slices - 1) / p.slices), slices(p.slices) {}
  // group g (row g / row_groups, columns 8 (g % row_groups) ..) belongs to block g % slices
  __device__ __forceinline__ void put(int source, int g, int i, float v) const {
    const int own = g / slices;
    push(base + (uint32_t)(((source * groups + own) * 8 + i) * 4), (uint32_t)(g - own * slices), v);
  }
};

// What this thread's first eight results need from memory, on its way to L2 while the weights come in.
template <typename ET, int kRowGroups>
__device__ __forceinline__ void prefetch_epilogue(const RowsParams& p, int rank, int col0) {
  const int g = threadIdx.x * p.slices + rank, row = g / kRowGroups, col = col0 + g % kRowGroups * 8;
  if (row >= p.M || col >= p.N) return;
  if (p.e.bias != nullptr) asm volatile("prefetch.global.L2 [%0];" ::"l"(p.e.bias + col));
  if (p.e.residual != nullptr)
    asm volatile("prefetch.global.L2 [%0];" ::"l"(static_cast<const ET*>(p.e.residual) + row * p.ld_out + col));
}

// After the pushes: the groups of this block.  `sources` per slice.
template <typename ET, int kRowGroups>
__device__ __forceinline__ void join_slices(const RowsParams& p, const float* sums, int sources, int rank, int col0) {
  const DropoutState rng = dropout_state(p.e.dropout);
  __syncwarp();                                       // (the aligned form wants whole warps)
  cluster_arrive();
  cluster_wait();
  const int groups = (kRowGroups * p.M + p.slices - 1) / p.slices;
  for (int own = threadIdx.x; own < groups; own += kThreads) {
    const int g = own * p.slices + rank, row = g / kRowGroups, col = col0 + g % kRowGroups * 8;
    if (row >= p.M || col >= p.N) continue;
    float x[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
#pragma unroll 4
    for (int s = 0; s < sources * p.slices; ++s) {
      const float4 a = *reinterpret_cast<const float4*>(sums + (s * groups + own) * 8);
      const float4 b = *reinterpret_cast<const float4*>(sums + (s * groups + own) * 8 + 4);
      x[0] += a.x; x[1] += a.y; x[2] += a.z; x[3] += a.w;
      x[4] += b.x; x[5] += b.y; x[6] += b.z; x[7] += b.w;
    }
    finish8<ET>(p.e, rng, p.out, p.ld_out, p.N, row, col, x);
  }
}

// kNK: W is stored [output column][contraction] (dx), else [contraction][output column].  NT: tiles of eight rows of x.
template <bool kNK, int NT, int kCols>
__global__ void __launch_bounds__(kThreads)
linear_rows_kernel(const RowsParams p) {
  constexpr int kColGroups = kCols / 16, kParts = 8 / kColGroups, kSteps = 4 / kParts;   // warps: columns x parts of the steps
  constexpr int kWBytes = kCols * kDepth * 2, kXBytes = NT * 8 * kDepth * 2, kStage = kWBytes + kXBytes;
  pdl_launch_dependents();
  extern __shared__ __align__(1024) uint8_t smem[];
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int rank = blockIdx.x % p.slices, col0 = (int)(blockIdx.x / p.slices) * kCols;
  const int first = rank * p.depth_per_slice;
  const int total = (int)((p.K + kDepth - 1) / kDepth), count = max(0, min(p.depth_per_slice, total - first));
  const __nv_bfloat16* x = static_cast<const __nv_bfloat16*>(p.x);
  const __nv_bfloat16* W = static_cast<const __nv_bfloat16*>(p.W);
  cluster_arrive();
  pdl_wait();
  if (p.status != nullptr && blockIdx.x == 0 && threadIdx.x < kStatusWords) p.status[threadIdx.x] = 0;
  // Tiles have rows of 128 bytes (W's of 32 columns, [step][column]: 64), their 16-byte pieces exchanged by the row.
  constexpr int kWRow = kNK || kCols == 64 ? 128 : 64;
  auto w_swap = [](int r) { return kWRow == 128 ? r & 7 : (r >> 1) & 3; };
  auto fetch = [&](int s) {
    const long long k0 = (long long)(first + s) * kDepth;
    const uint32_t w_dst = smem_at(smem) + (uint32_t)(s % kStages) * kStage, x_dst = w_dst + kWBytes;
#pragma unroll
    for (int i = 0; i < kCols * 8 / kThreads; ++i) {
      const int at = threadIdx.x + i * kThreads;
      const int r = kNK || kCols == 64 ? at >> 3 : at >> 2, piece = kNK || kCols == 64 ? at & 7 : at & 3;
      const long long outer = kNK ? (long long)col0 + r : k0 + r, inner = (kNK ? k0 : (long long)col0) + piece * 8;
      const long long outer_end = kNK ? p.N : p.K, inner_end = kNK ? p.K : p.N;
      const long long left = outer < outer_end ? inner_end - inner : 0;
      const int bytes = left >= 8 ? 16 : left > 0 ? (int)left * 2 : 0;
      copy16(w_dst + r * kWRow + ((piece ^ w_swap(r)) << 4), bytes > 0 ? W + outer * p.ldw + inner : W, bytes);
    }
    for (int at = threadIdx.x; at < NT * 64; at += kThreads) {
      const int r = at >> 3, piece = at & 7;
      const long long k = k0 + piece * 8, left = r < p.M ? p.K - k : 0;
      const int bytes = left >= 8 ? 16 : left > 0 ? (int)left * 2 : 0;
      copy16(x_dst + r * 128 + ((piece ^ (r & 7)) << 4), bytes > 0 ? x + r * p.ldx + k : x, bytes);
    }
  };
#pragma unroll
  for (int s = 0; s < kStages - 1; ++s) {
    if (s < count) fetch(s);
    asm volatile("cp.async.commit_group;" ::: "memory");
  }
  prefetch_epilogue<__nv_bfloat16, kCols / 8>(p, rank, col0);
  const int cg = warp % kColGroups, kh = warp / kColGroups;
  float acc[NT][4];
#pragma unroll
  for (int t = 0; t < NT; ++t)
#pragma unroll
    for (int i = 0; i < 4; ++i) acc[t][i] = 0.f;
  for (int s = 0; s < count; ++s) {
    asm volatile("cp.async.wait_group %0;" ::"n"(kStages - 2) : "memory");
    __syncthreads();                                  // stage s is there, and stage s - 1 has been used by all
    if (s + kStages - 1 < count) fetch(s + kStages - 1);
    asm volatile("cp.async.commit_group;" ::: "memory");
    const uint32_t w_src = smem_at(smem) + (uint32_t)(s % kStages) * kStage, x_src = w_src + kWBytes;
#pragma unroll
    for (int ks = 0; ks < kSteps; ++ks) {
      const int step = kSteps * kh + ks;                   // 16 steps of the contraction: pieces 2 step and 2 step + 1 of x's rows
      uint32_t a[4];
      if (kNK) {
        const int r = 16 * cg + (lane & 15), piece = 2 * step + (lane >> 4);
        ldm4(w_src + r * kWRow + ((piece ^ w_swap(r)) << 4), a);
      } else {
        const int r = 16 * step + (lane & 7) + ((lane >> 4) << 3), piece = 2 * cg + ((lane >> 3) & 1);
        ldm4_trans(w_src + r * kWRow + ((piece ^ w_swap(r)) << 4), a);
      }
      if constexpr (NT == 1) {
        uint32_t b[4];                                // (two of the four matrices are the same)
        const int r = lane & 7, piece = 2 * step + ((lane >> 3) & 1);
        ldm4(x_src + r * 128 + ((piece ^ (r & 7)) << 4), b);
        mma16816(acc[0], a, b[0], b[1]);
      } else {
#pragma unroll
        for (int t = 0; t < NT; t += 2) {
          uint32_t b[4];
          const int r = 8 * t + (lane & 7) + ((lane >> 4) << 3), piece = 2 * step + ((lane >> 3) & 1);
          ldm4(x_src + r * 128 + ((piece ^ (r & 7)) << 4), b);
          mma16816(acc[t], a, b[0], b[1]);
          mma16816(acc[t + 1], a, b[2], b[3]);
        }
      }
    }
  }
  const Sums sums(p, kCols / 8, smem_at(smem) + p.stages * kStage);
  __syncwarp();
  cluster_wait();                                     // every block of the cluster is there to be written to
#pragma unroll
  for (int t = 0; t < NT; ++t)
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int row = 8 * t + 2 * (lane & 3) + (i & 1), group = 2 * cg + (i >> 1);
      if (row < p.M) sums.put(kParts * rank + kh, kCols / 8 * row + group, lane >> 2, acc[t][i]);
    }
  join_slices<__nv_bfloat16, kCols / 8>(p, reinterpret_cast<const float*>(smem + p.stages * kStage), kParts, rank, col0);
}

// float32: thread = one column x a part of a stage's steps, MT rows in registers.
template <bool kNK, int MT, int kCols>
__global__ void __launch_bounds__(kThreads)
linear_rows_f32_kernel(const RowsParams p) {
  constexpr int kParts = kThreads / kCols, kSteps = kDepth / kParts;
  constexpr int kWBytes = kCols * kDepth * 4, kXBytes = MT * kDepth * 4, kStage = kWBytes + kXBytes;
  pdl_launch_dependents();
  extern __shared__ __align__(1024) uint8_t smem[];
  const int rank = blockIdx.x % p.slices, col0 = (int)(blockIdx.x / p.slices) * kCols;
  const int first = rank * p.depth_per_slice;
  const int total = (int)((p.K + kDepth - 1) / kDepth), count = max(0, min(p.depth_per_slice, total - first));
  const float* x = static_cast<const float*>(p.x);
  const float* W = static_cast<const float*>(p.W);
  cluster_arrive();
  pdl_wait();
  if (p.status != nullptr && blockIdx.x == 0 && threadIdx.x < kStatusWords) p.status[threadIdx.x] = 0;
  // W's tile has rows of 64 steps or kCols columns, their 16-byte pieces exchanged by the row where lanes read down a column of
  // pieces.
  constexpr int kWRow = kNK ? kDepth * 4 : kCols * 4;
  auto fetch = [&](int s) {
    const long long k0 = (long long)(first + s) * kDepth;
    const uint32_t w_dst = smem_at(smem) + (uint32_t)(s % kStagesF32) * kStage, x_dst = w_dst + kWBytes;
#pragma unroll
    for (int i = 0; i < kCols * 16 / kThreads; ++i) {
      const int at = threadIdx.x + i * kThreads;
      const int r = kNK || kCols == 64 ? at >> 4 : at >> 3, piece = kNK || kCols == 64 ? at & 15 : at & 7;
      const long long outer = kNK ? (long long)col0 + r : k0 + r, inner = (kNK ? k0 : (long long)col0) + piece * 4;
      const long long outer_end = kNK ? p.N : p.K, inner_end = kNK ? p.K : p.N;
      const long long left = outer < outer_end ? inner_end - inner : 0;
      const int bytes = left >= 4 ? 16 : left > 0 ? (int)left * 4 : 0;
      copy16(w_dst + r * kWRow + ((kNK ? piece ^ (r & 15) : piece) << 4), bytes > 0 ? W + outer * p.ldw + inner : W, bytes);
    }
    for (int at = threadIdx.x; at < MT * 16; at += kThreads) {
      const int r = at >> 4, piece = at & 15;
      const long long k = k0 + piece * 4, left = r < p.M ? p.K - k : 0;
      const int bytes = left >= 4 ? 16 : left > 0 ? (int)left * 4 : 0;
      copy16(x_dst + r * 256 + (piece << 4), bytes > 0 ? x + r * p.ldx + k : x, bytes);
    }
  };
#pragma unroll
  for (int s = 0; s < kStagesF32 - 1; ++s) {
    if (s < count) fetch(s);
    asm volatile("cp.async.commit_group;" ::: "memory");
  }
  prefetch_epilogue<float, kCols / 8>(p, rank, col0);
  const int c = threadIdx.x % kCols, kq = threadIdx.x / kCols;
  float acc[MT];
#pragma unroll
  for (int m = 0; m < MT; ++m) acc[m] = 0.f;
  for (int s = 0; s < count; ++s) {
    asm volatile("cp.async.wait_group %0;" ::"n"(kStagesF32 - 2) : "memory");
    __syncthreads();
    if (s + kStagesF32 - 1 < count) fetch(s + kStagesF32 - 1);
    asm volatile("cp.async.commit_group;" ::: "memory");
    const uint8_t* w_src = smem + (s % kStagesF32) * kStage;
    const uint8_t* x_src = w_src + kWBytes;
#pragma unroll
    for (int q = 0; q < kSteps / 4; ++q) {            // four steps at a time
      const int k = kSteps * kq + 4 * q;
      float w[4];
      if (kNK) {
        const float4 v = *reinterpret_cast<const float4*>(w_src + c * kWRow + (((k >> 2) ^ (c & 15)) << 4));
        w[0] = v.x; w[1] = v.y; w[2] = v.z; w[3] = v.w;
      } else {
#pragma unroll
        for (int i = 0; i < 4; ++i) w[i] = *reinterpret_cast<const float*>(w_src + (k + i) * kWRow + c * 4);
      }
#pragma unroll
      for (int m = 0; m < MT; ++m) {
        const float4 v = *reinterpret_cast<const float4*>(x_src + m * 256 + k * 4);
        acc[m] = fmaf(v.x, w[0], acc[m]);
        acc[m] = fmaf(v.y, w[1], acc[m]);
        acc[m] = fmaf(v.z, w[2], acc[m]);
        acc[m] = fmaf(v.w, w[3], acc[m]);
      }
    }
  }
  const Sums sums(p, kCols / 8, smem_at(smem) + p.stages * kStage);
  __syncwarp();
  cluster_wait();
#pragma unroll
  for (int m = 0; m < MT; ++m)
    if (m < p.M) sums.put(kParts * rank + kq, kCols / 8 * m + (c >> 3), c & 7, acc[m]);
  join_slices<float, kCols / 8>(p, reinterpret_cast<const float*>(smem + p.stages * kStage), kParts, rank, col0);
}

// dW = x^T dz of up to 64 rows, by fused multiply-adds: a block has 128 columns of dW, forms their dz itself, and takes 64 rows
// of dW after another, a thread 4 x 8 of them; the first block of each 128 columns also leaves the bias gradient, and dz for the
// product of dx (it alone, where dW is not wanted).  dW takes dz in float32, as it was formed; dx's tensor cores take it rounded.
// Latency and writing dW bound it (GELU): 9 rows, 540 x 372 5.6 us, 16 rows, 512 x 2880 7, where the pass over dz and the
// tensor-core product take two launches of 6 to 8.
constexpr int kDwRows = 64, kDwCols = 128, kDwPitch = kDwCols + 4;
template <typename ET>
__global__ void __launch_bounds__(kThreads)
linear_rows_dw_kernel(const RowsDw p) {
  pdl_launch_dependents();
  extern __shared__ __align__(16) float tile[];       // x [M][64], then dz [M][128 + 4]
  pdl_wait();
  if (p.status != nullptr && blockIdx.x == 0 && blockIdx.y == 0 && threadIdx.x < kStatusWords) p.status[threadIdx.x] = 0;
  float* const xs = tile;
  float* const gs = tile + p.M * kDwRows;
  const ET* x = static_cast<const ET*>(p.x);
  const ET* dy = static_cast<const ET*>(p.dy);
  const ET* pre = static_cast<const ET*>(p.pre);
  const long long col0 = (long long)blockIdx.x * kDwCols;
  const bool sums = blockIdx.y == 0 && p.dbias != nullptr;
  // Up to 64 rows of bfloat16 are two groups of eight of x and four of dy and z a thread, 16 of float32 one: all asked for first.
  constexpr int kX = sizeof(ET) == 2 ? 2 : 1, kG = sizeof(ET) == 2 ? 4 : 1;
  Raw8<ET> xr[kX], gr[kG], zr[kG];
  const int x_units = p.dW != nullptr ? p.M * (kDwRows / 8) : 0, g_units = p.M * (kDwCols / 8);
#pragma unroll
  for (int i = 0; i < kG; ++i) {
    const int u = threadIdx.x + i * kThreads, row = u / (kDwCols / 8);
    const long long col = col0 + u % (kDwCols / 8) * 8, at = row * p.ldy + col;
    if (u < g_units && col < p.N) {
      const int n = p.N - col < 8 ? (int)(p.N - col) : 8;
      gr[i].load(dy + at, n);
      if (p.act != SWITCH_MOE_ACT_NONE) zr[i].load(pre + at, n);
    }
  }
  auto fetch_x = [&](long long k0) {
#pragma unroll
    for (int i = 0; i < kX; ++i) {
      const int u = threadIdx.x + i * kThreads;
      const long long k = k0 + u % (kDwRows / 8) * 8;
      if (u < x_units && k < p.K) xr[i].load(x + u / (kDwRows / 8) * p.ldx + k, p.K - k < 8 ? (int)(p.K - k) : 8);
    }
  };
  fetch_x((long long)blockIdx.y * kDwRows);
  const DropoutState rng = dropout_state(p.dropout);
#pragma unroll
  for (int i = 0; i < kG; ++i) {
    const int u = threadIdx.x + i * kThreads, row = u / (kDwCols / 8), c = u % (kDwCols / 8) * 8;
    if (u >= g_units) break;
    float g[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f}, z[8];
    if (col0 + c < p.N) {
      gr[i].get(g);
      if (p.act != SWITCH_MOE_ACT_NONE) zr[i].get(z);
      dz8(p.act, p.dropout, rng, (unsigned long long)row * (unsigned)p.per_row + (unsigned)((col0 + c) >> 3), z, g);
      if (p.dz != nullptr && blockIdx.y == 0) store8(static_cast<ET*>(p.dz) + row * p.ldn + col0 + c, 8, g);
    }
    store8(gs + row * kDwPitch + c, 8, g);
  }
  __syncthreads();
  if (sums && threadIdx.x < kDwCols && col0 + threadIdx.x < p.N) {
    float s = 0.f;
    for (int m = 0; m < p.M; ++m) s += gs[m * kDwPitch + threadIdx.x];
    p.dbias[col0 + threadIdx.x] = s;
  }
  if (p.dW == nullptr) return;
  const int tx = threadIdx.x & 15, ty = threadIdx.x >> 4;                // columns 8 tx .., rows 4 ty ..
  const long long n = p.N - (col0 + 8 * tx), step = (long long)gridDim.y * kDwRows;
  for (long long k0 = (long long)blockIdx.y * kDwRows; k0 < p.K; k0 += step) {
#pragma unroll
    for (int i = 0; i < kX; ++i) {
      const int u = threadIdx.x + i * kThreads;
      float f[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
      if (u >= x_units) break;
      if (k0 + u % (kDwRows / 8) * 8 < p.K) xr[i].get(f);
      store8(xs + u * 8, 8, f);
    }
    __syncthreads();
    if (k0 + step < p.K) fetch_x(k0 + step);
    float acc[4][8];
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
      for (int j = 0; j < 8; ++j) acc[i][j] = 0.f;
#pragma unroll 2
    for (int m = 0; m < p.M; ++m) {
      const float4 a = *reinterpret_cast<const float4*>(xs + m * kDwRows + 4 * ty);
      float b[8];
      load8(gs + m * kDwPitch + 8 * tx, 8, b);
      const float av[4] = {a.x, a.y, a.z, a.w};
#pragma unroll
      for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int j = 0; j < 8; ++j) acc[i][j] = fmaf(av[i], b[j], acc[i][j]);
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const long long k = k0 + 4 * ty + i;
      if (k < p.K && n > 0) store8(static_cast<ET*>(p.dW) + k * p.ldw + col0 + 8 * tx, n < 8 ? (int)n : 8, acc[i]);
    }
    __syncthreads();                                   // x's tile has been used by all
  }
}

template <typename Kern>
int launch(Kern kernel, size_t stage, int most_stages, size_t sums, int cols, const RowsParams& p, bool* ready, cudaStream_t st) {
  int dev = 0;
  if (cudaGetDevice(&dev) != cudaSuccess) return SWITCH_MOE_CUDA_ERROR;
  if (dev < 0 || dev >= 64 || !ready[dev]) {
    if (cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)(most_stages * stage + sums)) != cudaSuccess)
      return SWITCH_MOE_CUDA_ERROR;
    if (dev >= 0 && dev < 64) ready[dev] = true;
  }
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3((unsigned)(((p.N + (long long)cols - 1) / cols) * p.slices));
  cfg.blockDim = dim3(kThreads);
  cfg.dynamicSmemBytes = p.stages * stage + sums;      // (with two or three blocks an SM where slices are short)
  cfg.stream = st;
  cudaLaunchAttribute attr[2];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  attr[1].id = cudaLaunchAttributeClusterDimension;
  attr[1].val.clusterDim.x = (unsigned)p.slices;
  attr[1].val.clusterDim.y = attr[1].val.clusterDim.z = 1;
  cfg.attrs = attr;
  cfg.numAttrs = 2;
  if (cudaLaunchKernelEx(&cfg, kernel, p) != cudaSuccess) launch_failed_flag() = true;
  return launch_status();
}

// Shared memory: the stages, then for every source the groups of eight of this block (rounded up).
constexpr size_t sum_bytes(int parts, int rows, int cols) { return (size_t)parts * (rows * cols / 8 + kMaxSlices) * 32; }

template <bool kNK, int NT, int kCols>
int launch_bf16(RowsParams p, cudaStream_t st) {
  static bool ready[64] = {false};
  p.stages = p.depth_per_slice < kStages ? p.depth_per_slice : kStages;
  return launch(linear_rows_kernel<kNK, NT, kCols>, kCols * kDepth * 2 + NT * 8 * kDepth * 2, kStages,
                sum_bytes(8 / (kCols / 16), NT * 8, kCols), kCols, p, ready, st);
}
template <bool kNK, int MT, int kCols>
int launch_f32(RowsParams p, cudaStream_t st) {
  static bool ready[64] = {false};
  p.stages = p.depth_per_slice < kStagesF32 ? p.depth_per_slice : kStagesF32;
  return launch(linear_rows_f32_kernel<kNK, MT, kCols>, kCols * kDepth * 4 + MT * kDepth * 4, kStagesF32,
                sum_bytes(kThreads / kCols, MT, kCols), kCols, p, ready, st);
}
template <bool kNK, int kCols>
int launch_cols(const DenseProduct& q, const RowsParams& p, cudaStream_t st) {
  if (q.f32) {
    if (q.rows <= 4) return launch_f32<kNK, 4, kCols>(p, st);
    return launch_f32<kNK, 16, kCols>(p, st);
  }
  if (q.rows <= 8) return launch_bf16<kNK, 1, kCols>(p, st);
  if (q.rows <= 16) return launch_bf16<kNK, 2, kCols>(p, st);
  return q.rows <= 32 ? launch_bf16<kNK, 4, kCols>(p, st) : launch_bf16<kNK, 8, kCols>(p, st);
}

}  // namespace

// `q.a.p` and `q.b.p` are the operands themselves, also of float32.  Slices: as many as fill the SMs about twice over, each
// of at least one stage, so that none is without work.
int launch_dense_rows(DenseKind kind, const DenseProduct& q, const DenseEpilogue& e, cudaStream_t st) {
  RowsParams p{};
  p.x = q.a.p; p.W = q.b.p; p.ldx = q.a.ld; p.ldw = q.b.ld; p.ld_out = q.ld_out;
  p.M = q.rows; p.N = q.cols; p.K = q.k; p.e = e; p.out = q.out;
  p.status = q.clear_status ? q.status : nullptr;
  const long long stages = ((long long)q.k + kDepth - 1) / kDepth;
  auto slices_for = [&](long long blocks) {
    long long slices = 2 * kChipSms / blocks;
    if (slices > kMaxSlices) slices = kMaxSlices;
    if (slices > stages) slices = stages;
    return slices < 1 ? 1ll : slices;
  };
  const long long wide = ((long long)q.cols + 63) / 64;
  const bool narrow = wide * slices_for(wide) < kChipSms;
  const long long blocks = narrow ? ((long long)q.cols + 31) / 32 : wide, slices = slices_for(blocks);
  p.depth_per_slice = (int)((stages + slices - 1) / slices);
  p.slices = (int)((stages + p.depth_per_slice - 1) / p.depth_per_slice);
  if (blocks * p.slices > 0x7fffffffll) return SWITCH_MOE_UNSUPPORTED_SHAPE;
  if (kind == kDenseDx) return narrow ? launch_cols<true, 32>(q, p, st) : launch_cols<true, 64>(q, p, st);
  return narrow ? launch_cols<false, 32>(q, p, st) : launch_cols<false, 64>(q, p, st);
}

int launch_rows_dw(bool f32, const RowsDw& d, cudaStream_t st) {
  const size_t smem = (size_t)d.M * (kDwRows + kDwPitch) * 4;        // 64 rows: 50 KB
  static bool ready[2][64] = {};
  int dev = 0;
  if (cudaGetDevice(&dev) != cudaSuccess) return SWITCH_MOE_CUDA_ERROR;
  auto kernel = f32 ? linear_rows_dw_kernel<float> : linear_rows_dw_kernel<__nv_bfloat16>;
  if (dev < 0 || dev >= 64 || !ready[f32][dev]) {
    const int most = 64 * (kDwRows + kDwPitch) * 4;
    if (cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, most) != cudaSuccess) return SWITCH_MOE_CUDA_ERROR;
    if (dev >= 0 && dev < 64) ready[f32][dev] = true;
  }
  // about three blocks an SM: more rows of dW per block beyond that
  const long long bx = ((long long)d.N + kDwCols - 1) / kDwCols, k_tiles = ((long long)d.K + kDwRows - 1) / kDwRows;
  long long by = 3 * kChipSms / bx;
  if (by > k_tiles) by = k_tiles;
  if (by < 1 || d.dW == nullptr) by = 1;
  launch_k(kernel, dim3((unsigned)bx, (unsigned)by), dim3(kThreads), smem, st, d);
  return launch_status();
}

}  // namespace swmoe
