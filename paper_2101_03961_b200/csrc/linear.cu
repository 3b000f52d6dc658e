// The dense layer's entry points (switch_moe_linear_*): argument checks, workspace, launch sequences, and the kernels
// around the products: dz = dropout(dy) . activation'(pre) with the bias gradient's sums, the bfloat16 parts of float32
// operands, the sum of a split contraction's parts.
#include <cstring>

#include "linear_common.cuh"

namespace swmoe {
namespace {

constexpr int kThreads = 256;
constexpr int kColsPerBlock = 256, kRowLanes = 8;    // 32 threads x 8 columns, 8 rows side by side,
constexpr int kRowsAhead = 2;                        // two of them per thread in flight
constexpr int kChunkRows = 64;                       // rows of a block, where that leaves at most 1024 of them

struct LinearShape {
  int M, K, N, act, q, site;
  bool f32;
  long long ldx, ldw, ldy, elt;
  long long ldn, ldk;                                // rows of N or K elements in the workspace, multiples of 8
  int chunks, chunk_rows;                            // row chunks of the dz kernel
  DenseTiling fwd, dx, dw;
  bool rows_kernel;                                  // few rows: the forward product and dx have a kernel of their own
};
struct LinearPlan {
  size_t status, x_parts, w_parts, dz, dz_parts, db_part, sums, total;
};

int resolve(const switch_moe_linear_config* cfg, bool backward, LinearShape* s) {
  if (cfg == nullptr) return SWITCH_MOE_INVALID_ARGUMENT;
  const switch_moe_linear_config& c = *cfg;
  if (c.M < 0 || c.K <= 0 || c.N <= 0 || c.ldx < 0 || c.ldw < 0 || c.ldy < 0 || c.reserved[0] != 0 || c.reserved[1] != 0)
    return SWITCH_MOE_INVALID_ARGUMENT;
  if ((c.ldx > 0 && c.ldx < c.K) || (c.ldw > 0 && c.ldw < c.N) || (c.ldy > 0 && c.ldy < c.N)) return SWITCH_MOE_INVALID_ARGUMENT;
  if (c.dtype != SWITCH_MOE_BF16 && c.dtype != SWITCH_MOE_F32) return SWITCH_MOE_INVALID_ARGUMENT;
  if (c.activation < SWITCH_MOE_ACT_NONE || c.activation > SWITCH_MOE_ACT_GELU) return SWITCH_MOE_INVALID_ARGUMENT;
  s->q = dropout_threshold(c.dropout);
  if (s->q < 0 || c.site < 0 || c.site > 65535) return SWITCH_MOE_INVALID_ARGUMENT;
  s->M = c.M; s->K = c.K; s->N = c.N; s->act = c.activation; s->site = c.site;
  s->f32 = c.dtype == SWITCH_MOE_F32;
  s->elt = s->f32 ? 4 : 2;
  s->ldx = c.ldx > 0 ? c.ldx : c.K;
  s->ldw = c.ldw > 0 ? c.ldw : c.N;
  s->ldy = c.ldy > 0 ? c.ldy : c.N;
  if (s->ldx * s->elt % 16 != 0 || s->ldw * s->elt % 16 != 0 || s->ldy * s->elt % 16 != 0) return SWITCH_MOE_UNSUPPORTED_SHAPE;
  if (c.M > kMaxExtent || c.K > kMaxExtent || c.N > kMaxExtent) return SWITCH_MOE_UNSUPPORTED_SHAPE;
  s->ldn = ((long long)c.N + 7) / 8 * 8;
  s->ldk = ((long long)c.K + 7) / 8 * 8;
  if ((long long)c.M * (s->ldn / 8) >= 1ll << 48) return SWITCH_MOE_UNSUPPORTED_SHAPE;
  // Chunks of 64 rows: many short blocks keep the SMs evenly busy; longer ones where that would be more than 1024 chunks.
  const long long col_blocks = ((long long)c.N + kColsPerBlock - 1) / kColsPerBlock;
  long long rows = ((long long)c.M + 1023) / 1024;
  if (rows < kChunkRows) {
    // (shorter ones where there would be fewer than four blocks an SM, down to what a thread has in flight; up to 64 rows
    // stay one chunk, whose sums need not be added up)
    const long long want = ((long long)c.M * col_blocks + 4 * kChipSms - 1) / (4 * kChipSms);
    rows = c.M <= kChunkRows || want > kChunkRows ? kChunkRows : want;
  }
  rows = (rows + kRowsAhead * kRowLanes - 1) / (kRowsAhead * kRowLanes) * (kRowsAhead * kRowLanes);
  s->chunk_rows = (int)rows;
  s->chunks = (int)(((long long)c.M + rows - 1) / rows);
  if (s->chunks > 65535 || col_blocks > 0x7fffffffll) return SWITCH_MOE_UNSUPPORTED_SHAPE;
  s->rows_kernel = few_rows(s->f32, c.M);
  const DenseTiling none{1, 256};
  s->fwd = backward || s->rows_kernel ? none : dense_tiling(kDenseFwd, s->f32, c.M, c.N, c.K);
  s->dx = !backward || s->rows_kernel ? none : dense_tiling(kDenseDx, s->f32, c.M, c.K, c.N);
  s->dw = !backward ? none : dense_tiling(kDenseDw, s->f32, c.K, c.N, c.M);
  return SWITCH_MOE_OK;
}

// The forward and the backward call lay the workspace out each for itself.
void make_plan(const LinearShape& s, bool backward, LinearPlan* p) {
  size_t off = 0;
  auto take = [&](size_t bytes) { size_t o = off; off = (off + bytes + 1023) / 1024 * 1024; return o; };
  auto part_bytes = [](const DenseTiling& g, size_t rows, size_t ld) { return g.splits > 1 ? g.splits * rows * ld * 4 : 0; };
  const size_t M = s.M, K = s.K;
  const bool own_dz = backward && (s.act != SWITCH_MOE_ACT_NONE || s.q > 0), parts = s.f32;
  p->status = take(kStatusWords * 4);
  p->x_parts = take(parts && (backward || !s.rows_kernel) ? 3 * M * s.ldk * 2 : 0);
  p->w_parts = take(parts && !s.rows_kernel ? 3 * K * s.ldn * 2 : 0);
  p->dz = take(own_dz ? M * s.ldn * s.elt : 0);
  p->dz_parts = take(backward && parts ? 3 * M * s.ldn * 2 : 0);
  p->db_part = take(backward ? (size_t)s.chunks * s.ldn * 4 : 0);
  const size_t fwd = part_bytes(s.fwd, M, s.ldn), dx = part_bytes(s.dx, M, s.ldk), dw = part_bytes(s.dw, K, s.ldn);
  p->sums = take(fwd + (dx > dw ? dx : dw));           // (fwd, or dx and then dw)
  p->total = off;
}

// x 2^24 = h + m + l: three arrays `plane` elements apart.  (A value beyond the parts' range makes m NaN, and with it the
// results that it meets, which the product then forms again.)
__device__ __forceinline__ void store_parts8(__nv_bfloat16* p, long long plane, const float* f) {
  float h[8], m[8], l[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const float x = f[i] * kPartUp;
    h[i] = __bfloat162float(__float2bfloat16(x));
    const float rest = x - h[i];
    m[i] = __bfloat162float(__float2bfloat16(rest));
    l[i] = rest - m[i];
  }
  store8(p, 8, h);
  store8(p + plane, 8, m);
  store8(p + 2 * plane, 8, l);
}

// dz and the bias gradient.  bfloat16: dz is rounded for the products, since the tensor cores take bfloat16 (two parts of it would
// double both products; dx's and dW's error against float64 is 0.0023 of the norm for 0.0017 with dz in float32); the column sums
// take it unrounded.  A block takes 256 columns of a chunk of rows: 32 threads x 8 columns, 8 rows side by side; a
// thread asks for two of its rows before it works on the first (32768 x 2048, GELU: 83 us; with a GELU' of 5 us less four rows
// ahead and three blocks an SM took 82, two ahead and five blocks 91, against 78).  Column sums go to `part`, from where they are
// added up in chunk order.  Bound by reading dy and pre and writing dz once (ReLU 16384 x 10240: 148 us, 6.8 TB/s); with GELU and
// dropout by instructions.
struct DzArgs {
  int M, N, act, chunk_rows, per_row;
  long long ldy, ldn;
  DropoutParams dropout;
};
template <typename ET, int kAct>
__global__ void __launch_bounds__(kThreads, sizeof(ET) == 2 ? 4 : 3)
linear_dz_kernel(const ET* __restrict__ dy, const ET* __restrict__ pre, DzArgs a, ET* dz, __nv_bfloat16* parts, float* part, int* status) {
  pdl_launch_dependents();
  pdl_wait();
  __shared__ float sums[kRowLanes][kColsPerBlock];
  if (status != nullptr && blockIdx.x == 0 && blockIdx.y == 0 && threadIdx.x < kStatusWords) status[threadIdx.x] = 0;
  const int cx = threadIdx.x & 31, ry = threadIdx.x >> 5;
  const long long col = (long long)blockIdx.x * kColsPerBlock + cx * 8;
  const int n = (int)(col < a.N ? (a.N - col < 8 ? a.N - col : 8) : 0);
  const DropoutState rng = dropout_state(a.dropout);
  float acc[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) acc[i] = 0.f;
  const long long row_end = min((long long)a.M, (long long)(blockIdx.y + 1) * a.chunk_rows);
  if (n > 0) {
#pragma unroll 1
    for (long long row0 = (long long)blockIdx.y * a.chunk_rows + ry; row0 < row_end; row0 += kRowsAhead * kRowLanes) {
      Raw8<ET> graw[kRowsAhead], zraw[kRowsAhead];
#pragma unroll
      for (int k = 0; k < kRowsAhead; ++k) {
        const long long row = row0 + k * kRowLanes;
        if (row < row_end) {
          graw[k].load(dy + row * a.ldy + col, n);
          if (kAct != SWITCH_MOE_ACT_NONE) zraw[k].load(pre + row * a.ldy + col, n);
        }
      }
#pragma unroll
      for (int k = 0; k < kRowsAhead; ++k) {
        const long long row = row0 + k * kRowLanes;
        if (row >= row_end) break;
        float g[8], z[8];
        graw[k].get(g);
        if (kAct != SWITCH_MOE_ACT_NONE) zraw[k].get(z);
        dz8(kAct, a.dropout, rng, (unsigned long long)row * (unsigned)a.per_row + (unsigned)(col >> 3), z, g);
#pragma unroll
        for (int i = 0; i < 8; ++i) acc[i] += g[i];
        if (dz != nullptr) store8(dz + row * a.ldn + col, 8, g);        // (the workspace's rows are multiples of 8)
        if (parts != nullptr) store_parts8(parts + row * a.ldn + col, (long long)a.M * a.ldn, g);
      }
    }
  }
  if (part == nullptr) return;
#pragma unroll
  for (int i = 0; i < 8; ++i) sums[ry][cx * 8 + i] = acc[i];
  __syncthreads();
  float s = 0.f;
#pragma unroll
  for (int r = 0; r < kRowLanes; ++r) s += sums[r][threadIdx.x];
  const long long c = (long long)blockIdx.x * kColsPerBlock + threadIdx.x;
  if (c < a.N) part[(long long)blockIdx.y * a.ldn + c] = s;
}

// db[c] = sum over chunks: 32 columns per block, 32 chunks at a time.
__global__ void __launch_bounds__(1024)
linear_db_kernel(const float* __restrict__ part, int chunks, int N, long long ldn, float* db) {
  pdl_launch_dependents();
  pdl_wait();
  __shared__ float sums[32][33];
  const int lane = threadIdx.x & 31, w = threadIdx.x >> 5;
  const long long c = (long long)blockIdx.x * 32 + lane;
  float s = 0.f;
  if (c < N) {
#pragma unroll 4
    for (int i = w; i < chunks; i += 32) s += part[(long long)i * ldn + c];
  }
  sums[w][lane] = s;
  __syncthreads();
  s = sums[lane][w];                                  // column w, the 32 lanes hold its parts
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) s += __shfl_xor_sync(0xffffffffu, s, o);
  const long long out = (long long)blockIdx.x * 32 + w;
  if (lane == 0 && out < N) db[out] = s;
}

// The parts of a float32 matrix, eight elements of a row per thread.
__global__ void __launch_bounds__(kThreads)
linear_parts_kernel(const float* __restrict__ src, long long ld, long long rows, int cols, long long ld_out, __nv_bfloat16* parts) {
  pdl_launch_dependents();
  pdl_wait();
  const long long per_row = ld_out / 8, total = rows * per_row;
  for (long long b = (long long)blockIdx.x * kThreads + threadIdx.x; b < total; b += (long long)gridDim.x * kThreads) {
    const long long row = b / per_row;
    const int col = (int)(b - row * per_row) * 8;
    float f[8];
    load8(src + row * ld + col, cols - col, f);
    store_parts8(parts + row * ld_out + col, rows * ld_out, f);
  }
}

// The sum of a split contraction's parts, in order, and what comes after the product.
template <typename ET>
__global__ void __launch_bounds__(kThreads)
linear_add_kernel(const float* __restrict__ part, int splits, long long rows, int cols, long long ld_part, DenseEpilogue e,
                  void* out, long long ld_out) {
  pdl_launch_dependents();
  pdl_wait();
  const DropoutState rng = dropout_state(e.dropout);
  const long long per_row = ld_part / 8, total = rows * per_row;
  for (long long b = (long long)blockIdx.x * kThreads + threadIdx.x; b < total; b += (long long)gridDim.x * kThreads) {
    const long long row = total <= 0x7fffffffll ? (long long)((unsigned)b / (unsigned)per_row) : b / per_row;
    const int col = (int)(b - row * per_row) * 8;
    float s[8];
    load8(part + row * ld_part + col, 8, s);          // (the parts' rows are whole eights; what is beyond cols is not stored)
#pragma unroll 4
    for (int i = 1; i < splits; ++i) {
      float f[8];
      load8(part + ((long long)i * rows + row) * ld_part + col, 8, f);
#pragma unroll
      for (int j = 0; j < 8; ++j) s[j] += f[j];
    }
    finish8<ET>(e, rng, out, ld_out, cols, row, col, s);
  }
}

unsigned flat_grid(long long threads) {
  const long long want = (threads + kThreads - 1) / kThreads, most = 16ll * kChipSms;
  return (unsigned)(want < most ? want : most);
}

int launch_parts(const void* src, long long ld, long long rows, int cols, long long ld_out, __nv_bfloat16* parts, cudaStream_t st) {
  launch_k(linear_parts_kernel, dim3(flat_grid(rows * (ld_out / 8))), dim3(kThreads), 0, st, static_cast<const float*>(src), ld,
           rows, cols, ld_out, parts);
  return launch_status();
}

// One product, split or not; `out` and `ld_out` are the result's.
int launch_product(DenseKind kind, DenseProduct q, const DenseTiling& g, const DenseEpilogue& e, float* sums, long long ld_sums,
                   void* out, long long ld_out, cudaStream_t st) {
  q.splits = g.splits; q.width = g.width;
  q.out = g.splits > 1 ? sums : out;
  q.ld_out = g.splits > 1 ? ld_sums : ld_out;
  const int rc = launch_dense(kind, q, g.splits > 1 ? DenseEpilogue{} : e, st);
  if (rc != SWITCH_MOE_OK || g.splits == 1) return rc;
  const dim3 grid(flat_grid((long long)q.rows * (ld_sums / 8)));
  launch_k(q.f32 ? linear_add_kernel<float> : linear_add_kernel<__nv_bfloat16>, grid, dim3(kThreads), 0, st,
           static_cast<const float*>(sums), g.splits, (long long)q.rows, q.cols, ld_sums, e, out, ld_out);
  return launch_status();
}

template <typename ET>
int launch_dz(const LinearShape& s, const void* dy, const void* pre, const uint64_t* rng, void* dz, __nv_bfloat16* parts,
              float* part, int* status, cudaStream_t st) {
  DzArgs a{s.M, s.N, s.act, s.chunk_rows, (int)(s.ldn / 8), s.ldy, s.ldn, dropout_params(rng, s.q, s.site)};
  const dim3 grid((unsigned)((s.N + kColsPerBlock - 1) / kColsPerBlock), s.chunks);
  const ET* g = static_cast<const ET*>(dy);
  const ET* z = static_cast<const ET*>(pre);
  if (s.act == SWITCH_MOE_ACT_RELU)
    launch_k(linear_dz_kernel<ET, SWITCH_MOE_ACT_RELU>, grid, dim3(kThreads), 0, st, g, z, a, static_cast<ET*>(dz), parts, part, status);
  else if (s.act == SWITCH_MOE_ACT_GELU)
    launch_k(linear_dz_kernel<ET, SWITCH_MOE_ACT_GELU>, grid, dim3(kThreads), 0, st, g, z, a, static_cast<ET*>(dz), parts, part, status);
  else
    launch_k(linear_dz_kernel<ET, SWITCH_MOE_ACT_NONE>, grid, dim3(kThreads), 0, st, g, z, a, static_cast<ET*>(dz), parts, part, status);
  return launch_status();
}

int check_workspace(const void* workspace, size_t have, size_t need) {
  if (workspace == nullptr) return SWITCH_MOE_INVALID_ARGUMENT;
  if ((reinterpret_cast<uintptr_t>(workspace) & 1023u) != 0) return SWITCH_MOE_UNSUPPORTED_SHAPE;
  return have < need ? SWITCH_MOE_WORKSPACE_TOO_SMALL : SWITCH_MOE_OK;
}

#define SWMOE_TRY(expr)                    \
  do {                                     \
    int rc__ = (expr);                     \
    if (rc__ != SWITCH_MOE_OK) return rc__; \
  } while (0)

}  // namespace
}  // namespace swmoe

using namespace swmoe;

extern "C" int switch_moe_linear_workspace_bytes(const switch_moe_linear_config* cfg, int32_t backward, size_t* bytes_out) {
  if (bytes_out == nullptr) return SWITCH_MOE_INVALID_ARGUMENT;
  size_t most = 0;
  for (int pass = 0; pass <= (backward != 0 ? 1 : 0); ++pass) {
    LinearShape s;
    SWMOE_TRY(resolve(cfg, pass == 1, &s));
    LinearPlan p;
    make_plan(s, pass == 1, &p);
    if (p.total > most) most = p.total;
  }
  *bytes_out = most;
  return SWITCH_MOE_OK;
}

extern "C" int switch_moe_linear_fwd(const switch_moe_linear_config* cfg, const void* x, const void* W, const float* bias,
                                     const void* residual, const uint64_t* rng, void* y, void* pre, void* workspace,
                                     size_t workspace_bytes, void* stream) {
  LinearShape s;
  SWMOE_TRY(resolve(cfg, false, &s));
  LinearPlan p;
  make_plan(s, false, &p);
  SWMOE_TRY(check_workspace(workspace, workspace_bytes, p.total));
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  int* status = ws_ptr<int>(workspace, p.status);
  if (s.M == 0)
    return cudaMemsetAsync(status, 0, kStatusWords * 4, st) == cudaSuccess ? SWITCH_MOE_OK : SWITCH_MOE_CUDA_ERROR;
  if (x == nullptr || W == nullptr || y == nullptr || (s.q > 0 && rng == nullptr)) return SWITCH_MOE_INVALID_ARGUMENT;
  if (!aligned16(x) || !aligned16(W) || !aligned16(y) || !aligned16(pre) || !aligned16(residual) || !aligned16(bias) ||
      (reinterpret_cast<uintptr_t>(rng) & 7u) != 0)
    return SWITCH_MOE_UNSUPPORTED_SHAPE;
  if (pre != nullptr && (pre == y || pre == residual)) return SWITCH_MOE_INVALID_ARGUMENT;   // z would meet y, or replace what is added
  DenseProduct q{};
  q.rows = s.M; q.cols = s.N; q.k = s.K; q.f32 = s.f32;
  q.a = {x, s.ldx, static_cast<const float*>(x), s.ldx, 1};
  q.b = {W, s.ldw, static_cast<const float*>(W), 1, s.ldw};
  q.out = y; q.ld_out = s.ldy; q.status = status; q.clear_status = true;
  const DenseEpilogue e{bias, residual, pre, s.act, (int)(s.ldn / 8), dropout_params(rng, s.q, s.site)};
  if (s.rows_kernel) return launch_dense_rows(kDenseFwd, q, e, st);
  if (s.f32) {
    __nv_bfloat16* xp = ws_ptr<__nv_bfloat16>(workspace, p.x_parts);
    __nv_bfloat16* wp = ws_ptr<__nv_bfloat16>(workspace, p.w_parts);
    SWMOE_TRY(launch_parts(x, s.ldx, s.M, s.K, s.ldk, xp, st));
    SWMOE_TRY(launch_parts(W, s.ldw, s.K, s.N, s.ldn, wp, st));
    q.a.p = xp; q.a.ld = s.ldk;
    q.b.p = wp; q.b.ld = s.ldn;
  }
  return launch_product(kDenseFwd, q, s.fwd, e, ws_ptr<float>(workspace, p.sums), s.ldn, y, s.ldy, st);
}

extern "C" int switch_moe_linear_bwd(const switch_moe_linear_config* cfg, const void* dy, const void* x, const void* W,
                                     const void* pre, const uint64_t* rng, void* workspace, size_t workspace_bytes,
                                     void* dx, void* dW, float* dbias, void* stream) {
  LinearShape s;
  SWMOE_TRY(resolve(cfg, true, &s));
  LinearPlan p;
  make_plan(s, true, &p);
  SWMOE_TRY(check_workspace(workspace, workspace_bytes, p.total));
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  if (!aligned16(dy) || !aligned16(x) || !aligned16(W) || !aligned16(pre) || !aligned16(dx) || !aligned16(dW) ||
      !aligned16(dbias) || (reinterpret_cast<uintptr_t>(rng) & 7u) != 0)
    return SWITCH_MOE_UNSUPPORTED_SHAPE;
  int* status = ws_ptr<int>(workspace, p.status);
  if (s.M == 0) {
    if (cudaMemsetAsync(status, 0, kStatusWords * 4, st) != cudaSuccess) return SWITCH_MOE_CUDA_ERROR;
    if (dW != nullptr && cudaMemset2DAsync(dW, s.ldw * s.elt, 0, s.N * s.elt, s.K, st) != cudaSuccess) return SWITCH_MOE_CUDA_ERROR;
    if (dbias != nullptr && cudaMemsetAsync(dbias, 0, (size_t)s.N * 4, st) != cudaSuccess) return SWITCH_MOE_CUDA_ERROR;
    return SWITCH_MOE_OK;
  }
  if (dy == nullptr || (dW != nullptr && x == nullptr) || (dx != nullptr && W == nullptr) ||
      (s.act != SWITCH_MOE_ACT_NONE && pre == nullptr) || (s.q > 0 && rng == nullptr))
    return SWITCH_MOE_INVALID_ARGUMENT;
  if (dx == nullptr && dW == nullptr && dbias == nullptr)
    return cudaMemsetAsync(status, 0, kStatusWords * 4, st) == cudaSuccess ? SWITCH_MOE_OK : SWITCH_MOE_CUDA_ERROR;
  if (s.rows_kernel && rows_dw_pays(s.M, s.K, s.N)) {
    // few rows: dW, the bias gradient and, for dx, dz itself in one launch (what is not wanted is left out, so that the rest
    // comes out the same)
    const bool keep_dz = dx != nullptr && (s.act != SWITCH_MOE_ACT_NONE || s.q > 0);
    RowsDw d{};
    d.dy = dy; d.pre = pre; d.x = x; d.dW = dW; d.dbias = dbias; d.dz = keep_dz ? ws_ptr<void>(workspace, p.dz) : nullptr;
    d.M = s.M; d.K = s.K; d.N = s.N; d.act = s.act; d.per_row = (int)(s.ldn / 8);
    d.ldx = s.ldx; d.ldw = s.ldw; d.ldy = s.ldy; d.ldn = s.ldn;
    d.dropout = dropout_params(rng, s.q, s.site);
    d.status = status;
    const bool any = dW != nullptr || dbias != nullptr || keep_dz;
    if (any) SWMOE_TRY(launch_rows_dw(s.f32, d, st));
    if (dx == nullptr) return SWITCH_MOE_OK;
    DenseProduct q{};
    q.rows = s.M; q.cols = s.K; q.k = s.N; q.f32 = s.f32;
    q.a.p = keep_dz ? d.dz : dy; q.a.ld = keep_dz ? s.ldn : s.ldy;
    q.b.p = W; q.b.ld = s.ldw;
    q.out = dx; q.ld_out = s.ldx; q.status = status; q.clear_status = !any;
    return launch_dense_rows(kDenseDx, q, DenseEpilogue{}, st);
  }
  const bool products = dx != nullptr || dW != nullptr, own_dz = s.act != SWITCH_MOE_ACT_NONE || s.q > 0;
  bool cleared = false;
  void* dz = own_dz && products ? ws_ptr<void>(workspace, p.dz) : nullptr;
  __nv_bfloat16* dz_parts = s.f32 && products ? ws_ptr<__nv_bfloat16>(workspace, p.dz_parts) : nullptr;
  float* db_part = dbias == nullptr || s.chunks == 1 ? dbias : ws_ptr<float>(workspace, p.db_part);   // one chunk: its sums are all
  if (dz != nullptr || dz_parts != nullptr || db_part != nullptr) {
    SWMOE_TRY(s.f32 ? launch_dz<float>(s, dy, pre, rng, dz, dz_parts, db_part, status, st)
                    : launch_dz<__nv_bfloat16>(s, dy, pre, rng, dz, dz_parts, db_part, status, st));
    cleared = true;
  }
  if (dbias != nullptr && s.chunks > 1) {
    launch_k(linear_db_kernel, dim3((unsigned)((s.N + 31) / 32)), dim3(1024), 0, st, static_cast<const float*>(db_part),
             s.chunks, s.N, s.ldn, dbias);
    SWMOE_TRY(launch_status());
  }
  const void* g = dz != nullptr ? dz : dy;
  const long long ldg = dz != nullptr ? s.ldn : s.ldy;
  DenseOperand go{s.f32 ? dz_parts : g, s.f32 ? s.ldn : ldg, static_cast<const float*>(g), 0, 0};
  if (dx != nullptr) {
    DenseProduct q{};
    q.rows = s.M; q.cols = s.K; q.k = s.N; q.f32 = s.f32;
    q.a = go; q.a.si = ldg; q.a.sk = 1;
    q.b = {W, s.ldw, static_cast<const float*>(W), s.ldw, 1};
    q.out = dx; q.ld_out = s.ldx; q.status = status; q.clear_status = !cleared;
    if (s.rows_kernel) {
      q.a.p = g; q.a.ld = ldg;
      SWMOE_TRY(launch_dense_rows(kDenseDx, q, DenseEpilogue{}, st));
    } else {
      if (s.f32) {
        __nv_bfloat16* wp = ws_ptr<__nv_bfloat16>(workspace, p.w_parts);
        SWMOE_TRY(launch_parts(W, s.ldw, s.K, s.N, s.ldn, wp, st));
        q.b.p = wp; q.b.ld = s.ldn;
      }
      SWMOE_TRY(launch_product(kDenseDx, q, s.dx, DenseEpilogue{}, ws_ptr<float>(workspace, p.sums), s.ldk, dx, s.ldx, st));
    }
    cleared = true;
  }
  if (dW != nullptr) {
    DenseProduct q{};
    q.rows = s.K; q.cols = s.N; q.k = s.M; q.f32 = s.f32;
    q.a = {x, s.ldx, static_cast<const float*>(x), 1, s.ldx};
    q.b = go; q.b.si = 1; q.b.sk = ldg;
    if (s.f32) {
      __nv_bfloat16* xp = ws_ptr<__nv_bfloat16>(workspace, p.x_parts);
      SWMOE_TRY(launch_parts(x, s.ldx, s.M, s.K, s.ldk, xp, st));
      q.a.p = xp; q.a.ld = s.ldk;
    }
    q.status = status; q.clear_status = !cleared;
    SWMOE_TRY(launch_product(kDenseDw, q, s.dw, DenseEpilogue{}, ws_ptr<float>(workspace, p.sums), s.ldn, dW, s.ldw, st));
  }
  return SWITCH_MOE_OK;
}

extern "C" int switch_moe_linear_check_device_status(const switch_moe_linear_config* cfg, void* workspace,
                                                     int32_t* info_out, void* stream) {
  LinearShape s;
  SWMOE_TRY(resolve(cfg, false, &s));
  SWMOE_TRY(check_workspace(workspace, ~(size_t)0, 0));
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  int32_t host[kStatusWords];
  if (cudaMemcpyAsync(host, workspace, sizeof(host), cudaMemcpyDeviceToHost, st) != cudaSuccess) return SWITCH_MOE_CUDA_ERROR;
  if (cudaStreamSynchronize(st) != cudaSuccess) return SWITCH_MOE_CUDA_ERROR;
  if (info_out != nullptr) std::memcpy(info_out, host, sizeof(host));
  return host[0] != 0 ? SWITCH_MOE_DEVICE_TIMEOUT : SWITCH_MOE_OK;
}
