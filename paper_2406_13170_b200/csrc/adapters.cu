// amph_project_adapters: a projection shared by all rows, and each row's own low-rank adapter beside it.
//
//   t[r][s][j] = sum_k x[r][k] a[i_r][s][j][k]                       the rows' low-rank products (down)
//   P          = x . w^T                                             the projection kernels, as split-K partial sums
//   y[r][s][o] = sum P + scale[i_r] sum_j t[r][s][j] b[i_r][s][o][j]  reduction of the partial sums, adapters' way back up (up)
#include <math.h>

#include <mutex>

#include "amph_internal.cuh"
#include "gemm_tc_common.cuh"

namespace amph {
namespace {

typedef __nv_bfloat16 bf16;

constexpr int kMaxRowsAll = 4 * kMaxRows;
constexpr int kThreads = 128;

__device__ __forceinline__ void put(bf16* p, float v) { *p = __float2bfloat16_rn(v); }

// Up to kTileRows rows of one adapter (or without any: adapter < 0), as adapter_down leaves them for adapter_up.
constexpr int kTileRows = 16;
struct __align__(16) RowTile {
  int adapter, n;
  uint16_t row[kTileRows];
};

struct AdapterArgs {
  const void *x, *a, *b;
  const float* scale;
  const int* row_adapter;
  RowTile* tiles;
  float* t;                // [splits][rows][n_seg * rank]
  void* y;
  int* status;
  int n_adapters, rank, n_seg, out, in, rows, splits;
};

// The row's adapter, -1 if it has none (or names one that does not exist, which is reported).
__device__ __forceinline__ int adapter_of(const AdapterArgs& p, int row) {
  const int a = p.row_adapter[row];
  if (a < p.n_adapters) return a < 0 ? -1 : a;
  if (p.status != nullptr) *p.status = AMPH_ERR_INVALID_ARG;
  return -1;
}

// fp32: one warp per (row, column of t).
__global__ void __launch_bounds__(kThreads) adapter_down_plain_kernel(const AdapterArgs p) {
  pdl_wait();
  pdl_launch_dependents();
  const int cols = p.n_seg * p.rank, lane = threadIdx.x & 31;
  const int row = blockIdx.y, col = blockIdx.x * (kThreads / 32) + (threadIdx.x >> 5);
  const int i = adapter_of(p, row);
  if (i < 0 || col >= cols) return;
  const float4* x = (const float4*)((const float*)p.x + (size_t)row * p.in);
  const float4* a = (const float4*)((const float*)p.a + ((size_t)i * cols + col) * p.in);
  float acc = 0.f;
#pragma unroll 4
  for (int k = lane; k < p.in / 4; k += 32) {
    const float4 u = x[k], v = a[k];
    acc += u.x * v.x; acc += u.y * v.y; acc += u.z * v.z; acc += u.w * v.w;
  }
#pragma unroll
  for (int d = 16; d; d >>= 1) acc += __shfl_xor_sync(~0u, acc, d);
  if (lane == 0) p.t[(size_t)row * cols + col] = acc;
}

// fp32: grid (128 columns, row), one column per thread.
__global__ void __launch_bounds__(kThreads) adapter_up_plain_kernel(const AdapterArgs p, const PartialView P) {
  pdl_wait();
  pdl_launch_dependents();
  __shared__ float t[kMaxK * AMPH_MAX_ADAPTER_RANK];
  const int cols = p.n_seg * p.rank, row = blockIdx.y, ld = p.n_seg * p.out;
  const int i = adapter_of(p, row);
  if (i >= 0) {
    const float scale = p.scale ? p.scale[i] : 1.f;
    for (int j = threadIdx.x; j < cols; j += kThreads) t[j] = scale * p.t[(size_t)row * cols + j];
  }
  __syncthreads();
  const int c = blockIdx.x * kThreads + threadIdx.x;
  if (c >= ld) return;
  float acc = P.p[(size_t)row * P.ld + c];
  if (i >= 0) {
    const int seg = c / p.out, o = c - seg * p.out;
    const float4* b = (const float4*)((const float*)p.b + (((size_t)i * p.n_seg + seg) * p.out + o) * p.rank);
    const float* ts = t + seg * p.rank;
    float low = 0.f;
#pragma unroll 4
    for (int j = 0; j < p.rank / 4; ++j) {
      const float4 v = b[j];
      low += ts[4 * j] * v.x; low += ts[4 * j + 1] * v.y; low += ts[4 * j + 2] * v.z; low += ts[4 * j + 3] * v.w;
    }
    acc += low;
  }
  ((float*)p.y)[(size_t)row * ld + c] = acc;
}

__device__ __forceinline__ void mma_16816(float (&d)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
  asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
               : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3]) : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}

// Tile `tile` of the call's rows: the rows of one adapter in their order, 16 at a time, tiles in the order of their first rows.  Every
// block finds its own (an adapter's rows may lie anywhere): row r is the c-th of its adapter, c = how many rows ahead of it name the same.
struct TileSmem {
  int adapter[kMaxRowsAll];
  short nth[kMaxRowsAll];
  int firsts[kMaxRowsAll / 32];
  int leader;
  RowTile tile;
};
__device__ __forceinline__ bool find_tile(const AdapterArgs& p, int tile, TileSmem& sm) {
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  for (int r = tid; r < p.rows; r += kThreads) sm.adapter[r] = adapter_of(p, r);
  if (tid == 0) { sm.leader = -1; sm.tile.n = 0; }
  __syncthreads();
  unsigned first[kMaxRowsAll / kThreads];
#pragma unroll
  for (int i = 0; i < kMaxRowsAll / kThreads; ++i) {
    const int r = i * kThreads + tid;
    first[i] = 0;
    if (i * kThreads >= p.rows) break;
    int c = 0, q = 0;
    if (r < p.rows) {
      const int a = sm.adapter[r];
      for (; q + 4 <= r; q += 4) {
        const int4 v = *reinterpret_cast<const int4*>(&sm.adapter[q]);
        c += (v.x == a) + (v.y == a) + (v.z == a) + (v.w == a);
      }
      for (; q < r; ++q) c += sm.adapter[q] == a;
      sm.nth[r] = (short)c;
    }
    first[i] = __ballot_sync(~0u, r < p.rows && c % kTileRows == 0);
    if (lane == 0) sm.firsts[i * (kThreads / 32) + warp] = __popc(first[i]);
  }
  __syncthreads();
#pragma unroll
  for (int i = 0; i < kMaxRowsAll / kThreads; ++i) {
    if (i * kThreads >= p.rows) break;
    if ((first[i] >> lane) & 1) {
      int at = __popc(first[i] & ((1u << lane) - 1u));
      for (int w = 0; w < i * (kThreads / 32) + warp; ++w) at += sm.firsts[w];
      if (at == tile) sm.leader = i * kThreads + tid;
    }
  }
  __syncthreads();
  const int leader = sm.leader;
  if (leader < 0) return false;
  const int a = sm.adapter[leader], c0 = sm.nth[leader];
  for (int r = tid; r < p.rows; r += kThreads) {
    const int c = sm.nth[r] - c0;
    if (sm.adapter[r] == a && c >= 0 && c < kTileRows) {
      sm.tile.row[c] = (uint16_t)r;
      atomicMax(&sm.tile.n, c + 1);
    }
  }
  if (tid == 0) sm.tile.adapter = a;
  __syncthreads();
  return true;
}

// t of one tile of rows: grid (tile, K range, 64 columns of t), MMA with the rows as A (M = 16) and the adapter's rows as B, both straight
// from global memory: the sum over k may run in any order that both share, so a lane takes 16 contiguous bytes for two steps.  The
// four warps take turns at 64 columns of k and meet in shared memory.
// Bound: latency for a few rows, the adapters' bytes for many tenants.
constexpr int kDownCols = 64;
__global__ void __launch_bounds__(kThreads) adapter_down_kernel(const AdapterArgs p) {
  pdl_wait();
  pdl_launch_dependents();
  __shared__ TileSmem sm;
  __shared__ float red[kThreads / 32][kTileRows][kDownCols + 2];
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31, g = lane >> 2, t = lane & 3;
  const bool any = find_tile(p, blockIdx.x, sm);
  const int n = any ? sm.tile.n : 0;
  if (blockIdx.y == 0 && blockIdx.z == 0 && tid == 0) {
    if (!any) sm.tile.adapter = -1;
    p.tiles[blockIdx.x] = sm.tile;
  }
  if (!any || sm.tile.adapter < 0) return;
  const int cols = p.n_seg * p.rank, col0 = blockIdx.z * kDownCols;
  const int nt = min(kDownCols, cols - col0) / 8;
  const int steps = (p.in + 63) / 64;
  const int s0 = steps * (int)blockIdx.y / p.splits, s1 = steps * ((int)blockIdx.y + 1) / p.splits;
  const bf16* x[2];
  x[0] = g < n ? (const bf16*)p.x + (size_t)sm.tile.row[g] * p.in : nullptr;
  x[1] = g + 8 < n ? (const bf16*)p.x + (size_t)sm.tile.row[g + 8] * p.in : nullptr;
  const bf16* a = (const bf16*)p.a + ((size_t)sm.tile.adapter * cols + col0 + g) * p.in;
  float acc[kDownCols / 8][4];
#pragma unroll
  for (int j = 0; j < kDownCols / 8; ++j) acc[j][0] = acc[j][1] = acc[j][2] = acc[j][3] = 0.f;
  const uint4 zero = make_uint4(0u, 0u, 0u, 0u);
  for (int s = s0 + warp; s < s1; s += kThreads / 32) {
    uint4 xv[2][2], av[kDownCols / 8][2];
#pragma unroll
    for (int c = 0; c < 2; ++c) {
      const int k = s * 64 + c * 32 + t * 8;
#pragma unroll
      for (int i = 0; i < 2; ++i) xv[i][c] = x[i] != nullptr && k < p.in ? *reinterpret_cast<const uint4*>(x[i] + k) : zero;
#pragma unroll
      for (int j = 0; j < kDownCols / 8; ++j)
        av[j][c] = j < nt && k < p.in ? *reinterpret_cast<const uint4*>(a + (size_t)j * 8 * p.in + k) : zero;
    }
#pragma unroll
    for (int j = 0; j < kDownCols / 8; ++j)
      if (j < nt)
#pragma unroll
        for (int c = 0; c < 2; ++c) {
          mma_16816(acc[j], xv[0][c].x, xv[1][c].x, xv[0][c].y, xv[1][c].y, av[j][c].x, av[j][c].y);
          mma_16816(acc[j], xv[0][c].z, xv[1][c].z, xv[0][c].w, xv[1][c].w, av[j][c].z, av[j][c].w);
        }
  }
#pragma unroll
  for (int j = 0; j < kDownCols / 8; ++j)
    if (j < nt) {
      *reinterpret_cast<float2*>(&red[warp][g][j * 8 + 2 * t]) = make_float2(acc[j][0], acc[j][1]);
      *reinterpret_cast<float2*>(&red[warp][g + 8][j * 8 + 2 * t]) = make_float2(acc[j][2], acc[j][3]);
    }
  __syncthreads();
  for (int i = tid; i < n * nt * 8; i += kThreads) {
    const int r = i / (nt * 8), c = i - r * (nt * 8);
    float v = red[0][r][c];
#pragma unroll
    for (int w = 1; w < kThreads / 32; ++w) v += red[w][r][c];
    p.t[((size_t)blockIdx.y * p.rows + sm.tile.row[r]) * cols + col0 + c] = v;
  }
}

__device__ __forceinline__ uint32_t pack(float lo, float hi) {
  const __nv_bfloat162 h = __floats2bfloat162_rn(lo, hi);
  return *reinterpret_cast<const uint32_t*>(&h);
}
// what rounding `v` to the bf16 in the upper half of `h` loses (nothing where that is an infinity)
__device__ __forceinline__ float lost(float v, uint32_t h) {
  const float d = v - __uint_as_float(h & 0xffff0000u);
  return fabsf(d) < INFINITY ? d : 0.f;
}
__device__ __forceinline__ void add4(float4& a, const float4 v) { a.x += v.x; a.y += v.y; a.z += v.z; a.w += v.w; }
// four values from `left` on (all four where `vec`)
__device__ __forceinline__ float4 get4(const float* p, int vec, int left) {
  if (vec) return *reinterpret_cast<const float4*>(p);
  float4 v = make_float4(p[0], 0.f, 0.f, 0.f);
  if (left > 1) v.y = p[1];
  if (left > 2) v.z = p[2];
  if (left > 3) v.w = p[3];
  return v;
}
__device__ __forceinline__ void put4(float* p, float4 v, int vec, int left) {
  if (vec) { *reinterpret_cast<float4*>(p) = v; return; }
  p[0] = v.x;
  if (left > 1) p[1] = v.y;
  if (left > 2) p[2] = v.z;
  if (left > 3) p[3] = v.w;
}
__device__ __forceinline__ void put4(bf16* p, float4 v, int vec, int left) {
  if (vec) { *reinterpret_cast<uint2*>(p) = make_uint2(pack(v.x, v.y), pack(v.z, v.w)); return; }
  put(p, v.x);
  if (left > 1) put(p + 1, v.y);
  if (left > 2) put(p + 2, v.z);
  if (left > 3) put(p + 3, v.w);
}

// Reduction of the projection's partial sums, the adapters' way back up, one rounding: grid (columns, tile, segment), a warp has 16
// columns of the tile's rows at a time.  MMA with t as A and b as B; t is split in two bf16 halves (16 bits of it, 2^-17 of the
// adapter's share), its partial sums are added once per block.  A lane's two output tiles are numbered so that it owns four neighbouring
// columns.  CHUNKS: 16 columns of t each.  Bound: L2 (partial sums) and the bytes of b and y.
template <int CHUNKS, typename TY>
__global__ void __launch_bounds__(kThreads) adapter_up_kernel(const AdapterArgs p, const PartialView P, int steps, int vec) {
  pdl_wait();
  pdl_launch_dependents();
  const RowTile& tile = p.tiles[blockIdx.y];
  const int n = tile.n, adapter = tile.adapter, seg = blockIdx.z;
  if (n == 0) return;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, g = lane >> 2, t = lane & 3;
  const int cols = p.n_seg * p.rank;
  int row[2];
  row[0] = g < n ? tile.row[g] : -1;
  row[1] = g + 8 < n ? tile.row[g + 8] : -1;
  uint32_t hi[CHUNKS][4], lo[CHUNKS][4];
  if (adapter >= 0) {
    const float scale = p.scale ? p.scale[adapter] : 1.f;
#pragma unroll
    for (int c = 0; c < CHUNKS; ++c)
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        float4 v = make_float4(0.f, 0.f, 0.f, 0.f);
        const int j = c * 16 + t * 4;
        if (row[i] >= 0 && j < p.rank) {
          const float* src = p.t + (size_t)row[i] * cols + seg * p.rank + j;
#pragma unroll 8
          for (int s = 0; s < p.splits; ++s) add4(v, *reinterpret_cast<const float4*>(src + (size_t)s * p.rows * cols));
        }
        v.x *= scale; v.y *= scale; v.z *= scale; v.w *= scale;
        const uint32_t h0 = pack(v.x, v.y), h1 = pack(v.z, v.w);
        hi[c][i] = h0;
        hi[c][2 + i] = h1;
        lo[c][i] = pack(lost(v.x, h0 << 16), lost(v.y, h0));
        lo[c][2 + i] = pack(lost(v.z, h1 << 16), lost(v.w, h1));
      }
  }
  const bf16* b = (const bf16*)p.b + ((size_t)(adapter < 0 ? 0 : adapter) * p.n_seg + seg) * p.out * p.rank;
  for (int step = 0; step < steps; ++step) {
    const int c0 = ((blockIdx.x * steps + step) * (kThreads / 32) + warp) * 16;
    if (c0 >= p.out) return;
    const int col = c0 + 4 * t, left = p.out - col;
    float4 sum[2];
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      sum[i] = make_float4(0.f, 0.f, 0.f, 0.f);
      if (row[i] >= 0 && left > 0) {
        const float* src = P.p + (size_t)row[i] * P.ld + seg * p.out + col;
#pragma unroll 8
        for (int s = 0; s < P.splits; ++s) add4(sum[i], get4(src + s * P.split_stride, vec, left));
      }
    }
    if (adapter >= 0) {
      float acc[2][4];
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        acc[i][0] = acc[i][1] = acc[i][2] = acc[i][3] = 0.f;
        const int o = c0 + 4 * (g >> 1) + 2 * i + (g & 1);
        const bf16* src = b + (size_t)o * p.rank + t * 4;
#pragma unroll
        for (int c = 0; c < CHUNKS; ++c) {
          const uint2 v = o < p.out && c * 16 + t * 4 < p.rank ? *reinterpret_cast<const uint2*>(src + c * 16) : make_uint2(0u, 0u);
          mma_16816(acc[i], lo[c][0], lo[c][1], lo[c][2], lo[c][3], v.x, v.y);
          mma_16816(acc[i], hi[c][0], hi[c][1], hi[c][2], hi[c][3], v.x, v.y);
        }
      }
      add4(sum[0], make_float4(acc[0][0], acc[0][1], acc[1][0], acc[1][1]));
      add4(sum[1], make_float4(acc[0][2], acc[0][3], acc[1][2], acc[1][3]));
    }
#pragma unroll
    for (int i = 0; i < 2; ++i)
      if (row[i] >= 0 && left > 0) put4((TY*)p.y + (size_t)row[i] * P.ld + seg * p.out + col, sum[i], vec, left);
  }
}

constexpr int kMaxDevices = 64;
std::mutex g_mutex;
TcGemm* g_plans[kMaxDevices];            // tensor-map encoder and kernel attributes of a device; no call's data

size_t round256(size_t n) { return (n + 255) / 256 * 256; }
int padded(int rows) { return rows <= 128 ? (rows + 15) / 16 * 16 : (rows + 127) / 128 * 128; }
// K ranges that the projection kernels make of a launch (about two blocks per SM, at most 16), bounded from above
int most_splits(int n_seg, int out) {
  const int tiles = (n_seg * out + 127) / 128;
  const int s = (320 + tiles - 1) / tiles;
  return s > 16 ? 16 : s;
}
// Tiles of rows that n_adapters adapters can make: each adapter, and the rows without one, rounds up once.
int most_tiles(int rows, int n_adapters) {
  const int64_t n = (int64_t)n_adapters + 1 + rows / kTileRows;
  return n < rows ? (int)n : rows;
}
constexpr int kMaxDownSplits = 16;
// K ranges of adapter_down: about two blocks per SM, 64 columns of k for each warp at least
int down_splits(int in, int blocks) {
  const int most = (in + 255) / 256, want = (296 + blocks - 1) / blocks;
  const int s = want < most ? want : most;
  return s > kMaxDownSplits ? kMaxDownSplits : s;
}
size_t tiles_bytes(int rows) { return round256(sizeof(RowTile) * rows); }

amph_status bad_shape(int n_seg, int out, int rows, int rank) {
  if (n_seg < 1 || n_seg > kMaxK || out < 1 || rows < 1 || rows > kMaxRowsAll) return api_fail(AMPH_ERR_SHAPE, "bad projection shape");
  if ((int64_t)n_seg * out > 0x7fffffff / 4) return api_fail(AMPH_ERR_SHAPE, "too many output features");
  if (rank < 8 || rank > AMPH_MAX_ADAPTER_RANK || rank % 8)
    return api_fail(AMPH_ERR_SHAPE, "rank must be a multiple of 8 in 8..%d (got %d)", AMPH_MAX_ADAPTER_RANK, rank);
  return AMPH_OK;
}
size_t t_bytes(int n_seg, int rows, int rank) { return round256((size_t)kMaxDownSplits * rows * n_seg * rank * sizeof(float)); }

template <typename TY>
cudaError_t run_up(const AdapterArgs& p, const PartialView& pv, int tiles, cudaStream_t st) {
  // a block's columns: 64, or more where that still leaves several blocks per SM
  const int groups = (p.out + 63) / 64;
  int steps = (int)((int64_t)groups * tiles * p.n_seg / (148 * 8));
  steps = steps < 1 ? 1 : (steps > 4 ? 4 : steps);
  const dim3 grid((groups + steps - 1) / steps, tiles, p.n_seg);
  const int vec = p.out % 4 == 0;
  if (p.rank <= 16) return launch_pdl(adapter_up_kernel<1, TY>, grid, dim3(kThreads), 0, st, p, pv, steps, vec);
  if (p.rank <= 32) return launch_pdl(adapter_up_kernel<2, TY>, grid, dim3(kThreads), 0, st, p, pv, steps, vec);
  if (p.rank <= 64) return launch_pdl(adapter_up_kernel<4, TY>, grid, dim3(kThreads), 0, st, p, pv, steps, vec);
  return launch_pdl(adapter_up_kernel<8, TY>, grid, dim3(kThreads), 0, st, p, pv, steps, vec);
}

amph_status project_adapters(const void* x_dev, int32_t x_rows_cap, const void* const* w, int32_t n_seg, int32_t out, int32_t in,
                             int32_t rows, int32_t dtype, int32_t use_tensor_core, const amph_adapters* ad, const int32_t* row_adapter,
                             void* y_dev, int32_t y_dtype, void* ws_dev, size_t ws_bytes, int32_t* status_dev, cudaStream_t st) {
  if (!x_dev || !w || !ad || !ad->a || !ad->b || !row_adapter || !y_dev) return api_fail(AMPH_ERR_INVALID_ARG, "NULL pointer");
  amph_status rc = bad_shape(n_seg, out, rows, ad->rank);
  if (rc != AMPH_OK) return rc;
  for (int s = 0; s < n_seg; ++s)
    if (!w[s]) return api_fail(AMPH_ERR_INVALID_ARG, "NULL pointer");
  if (in < 8 || x_rows_cap < rows || ad->n_adapters < 1) return api_fail(AMPH_ERR_SHAPE, "bad projection shape");
  if ((dtype != AMPH_DTYPE_F32 && dtype != AMPH_DTYPE_BF16) || in % (dtype == AMPH_DTYPE_F32 ? 4 : 8))
    return api_fail(AMPH_ERR_SHAPE, "unknown dtype, or a row of `in` elements is not a multiple of 16 bytes");
  if (y_dtype != AMPH_DTYPE_F32 && (y_dtype != AMPH_DTYPE_BF16 || dtype != AMPH_DTYPE_BF16))
    return api_fail(AMPH_ERR_SHAPE, "y_dtype must be fp32, or bf16 with bf16 weights");
  uintptr_t all = (uintptr_t)x_dev | (uintptr_t)ad->a | (uintptr_t)ad->b | (uintptr_t)y_dev;
  for (int s = 0; s < n_seg; ++s) all |= (uintptr_t)w[s];
  if (all & 15) return api_fail(AMPH_ERR_INVALID_ARG, "x, w, the adapters and y must be 16-byte aligned");
  size_t need = 0;
  amph_project_adapters_bytes(n_seg, out, rows, ad->rank, &need);
  if (!ws_dev || ws_bytes < need || ((uintptr_t)ws_dev & 255))
    return api_fail(AMPH_ERR_WORKSPACE, "scratch: %zu bytes needed, 256-byte aligned", need);
  const size_t ld = (size_t)n_seg * out, tb = tiles_bytes(rows) + t_bytes(n_seg, rows, ad->rank);
  const int cols = n_seg * ad->rank, tiles = most_tiles(rows, ad->n_adapters), col_blocks = (cols + kDownCols - 1) / kDownCols;
  AdapterArgs p;
  p.x = x_dev; p.a = ad->a; p.b = ad->b; p.scale = ad->scale;
  p.row_adapter = row_adapter;
  p.tiles = (RowTile*)ws_dev;
  p.t = (float*)((char*)ws_dev + tiles_bytes(rows));
  p.y = y_dev;
  p.status = status_dev;
  p.n_adapters = ad->n_adapters; p.rank = ad->rank; p.n_seg = n_seg; p.out = out; p.in = in; p.rows = rows; p.splits = dtype == AMPH_DTYPE_F32 ? 1 : down_splits(in, tiles * col_blocks);
  PartialView pv;
  pv.p = (float*)((char*)ws_dev + tb);
  pv.ld = (int)ld;
  pv.splits = 1;
  pv.split_stride = 0;
  float* P = (float*)((char*)ws_dev + tb);
  const size_t p_floats = (ws_bytes - tb) / sizeof(float);

  std::unique_lock<std::mutex> lock(g_mutex, std::defer_lock);
  TcGemm* g = nullptr;
  if (use_tensor_core) {
    if (dtype != AMPH_DTYPE_BF16 || out % 128 || in % 64 || x_rows_cap < padded(rows))
      return api_fail(AMPH_ERR_SHAPE, "shape not covered by the tensor-core kernel");
    int dev = -1;
    if (cudaGetDevice(&dev) != cudaSuccess || dev < 0 || dev >= kMaxDevices) {
      cudaGetLastError();
      return api_fail(AMPH_ERR_CUDA, "no usable current device");
    }
    void* xb[1] = {const_cast<void*>(x_dev)};
    const int xr[1] = {x_rows_cap}, xc[1] = {in};
    lock.lock();
    if (!g_plans[dev]) {
      g_plans[dev] = tc_gemm_create(xb, xr, xc, 1, status_dev);
      if (g_plans[dev]) tc_wide_init(g_plans[dev]);
    }
    g = g_plans[dev];
    if (!g) return api_fail(AMPH_ERR_CUDA, "tensor-map encoder unavailable or not an sm_100 device");
    g->cache.clear();                       // tensor maps are made for each call
    tc_gemm_rebind(g, 0, xb[0], x_rows_cap, in, status_dev);
  }
  cudaError_t e;
  if (dtype == AMPH_DTYPE_F32)
    e = launch_pdl(adapter_down_plain_kernel, dim3((cols + 3) / 4, rows), dim3(kThreads), 0, st, p);
  else
    e = launch_pdl(adapter_down_kernel, dim3(tiles, p.splits, col_blocks), dim3(kThreads), 0, st, p);
  if (e == cudaSuccess) {
    if (g) {
      int splits = 0;
      size_t stride = 0;
      // The weights are fetched while the kernel ahead still runs: that is adapter_down, which starts its successor only when
      // everything ahead of itself is done.
      if (!tc_gemm_launch(g, 0, w, n_seg, out, in, rows, P, p_floats, &splits, &stride, st))
        return api_fail(AMPH_ERR_SHAPE, "shape not covered by the tensor-core kernel");
      pv.splits = splits;
      pv.split_stride = stride;
    } else {
      // the plain kernel takes blocks of up to kMaxRows rows as the context's passes do
      GemmSeg segs[kMaxK];
      for (int s = 0; s < n_seg; ++s) segs[s].w = w[s];
      launch_gemm_generic(x_dev, in, segs, n_seg, out, in, P, (int)ld, rows, dtype, st);
    }
    if (dtype == AMPH_DTYPE_F32)
      e = launch_pdl(adapter_up_plain_kernel, dim3((unsigned)((ld + kThreads - 1) / kThreads), rows), dim3(kThreads), 0, st, p, pv);
    else
      e = y_dtype == AMPH_DTYPE_F32 ? run_up<float>(p, pv, tiles, st) : run_up<bf16>(p, pv, tiles, st);
  }
  const cudaError_t last = cudaGetLastError();
  if (e == cudaSuccess) e = last;
  if (e != cudaSuccess) return api_fail(AMPH_ERR_CUDA, "amph_project_adapters: %s", cudaGetErrorString(e));
  return AMPH_OK;
}

}  // namespace
}  // namespace amph

using namespace amph;

extern "C" {

amph_status amph_project_adapters_bytes(int32_t n_seg, int32_t out, int32_t rows, int32_t rank, size_t* ws_bytes) {
  if (!ws_bytes) return api_fail(AMPH_ERR_INVALID_ARG, "ws_bytes must not be NULL");
  const amph_status rc = bad_shape(n_seg, out, rows, rank);
  if (rc != AMPH_OK) return rc;
  *ws_bytes = tiles_bytes(rows) + t_bytes(n_seg, rows, rank) + round256((size_t)most_splits(n_seg, out) * padded(rows) * n_seg * out * sizeof(float));
  return AMPH_OK;
}

amph_status amph_project_adapters(const void* x_dev, int32_t x_rows_cap, const void* const* w, int32_t n_seg, int32_t out,
                                  int32_t in, int32_t rows, int32_t dtype, int32_t use_tensor_core, const amph_adapters* adapters,
                                  const int32_t* row_adapter, void* y_dev, int32_t y_dtype, void* ws_dev, size_t ws_bytes,
                                  int32_t* status_dev, void* stream) {
  try {                                     // the tensor maps live in a container of the host's
    return project_adapters(x_dev, x_rows_cap, w, n_seg, out, in, rows, dtype, use_tensor_core, adapters, row_adapter, y_dev, y_dtype,
                            ws_dev, ws_bytes, status_dev, (cudaStream_t)stream);
  } catch (...) {
    return AMPH_ERR_CUDA;
  }
}

}  // extern "C"
