// amph_project_adapters: a projection shared by all rows, and each row's own low-rank adapter beside it.
//
//   t[r][s][j] = sum_k x[r][k] a[i_r][s][j][k]                       the rows' low-rank products (down)
//   P          = x . w^T                                             the projection kernels, as split-K partial sums
//   y[r][s][o] = sum P + scale[i_r] sum_j t[r][s][j] b[i_r][s][o][j]  reduction of the partial sums, adapters' way back up (up)
//
// Small projections and those that the tensor-core kernels do not take: down, then all of y in one kernel (whole; fp32: the plain
// projection's epilogue).  A few rows: down and up in one kernel (few).
#include <math.h>

#include <mutex>

#include "amph_internal.cuh"
#include "gemm_tc_common.cuh"

namespace amph {
namespace {

typedef __nv_bfloat16 bf16;

constexpr int kMaxRowsAll = 4 * kMaxRows;
constexpr int kThreads = 128;

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
  float* t;                // fp32: [rows][n_seg * rank]
  bf16 *t_hi, *t_lo;       // bf16: the same, times scale, in two halves
  void* y;
  int* status;
  int n_adapters, rank, n_seg, out, in, rows, splits;
  int beside;              // bf16: adapter_down runs beside the kernel ahead of it (the projection)
};

// The row's adapter, -1 if it has none (or names one that does not exist, which is reported).
__device__ __forceinline__ int adapter_of(const AdapterArgs& p, int row) {
  const int a = __ldcg(p.row_adapter + row);
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

__device__ __forceinline__ void mma_16816(float (&d)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
  asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
               : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3]) : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}

// Tile `want` of the call's rows: the rows of one adapter in their order, 16 at a time, tiles in the order of their first rows.  Every
// block finds its own (an adapter's rows may lie anywhere): row r is the c-th of its adapter, c = how many rows ahead of it name the same.
// The adapters get slots of a hash table (twice as many as rows), a strip of 32 rows counts its own per slot, a row adds up the strips
// ahead of its own.  (Comparing every row with all rows ahead of it: 4.7 us more per block at 512 rows, the same at 64.)
constexpr int kStrips = kMaxRowsAll / 32, kSlots = 2 * kMaxRowsAll;
struct __align__(16) TileSmem {
  uint8_t count[kSlots][kStrips];
  int key[kSlots];
  short slot[kMaxRowsAll], nth[kMaxRowsAll];
  int firsts[kStrips];
};
static_assert(kStrips == 16, "a slot's counts are one 16-byte word");
constexpr int kDownThreads = 256, kDownWarps = kDownThreads / 32;
__device__ __forceinline__ bool find_tile(const AdapterArgs& p, int want, TileSmem& sm, RowTile& tile, int& leader) {
  constexpr int kNoKey = -2;                 // (adapter_of() answers -1 or more)
  constexpr int kPer = kMaxRowsAll / kDownThreads;
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  const unsigned ahead = (1u << lane) - 1u;
  int slots = 64;
  while (slots < 2 * p.rows) slots *= 2;
  int adapter[kPer];
#pragma unroll
  for (int i = 0; i < kPer; ++i) {
    const int r = i * kDownThreads + tid;
    adapter[i] = r < p.rows ? adapter_of(p, r) : kNoKey;
  }
  for (int i = tid; i < slots; i += kDownThreads) {
    sm.key[i] = kNoKey;
    *reinterpret_cast<uint4*>(sm.count[i]) = make_uint4(0u, 0u, 0u, 0u);
  }
  if (tid == 0) { leader = -1; tile.n = 0; tile.adapter = -1; }
  __syncthreads();
  unsigned same[kPer];
#pragma unroll
  for (int i = 0; i < kPer; ++i) {
    const int strip = i * kDownWarps + warp;
    if (strip * 32 >= p.rows) break;
    same[i] = __match_any_sync(~0u, adapter[i]);
    const int first = __ffs(same[i]) - 1;
    int at = 0;
    if (lane == first && adapter[i] != kNoKey) {
      at = (int)((uint32_t)adapter[i] * 2654435769u >> 16) & (slots - 1);
      for (;;) {
        const int was = atomicCAS(&sm.key[at], kNoKey, adapter[i]);
        if (was == kNoKey || was == adapter[i]) break;
        at = (at + 1) & (slots - 1);
      }
      sm.count[at][strip] = (uint8_t)__popc(same[i]);
    }
    at = __shfl_sync(~0u, at, first);
    sm.slot[strip * 32 + lane] = (short)at;              // (rows behind the last: not read)
  }
  __syncthreads();
  unsigned firsts[kPer];
#pragma unroll
  for (int i = 0; i < kPer; ++i) {
    const int strip = i * kDownWarps + warp, r = strip * 32 + lane;
    firsts[i] = 0;
    if (strip * 32 >= p.rows) break;
    int c = __popc(same[i] & ahead);
    if (r < p.rows) {
      const uint4 n = *reinterpret_cast<const uint4*>(sm.count[sm.slot[r]]);
      const unsigned words[4] = {n.x, n.y, n.z, n.w};
#pragma unroll
      for (int w = 0; w < 4; ++w) {
        const int left = strip - 4 * w;                  // strips of this word that are ahead
        const unsigned mask = left >= 4 ? 0xffffffffu : left <= 0 ? 0u : (1u << (8 * left)) - 1u;
        c = (int)__dp4a(words[w] & mask, 0x01010101u, (unsigned)c);
      }
      sm.nth[r] = (short)c;
    }
    firsts[i] = __ballot_sync(~0u, r < p.rows && c % kTileRows == 0);
    if (lane == 0) sm.firsts[strip] = __popc(firsts[i]);
  }
  __syncthreads();
#pragma unroll
  for (int i = 0; i < kPer; ++i) {
    const int strip = i * kDownWarps + warp;
    if ((firsts[i] >> lane) & 1) {
      int at = __popc(firsts[i] & ahead);
      for (int w = 0; w < strip; ++w) at += sm.firsts[w];
      if (at == want) leader = strip * 32 + lane;
    }
    if (strip * 32 >= p.rows) break;
  }
  __syncthreads();
  const int lead = leader;
  if (lead < 0) return false;
  const int slot = sm.slot[lead], c0 = sm.nth[lead];
  if (tid == 0) tile.adapter = sm.key[slot];
  for (int r = tid; r < p.rows; r += kDownThreads) {
    const int c = sm.nth[r] - c0;
    if (sm.slot[r] == slot && c >= 0 && c < kTileRows) {
      tile.row[c] = (uint16_t)r;
      atomicMax(&tile.n, c + 1);
    }
  }
  __syncthreads();
  return true;
}

// bf16 of a value, and what that loses (nothing where it is an infinity): 16 bits of the value in two halves.
__device__ __forceinline__ void halves(float v, bf16& hi, bf16& lo) {
  hi = __float2bfloat16_rn(v);
  const float d = v - __bfloat162float(hi);
  lo = __float2bfloat16_rn(fabsf(d) < INFINITY ? d : 0.f);
}

// t of one tile of rows: grid (tile, K range, 32 columns of t), a cluster holds the K ranges.  MMA with the rows as A (M = 16) and the
// adapter's rows as B, both straight from global memory: the sum over k may run in any order that both share, so a lane takes 16
// contiguous bytes for two steps.  The warps take turns at 64 columns of k and meet in shared memory, the ranges in that of the cluster's
// first block; what leaves is scale * t as two bf16 halves (2^-17 of the adapter's share), the way adapter_up's MMA takes it.
// `beside`: the kernel ahead is the tensor-core projection, which starts this one once everything ahead of itself is done, so it takes
// the SMs and the shared memory that the projection leaves; what it reads is older than the projection (and past L1, see pdl_wait); only the first block
// waits for the projection, so that both are done when this one is.  (Ahead of the projection, q / k / v of 64 rows of 24
// tenants took 36.1 us in all, 28.0 now; gate / up of 37 rows at rank 64 48.5, 42.9 now; 512 rows, see down_splits, 59 and 48.7.)  72 registers:
// beside a CTA of the pair kernel an SM's schedulers have room for two such warps each, not for two of 80.
// Bound: latency for a few rows, the adapters' bytes for many tenants.
constexpr int kDownCols = 32;
constexpr int kMaxDownSplits = 8;
__global__ void __maxnreg__(72) adapter_down_kernel(const AdapterArgs p) {
  __shared__ union {
    TileSmem find;
    float red[kDownWarps][kTileRows][kDownCols + 2];
    float part[kMaxDownSplits - 1][kTileRows * kDownCols];               // of the cluster's other blocks, in the first one
  } sm;
  __shared__ RowTile tile;
  __shared__ int leader;
  const bool alone = p.splits == 1;
  if (!p.beside) pdl_wait();
  pdl_launch_dependents();
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31, g = lane >> 2, t = lane & 3;
  const bool waits = p.beside && blockIdx.x == 0 && blockIdx.y == 0 && blockIdx.z == 0;
  const bool any = find_tile(p, blockIdx.x, sm.find, tile, leader);
  if (blockIdx.y == 0 && blockIdx.z == 0 && tid == 0) p.tiles[blockIdx.x] = tile;
  const int n = any && tile.adapter >= 0 ? tile.n : 0;               // the same in the whole cluster
  const int cols = p.n_seg * p.rank, col0 = blockIdx.z * kDownCols;
  const int nt = min(kDownCols, cols - col0) / 8, width = nt * 8;
  if (n > 0) {
    const int steps = (p.in + 63) / 64;
    const int s0 = steps * (int)blockIdx.y / p.splits, s1 = steps * ((int)blockIdx.y + 1) / p.splits;
    const bf16* x[2];
    x[0] = g < n ? (const bf16*)p.x + (size_t)tile.row[g] * p.in : nullptr;
    x[1] = g + 8 < n ? (const bf16*)p.x + (size_t)tile.row[g + 8] * p.in : nullptr;
    const bf16* a = (const bf16*)p.a + ((size_t)tile.adapter * cols + col0 + g) * p.in;
    float acc[kDownCols / 8][4];
#pragma unroll
    for (int j = 0; j < kDownCols / 8; ++j) acc[j][0] = acc[j][1] = acc[j][2] = acc[j][3] = 0.f;
    const uint4 zero = make_uint4(0u, 0u, 0u, 0u);
#pragma unroll 2
    for (int s = s0 + warp; s < s1; s += kDownWarps) {
      uint4 xv[2][2], av[kDownCols / 8][2];
#pragma unroll
      for (int c = 0; c < 2; ++c) {
        const int k = s * 64 + c * 32 + t * 8;
#pragma unroll
        for (int i = 0; i < 2; ++i) xv[i][c] = x[i] != nullptr && k < p.in ? __ldcg(reinterpret_cast<const uint4*>(x[i] + k)) : zero;
#pragma unroll
        for (int j = 0; j < kDownCols / 8; ++j)
          av[j][c] = j < nt && k < p.in ? __ldcg(reinterpret_cast<const uint4*>(a + (size_t)j * 8 * p.in + k)) : zero;
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
        *reinterpret_cast<float2*>(&sm.red[warp][g][j * 8 + 2 * t]) = make_float2(acc[j][0], acc[j][1]);
        *reinterpret_cast<float2*>(&sm.red[warp][g + 8][j * 8 + 2 * t]) = make_float2(acc[j][2], acc[j][3]);
      }
  }
  __syncthreads();
  float mine[kTileRows * kDownCols / kDownThreads];
#pragma unroll
  for (int q = 0; q < kTileRows * kDownCols / kDownThreads; ++q) {
    const int i = q * kDownThreads + tid, r = i / width, c = i - r * width;
    mine[q] = 0.f;
    if (i < n * width) {
      mine[q] = sm.red[0][r][c];
#pragma unroll
      for (int w = 1; w < kDownWarps; ++w) mine[q] += sm.red[w][r][c];
    }
  }
  if (!alone) {
    __syncwarp();                                                    // every block has read its warps' sums
    asm volatile("barrier.cluster.arrive.release.aligned;\nbarrier.cluster.wait.acquire.aligned;" ::: "memory");
    if (blockIdx.y > 0) {
#pragma unroll
      for (int q = 0; q < kTileRows * kDownCols / kDownThreads; ++q) {
        const int i = q * kDownThreads + tid;
        if (i < n * width) {
          uint32_t there;
          asm volatile("mapa.shared::cluster.u32 %0, %1, 0;" : "=r"(there) : "r"((uint32_t)__cvta_generic_to_shared(&sm.part[blockIdx.y - 1][i])));
          asm volatile("st.shared::cluster.f32 [%0], %1;" ::"r"(there), "f"(mine[q]) : "memory");
        }
      }
    }
    __syncwarp();
    asm volatile("barrier.cluster.arrive.release.aligned;\nbarrier.cluster.wait.acquire.aligned;" ::: "memory");
    if (blockIdx.y > 0) return;
  }
  if (n == 0) {
    if (waits) pdl_wait();
    return;
  }
  const float scale = p.scale ? __ldcg(p.scale + tile.adapter) : 1.f;
#pragma unroll
  for (int q = 0; q < kTileRows * kDownCols / kDownThreads; ++q) {
    const int i = q * kDownThreads + tid, r = i / width, c = i - r * width;
    if (i < n * width) {
      float v = mine[q];
#pragma unroll
      for (int k = 1; k < kMaxDownSplits; ++k)
        if (k < p.splits) v += sm.part[k - 1][i];
      const size_t at = (size_t)tile.row[r] * cols + col0 + c;
      halves(scale * v, p.t_hi[at], p.t_lo[at]);
    }
  }
  if (waits) pdl_wait();
}

__device__ __forceinline__ uint32_t pack(float lo, float hi) {
  const __nv_bfloat162 h = __floats2bfloat162_rn(lo, hi);
  return *reinterpret_cast<const uint32_t*>(&h);
}
__device__ __forceinline__ void add4(float4& a, const float4 v) { a.x += v.x; a.y += v.y; a.z += v.z; a.w += v.w; }
__device__ __forceinline__ float4 get4(const float* p) { return *reinterpret_cast<const float4*>(p); }
__device__ __forceinline__ void put(float* p, float v) { *p = v; }
__device__ __forceinline__ void put(bf16* p, float v) { *p = __float2bfloat16_rn(v); }
__device__ __forceinline__ void put_all(float* p, float4 v) { *reinterpret_cast<float4*>(p) = v; }
__device__ __forceinline__ void put_all(bf16* p, float4 v) { *reinterpret_cast<uint2*>(p) = make_uint2(pack(v.x, v.y), pack(v.z, v.w)); }
// four values (VEC), or the first `left` of them
template <bool VEC, typename TY>
__device__ __forceinline__ void put4(TY* p, float4 v, int left) {
  if constexpr (VEC) { put_all(p, v); return; }
  put(p, v.x);
  if (left > 1) put(p + 1, v.y);
  if (left > 2) put(p + 2, v.z);
  if (left > 3) put(p + 3, v.w);
}

// Reduction of the projection's partial sums, the adapters' way back up, one rounding: grid (columns, tile, segment), a warp has 16
// columns of the tile's rows at a time.  MMA with t's halves as A and b as B.  As in adapter_down the sum over j may run in any order: a
// lane takes four (rank up to 16: QUADS = 0) or eight neighbouring j, QUADS is how many times 32 of them.  A lane's two output tiles are
// numbered so that it owns four neighbouring columns.  A lane without a row reads row 0's sums, unconditionally (loads behind a branch are
// waited for one by one: 7.4 us instead of 3.6 for one row of 4096), and writes nothing.  out is a multiple of 128 (as the projection wants it),
// so a warp's columns are there or not as a whole.  Bound: L2 (partial sums) and the bytes of b and y.
__host__ __device__ constexpr int up_groups(int quads) { return quads <= 2 ? 2 : 1; }        // 16 columns each, whose loads are in flight together
template <int QUADS, typename TY>
__global__ void __launch_bounds__(kThreads) adapter_up_kernel(const AdapterArgs p, const PartialView P, int steps) {
  pdl_wait();
  pdl_launch_dependents();
  constexpr int CHUNKS = QUADS ? QUADS : 1, J = QUADS ? 8 : 4;           // j of a lane per chunk of 4 J
  constexpr int GROUPS = up_groups(QUADS);
  const RowTile& tile = p.tiles[blockIdx.y];
  const int n = tile.n, adapter = tile.adapter, seg = blockIdx.z;
  if (n == 0) return;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, g = lane >> 2, t = lane & 3;
  const int cols = p.n_seg * p.rank;
  int row[2];
  row[0] = g < n ? tile.row[g] : -1;
  row[1] = g + 8 < n ? tile.row[g + 8] : -1;
  uint32_t hi[2][CHUNKS][J / 2], lo[2][CHUNKS][J / 2];                   // [row][chunk][pair of j]
  auto load_j = [&](const bf16* src, bool there, uint32_t (&v)[J / 2]) {
    if constexpr (J == 8) {
      const uint4 u = there ? *reinterpret_cast<const uint4*>(src) : make_uint4(0u, 0u, 0u, 0u);
      v[0] = u.x; v[1] = u.y; v[2] = u.z; v[3] = u.w;
    } else {
      const uint2 u = there ? *reinterpret_cast<const uint2*>(src) : make_uint2(0u, 0u);
      v[0] = u.x; v[1] = u.y;
    }
  };
  if (adapter >= 0) {
#pragma unroll
    for (int c = 0; c < CHUNKS; ++c)
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        const int j = (c * 4 + t) * J;
        const size_t at = (size_t)(row[i] < 0 ? 0 : row[i]) * cols + seg * p.rank + j;
        load_j(p.t_hi + at, row[i] >= 0 && j < p.rank, hi[i][c]);
        load_j(p.t_lo + at, row[i] >= 0 && j < p.rank, lo[i][c]);
      }
  }
  const bf16* b = (const bf16*)p.b + ((size_t)(adapter < 0 ? 0 : adapter) * p.n_seg + seg) * p.out * p.rank;
  for (int step = 0; step < steps; ++step) {
    const int c0 = ((blockIdx.x * steps + step) * (kThreads / 32) + warp) * 16 * GROUPS;
    if (c0 >= p.out) return;
    uint32_t bv[GROUPS][2][CHUNKS][J / 2];
    if (adapter >= 0) {
#pragma unroll
      for (int q = 0; q < GROUPS; ++q)
#pragma unroll
        for (int i = 0; i < 2; ++i) {
          const int o = c0 + q * 16 + 4 * (g >> 1) + 2 * i + (g & 1);
#pragma unroll
          for (int c = 0; c < CHUNKS; ++c) {
            const int j = (c * 4 + t) * J;
            load_j(b + (size_t)o * p.rank + j, j < p.rank, bv[q][i][c]);
          }
        }
    }
    float4 sum[GROUPS][2];
#pragma unroll
    for (int q = 0; q < GROUPS; ++q)
#pragma unroll
      for (int i = 0; i < 2; ++i) sum[q][i] = make_float4(0.f, 0.f, 0.f, 0.f);
    const float* src[GROUPS][2];
#pragma unroll
    for (int q = 0; q < GROUPS; ++q)
#pragma unroll
      for (int i = 0; i < 2; ++i) src[q][i] = P.p + (size_t)max(row[i], 0) * P.ld + seg * p.out + c0 + q * 16 + 4 * t;
#pragma unroll 4
    for (int s = 0; s < P.splits; ++s)
#pragma unroll
      for (int q = 0; q < GROUPS; ++q)
#pragma unroll
        for (int i = 0; i < 2; ++i) add4(sum[q][i], get4(src[q][i] + s * P.split_stride));
    if (adapter >= 0) {
#pragma unroll
      for (int q = 0; q < GROUPS; ++q) {
        float acc[2][4];
#pragma unroll
        for (int i = 0; i < 2; ++i) {
          acc[i][0] = acc[i][1] = acc[i][2] = acc[i][3] = 0.f;
#pragma unroll
          for (int c = 0; c < CHUNKS; ++c)
#pragma unroll
            for (int k = 0; k < J / 2; k += 2) {
              mma_16816(acc[i], lo[0][c][k], lo[1][c][k], lo[0][c][k + 1], lo[1][c][k + 1], bv[q][i][c][k], bv[q][i][c][k + 1]);
              mma_16816(acc[i], hi[0][c][k], hi[1][c][k], hi[0][c][k + 1], hi[1][c][k + 1], bv[q][i][c][k], bv[q][i][c][k + 1]);
            }
        }
        add4(sum[q][0], make_float4(acc[0][0], acc[0][1], acc[1][0], acc[1][1]));
        add4(sum[q][1], make_float4(acc[0][2], acc[0][3], acc[1][2], acc[1][3]));
      }
    }
#pragma unroll
    for (int q = 0; q < GROUPS; ++q)
#pragma unroll
      for (int i = 0; i < 2; ++i)
        if (row[i] >= 0) put_all((TY*)p.y + (size_t)row[i] * P.ld + seg * p.out + c0 + q * 16 + 4 * t, sum[q][i]);
  }
}

// adapter_down and adapter_up in one for a few rows (kFewRows) and a small rank: grid (128 columns, tile, segment), a block works out its
// tile's t itself while the projection ahead still runs (which has started it once everything ahead of itself was done, see pdl_wait), holds b in registers,
// waits, and adds the partial sums.  Its warps share K for t and have 16 columns each for y.  (One row of 4096 x 4096, rank 16: 9.4 us, 11.3
// with the two kernels, and one launch less for the host.)
constexpr int kFewRows = 16, kFewRank = 32;
template <int QUADS, typename TY>
__global__ void __launch_bounds__(kDownThreads) adapter_few_kernel(const __grid_constant__ AdapterArgs p, const PartialView P) {
  constexpr int J = QUADS ? 8 : 4, NT = J / 2;                           // j of a lane; eights of the rank
  __shared__ __align__(16) float red[kDownWarps][kTileRows][8 * NT + 4];
  __shared__ __align__(16) bf16 t_hi[kTileRows][8 * NT], t_lo[kTileRows][8 * NT];
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31, g = lane >> 2, t = lane & 3, seg = blockIdx.z;
  // the tile: an adapter's rows, adapters in the order of their first rows; every warp finds it
  const int mine = lane < p.rows ? adapter_of(p, lane) : -2;
  const unsigned same = __match_any_sync(~0u, mine);
  const unsigned firsts = __ballot_sync(~0u, mine != -2 && __ffs(same) - 1 == lane);
  const int first = __fns(firsts, 0, blockIdx.y + 1);                     // lane of this tile's first row
  if ((int)blockIdx.y >= __popc(firsts)) {
    pdl_wait();
    return;
  }
  const int adapter = __shfl_sync(~0u, mine, first);
  const unsigned rows = __shfl_sync(~0u, same, first);
  const int n = __popc(rows);
  int row[2];
#pragma unroll
  for (int i = 0; i < 2; ++i) row[i] = __fns(rows, 0, (g + 8 * i < n ? g + 8 * i : 0) + 1);
  const int c0 = (blockIdx.x * kDownWarps + warp) * 16;
  uint32_t hi[2][J / 2], lo[2][J / 2], b[2][J / 2];
  if (adapter >= 0) {
    const bf16* bs = (const bf16*)p.b + ((size_t)adapter * p.n_seg + seg) * p.out * p.rank;
    const bool is = t * J < p.rank;
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      const bf16* src = bs + (size_t)(c0 + 4 * (g >> 1) + 2 * i + (g & 1)) * p.rank + (is ? t * J : 0);
#pragma unroll
      for (int k = 0; k < J / 2; k += 2) {
        const uint2 u = __ldcg(reinterpret_cast<const uint2*>(src + 2 * k));
        b[i][k] = is ? u.x : 0u;
        b[i][k + 1] = is ? u.y : 0u;
      }
    }
    const bf16* a = (const bf16*)p.a + (((size_t)adapter * p.n_seg + seg) * p.rank) * p.in;
    const int nt = p.rank / 8, steps = p.in / 64;
    float acc[NT][4];
#pragma unroll
    for (int j = 0; j < NT; ++j) acc[j][0] = acc[j][1] = acc[j][2] = acc[j][3] = 0.f;
#pragma unroll 2
    for (int s = warp; s < steps; s += kDownWarps) {
      uint4 xv[2][2], av[NT][2];
#pragma unroll
      for (int c = 0; c < 2; ++c) {
        const int k = s * 64 + c * 32 + t * 8;
#pragma unroll
        for (int i = 0; i < 2; ++i) xv[i][c] = __ldcg(reinterpret_cast<const uint4*>((const bf16*)p.x + (size_t)row[i] * p.in + k));
#pragma unroll
        for (int j = 0; j < NT; ++j) av[j][c] = __ldcg(reinterpret_cast<const uint4*>(a + (size_t)((j < nt ? j : 0) * 8 + g) * p.in + k));
      }
#pragma unroll
      for (int j = 0; j < NT; ++j)
#pragma unroll
        for (int c = 0; c < 2; ++c) {
          mma_16816(acc[j], xv[0][c].x, xv[1][c].x, xv[0][c].y, xv[1][c].y, av[j][c].x, av[j][c].y);
          mma_16816(acc[j], xv[0][c].z, xv[1][c].z, xv[0][c].w, xv[1][c].w, av[j][c].z, av[j][c].w);
        }
    }
#pragma unroll
    for (int j = 0; j < NT; ++j) {
      *reinterpret_cast<float2*>(&red[warp][g][j * 8 + 2 * t]) = make_float2(acc[j][0], acc[j][1]);
      *reinterpret_cast<float2*>(&red[warp][g + 8][j * 8 + 2 * t]) = make_float2(acc[j][2], acc[j][3]);
    }
    __syncthreads();
    const float scale = p.scale ? __ldcg(p.scale + adapter) : 1.f;
    for (int i = tid; i < kTileRows * 8 * NT; i += kDownThreads) {
      const int q = i / (8 * NT), j = i % (8 * NT);
      float v = 0.f;
#pragma unroll
      for (int w = 0; w < kDownWarps; ++w) v += red[w][q][j];
      halves(j < p.rank ? scale * v : 0.f, t_hi[q][j], t_lo[q][j]);
    }
    __syncthreads();
#pragma unroll
    for (int i = 0; i < 2; ++i)
#pragma unroll
      for (int k = 0; k < J / 2; k += 2) {
        const uint2 u = *reinterpret_cast<const uint2*>(&t_hi[g + 8 * i][t * J + 2 * k]), v = *reinterpret_cast<const uint2*>(&t_lo[g + 8 * i][t * J + 2 * k]);
        hi[i][k] = u.x; hi[i][k + 1] = u.y;
        lo[i][k] = v.x; lo[i][k + 1] = v.y;
      }
  }
  pdl_wait();                                                             // the partial sums
  pdl_launch_dependents();
  const int col = c0 + 4 * t;
  float4 sum[2] = {make_float4(0.f, 0.f, 0.f, 0.f), make_float4(0.f, 0.f, 0.f, 0.f)};
  const float* src[2];
#pragma unroll
  for (int i = 0; i < 2; ++i) src[i] = P.p + (size_t)row[i] * P.ld + seg * p.out + col;
#pragma unroll 8
  for (int s = 0; s < P.splits; ++s)
#pragma unroll
    for (int i = 0; i < 2; ++i) add4(sum[i], get4(src[i] + s * P.split_stride));
  if (adapter >= 0) {
    float acc[2][4];
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      acc[i][0] = acc[i][1] = acc[i][2] = acc[i][3] = 0.f;
#pragma unroll
      for (int k = 0; k < J / 2; k += 2) {
        mma_16816(acc[i], lo[0][k], lo[1][k], lo[0][k + 1], lo[1][k + 1], b[i][k], b[i][k + 1]);
        mma_16816(acc[i], hi[0][k], hi[1][k], hi[0][k + 1], hi[1][k + 1], b[i][k], b[i][k + 1]);
      }
    }
    add4(sum[0], make_float4(acc[0][0], acc[0][1], acc[1][0], acc[1][1]));
    add4(sum[1], make_float4(acc[0][2], acc[0][3], acc[1][2], acc[1][3]));
  }
#pragma unroll
  for (int i = 0; i < 2; ++i)
    if (g + 8 * i < n) put_all((TY*)p.y + (size_t)row[i] * P.ld + seg * p.out + col, sum[i]);
}

// The whole of y behind adapter_down, for projections that are small or that the tensor-core kernels do not take: grid (32 columns, tile,
// segment).  A block's warps share K, 64 of it at a time, and the rank, 32 of it at a time; both are terms of one sum of MMAs (rows as A,
// weights or b as B, t in two halves), which meets in shared memory.  Every tile reads the weights again.  Bound: latency for small shapes,
// else L2.
struct Weights { const void* w[kMaxK]; };
constexpr int kWholeCols = 32;
template <bool VEC, typename TY>
__global__ void __launch_bounds__(kThreads) adapter_whole_kernel(const __grid_constant__ AdapterArgs p, const __grid_constant__ Weights ws) {
  pdl_wait();
  pdl_launch_dependents();
  constexpr int WARPS = kThreads / 32;
  __shared__ __align__(16) float red[WARPS][kTileRows][kWholeCols + 4];
  const RowTile& tile = p.tiles[blockIdx.y];
  const int n = tile.n, adapter = tile.adapter, seg = blockIdx.z, c0 = blockIdx.x * kWholeCols;
  if (n == 0) return;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, g = lane >> 2, t = lane & 3;
  const int cols = p.n_seg * p.rank;
  const uint4 zero = make_uint4(0u, 0u, 0u, 0u);
  auto load = [](const bf16* q) { return __ldg(reinterpret_cast<const uint4*>(q)); };
  // Unconditional loads, as in adapter_up: a lane without a row or column reads the first row's or the last column's and writes nothing.
  int row[2], o[4];
#pragma unroll
  for (int i = 0; i < 2; ++i) row[i] = tile.row[g + 8 * i < n ? g + 8 * i : 0];
#pragma unroll
  for (int i = 0; i < 4; ++i) o[i] = min(c0 + (i >> 1) * 16 + 4 * (g >> 1) + 2 * (i & 1) + (g & 1), p.out - 1);
  float acc[4][4];
#pragma unroll
  for (int i = 0; i < 4; ++i) acc[i][0] = acc[i][1] = acc[i][2] = acc[i][3] = 0.f;
  const bf16 *x = (const bf16*)p.x, *w = (const bf16*)ws.w[seg];
  const int steps = (p.in + 63) / 64;
  for (int s = warp; s < steps; s += WARPS) {
    uint4 xv[2][2], wv[4][2];
#pragma unroll
    for (int c = 0; c < 2; ++c) {
      const int k = min(s * 64 + c * 32 + t * 8, p.in - 8);
#pragma unroll
      for (int i = 0; i < 2; ++i) xv[i][c] = load(x + (size_t)row[i] * p.in + k);
#pragma unroll
      for (int i = 0; i < 4; ++i) wv[i][c] = load(w + (size_t)o[i] * p.in + k);
    }
    if (s * 64 + 64 > p.in) {
#pragma unroll
      for (int c = 0; c < 2; ++c)
        if (s * 64 + c * 32 + t * 8 >= p.in) {
          xv[0][c] = xv[1][c] = zero;
#pragma unroll
          for (int i = 0; i < 4; ++i) wv[i][c] = zero;
        }
    }
#pragma unroll
    for (int c = 0; c < 2; ++c)
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        mma_16816(acc[i], xv[0][c].x, xv[1][c].x, xv[0][c].y, xv[1][c].y, wv[i][c].x, wv[i][c].y);
        mma_16816(acc[i], xv[0][c].z, xv[1][c].z, xv[0][c].w, xv[1][c].w, wv[i][c].z, wv[i][c].w);
      }
  }
  const int j = (warp * 4 + t) * 8;                     // rank is at most 32 for each of the four warps
  static_assert(WARPS * 32 >= AMPH_MAX_ADAPTER_RANK, "every j has a warp");
  if (adapter >= 0 && warp * 32 < p.rank) {
    const bool is = j < p.rank;
    const bf16* b = (const bf16*)p.b + ((size_t)adapter * p.n_seg + seg) * p.out * p.rank;
    const int at = seg * p.rank + (is ? j : 0);
    uint4 hi[2], lo[2], bv[4];
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      hi[i] = *reinterpret_cast<const uint4*>(p.t_hi + (size_t)row[i] * cols + at);
      lo[i] = *reinterpret_cast<const uint4*>(p.t_lo + (size_t)row[i] * cols + at);
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) bv[i] = load(b + (size_t)o[i] * p.rank + (is ? j : 0));
    if (!is) {
      hi[0] = hi[1] = lo[0] = lo[1] = zero;
#pragma unroll
      for (int i = 0; i < 4; ++i) bv[i] = zero;
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      mma_16816(acc[i], lo[0].x, lo[1].x, lo[0].y, lo[1].y, bv[i].x, bv[i].y);
      mma_16816(acc[i], lo[0].z, lo[1].z, lo[0].w, lo[1].w, bv[i].z, bv[i].w);
      mma_16816(acc[i], hi[0].x, hi[1].x, hi[0].y, hi[1].y, bv[i].x, bv[i].y);
      mma_16816(acc[i], hi[0].z, hi[1].z, hi[0].w, hi[1].w, bv[i].z, bv[i].w);
    }
  }
#pragma unroll
  for (int q = 0; q < 2; ++q)
#pragma unroll
    for (int i = 0; i < 2; ++i)
      *reinterpret_cast<float4*>(&red[warp][g + 8 * i][q * 16 + 4 * t]) =
          make_float4(acc[2 * q][2 * i], acc[2 * q][2 * i + 1], acc[2 * q + 1][2 * i], acc[2 * q + 1][2 * i + 1]);
  __syncthreads();
  static_assert(kThreads * 4 == kTileRows * kWholeCols, "four sums a thread");
  const int r = threadIdx.x / (kWholeCols / 4), c = threadIdx.x % (kWholeCols / 4) * 4, col = c0 + c;
  float4 sum = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
  for (int q = 0; q < WARPS; ++q) add4(sum, *reinterpret_cast<const float4*>(&red[q][r][c]));
  if (r < n && col < p.out) put4<VEC>((TY*)p.y + (size_t)tile.row[r] * ((size_t)p.n_seg * p.out) + seg * p.out + col, sum, p.out - col);
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
// Weights that adapter_whole's tiles may read in all.  Up to there its two launches take no longer than the tensor-core kernel's three and cost
// the host 2.5 us less (three matrices of 512 x 512: 1 row 6.4 us, 6.8 with three; 128 rows, 19 MB, 8.3 and 8.5; 256 rows, 31 MB, 11.4 and 10.7).
constexpr int64_t kWholeBytes = 24 << 20;
// Tiles of rows that n_adapters adapters can make: each adapter, and the rows without one, rounds up once.
int most_tiles(int rows, int n_adapters) {
  const int64_t n = (int64_t)n_adapters + 1 + rows / kTileRows;
  return n < rows ? (int)n : rows;
}
// K ranges of adapter_down, a cluster: at most `most` blocks in all, 64 columns of k for each warp at least.  444: three blocks per SM; 168
// beside the pair kernel, which leaves room for one block on each SM that it uses (512 rows, out 4096, in 11008, rank 32: 48.7 us, 52.9 with 444;
// 128 rows, three matrices of 5120 x 5120, rank 16, 32 adapters: 43.7 us, 54.3 with 148 and so no cluster).
int down_splits(int in, int blocks, int most) {
  int s = 1;
  while (s < kMaxDownSplits && s * kDownWarps * 64 < in && 2 * s * blocks <= most) s *= 2;
  return s;
}
size_t tiles_bytes(int rows) { return round256(sizeof(RowTile) * rows); }

amph_status bad_shape(int n_seg, int out, int rows, int rank) {
  if (n_seg < 1 || n_seg > kMaxK || out < 1 || rows < 1 || rows > kMaxRowsAll) return api_fail(AMPH_ERR_SHAPE, "bad projection shape");
  if ((int64_t)n_seg * out > 0x7fffffff / 4) return api_fail(AMPH_ERR_SHAPE, "too many output features");
  if (rank < 8 || rank > AMPH_MAX_ADAPTER_RANK || rank % 8)
    return api_fail(AMPH_ERR_SHAPE, "rank must be a multiple of 8 in 8..%d (got %d)", AMPH_MAX_ADAPTER_RANK, rank);
  return AMPH_OK;
}
size_t t_bytes(int n_seg, int rows, int rank) { return round256((size_t)rows * n_seg * rank * sizeof(float)); }

template <int QUADS, typename TY>
cudaError_t run_up(const AdapterArgs& p, const PartialView& pv, int tiles, cudaStream_t st) {
  // a warp's columns: 16 or 32, or several times as many where that still leaves several blocks per SM
  const int cols = kThreads / 32 * 16 * up_groups(QUADS), blocks = (p.out + cols - 1) / cols;
  int steps = (int)((int64_t)blocks * tiles * p.n_seg / (148 * 8));
  steps = steps < 1 ? 1 : (steps > 4 ? 4 : steps);
  const dim3 grid((blocks + steps - 1) / steps, tiles, p.n_seg);
  return launch_pdl(adapter_up_kernel<QUADS, TY>, grid, dim3(kThreads), 0, st, p, pv, steps);
}
template <typename TY>
cudaError_t run_up(const AdapterArgs& p, const PartialView& pv, int tiles, cudaStream_t st) {
  if (p.rank <= 16) return run_up<0, TY>(p, pv, tiles, st);
  if (p.rank <= 32) return run_up<1, TY>(p, pv, tiles, st);
  if (p.rank <= 64) return run_up<2, TY>(p, pv, tiles, st);
  return run_up<4, TY>(p, pv, tiles, st);
}

// Bytes of a that adapter_few's blocks may read in all (5 rows of as many adapters, 13824 x 5120, rank 24: 43 us with 130 MB, 26.3 with the two kernels; 12 rows,
// 17 MB: 21.3 and 18.6; 16 rows, 11 MB: 19.4 and 19.5)
constexpr int64_t kFewBytes = 16 << 20;
template <int QUADS, typename TY>
cudaError_t run_few(const AdapterArgs& p, const PartialView& pv, int tiles, cudaStream_t st) {
  static_assert(kDownWarps * 16 == 128, "out is a multiple of a block's columns");
  return launch_pdl(adapter_few_kernel<QUADS, TY>, dim3(p.out / 128, tiles, p.n_seg), dim3(kDownThreads), 0, st, p, pv);
}

template <typename TY>
cudaError_t run_whole(const AdapterArgs& p, const void* const* w, int tiles, cudaStream_t st) {
  Weights ws = {};
  for (int s = 0; s < p.n_seg; ++s) ws.w[s] = w[s];
  const dim3 grid((p.out + kWholeCols - 1) / kWholeCols, tiles, p.n_seg);
  return p.out % 4 == 0 ? launch_pdl(adapter_whole_kernel<true, TY>, grid, dim3(kThreads), 0, st, p, ws)
                        : launch_pdl(adapter_whole_kernel<false, TY>, grid, dim3(kThreads), 0, st, p, ws);
}

cudaError_t run_down(const AdapterArgs& p, int tiles, int col_blocks, cudaStream_t st) {
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(tiles, p.splits, col_blocks);
  cfg.blockDim = dim3(kDownThreads);
  cfg.stream = st;
  cudaLaunchAttribute at[2];
  at[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  at[0].val.programmaticStreamSerializationAllowed = 1;
  at[1].id = cudaLaunchAttributeClusterDimension;
  at[1].val.clusterDim.x = 1;
  at[1].val.clusterDim.y = p.splits;
  at[1].val.clusterDim.z = 1;
  cfg.attrs = at;
  cfg.numAttrs = 2;
  return cudaLaunchKernelEx(&cfg, adapter_down_kernel, p);
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
  // Small projections: adapter_whole instead of the tensor-core kernel and adapter_up (kWholeBytes).
  const bool whole = dtype == AMPH_DTYPE_BF16 && (!use_tensor_core || (int64_t)tiles * n_seg * out * in * 2 <= kWholeBytes);
  AdapterArgs p;
  p.x = x_dev; p.a = ad->a; p.b = ad->b; p.scale = ad->scale;
  p.row_adapter = row_adapter;
  p.tiles = (RowTile*)ws_dev;
  p.t = (float*)((char*)ws_dev + tiles_bytes(rows));
  p.t_hi = (bf16*)p.t;
  p.t_lo = p.t_hi + (size_t)rows * cols;
  p.y = y_dev;
  p.status = status_dev;
  p.n_adapters = ad->n_adapters; p.rank = ad->rank; p.n_seg = n_seg; p.out = out; p.in = in; p.rows = rows;
  p.splits = dtype == AMPH_DTYPE_F32 ? 1 : down_splits(in, tiles * col_blocks, !whole && rows > kWideFrom ? 168 : 444);
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
  }
  if (use_tensor_core && !whole) {
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
      if (g_plans[dev]) {
        tc_wide_init(g_plans[dev]);
        tc_gemm_wait_first(g_plans[dev]);      // a call's weights may be an earlier call's output
        tc_gemm_late_trigger(g_plans[dev]);
      }
    }
    g = g_plans[dev];
    if (!g) return api_fail(AMPH_ERR_CUDA, "tensor-map encoder unavailable or not an sm_100 device");
    g->cache.clear();                       // tensor maps are made for each call
    tc_gemm_rebind(g, 0, xb[0], x_rows_cap, in, status_dev);
  }
  cudaError_t e = cudaSuccess;
  p.beside = g != nullptr;
  if (g) {
    int splits = 0;
    size_t stride = 0;
    if (!tc_gemm_launch(g, 0, w, n_seg, out, in, rows, P, p_floats, &splits, &stride, st))
      return api_fail(AMPH_ERR_SHAPE, "shape not covered by the tensor-core kernel");
    pv.splits = splits;
    pv.split_stride = stride;
  }
  const bool few = g && rows <= kFewRows && ad->rank <= kFewRank &&
                   (int64_t)((out + 127) / 128) * tiles * n_seg * ad->rank * in * 2 <= kFewBytes;
  if (few)
    e = ad->rank <= 16 ? (y_dtype == AMPH_DTYPE_F32 ? run_few<0, float>(p, pv, tiles, st) : run_few<0, bf16>(p, pv, tiles, st))
                       : (y_dtype == AMPH_DTYPE_F32 ? run_few<1, float>(p, pv, tiles, st) : run_few<1, bf16>(p, pv, tiles, st));
  else if (dtype == AMPH_DTYPE_F32)
    e = launch_pdl(adapter_down_plain_kernel, dim3((cols + 3) / 4, rows), dim3(kThreads), 0, st, p);
  else
    e = run_down(p, tiles, col_blocks, st);
  if (e == cudaSuccess && !few) {
    if (dtype == AMPH_DTYPE_F32)
      e = launch_plain_adapters(x_dev, w, n_seg, out, in, (float*)y_dev, rows, {p.t, (const float*)p.b, p.scale, row_adapter, p.n_adapters, p.rank}, st);
    else if (whole)
      e = y_dtype == AMPH_DTYPE_F32 ? run_whole<float>(p, w, tiles, st) : run_whole<bf16>(p, w, tiles, st);
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
