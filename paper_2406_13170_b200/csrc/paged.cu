// Paged key / value caches: amph_paged_write (rotary embedding, keys and values into their pages) and amph_paged_attention
// (one new token of every sequence against its pages).
#include <math.h>
#include <string.h>

#include <atomic>
#include <new>

#include "amph_internal.cuh"
#include "line.cuh"

namespace amph {
namespace {

typedef __nv_bfloat16 bf16;

// eight values as they lie in memory, and as fp32
template <typename T> struct Raw8 { uint4 u[sizeof(T) / 2]; };
template <typename T>
__device__ __forceinline__ Raw8<T> load8(const T* p) {
  Raw8<T> r;
#pragma unroll
  for (int i = 0; i < (int)sizeof(T) / 2; ++i) r.u[i] = reinterpret_cast<const uint4*>(p)[i];
  return r;
}
__device__ __forceinline__ void values(const Raw8<float>& r, float (&v)[8]) {
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    v[4 * i] = __uint_as_float(r.u[i].x); v[4 * i + 1] = __uint_as_float(r.u[i].y);
    v[4 * i + 2] = __uint_as_float(r.u[i].z); v[4 * i + 3] = __uint_as_float(r.u[i].w);
  }
}
__device__ __forceinline__ void values(const Raw8<bf16>& r, float (&v)[8]) {
  const uint32_t w[4] = {r.u[0].x, r.u[0].y, r.u[0].z, r.u[0].w};
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    v[2 * i] = __uint_as_float(w[i] << 16);
    v[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u);
  }
}
__device__ __forceinline__ void store8(float* p, const float (&v)[8]) {
  *reinterpret_cast<float4*>(p) = make_float4(v[0], v[1], v[2], v[3]);
  *reinterpret_cast<float4*>(p + 4) = make_float4(v[4], v[5], v[6], v[7]);
}
__device__ __forceinline__ void store8(bf16* p, const float (&v)[8]) {
  uint32_t w[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const __nv_bfloat162 h = __floats2bfloat162_rn(v[2 * i], v[2 * i + 1]);
    w[i] = *reinterpret_cast<const uint32_t*>(&h);
  }
  *reinterpret_cast<uint4*>(p) = make_uint4(w[0], w[1], w[2], w[3]);
}

// ---------------------------------------------------------------------------------------------------------------------
// amph_paged_write
// ---------------------------------------------------------------------------------------------------------------------
constexpr int kWriteThreads = 256;       // at most

struct WriteParams {
  const void *q, *k, *v;
  int64_t q_stride, k_stride, v_stride;
  void *q_out, *k_pages, *v_pages;
  const int *row_seq, *row_pos, *table;
  int* status;
  int n_seqs, table_stride, n_heads, n_kv, dh, page_shift, n_pages;
  u64 turn[64];            // theta^(-2 i / dh) / (2 pi) as a fraction of 2^64: the share of a turn per position
};

// cos and sin of the angle whose share of a full turn is phase / 2^64.  The product position * turn wraps at whole turns, so the
// phase of any position is exact to 2^-64 * position; what fp32 rounds is an angle of at most pi / 4.
__device__ __forceinline__ float2 cos_sin_of_phase(u64 phase) {
  const uint32_t top = (uint32_t)(phase >> 32);
  const uint32_t quadrant = (top + 0x20000000u) >> 30;
  const int rest = (int)(top - (quadrant << 30));                    // [-2^29, 2^29): an eighth of a turn either way
  float s, c;
  sincospif((float)rest * 4.656612873077393e-10f, &s, &c);           // 2^-31: in units of half a turn
  if (quadrant & 1) { const float x = s; s = c; c = -x; }
  if (quadrant & 2) { s = -s; c = -c; }
  return make_float2(c, s);
}

// Grid (row, part of the row's heads); an item is eight rotation pairs of one head (eight values twice for v), a thread has ITEMS, whose
// loads are under way while the row's place in the cache is looked up.  A thread writes what it has read and nobody else reads, so q_out may be q.  Bound: HBM for many rows, latency for few (see run_write).
template <typename TS, typename TD, int ITEMS>
__global__ void __launch_bounds__(kWriteThreads) paged_write_kernel(const __grid_constant__ WriteParams p) {
  pdl_wait();
  pdl_launch_dependents();
  __shared__ float2 cs[64];
  const int row = blockIdx.x, half = p.dh >> 1;
  const int seq = p.row_seq[row], pos = p.row_pos[row];
  const int per_head = half >> 3, shift = p.dh == 128 ? 3 : 2;
  const int items = (p.n_heads + 2 * p.n_kv) * per_head, item0 = blockIdx.y * ITEMS * blockDim.x + threadIdx.x;
  Raw8<TS> lo[ITEMS], hi[ITEMS];
#pragma unroll
  for (int n = 0; n < ITEMS; ++n) {
    const int it = item0 + n * blockDim.x;
    if (it >= items) break;
    const int head = it >> shift, i = (it & (per_head - 1)) * 8, hk = head - p.n_heads;
    const TS* src = head < p.n_heads ? (const TS*)p.q + row * p.q_stride + head * p.dh
                    : hk < p.n_kv    ? (const TS*)p.k + row * p.k_stride + hk * p.dh
                                     : (const TS*)p.v + row * p.v_stride + (hk - p.n_kv) * p.dh;
    lo[n] = load8(src + i);
    hi[n] = load8(src + half + i);
  }
  if (seq < 0) return;
  bool ok = seq < p.n_seqs && pos >= 0 && (pos >> p.page_shift) < p.table_stride;
  int page = 0;
  if (ok) {
    page = p.table[(int64_t)seq * p.table_stride + (pos >> p.page_shift)];
    ok = page >= 0 && page < p.n_pages;
  }
  if (!ok) {
    if (p.status != nullptr && threadIdx.x == 0) *p.status = AMPH_ERR_INVALID_ARG;
    return;
  }
  for (int i = threadIdx.x; i < half; i += blockDim.x) cs[i] = cos_sin_of_phase((u64)pos * p.turn[i]);
  __syncthreads();
  const int64_t slot = pos & ((1 << p.page_shift) - 1);
#pragma unroll
  for (int n = 0; n < ITEMS; ++n) {
    const int it = item0 + n * blockDim.x;
    if (it >= items) break;
    const int head = it >> shift, i = (it & (per_head - 1)) * 8, h = head - p.n_heads, is_v = h >= p.n_kv, hk = is_v ? h - p.n_kv : h;
    TD* dst = head < p.n_heads ? (TD*)p.q_out + ((int64_t)row * p.n_heads + head) * p.dh
                               : (TD*)(is_v ? p.v_pages : p.k_pages) + ((((int64_t)page * p.n_kv + hk) << p.page_shift) + slot) * p.dh;
    float a[8], b[8];
    values(lo[n], a);
    values(hi[n], b);
    if (h < p.n_kv) {
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        const float2 t = cs[i + j];
        const float x = a[j] * t.x - b[j] * t.y;
        b[j] = b[j] * t.x + a[j] * t.y;
        a[j] = x;
      }
    }
    store8(dst + i, a);
    store8(dst + half + i, b);
  }
}

// ---------------------------------------------------------------------------------------------------------------------
// amph_paged_attention
//
// The work is a line of units of kUnit keys: sequence by sequence, in a sequence item by item (a key / value head and up to kHeads of
// the query heads that share it), in an item unit by unit, with one unit more ahead of each item for what an item costs whatever its length
// (the pipeline fills, the warps' sums are joined).  The grid is as many blocks as the device runs at a time, and
// block c of n (the grid, or fewer where there is little) takes units [total * c / n, total * (c + 1) / n): every length mix is spread evenly, and the host needs no length.  An item
// inside one block is finished there.  Of an item cut over blocks each leaves its part (running maximum, sum, weighted values)
// in scratch.  Of every kGroup neighbouring parts the block that arrives last adds them in the order of the blocks, and of the groups the
// one that is done last adds those: no block waits, and the bits do not depend on who is last.  Statistics and sums are fp32.
// ---------------------------------------------------------------------------------------------------------------------
constexpr int kUnit = 64;                // keys: 16 for each warp
constexpr int kAttWarps = 4;
constexpr int kAttThreads = kAttWarps * 32;
// blocks per SM: 168 or 128 registers a thread; those of 64 columns have half the bytes in flight (16 sequences up to 4000, 32 heads: 54.5 us, 60.3
// with three)
template <int DH> constexpr int kAttResident = DH == 64 ? 4 : 3;
constexpr int kHeads = 8;                // query heads of an item
constexpr int kMaxBlocks = 592;
constexpr int kGroup = 8;                // parts that one block adds at a time: as many as it has loads in flight
constexpr float kLog2e = 1.4426950408889634f;

struct AttendParams {
  const void *q, *k, *v;
  const int *lens, *table;
  void* out;
  float* lse;
  int* counters;           // [2][kMaxBlocks]: parts that arrived of the group that begins in block c | groups of the item that begins there
  float* parts;            // [kMaxBlocks][2][part_floats]: block c's part of an item that began before it | begins in it
  int* status;
  int part_floats;
  int n_seqs, table_stride, n_heads, n_kv, group, head_blocks, page_shift, n_pages;
  int cap;                 // positions a table row has room for
  float scale_log2;
};

template <int DH>
struct __align__(16) MergeSmem {
  float o[kAttWarps][kHeads][DH];
  float m[kAttWarps][kHeads], l[kAttWarps][kHeads];
};

__device__ __forceinline__ int clamped_len(const AttendParams& p, int s) {
  const int n = p.lens[s];
  return n < 0 ? 0 : (n > p.cap ? p.cap : n);
}

// exp2(x - m) of a running maximum m that may still be -inf (nothing seen)
__device__ __forceinline__ float weight(float x, float m) { return exp2f(x - (m == -INFINITY ? 0.f : m)); }

// First key of the 16 at `key` (page_size >= 16: they share a page); a page that does not exist is reported and counts as absent.
__device__ __forceinline__ int page_of(const AttendParams& p, int seq, int key) {
  const int page = p.table[(int64_t)seq * p.table_stride + (key >> p.page_shift)];
  if (page >= 0 && page < p.n_pages) return page;
  if (p.status != nullptr) *p.status = AMPH_ERR_INVALID_ARG;
  return -1;
}

__device__ __forceinline__ void load_n(const float* p, float (&v)[4]) {
  const float4 a = *reinterpret_cast<const float4*>(p);
  v[0] = a.x; v[1] = a.y; v[2] = a.z; v[3] = a.w;
}
__device__ __forceinline__ void load_n(const float* p, float (&v)[2]) {
  const float2 a = *reinterpret_cast<const float2*>(p);
  v[0] = a.x; v[1] = a.y;
}
// 16 bytes to shared memory, zeros where `there` is false
__device__ __forceinline__ void copy_async(float* dst, const float* src, bool there) {
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"((uint32_t)__cvta_generic_to_shared(dst)), "l"(src), "r"(there ? 16 : 0) : "memory");
}
__device__ __forceinline__ void commit_copies() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int N> __device__ __forceinline__ void wait_copies() { asm volatile("cp.async.wait_group %0;" ::"n"(N) : "memory"); }

// The 16 keys at key0 as lanes see them: lane j (and j + 16) knows the page of key j, -1 where there is none.
__device__ __forceinline__ int find_page(const AttendParams& p, int seq, int key0, int k1) {
  const int key = key0 + (threadIdx.x & 15);
  return key < k1 ? page_of(p, seq, key) : -1;
}
// Element offset of key j's row, from what find_page gave the lanes (all of them call)
template <int DH>
__device__ __forceinline__ int64_t row_of(const AttendParams& p, int kv, int key0, int page, int j) {
  const int from = __shfl_sync(~0u, page, p.page_shift >= 4 ? 0 : j);           // pages of 16 slots or more: 16 keys share one
  return ((((int64_t)from * p.n_kv + kv) << p.page_shift) + ((key0 + j) & ((1 << p.page_shift) - 1))) * DH;
}

// Keys [k0, k1) of one fp32 item by CUDA cores, 16 keys of a warp at a time through shared memory of its own: the next keys are copied while
// these values are worked on, and the other way round.
//   Scores   eight lanes share a key, four keys at a time of 16 held in registers, so that a query is read once for all of them
//   Values   every lane has its own columns
// Bound: HBM with few heads to a key, the issue of FMAs with eight (1300 instructions per 16 keys of 16 KB).  Eight ragged sequences of 40 heads
// up to 2048 tokens: 78 us, 4.5 TB/s (185 us with every key loaded when it was needed).
template <int DH>
struct PlainItem {
  struct Smem {
    union {
      MergeSmem<DH> mg;
      float kv[kAttWarps][2][16][DH];
    };
    float q[kHeads][DH];
    float s[kAttWarps][kHeads][16];
    float alpha[kAttWarps][kHeads];
  };
  static __device__ __forceinline__ void run(const AttendParams& p, Smem& sm, int seq, int kv, int head0, int heads, int k0, int k1) {
    constexpr int C = DH / 32, PER = 128 / DH;        // 128-byte parts of a key; keys that a warp copies at a time
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    const float* kp = (const float*)p.k;
    const float* vp = (const float*)p.v;
    auto copy = [&](int which, int key0, int page, unsigned there) {
      const float* src = which ? vp : kp;
      const int mine = lane / (DH / 4), col = lane % (DH / 4) * 4;
#pragma unroll
      for (int j0 = 0; j0 < 16; j0 += PER) {
        const int j = j0 + mine;
        const int64_t at = row_of<DH>(p, kv, key0, page, j);
        const bool is = (there >> j) & 1;
        copy_async(&sm.kv[warp][which][j][col], is ? src + at + col : src, is);
      }
      commit_copies();
    };
    int key0 = k0 + warp * 16;
    int page = find_page(p, seq, key0, k1);
    unsigned there = __ballot_sync(~0u, page >= 0);
    copy(0, key0, page, there);
    copy(1, key0, page, there);
    page = find_page(p, seq, key0 + kUnit, k1);
    for (int i = tid; i < heads * DH; i += kAttThreads)
      sm.q[i / DH][i % DH] = ((const float*)p.q)[((int64_t)seq * p.n_heads + head0) * DH + i];
    __syncthreads();
    float o[kHeads][C];
#pragma unroll
    for (int h = 0; h < kHeads; ++h)
#pragma unroll
      for (int c = 0; c < C; ++c) o[h][c] = 0.f;
    float m_run = -INFINITY, l_run = 0.f;
    const int my_head = lane >> 2, part = lane & 7;
    for (; key0 < k1; key0 += kUnit) {
      wait_copies<1>();
      __syncwarp();
      const unsigned now = there;
      there = __ballot_sync(~0u, page >= 0);
      float kf[4][C][4];                               // keys 4 i + lane / 8
#pragma unroll
      for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int c = 0; c < C; ++c) load_n(&sm.kv[warp][0][4 * i + (lane >> 3)][c * 32 + part * 4], kf[i][c]);
      __syncwarp();
      copy(0, key0 + kUnit, page, there);
      for (int h = 0; h < heads; ++h) {
        float acc[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int c = 0; c < C; ++c) {
          const float4 qv = *reinterpret_cast<const float4*>(&sm.q[h][c * 32 + part * 4]);
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            acc[i] += kf[i][c][0] * qv.x; acc[i] += kf[i][c][1] * qv.y; acc[i] += kf[i][c][2] * qv.z; acc[i] += kf[i][c][3] * qv.w;
          }
        }
        // sums over the eight lanes; bits 0 and 1 of the lane end up choosing which of the four keys it has
#pragma unroll
        for (int i = 0; i < 2; ++i) {
          const float give = part & 1 ? acc[2 * i] : acc[2 * i + 1], keep = part & 1 ? acc[2 * i + 1] : acc[2 * i];
          acc[i] = keep + __shfl_xor_sync(~0u, give, 1);
        }
        const float give = part & 2 ? acc[0] : acc[1], keep = part & 2 ? acc[1] : acc[0];
        float x = keep + __shfl_xor_sync(~0u, give, 2);
        x += __shfl_xor_sync(~0u, x, 4);
        const int j = 4 * ((part & 2) + (part & 1)) + (lane >> 3);
        if (part < 4) sm.s[warp][h][j] = (now >> j) & 1 ? x * p.scale_log2 : -INFINITY;
      }
      __syncwarp();
      if (my_head < heads) {
        float4 s = *reinterpret_cast<float4*>(&sm.s[warp][my_head][(lane & 3) * 4]);
        float mx = fmaxf(fmaxf(s.x, s.y), fmaxf(s.z, s.w));
        const unsigned quad = 0xfu << (lane & ~3);
        mx = fmaxf(mx, __shfl_xor_sync(quad, mx, 1));
        mx = fmaxf(mx, __shfl_xor_sync(quad, mx, 2));
        mx = fmaxf(mx, m_run);
        const float alpha = weight(m_run, mx);
        s.x = weight(s.x, mx); s.y = weight(s.y, mx); s.z = weight(s.z, mx); s.w = weight(s.w, mx);
        l_run = l_run * alpha + (s.x + s.y + s.z + s.w);
        m_run = mx;
        *reinterpret_cast<float4*>(&sm.s[warp][my_head][(lane & 3) * 4]) = s;
        if ((lane & 3) == 0) sm.alpha[warp][my_head] = alpha;
      }
      wait_copies<1>();
      __syncwarp();
#pragma unroll
      for (int h = 0; h < kHeads; ++h)
        if (h < heads) {
          const float alpha = sm.alpha[warp][h];
#pragma unroll
          for (int c = 0; c < C; ++c) o[h][c] *= alpha;
        }
#pragma unroll
      for (int j0 = 0; j0 < 16; j0 += 4) {
        float vf[4][C];
#pragma unroll
        for (int j = 0; j < 4; ++j) load_n(&sm.kv[warp][1][j0 + j][lane * C], vf[j]);
#pragma unroll
        for (int h = 0; h < kHeads; ++h)
          if (h < heads) {
            const float4 w = *reinterpret_cast<const float4*>(&sm.s[warp][h][j0]);
#pragma unroll
            for (int c = 0; c < C; ++c) {
              o[h][c] += w.x * vf[0][c]; o[h][c] += w.y * vf[1][c]; o[h][c] += w.z * vf[2][c]; o[h][c] += w.w * vf[3][c];
            }
          }
      }
      __syncwarp();
      copy(1, key0 + kUnit, page, there);
      page = find_page(p, seq, key0 + 2 * kUnit, k1);
    }
    wait_copies<0>();
    __syncthreads();                                   // the copies' place becomes the warps' results'
#pragma unroll
    for (int h = 0; h < kHeads; ++h)
      if (h < heads)
#pragma unroll
        for (int c = 0; c < C; ++c) sm.mg.o[warp][h][lane * C + c] = o[h][c];
    l_run += __shfl_xor_sync(~0u, l_run, 1);
    l_run += __shfl_xor_sync(~0u, l_run, 2);
    if ((lane & 3) == 0) {
      sm.mg.m[warp][my_head] = m_run;
      sm.mg.l[warp][my_head] = l_run;
    }
    __syncthreads();
  }
};

// 32 or 16 bytes that no other thread of the block reads
__device__ __forceinline__ void load_once(const bf16* p, uint32_t (&v)[8]) {
  asm volatile("ld.global.nc.L1::no_allocate.v8.b32 {%0, %1, %2, %3, %4, %5, %6, %7}, [%8];"
               : "=r"(v[0]), "=r"(v[1]), "=r"(v[2]), "=r"(v[3]), "=r"(v[4]), "=r"(v[5]), "=r"(v[6]), "=r"(v[7]) : "l"(p));
}
__device__ __forceinline__ void load_once(const bf16* p, uint32_t (&v)[4]) {
  asm volatile("ld.global.nc.L1::no_allocate.v4.b32 {%0, %1, %2, %3}, [%4];" : "=r"(v[0]), "=r"(v[1]), "=r"(v[2]), "=r"(v[3]) : "l"(p));
}
__device__ __forceinline__ void mma_16816(float (&d)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
  asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
               : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3]) : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}
__device__ __forceinline__ uint32_t pack(float lo, float hi) {
  const __nv_bfloat162 h = __floats2bfloat162_rn(lo, hi);
  return *reinterpret_cast<const uint32_t*>(&h);
}

// Keys [k0, k1) of one bf16 item on the warp-level tensor cores, 16 keys of a warp at a time, straight from the pages to registers:
// no shared memory, no barrier, the next 16 keys' loads in flight while these are worked on.
//   Scores   S[head][key]: A = queries (rows 0-7; rows 8-15 zero), B = keys.  The sum over head_dim may run in any order that both
//            operands share, so a lane takes 32 contiguous bytes of its key for four steps.
//   Values   O[head][column]: A = weights, B = values.  Rows 8-15 carry what the weights of rows 0-7 lose when they are rounded to
//            bf16, so 16 bits of every weight enter at no further cost; columns may be numbered in any order, so a lane takes
//            head_dim / 8 contiguous ones of four keys and pairs them with byte permutes.
// Bound: HBM.  A key's 4 head_dim bytes cost at most 16 head_dim * 4 flops, a tenth of what the tensor pipe does meanwhile.
template <int DH>
struct MmaItem {
  struct Smem {
    MergeSmem<DH> mg;
  };
  static __device__ __forceinline__ void run(const AttendParams& p, Smem& sm, int seq, int kv, int head0, int heads, int k0, int k1) {
    constexpr int C = DH / 64, W = DH / 16;          // 128-byte parts of a key; 32-bit words of a value row that a lane takes
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, g = lane >> 2, t = lane & 3;
    const bf16* kp = (const bf16*)p.k;
    const bf16* vp = (const bf16*)p.v;
    uint32_t q[C][8];
#pragma unroll
    for (int c = 0; c < C; ++c)
#pragma unroll
      for (int i = 0; i < 8; i += 4) {
        uint4 v = make_uint4(0u, 0u, 0u, 0u);
        if (g < heads)
          v = *reinterpret_cast<const uint4*>((const bf16*)p.q + ((int64_t)seq * p.n_heads + head0 + g) * DH + c * 64 + t * 16 + i * 2);
        q[c][i] = v.x; q[c][i + 1] = v.y; q[c][i + 2] = v.z; q[c][i + 3] = v.w;
      }
    float o[2 * W][4];
#pragma unroll
    for (int j = 0; j < 2 * W; ++j) o[j][0] = o[j][1] = o[j][2] = o[j][3] = 0.f;
    float m_run = -INFINITY, l_run = 0.f;

    uint32_t kr[2][C][8], vr[4][W];
    auto load_k = [&](int key0, int page, unsigned there) {
#pragma unroll
      for (int n = 0; n < 2; ++n) {
        const int j = n * 8 + g;
        const bf16* src = kp + row_of<DH>(p, kv, key0, page, j) + t * 16;
#pragma unroll
        for (int c = 0; c < C; ++c) {
          if ((there >> j) & 1) {
            load_once(src + c * 64, kr[n][c]);
          } else {
#pragma unroll
            for (int i = 0; i < 8; ++i) kr[n][c][i] = 0u;
          }
        }
      }
    };
    auto load_v = [&](int key0, int page, unsigned there) {
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const int j = 2 * t + (i & 1) + (i >> 1) * 8;
        const bf16* src = vp + row_of<DH>(p, kv, key0, page, j) + g * 2 * W;
        if ((there >> j) & 1) {
          load_once(src, vr[i]);
        } else {
#pragma unroll
          for (int w = 0; w < W; ++w) vr[i][w] = 0u;
        }
      }
    };
    int key0 = k0 + warp * 16;
    int page = find_page(p, seq, key0, k1);
    unsigned there = __ballot_sync(~0u, page >= 0);
    load_k(key0, page, there);
    load_v(key0, page, there);
    int page_next = find_page(p, seq, key0 + kUnit, k1);
    for (; key0 < k1; key0 += kUnit) {
      float s[2][4];
#pragma unroll
      for (int n = 0; n < 2; ++n) {
        s[n][0] = s[n][1] = s[n][2] = s[n][3] = 0.f;
#pragma unroll
        for (int c = 0; c < C; ++c)
#pragma unroll
          for (int i = 0; i < 8; i += 2) mma_16816(s[n], q[c][i], 0u, q[c][i + 1], 0u, kr[n][c][i], kr[n][c][i + 1]);
      }
      const unsigned now = there;
      there = __ballot_sync(~0u, page_next >= 0);
      load_k(key0 + kUnit, page_next, there);
      float w[2][2];
      float mx = m_run;
#pragma unroll
      for (int n = 0; n < 2; ++n)
#pragma unroll
        for (int i = 0; i < 2; ++i) {
          w[n][i] = (now >> (n * 8 + 2 * t + i)) & 1 ? s[n][i] * p.scale_log2 : -INFINITY;
          mx = fmaxf(mx, w[n][i]);
        }
      mx = fmaxf(mx, __shfl_xor_sync(~0u, mx, 1));
      mx = fmaxf(mx, __shfl_xor_sync(~0u, mx, 2));
      if (__any_sync(~0u, mx != m_run)) {
        const float alpha = weight(m_run, mx);
        l_run *= alpha;
#pragma unroll
        for (int j = 0; j < 2 * W; ++j)
#pragma unroll
          for (int i = 0; i < 4; ++i) o[j][i] *= alpha;
        m_run = mx;
      }
      uint32_t hi[2], lo[2];
#pragma unroll
      for (int n = 0; n < 2; ++n) {
        w[n][0] = weight(w[n][0], mx);
        w[n][1] = weight(w[n][1], mx);
        l_run += w[n][0] + w[n][1];
        hi[n] = pack(w[n][0], w[n][1]);
        lo[n] = pack(w[n][0] - __uint_as_float(hi[n] << 16), w[n][1] - __uint_as_float(hi[n] & 0xffff0000u));
      }
#pragma unroll
      for (int j = 0; j < 2 * W; ++j) {
        const uint32_t pick = j & 1 ? 0x7632u : 0x5410u;
        mma_16816(o[j], hi[0], lo[0], hi[1], lo[1], __byte_perm(vr[0][j >> 1], vr[1][j >> 1], pick), __byte_perm(vr[2][j >> 1], vr[3][j >> 1], pick));
      }
      load_v(key0 + kUnit, page_next, there);
      page_next = find_page(p, seq, key0 + 2 * kUnit, k1);
    }
    l_run += __shfl_xor_sync(~0u, l_run, 1);
    l_run += __shfl_xor_sync(~0u, l_run, 2);
    if (g < heads) {
#pragma unroll
      for (int j = 0; j < 2 * W; j += 4)
#pragma unroll
        for (int i = 0; i < 2; ++i)                   // columns 2 W n + j of n = 2 t + i
          *reinterpret_cast<float4*>(&sm.mg.o[warp][g][2 * W * (2 * t + i) + j]) =
              make_float4(o[j][i] + o[j][i + 2], o[j + 1][i] + o[j + 1][i + 2], o[j + 2][i] + o[j + 2][i + 2], o[j + 3][i] + o[j + 3][i + 2]);
      if (t == 0) {
        sm.mg.m[warp][g] = m_run;
        sm.mg.l[warp][g] = l_run;
      }
    }
    __syncthreads();
  }
};

__device__ __forceinline__ void store4(float* p, float4 v) { *reinterpret_cast<float4*>(p) = v; }
__device__ __forceinline__ void store4(bf16* p, float4 v) { *reinterpret_cast<uint2*>(p) = make_uint2(pack(v.x, v.y), pack(v.z, v.w)); }

// Sums of one (or more) sets of weights that share the maximum m: sum of w V in o, sum of w in l.
struct Sums {
  float4 o;
  float m, l;
};
__device__ __forceinline__ void add_scaled(Sums& a, float f, float4 o, float l) {
  a.o.x += f * o.x; a.o.y += f * o.y; a.o.z += f * o.z; a.o.w += f * o.w;
  a.l += f * l;
}
template <typename T, int DH>
__device__ __forceinline__ void write_row(const AttendParams& p, int seq, int head, int col, const Sums& a) {
  const int64_t at = (int64_t)seq * p.n_heads + head;
  const float4 o = a.l == 0.f ? make_float4(0.f, 0.f, 0.f, 0.f) : make_float4(a.o.x / a.l, a.o.y / a.l, a.o.z / a.l, a.o.w / a.l);   // l = 0: no key at all
  store4((T*)p.out + at * DH + col, o);
  if (p.lse != nullptr && col == 0) p.lse[at] = a.l == 0.f ? -INFINITY : (a.m == -INFINITY ? 0.f : a.m) / kLog2e + logf(a.l);
}

// Columns 4 i .. 4 i + 3 of an item (i counts over its heads) from `count` parts, `stride` floats apart, of which this thread adds first,
// first + step, ... in their order.  The item's first part lies `ahead` floats further on than the others.  Eight parts' loads are in flight at a time.
__device__ __noinline__ Sums add_parts(const float* all, size_t stride, int ahead, int dh, int i, int first, int step, int count) {
  Sums a = {make_float4(0.f, 0.f, 0.f, 0.f), -INFINITY, 0.f};
  const int ml_at = kHeads * dh + 2 * (4 * i / dh);
  for (int c = first; c < count; c += kGroup * step) {
    float4 o[kGroup];
    float2 ml[kGroup];
#pragma unroll
    for (int q = 0; q < kGroup; ++q) {
      const int k = min(c + q * step, count - 1);
      const float* x = all + k * stride + (k == 0 ? ahead : 0);
      ml[q] = __ldcg(reinterpret_cast<const float2*>(x + ml_at));
      o[q] = __ldcg(reinterpret_cast<const float4*>(x) + i);
    }
    float m = a.m;
#pragma unroll
    for (int q = 0; q < kGroup; ++q)
      if (c + q * step < count) m = fmaxf(m, ml[q].x);
    const Sums old = a;
    a = {make_float4(0.f, 0.f, 0.f, 0.f), m, 0.f};
    if (c != first) add_scaled(a, weight(old.m, m), old.o, old.l);
#pragma unroll
    for (int q = 0; q < kGroup; ++q)
      if (c + q * step < count) add_scaled(a, weight(ml[q].x, m), o[q], ml[q].y);
  }
  return a;
}

// Columns 4 i .. 4 i + 3 of an item from a block's warps
template <int DH>
__device__ __forceinline__ Sums join_warps(const MergeSmem<DH>& mg, int i) {
  const int h = 4 * i / DH, c = 4 * i % DH;
  Sums a = {make_float4(0.f, 0.f, 0.f, 0.f), mg.m[0][h], 0.f};
#pragma unroll
  for (int w = 1; w < kAttWarps; ++w) a.m = fmaxf(a.m, mg.m[w][h]);
#pragma unroll
  for (int w = 0; w < kAttWarps; ++w)
    add_scaled(a, weight(mg.m[w][h], a.m), *reinterpret_cast<const float4*>(&mg.o[w][h][c]), mg.l[w][h]);
  return a;
}

// A few short sequences, where latency counts: grid (part, item, sequence), a cluster holds an item's parts and joins them through its
// shared memory, every block an equal share of the columns.  No scratch, no line to find one's place on.  (One sequence of 640 tokens, 32 heads:
// 6.1 us, 9.0 with the line; see kShortKeys.)
constexpr int kMaxParts = 16;
template <typename T, int DH, typename Item>
__global__ void __launch_bounds__(kAttThreads, kAttResident<DH>) paged_attention_cluster_kernel(const __grid_constant__ AttendParams p) {
  pdl_wait();
  pdl_launch_dependents();
  extern __shared__ __align__(16) unsigned char smem_raw[];
  typename Item::Smem& sm = *reinterpret_cast<typename Item::Smem*>(smem_raw);
  constexpr int kMost = kHeads * DH / 4;
  __shared__ __align__(16) float4 o_in[kMost + kMaxParts];             // [part][share]
  __shared__ float2 ml_in[kMost + kMaxParts];
  const int tid = threadIdx.x, parts = gridDim.x, part = blockIdx.x, seq = blockIdx.z;
  const int kv = blockIdx.y / p.head_blocks, block0 = (blockIdx.y - kv * p.head_blocks) * kHeads;
  const int head0 = kv * p.group + block0, heads = min(kHeads, p.group - block0), slots = heads * DH / 4;
  const int raw = p.lens[seq], len = raw < 0 ? 0 : min(raw, p.cap);
  if (raw != len && p.status != nullptr && tid == 0) *p.status = AMPH_ERR_INVALID_ARG;
  if (len == 0) {                                                      // the same in the whole cluster
    if (part == 0)
      for (int i = tid; i < slots; i += kAttThreads) write_row<T, DH>(p, seq, head0 + 4 * i / DH, 4 * i % DH, Sums{});
    return;
  }
  asm volatile("barrier.cluster.arrive.relaxed.aligned;" ::: "memory");
  const int units = (len + kUnit - 1) / kUnit, k0 = units * part / parts * kUnit, k1 = min(len, units * (part + 1) / parts * kUnit);
  if (k0 < k1) Item::run(p, sm, seq, kv, head0, heads, k0, k1);
  asm volatile("barrier.cluster.wait.aligned;" ::: "memory");          // every block has begun
  const int share = (slots + parts - 1) / parts;
  for (int i = tid; i < slots; i += kAttThreads) {
    Sums a = {make_float4(0.f, 0.f, 0.f, 0.f), -INFINITY, 0.f};
    if (k0 < k1) a = join_warps<DH>(sm.mg, i);
    const int to = i / share, at = part * share + i - to * share;
    uint32_t o_at, ml_at;
    asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(o_at) : "r"((uint32_t)__cvta_generic_to_shared(&o_in[at])), "r"(to));
    asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(ml_at) : "r"((uint32_t)__cvta_generic_to_shared(&ml_in[at])), "r"(to));
    asm volatile("st.shared::cluster.v4.f32 [%0], {%1, %2, %3, %4};" ::"r"(o_at), "f"(a.o.x), "f"(a.o.y), "f"(a.o.z), "f"(a.o.w) : "memory");
    asm volatile("st.shared::cluster.v2.f32 [%0], {%1, %2};" ::"r"(ml_at), "f"(a.m), "f"(a.l) : "memory");
  }
  __syncwarp();
  asm volatile("barrier.cluster.arrive.release.aligned;\nbarrier.cluster.wait.acquire.aligned;" ::: "memory");
  for (int j = tid; j < share; j += kAttThreads) {
    const int i = part * share + j;
    if (i >= slots) break;
    float m = -INFINITY;
    for (int k = 0; k < parts; ++k) m = fmaxf(m, ml_in[k * share + j].x);
    Sums a = {make_float4(0.f, 0.f, 0.f, 0.f), m, 0.f};
    for (int k = 0; k < parts; ++k) add_scaled(a, weight(ml_in[k * share + j].x, m), o_in[k * share + j], ml_in[k * share + j].y);
    write_row<T, DH>(p, seq, head0 + 4 * i / DH, 4 * i % DH, a);
  }
}

// A sequence's units per item.
__device__ __forceinline__ int span_of(int len) { return len == 0 ? 0 : (len + kUnit - 1) / kUnit + 1; }

template <typename T, int DH, typename Item>
__global__ void __launch_bounds__(kAttThreads, kAttResident<DH>) paged_attention_kernel(const __grid_constant__ AttendParams p) {
  pdl_wait();
  pdl_launch_dependents();
  extern __shared__ __align__(16) unsigned char smem_raw[];
  typename Item::Smem& sm = *reinterpret_cast<typename Item::Smem*>(smem_raw);
  MergeSmem<DH>& mg = sm.mg;
  __shared__ long long s_sum[kAttWarps], s_before;
  __shared__ int s_seq, s_last;
  __shared__ float2 s_ml[kAttThreads];
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  const int items = p.n_kv * p.head_blocks;

  // Units ahead of every sequence: a thread adds up a run of sequences, a scan over the threads does the rest.
  const int per = (p.n_seqs + kAttThreads - 1) / kAttThreads;
  const int s0 = min(tid * per, p.n_seqs), s1 = min(s0 + per, p.n_seqs);
  long long mine = 0;
  for (int s = s0; s < s1; ++s) {
    const int raw = p.lens[s];
    if ((raw < 0 || raw > p.cap) && p.status != nullptr) *p.status = AMPH_ERR_INVALID_ARG;
    mine += span_of(clamped_len(p, s));
  }
  mine *= items;
  long long upto = mine;
#pragma unroll
  for (int d = 1; d < 32; d <<= 1) {
    const long long x = __shfl_up_sync(~0u, upto, d);
    if (lane >= d) upto += x;
  }
  if (lane == 31) s_sum[warp] = upto;
  __syncthreads();
  long long total = 0, ahead = 0;
#pragma unroll
  for (int w = 0; w < kAttWarps; ++w) {
    if (w < warp) ahead += s_sum[w];
    total += s_sum[w];
  }
  const long long before = ahead + upto - mine;

  // sequences without keys
  for (int s = blockIdx.x; s < p.n_seqs; s += gridDim.x)
    if (clamped_len(p, s) == 0)
      for (int i = tid; i < p.n_heads * DH / 4; i += kAttThreads) write_row<T, DH>(p, s, 4 * i / DH, 4 * i % DH, Sums{});

  const int n = (int)(total < 2 * gridDim.x ? (total + 1) / 2 : gridDim.x);       // two units a block at least: fewer parts
  if ((int)blockIdx.x >= n) return;
  const long long u0 = mul_div(total, blockIdx.x, n), u1 = mul_div(total, blockIdx.x + 1, n);
  if (u0 >= before && u0 < before + mine) {
    long long at = before;
    int s = s0;
    for (;; ++s) {
      const long long here = (long long)span_of(clamped_len(p, s)) * items;
      if (u0 < at + here) break;
      at += here;
    }
    s_seq = s;
    s_before = at;
  }
  __syncthreads();
  int seq = s_seq;
  long long u = u0;
  int len = clamped_len(p, seq), span = span_of(len);
  int item = (int)mul_div(u0 - s_before, 1, span), at = (int)(u0 - s_before - (long long)item * span);
  while (u < u1) {
    const int take = (int)(u1 - u < span - at ? u1 - u : span - at), tiles = span - 1;
    const int t0 = max(at - 1, 0), t1 = at + take - 1;                  // keys [t0, t1) * kUnit
    const long long first = u - at + 1;                                  // tile 0's place on the line
    u += take;
    at += take;
    const int kv = item / p.head_blocks, block0 = (item - kv * p.head_blocks) * kHeads;
    const int head0 = kv * p.group + block0, heads = min(kHeads, p.group - block0);
    const int k0 = t0 * kUnit, k1 = min(len, t1 * kUnit), now = seq;
    if (at == span) {
      at = 0;
      if (++item == items) {
        item = 0;
        if (u < u1) {
          do ++seq; while ((len = clamped_len(p, seq)) == 0);
          span = span_of(len);
        }
      }
    }
    if (t0 >= t1) continue;
    Item::run(p, sm, now, kv, head0, heads, k0, k1);
    const bool whole = t1 - t0 == tiles;
    float* part = p.parts + ((size_t)blockIdx.x * 2 + (t0 == 0 ? 1 : 0)) * p.part_floats;
    const int slots = heads * DH / 4;
    for (int i = tid; i < slots; i += kAttThreads) {
      const int h = 4 * i / DH, c = 4 * i % DH;
      const Sums a = join_warps<DH>(mg, i);
      if (whole) {
        write_row<T, DH>(p, now, head0 + h, c, a);
      } else {
        reinterpret_cast<float4*>(part)[i] = a.o;
        if (c == 0) *reinterpret_cast<float2*>(part + kHeads * DH + 2 * h) = make_float2(a.m, a.l);
      }
    }
    if (!whole) {
      // The blocks of a group are neighbours; the last group has what is left, at least two blocks, so that no group begins where the next
      // item may.
      const int c0 = block_of(first, total, n), c1 = block_of(first + tiles - 1, total, n), count = c1 - c0 + 1;
      const int groups = max(1, (count - 1) / kGroup), group = min(((int)blockIdx.x - c0) / kGroup, groups - 1);
      const int g0 = c0 + group * kGroup, in_group = group == groups - 1 ? c1 - g0 + 1 : kGroup;
      // adds up `parts` parts of p.counters[which]'s item or group if this block is the last one to get there
      auto join = [&](int* counter, int parts, int from, int blocks_apart, bool done) {
        __threadfence();
        __syncthreads();
        if (tid == 0) {
          s_last = atomicAdd(counter, 1) == parts - 1;
          if (s_last) *counter = 0;
        }
        __syncthreads();
        if (!s_last) return false;
        __threadfence();
        float* all = p.parts + (size_t)from * 2 * p.part_floats;
        const size_t stride = (size_t)blocks_apart * 2 * p.part_floats;
        const int ahead = from == c0 ? p.part_floats : 0;
        const int sharers = slots * 2 <= kAttThreads ? kAttThreads / slots : 1;      // few columns: several threads share the parts
        for (int i0 = 0; i0 < slots; i0 += kAttThreads) {
          const int sharer = sharers > 1 ? tid / slots : 0, i = sharers > 1 ? tid - sharer * slots : i0 + tid;
          const bool mine_too = sharer < sharers && i < slots;
          Sums a = {make_float4(0.f, 0.f, 0.f, 0.f), -INFINITY, 0.f};
          if (mine_too) a = add_parts(all, stride, ahead, DH, i, sharer, sharers, parts);
          if (sharers > 1) {
            reinterpret_cast<float4*>(mg.o)[tid] = a.o;
            s_ml[tid] = make_float2(a.m, a.l);
          }
          __syncthreads();                           // the parts have been read
          if (mine_too && sharer == 0) {
            if (sharers > 1) {
              float m = a.m;
              for (int k = 1; k < sharers; ++k) m = fmaxf(m, s_ml[k * slots + i].x);
              a = {make_float4(0.f, 0.f, 0.f, 0.f), m, 0.f};
              for (int k = 0; k < sharers; ++k) {
                const float2 ml = s_ml[k * slots + i];
                add_scaled(a, weight(ml.x, m), reinterpret_cast<const float4*>(mg.o)[k * slots + i], ml.y);
              }
            }
            if (done) {
              write_row<T, DH>(p, now, head0 + 4 * i / DH, 4 * i % DH, a);
            } else {
              reinterpret_cast<float4*>(all + ahead)[i] = a.o;
              if (4 * i % DH == 0) *reinterpret_cast<float2*>(all + ahead + kHeads * DH + 2 * (4 * i / DH)) = make_float2(a.m, a.l);
            }
          }
        }
        return true;
      };
      if (join(&p.counters[g0], in_group, g0, 1, groups == 1) && groups > 1) join(&p.counters[kMaxBlocks + c0], groups, c0, kGroup, true);
    }
    __syncthreads();
  }
}

bool aligned16(const void* p) { return ((uintptr_t)p & 15) == 0; }

// AMPH_OK if the cache is one that the kernels take; *shift: log2 of its page size.
amph_status check_cache(const amph_paged_cache* c, int32_t n_seqs, int32_t table_stride, int* shift) {
  if (!c || !c->k_pages || !c->v_pages) return api_fail(AMPH_ERR_INVALID_ARG, "cache and its pages must not be NULL");
  if (c->dtype != AMPH_DTYPE_F32 && c->dtype != AMPH_DTYPE_BF16) return api_fail(AMPH_ERR_SHAPE, "unknown dtype %d", c->dtype);
  if (c->head_dim != 64 && c->head_dim != 128) return api_fail(AMPH_ERR_SHAPE, "head_dim must be 64 or 128 (got %d)", c->head_dim);
  if (c->n_kv_heads < 1 || c->n_kv_heads > 1024 || c->n_pages < 1)
    return api_fail(AMPH_ERR_SHAPE, "n_kv_heads must be in 1..1024 and n_pages positive");
  if (c->page_size < 1 || c->page_size > 65536 || (c->page_size & (c->page_size - 1)))
    return api_fail(AMPH_ERR_SHAPE, "page_size must be a power of two, at most 65536 (got %d)", c->page_size);
  if (n_seqs < 0 || table_stride < 1) return api_fail(AMPH_ERR_SHAPE, "n_seqs must not be negative and table_stride positive");
  if (((uintptr_t)c->k_pages | (uintptr_t)c->v_pages) & 31) return api_fail(AMPH_ERR_INVALID_ARG, "the pages must be 32-byte aligned");
  *shift = 0;
  while ((1 << *shift) < c->page_size) ++*shift;
  return AMPH_OK;
}

amph_status launched(cudaError_t e, const char* what) {
  if (e == cudaSuccess) return AMPH_OK;
  cudaGetLastError();
  return api_fail(AMPH_ERR_CUDA, "%s: %s", what, cudaGetErrorString(e));
}

// theta^(-2 i / dh) / (2 pi) for every pair, kept per thread for the last (theta, dh).
void fill_turns(float theta, int dh, u64* turn) {
  struct Kept { float theta = 0.f; int dh = 0; u64 turn[64]; };
  static thread_local Kept kept;
  if (kept.theta != theta || kept.dh != dh) {
    const long double two_pi = 6.283185307179586476925286766559005768L;
    for (int i = 0; i < dh / 2; ++i) {
      const long double share = powl((long double)theta, -2.0L * i / dh) / two_pi;
      kept.turn[i] = (u64)((share - floorl(share)) * 18446744073709551616.0L);
    }
    kept.theta = theta;
    kept.dh = dh;
  }
  memcpy(turn, kept.turn, sizeof(u64) * (dh / 2));
}

// One item a thread while all blocks run at once (8 rows of 32 heads: 2.4 us, 2.9 with three), three beyond (6,850 rows of 32 / 8 heads in
// bf16: 30.0 us, 5.6 TB/s; 34.7 with one or two, 31.5 with four).
template <typename TS, typename TD, int ITEMS>
cudaError_t run_write_items(const WriteParams& p, int rows, int items, cudaStream_t st) {
  // blocks of one row's parts, all of the same size
  const int parts = (items + ITEMS * kWriteThreads - 1) / (ITEMS * kWriteThreads);
  const int threads = ((items + parts * ITEMS - 1) / (parts * ITEMS) + 31) / 32 * 32;
  return launch_pdl(paged_write_kernel<TS, TD, ITEMS>, dim3(rows, parts), dim3(threads), 0, st, p);
}
template <typename TS, typename TD>
cudaError_t run_write(const WriteParams& p, int rows, cudaStream_t st) {
  const int items = (p.n_heads + 2 * p.n_kv) * (p.dh / 16);
  return (int64_t)rows * items <= 148 * 4 * kWriteThreads ? run_write_items<TS, TD, 1>(p, rows, items, st) : run_write_items<TS, TD, 3>(p, rows, items, st);
}

// What the table has room for, up to which an item gets a cluster: keys of a block, bytes of all keys and values.  Captured, line / cluster: one
// sequence of 640 tokens, 32 heads 9.0 / 6.1 us, 16 of 800 with 8 heads to one of 64 8.2 / 5.0, one of 2000 with 8 heads to one 14.0 / 6.0, of
// 8000 16.7 / 13.0, of 30000 26 / 37; room for 33 MB (32 of 2000, 8 / 2 heads of 64) 11.6 / 8.1, 43 MB (two of 1300, 32 heads) 15.5 / 14.8, 65 MB
// (8 of 2000, 32 / 8 heads) 15.5 / 18.6.
constexpr int kShortKeys = 8 * kUnit;
constexpr int64_t kShortBytes = 40 << 20;
// Launches the kernel in clusters of `blocks`, or, with `active`, asks how many of them run at a time.
cudaError_t launch_cluster(void (*kernel)(AttendParams), dim3 grid, int blocks, size_t smem, cudaStream_t st, const AttendParams& p, int* active = nullptr) {
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = grid;
  cfg.blockDim = dim3(kAttThreads);
  cfg.dynamicSmemBytes = smem;
  cfg.stream = st;
  cudaLaunchAttribute at[2];
  at[0].id = cudaLaunchAttributeClusterDimension;
  at[0].val.clusterDim.x = blocks;
  at[0].val.clusterDim.y = 1;
  at[0].val.clusterDim.z = 1;
  at[1].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  at[1].val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = at;
  cfg.numAttrs = active != nullptr ? 1 : 2;
  if (active != nullptr) return cudaOccupancyMaxActiveClusters(active, kernel, &cfg);
  return cudaLaunchKernelEx(&cfg, kernel, p);
}
// What a device runs at a time: blocks of the line, clusters of 1, 2, ... blocks (a cluster lies within a group of some 18 SMs, so that clusters
// of 13 leave a third of the device idle: one sequence of 1000 tokens, 32 heads 12.5 us with 13 parts, in two rounds, 7.6 with eight).
struct Limits {
  int blocks, clusters[kMaxParts + 1];
};
template <typename T, int DH, typename Item>
cudaError_t ask_limits(int dev, Limits& l) {
  constexpr size_t smem = sizeof(typename Item::Smem);
  int sms = 0;
  cudaError_t e = cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, dev);
  if (e == cudaSuccess) e = cudaFuncSetAttribute(paged_attention_cluster_kernel<T, DH, Item>, cudaFuncAttributeNonPortableClusterSizeAllowed, 1);
  if (e == cudaSuccess) e = cudaFuncSetAttribute(paged_attention_cluster_kernel<T, DH, Item>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem);
  if (e == cudaSuccess) e = cudaFuncSetAttribute(paged_attention_kernel<T, DH, Item>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem);
  l.blocks = sms * kAttResident<DH> < kMaxBlocks ? sms * kAttResident<DH> : kMaxBlocks;
  l.clusters[0] = 0;
  for (int i = 1; i <= kMaxParts && e == cudaSuccess; ++i)
    e = launch_cluster(paged_attention_cluster_kernel<T, DH, Item>, dim3(i), i, smem, nullptr, AttendParams{}, &l.clusters[i]);
  return e;
}
template <typename T, int DH, typename Item>
cudaError_t run_attention(const AttendParams& p, cudaStream_t st) {
  int dev = 0;
  cudaError_t e = cudaGetDevice(&dev);
  if (e != cudaSuccess) return e;
  constexpr size_t smem = sizeof(typename Item::Smem);
  static std::atomic<const Limits*> known[64];         // asked once; a device has them for good
  const Limits* l = dev < 64 ? known[dev].load() : nullptr;
  Limits now;
  if (l == nullptr) {
    e = ask_limits<T, DH, Item>(dev, now);
    if (e != cudaSuccess) return e;
    l = &now;
    if (dev < 64) known[dev].store(new (std::nothrow) Limits(now));
  }
  // A cluster for each item where all of them run at once and the tables have room for few keys
  const int64_t items = (int64_t)p.n_seqs * p.n_kv * p.head_blocks;
  int parts = items <= l->blocks ? (int)(l->blocks / items) : 0;
  if (parts > (p.cap + kUnit - 1) / kUnit) parts = (p.cap + kUnit - 1) / kUnit;
  if (parts > kMaxParts) parts = kMaxParts;
  while (parts > 0 && l->clusters[parts] < items) --parts;
  if (p.cap <= parts * kShortKeys && (int64_t)p.n_seqs * p.n_kv * p.cap * DH * (2 * sizeof(T)) <= kShortBytes)
    return launch_cluster(paged_attention_cluster_kernel<T, DH, Item>, dim3(parts, p.n_kv * p.head_blocks, p.n_seqs), parts, smem, st, p);
  return launch_pdl(paged_attention_kernel<T, DH, Item>, dim3(l->blocks), dim3(kAttThreads), smem, st, p);
}

static_assert(2 * kMaxBlocks * sizeof(int) <= AMPH_PAGED_WS_COUNTERS, "counters");
static_assert(AMPH_PAGED_WS_COUNTERS + (size_t)kMaxBlocks * 2 * kHeads * (128 + 2) * sizeof(float) <= AMPH_PAGED_WS_BYTES, "parts");

}  // namespace
}  // namespace amph

using namespace amph;

extern "C" {

amph_status amph_paged_write(const amph_paged_cache* cache, const void* q, int64_t q_stride, const void* k, int64_t k_stride,
                             const void* v, int64_t v_stride, int32_t src_dtype, int32_t n_heads, int32_t rows,
                             const int32_t* row_seq, const int32_t* row_pos, const int32_t* table, int32_t n_seqs,
                             int32_t table_stride, float theta, void* q_out, int32_t* status_dev, void* stream) {
  int shift = 0;
  const amph_status rc = check_cache(cache, n_seqs, table_stride, &shift);
  if (rc != AMPH_OK) return rc;
  if (!k || !v || !row_seq || !row_pos || !table || (n_heads != 0) != (q != nullptr) || (q != nullptr) != (q_out != nullptr))
    return api_fail(AMPH_ERR_INVALID_ARG, "k, v, row_seq, row_pos and table must not be NULL; q and q_out go together, with n_heads > 0");
  if (src_dtype != AMPH_DTYPE_F32 && src_dtype != AMPH_DTYPE_BF16) return api_fail(AMPH_ERR_SHAPE, "unknown src_dtype %d", src_dtype);
  if (n_heads < 0 || n_heads > 1024 || rows < 0) return api_fail(AMPH_ERR_SHAPE, "n_heads must be in 0..1024 and rows not negative");
  if (!(theta > 0.f) || !isfinite(theta)) return api_fail(AMPH_ERR_INVALID_ARG, "theta must be positive and finite");
  const int dh = cache->head_dim, esz = src_dtype == AMPH_DTYPE_F32 ? 4 : 2;
  if ((q && q_stride < (int64_t)n_heads * dh) || k_stride < (int64_t)cache->n_kv_heads * dh || v_stride < (int64_t)cache->n_kv_heads * dh)
    return api_fail(AMPH_ERR_SHAPE, "a row stride is shorter than the row");
  if (!aligned16(q) || !aligned16(k) || !aligned16(v) || !aligned16(q_out) || ((q ? q_stride : 0) | k_stride | v_stride) * esz % 16)
    return api_fail(AMPH_ERR_INVALID_ARG, "q, k, v and q_out must be 16-byte aligned, their row strides multiples of 16 bytes");
  if (rows == 0) return AMPH_OK;
  WriteParams p;
  p.q = q; p.k = k; p.v = v;
  p.q_stride = q_stride; p.k_stride = k_stride; p.v_stride = v_stride;
  p.q_out = q_out; p.k_pages = cache->k_pages; p.v_pages = cache->v_pages;
  p.row_seq = row_seq; p.row_pos = row_pos; p.table = table;
  p.status = status_dev;
  p.n_seqs = n_seqs; p.table_stride = table_stride; p.n_heads = n_heads; p.n_kv = cache->n_kv_heads;
  p.dh = dh; p.page_shift = shift; p.n_pages = cache->n_pages;
  fill_turns(theta, dh, p.turn);
  cudaStream_t st = (cudaStream_t)stream;
  const bool sf = src_dtype == AMPH_DTYPE_F32, df = cache->dtype == AMPH_DTYPE_F32;
  return launched(sf ? (df ? run_write<float, float>(p, rows, st) : run_write<float, bf16>(p, rows, st))
                     : (df ? run_write<bf16, float>(p, rows, st) : run_write<bf16, bf16>(p, rows, st)), "amph_paged_write");
}

amph_status amph_paged_attention(const amph_paged_cache* cache, const void* q, int32_t n_heads, const int32_t* lens,
                                 const int32_t* table, int32_t n_seqs, int32_t table_stride, float scale, void* out, float* lse,
                                 void* ws_dev, size_t ws_bytes, int32_t ws_clean, int32_t* status_dev, void* stream) {
  int shift = 0;
  const amph_status rc = check_cache(cache, n_seqs, table_stride, &shift);
  if (rc != AMPH_OK) return rc;
  if (!q || !lens || !table || !out || q == out) return api_fail(AMPH_ERR_INVALID_ARG, "q, lens, table and out must not be NULL, and out not q");
  if (n_heads < 1 || n_heads > 1024 || n_heads % cache->n_kv_heads)
    return api_fail(AMPH_ERR_SHAPE, "n_heads (%d) must be a multiple of n_kv_heads (%d), at most 1024", n_heads, cache->n_kv_heads);
  if (n_seqs > AMPH_PAGED_MAX_SEQS) return api_fail(AMPH_ERR_SHAPE, "n_seqs must be at most %d (got %d)", AMPH_PAGED_MAX_SEQS, n_seqs);
  const uintptr_t q_at = (uintptr_t)q, out_at = (uintptr_t)out, bytes = (uintptr_t)n_seqs * n_heads * cache->head_dim * (cache->dtype == AMPH_DTYPE_F32 ? 4 : 2);
  if (q_at < out_at + bytes && out_at < q_at + bytes) return api_fail(AMPH_ERR_INVALID_ARG, "out must not overlap q");
  const float scale_log2 = (scale == 0.f ? 1.0f / sqrtf((float)cache->head_dim) : scale) * kLog2e;
  if (!isfinite(scale_log2)) return api_fail(AMPH_ERR_INVALID_ARG, "scale must be finite, also times log2(e)");
  if (!aligned16(q) || !aligned16(out)) return api_fail(AMPH_ERR_INVALID_ARG, "q and out must be 16-byte aligned");
  if (!ws_dev || ((uintptr_t)ws_dev & 255) || ws_bytes < AMPH_PAGED_WS_BYTES)
    return api_fail(AMPH_ERR_WORKSPACE, "scratch: %u bytes needed, 256-byte aligned", AMPH_PAGED_WS_BYTES);
  if (n_seqs == 0) return AMPH_OK;
  AttendParams p;
  p.q = q; p.k = cache->k_pages; p.v = cache->v_pages;
  p.lens = lens; p.table = table; p.out = out; p.lse = lse;
  p.counters = (int*)ws_dev;
  p.parts = (float*)((char*)ws_dev + AMPH_PAGED_WS_COUNTERS);
  p.status = status_dev;
  p.part_floats = kHeads * (cache->head_dim + 2);
  p.n_seqs = n_seqs; p.table_stride = table_stride; p.n_heads = n_heads; p.n_kv = cache->n_kv_heads;
  p.group = n_heads / cache->n_kv_heads;
  p.head_blocks = (p.group + kHeads - 1) / kHeads;
  p.page_shift = shift; p.n_pages = cache->n_pages;
  const int64_t cap = (int64_t)table_stride << shift;
  p.cap = cap > 0x7fff0000 ? 0x7fff0000 : (int)cap;
  p.scale_log2 = scale_log2;
  cudaStream_t st = (cudaStream_t)stream;
  if (!ws_clean) {
    const cudaError_t e = cudaMemsetAsync(ws_dev, 0, AMPH_PAGED_WS_COUNTERS, st);
    if (e != cudaSuccess) return launched(e, "amph_paged_attention");
  }
  const bool d64 = cache->head_dim == 64;
  if (cache->dtype == AMPH_DTYPE_F32)
    return launched(d64 ? run_attention<float, 64, PlainItem<64>>(p, st) : run_attention<float, 128, PlainItem<128>>(p, st),
                    "amph_paged_attention");
  return launched(d64 ? run_attention<bf16, 64, MmaItem<64>>(p, st) : run_attention<bf16, 128, MmaItem<128>>(p, st),
                  "amph_paged_attention");
}

}  // extern "C"
