// amph_project_adapters: a projection shared by all rows, and each row's own low-rank adapter beside it.
//
//   t[r][s][j] = sum_k x[r][k] a[i_r][s][j][k]                       the rows' low-rank products (down)
//   P          = x . w^T                                             the projection kernels, as split-K partial sums
//   y[r][s][o] = sum P + scale[i_r] sum_j t[r][s][j] b[i_r][s][o][j]  reduction of the partial sums, adapters' way back up (up)
#include <mutex>

#include "amph_internal.cuh"
#include "gemm_tc_common.cuh"

namespace amph {
namespace {

typedef __nv_bfloat16 bf16;

constexpr int kMaxRowsAll = 4 * kMaxRows;
constexpr int kThreads = 128;

__device__ __forceinline__ float to_f(float v) { return v; }
__device__ __forceinline__ float to_f(bf16 v) { return __bfloat162float(v); }
__device__ __forceinline__ void put(float* p, float v) { *p = v; }
__device__ __forceinline__ void put(bf16* p, float v) { *p = __float2bfloat16_rn(v); }

struct AdapterArgs {
  const void *x, *a, *b;
  const float* scale;
  const int* row_adapter;
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

// One warp per (row, column of t).
template <typename T>
__global__ void __launch_bounds__(kThreads) adapter_down_plain_kernel(const AdapterArgs p) {
  pdl_wait();
  pdl_launch_dependents();
  const int cols = p.n_seg * p.rank, lane = threadIdx.x & 31;
  const int row = blockIdx.y, col = blockIdx.x * (kThreads / 32) + (threadIdx.x >> 5);
  const int i = adapter_of(p, row);
  if (i < 0 || col >= cols) return;
  const T* x = (const T*)p.x + (size_t)row * p.in;
  const T* a = (const T*)p.a + ((size_t)i * cols + col) * p.in;
  float acc = 0.f;
  for (int k = lane; k < p.in; k += 32) acc += to_f(x[k]) * to_f(a[k]);
#pragma unroll
  for (int d = 16; d; d >>= 1) acc += __shfl_xor_sync(~0u, acc, d);
  if (lane == 0) p.t[(size_t)row * cols + col] = acc;
}

// Grid (128 columns, row), one column per thread.
template <typename T, typename TY>
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
  const float* src = P.p + (size_t)row * P.ld + c;
  float acc = src[0];
  for (int s = 1; s < P.splits; ++s) acc += src[s * P.split_stride];
  if (i >= 0) {
    const int seg = c / p.out, o = c - seg * p.out;
    const T* b = (const T*)p.b + (((size_t)i * p.n_seg + seg) * p.out + o) * p.rank;
    float low = 0.f;
    for (int j = 0; j < p.rank; ++j) low += t[seg * p.rank + j] * to_f(b[j]);
    acc += low;
  }
  put((TY*)p.y + (size_t)row * ld + c, acc);
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
int down_splits(int rows) { (void)rows; return 1; }

amph_status bad_shape(int n_seg, int out, int rows, int rank) {
  if (n_seg < 1 || n_seg > kMaxK || out < 1 || rows < 1 || rows > kMaxRowsAll) return api_fail(AMPH_ERR_SHAPE, "bad projection shape");
  if ((int64_t)n_seg * out > 0x7fffffff / 4) return api_fail(AMPH_ERR_SHAPE, "too many output features");
  if (rank < 8 || rank > AMPH_MAX_ADAPTER_RANK || rank % 8)
    return api_fail(AMPH_ERR_SHAPE, "rank must be a multiple of 8 in 8..%d (got %d)", AMPH_MAX_ADAPTER_RANK, rank);
  return AMPH_OK;
}
size_t t_bytes(int n_seg, int rows, int rank) { return round256((size_t)down_splits(rows) * rows * n_seg * rank * 4); }

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
  const size_t ld = (size_t)n_seg * out, tb = t_bytes(n_seg, rows, ad->rank);
  AdapterArgs p;
  p.x = x_dev; p.a = ad->a; p.b = ad->b; p.scale = ad->scale;
  p.row_adapter = row_adapter;
  p.t = (float*)ws_dev;
  p.y = y_dev;
  p.status = status_dev;
  p.n_adapters = ad->n_adapters; p.rank = ad->rank; p.n_seg = n_seg; p.out = out; p.in = in; p.rows = rows; p.splits = down_splits(rows);
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
  const int cols = n_seg * ad->rank;
  cudaError_t e;
  {
    const dim3 grid((cols + 3) / 4, rows);
    e = dtype == AMPH_DTYPE_F32 ? launch_pdl(adapter_down_plain_kernel<float>, grid, dim3(kThreads), 0, st, p)
                                : launch_pdl(adapter_down_plain_kernel<bf16>, grid, dim3(kThreads), 0, st, p);
  }
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
    const dim3 grid((unsigned)((ld + kThreads - 1) / kThreads), rows);
    if (dtype == AMPH_DTYPE_F32) e = launch_pdl(adapter_up_plain_kernel<float, float>, grid, dim3(kThreads), 0, st, p, pv);
    else if (y_dtype == AMPH_DTYPE_F32) e = launch_pdl(adapter_up_plain_kernel<bf16, float>, grid, dim3(kThreads), 0, st, p, pv);
    else e = launch_pdl(adapter_up_plain_kernel<bf16, bf16>, grid, dim3(kThreads), 0, st, p, pv);
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
  *ws_bytes = t_bytes(n_seg, rows, rank) + round256((size_t)most_splits(n_seg, out) * padded(rows) * n_seg * out * sizeof(float));
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
