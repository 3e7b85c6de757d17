// The paged key-value cache: the handle, the write of new tokens (rotation, quantisation and placement in one pass), and
// reading cached tokens back.
//
// Both kernels are bound by memory: every input row is read once and every cached row written once (or the reverse). A
// token's angles and its place are found once and serve all its heads.
#include <new>

#include "kv_attend.cuh"

namespace lc {
namespace {

constexpr int kRowThreads = 256;

struct AppendArgs {
  int64_t n;
  const int32_t* seq;
  const int32_t* pos;
  const int32_t* rope_pos;
  Table table;
  int q_heads, kv_heads, chunks, lanes, page_size, rotate;
  int64_t pages;
  Rows k, v, q, q_out;
  void* pk;
  void* pv;
  float* ks;
  float* vs;
  unsigned int* status;
};

// Element (0, head, slot) of a cached row, as bytes from the pool's start.
template <int FMT>
__device__ __forceinline__ int64_t cached_at(int64_t row, int chunks) {
  return row * chunks * (FMT == LACACHE_KV_E4M3 || FMT == LACACHE_KV_INT8 ? 8 : 16);
}

template <int FMT>
__device__ __forceinline__ void store_cached(void* pool, float* scales, int64_t row, int chunks, int c, bool live, int lanes,
                                             const float (&x)[8]) {
  unsigned char* p = static_cast<unsigned char*>(pool) + cached_at<FMT>(row, chunks);
  if constexpr (FMT == LACACHE_KV_BF16) {
    if (live) store8(reinterpret_cast<__nv_bfloat16*>(p) + c * 8, x);
  } else if constexpr (FMT == LACACHE_KV_F16) {
    if (live) store8(reinterpret_cast<__half*>(p) + c * 8, x);
  } else {
    const float scale = row_scale<FMT>(x, lanes);
    if (live) {
      reinterpret_cast<uint2*>(p)[c] = quantise8<FMT>(x, scale);
      if (c == 0) scales[row] = scale;
    }
  }
}

// One token a block pass; its rows (q, then k, then v) go to the warps, 32 / lanes rows a warp at a time.
template <typename T, int FMT>
__global__ void __launch_bounds__(kRowThreads)
    append_kernel(const __grid_constant__ lacache_rope rope, const __grid_constant__ AppendArgs a) {
  __shared__ float2 cs[kMaxHeadDim / 2];
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const int rows_warp = 32 / a.lanes, c = lane & (a.lanes - 1), sub = lane / a.lanes;
  const int rows = a.q_heads + 2 * a.kv_heads;
  for (int64_t t = blockIdx.x; t < a.n; t += gridDim.x) {
    const int64_t place = slot_row(a.table, a.seq[t], a.pos[t], a.kv_heads, a.page_size, a.pages,
                                   threadIdx.x == 0 ? a.status : nullptr);
    __syncthreads();
    if (place < 0) continue;
    if (a.rotate && threadIdx.x < rope.rot_dim / 2)
      cs[threadIdx.x] = rope_angle(rope, threadIdx.x, a.rope_pos[t], 1.f);
    __syncthreads();
    for (int r0 = warp * rows_warp; r0 < rows; r0 += (kRowThreads / 32) * rows_warp) {
      const int r = r0 + sub;
      const bool live = r < rows && c < a.chunks;
      const int kind = r < a.q_heads ? 0 : r < a.q_heads + a.kv_heads ? 1 : 2;
      const int h = r - (kind == 0 ? 0 : kind == 1 ? a.q_heads : a.q_heads + a.kv_heads);
      const Rows& src = kind == 0 ? a.q : kind == 1 ? a.k : a.v;
      const T* row = reinterpret_cast<const T*>(src.p + t * src.token + (r < rows ? h : 0) * src.head);
      float x[8] = {};
      if (live) load8(row + c * 8, x);
      // every lane takes part in the exchange; rows of v rotate a copy and keep their own elements
      if (a.rotate) {
        float y[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) y[i] = x[i];
        rotate8(y, c, a.lanes, rope.rot_dim, rope.layout, cs, row);
#pragma unroll
        for (int i = 0; i < 8; ++i) x[i] = kind == 2 ? x[i] : y[i];
      }
      __syncwarp();
      if (live && kind == 0)
        store8(reinterpret_cast<T*>(a.q_out.p + t * a.q_out.token + h * a.q_out.head) + c * 8, x);
      const int64_t at = place + (int64_t)h * a.page_size;
      store_cached<FMT>(kind == 2 ? a.pv : a.pk, kind == 2 ? a.vs : a.ks, at, a.chunks, c, live && kind != 0, a.lanes, x);
    }
  }
}

struct ReadArgs {
  int64_t n;
  const int32_t* seq;
  const int32_t* pos;
  Table table;
  int kv_heads, chunks, lanes, page_size;
  int64_t pages;
  Rows k, v;   // p == nullptr: not wanted
  const void* pk;
  const void* pv;
  const float* ks;
  const float* vs;
  unsigned int* status;
};

template <typename T, int FMT>
__global__ void __launch_bounds__(kRowThreads) read_kernel(const __grid_constant__ ReadArgs a) {
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const int rows_warp = 32 / a.lanes, c = lane & (a.lanes - 1), sub = lane / a.lanes;
  const int rows = 2 * a.kv_heads;
  for (int64_t t = blockIdx.x; t < a.n; t += gridDim.x) {
    const int64_t place = slot_row(a.table, a.seq[t], a.pos[t], a.kv_heads, a.page_size, a.pages,
                                   threadIdx.x == 0 ? a.status : nullptr);
    if (place < 0) continue;
    for (int r = warp * rows_warp + sub; r < rows; r += (kRowThreads / 32) * rows_warp) {
      const bool is_v = r >= a.kv_heads;
      const int h = is_v ? r - a.kv_heads : r;
      const Rows& dst = is_v ? a.v : a.k;
      if (!dst.p || c >= a.chunks) continue;
      const int64_t at = place + (int64_t)h * a.page_size;
      const unsigned char* p = static_cast<const unsigned char*>(is_v ? a.pv : a.pk) + cached_at<FMT>(at, a.chunks);
      float x[8];
      if constexpr (FMT == LACACHE_KV_BF16)
        load8(reinterpret_cast<const __nv_bfloat16*>(p) + c * 8, x);
      else if constexpr (FMT == LACACHE_KV_F16)
        load8(reinterpret_cast<const __half*>(p) + c * 8, x);
      else
        dequantise8<FMT>(reinterpret_cast<const uint2*>(p)[c], (is_v ? a.vs : a.ks)[at], x);
      store8(reinterpret_cast<T*>(dst.p + t * dst.token + h * dst.head) + c * 8, x);
    }
  }
}

template <typename T>
void launch_append(int format, const lacache_rope& rope, const AppendArgs& a, unsigned grid, cudaStream_t st) {
  switch (format) {
    case LACACHE_KV_BF16: append_kernel<T, LACACHE_KV_BF16><<<grid, kRowThreads, 0, st>>>(rope, a); break;
    case LACACHE_KV_F16: append_kernel<T, LACACHE_KV_F16><<<grid, kRowThreads, 0, st>>>(rope, a); break;
    case LACACHE_KV_E4M3: append_kernel<T, LACACHE_KV_E4M3><<<grid, kRowThreads, 0, st>>>(rope, a); break;
    default: append_kernel<T, LACACHE_KV_INT8><<<grid, kRowThreads, 0, st>>>(rope, a); break;
  }
}
template <typename T>
void launch_read(int format, const ReadArgs& a, unsigned grid, cudaStream_t st) {
  switch (format) {
    case LACACHE_KV_BF16: read_kernel<T, LACACHE_KV_BF16><<<grid, kRowThreads, 0, st>>>(a); break;
    case LACACHE_KV_F16: read_kernel<T, LACACHE_KV_F16><<<grid, kRowThreads, 0, st>>>(a); break;
    case LACACHE_KV_E4M3: read_kernel<T, LACACHE_KV_E4M3><<<grid, kRowThreads, 0, st>>>(a); break;
    default: read_kernel<T, LACACHE_KV_INT8><<<grid, kRowThreads, 0, st>>>(a); break;
  }
}

size_t round_up(size_t n, size_t to) { return (n + to - 1) / to * to; }

}  // namespace
}  // namespace lc

extern "C" lacache_status lacache_kv_create(const lacache_kv_config* cfg, lacache_kv_t** out) {
  lc::NvtxRange nvtx("lacache_kv_create");
  if (!out) return LACACHE_ERR_INVALID_ARG;
  *out = nullptr;
  if (!cfg || cfg->layers < 1 || cfg->kv_heads < 1 || cfg->head_dim < 1 || cfg->page_size < 1 || cfg->pages < 1 ||
      cfg->pages > INT32_MAX || cfg->format < LACACHE_KV_BF16 || cfg->format > LACACHE_KV_INT8 || cfg->device < 0)
    return LACACHE_ERR_INVALID_ARG;
  if (cfg->head_dim % 16 || cfg->head_dim > lc::kMaxHeadDim || cfg->page_size % 16 || cfg->kv_heads > 65535)
    return LACACHE_ERR_UNSUPPORTED;
  const bool quantised = lc::is_quantised(cfg->format);
  // sizes in 64 bits: pages < 2^31, heads < 2^16, page sizes < 2^31, layers < 2^31, checked against 2^46 bytes in doubles
  const double rows_d = (double)cfg->pages * cfg->kv_heads * cfg->page_size;
  if (rows_d * cfg->layers * cfg->head_dim * 4.0 > 70368744177664.0) return LACACHE_ERR_OOM;
  const size_t rows = (size_t)cfg->pages * cfg->kv_heads * cfg->page_size;
  lacache_kv* h = new (std::nothrow) lacache_kv();
  if (!h) return LACACHE_ERR_OOM;
  h->cfg = *cfg;
  h->layer_bytes = rows * cfg->head_dim * (quantised ? 1 : 2);   // a multiple of 256: 16 slots of 16 elements or more
  h->layer_scales = quantised ? rows : 0;
  const size_t pool = h->layer_bytes * cfg->layers, scales = lc::round_up(h->layer_scales * cfg->layers * 4, 256);
  lc::DeviceGuard guard(cfg->device);
  lacache_status status = LACACHE_OK;
  if (!guard.ok() || cudaDeviceGetAttribute(&h->num_sms, cudaDevAttrMultiProcessorCount, cfg->device) != cudaSuccess) {
    status = LACACHE_ERR_CUDA;
  }
  const size_t blocks = (size_t)lc::kMaxBlocksPerSm * h->num_sms;
  const size_t partial = lc::round_up(blocks * 2 * lc::partial_floats(lc::padded_dim(cfg->head_dim)) * 4, 256);
  const size_t words = lc::round_up((blocks + 1) * 4, 256);   // counters and the status word: zeroed
  if (status == LACACHE_OK &&
      cudaMalloc(reinterpret_cast<void**>(&h->arena), 2 * pool + 2 * scales + partial + words) != cudaSuccess) {
    cudaGetLastError();   // the failed allocation is this call's to report, not a later one's
    status = LACACHE_ERR_OOM;
  }
  if (status == LACACHE_OK) {
    h->k = h->arena;
    h->v = h->k + pool;
    h->ks = quantised ? reinterpret_cast<float*>(h->v + pool) : nullptr;
    h->vs = quantised ? reinterpret_cast<float*>(h->v + pool + scales) : nullptr;
    h->partial = reinterpret_cast<float*>(h->v + pool + 2 * scales);
    h->arrived = reinterpret_cast<unsigned int*>(h->v + pool + 2 * scales + partial);
    h->dev_status = h->arrived + blocks;
    if (cudaMemset(h->arrived, 0, words) != cudaSuccess || cudaDeviceSynchronize() != cudaSuccess) {
      cudaFree(h->arena);
      status = LACACHE_ERR_CUDA;
    }
  }
  if (status != LACACHE_OK) {
    delete h;
    return status;
  }
  *out = h;
  return LACACHE_OK;
}

extern "C" lacache_status lacache_kv_destroy(lacache_kv_t* h) {
  if (!h) return LACACHE_OK;
  lc::DeviceGuard guard(h->cfg.device);
  cudaDeviceSynchronize();
  const cudaError_t e = cudaFree(h->arena);
  delete h;
  return lc::from_cuda(e);
}

extern "C" lacache_status lacache_kv_get_pool(const lacache_kv_t* h, int32_t layer, lacache_kv_pool* out) {
  if (!h || !out || layer < 0 || layer >= h->cfg.layers) return LACACHE_ERR_INVALID_ARG;
  out->k = h->k + h->layer_bytes * layer;
  out->v = h->v + h->layer_bytes * layer;
  out->k_scale = h->ks ? h->ks + h->layer_scales * layer : nullptr;
  out->v_scale = h->vs ? h->vs + h->layer_scales * layer : nullptr;
  return LACACHE_OK;
}

extern "C" lacache_status lacache_kv_append(lacache_kv_t* h, int32_t layer, const lacache_kv_table* table, int64_t n,
                                            const int32_t* seq_dev, const int32_t* pos_dev, const lacache_rope* rope,
                                            const int32_t* rope_pos_dev, int32_t dtype, const lacache_rows* k,
                                            const lacache_rows* v, int32_t q_heads, const lacache_rows* q,
                                            const lacache_rows* q_out, void* cuda_stream) {
  lc::NvtxRange nvtx("lacache_kv_append");
  lc::AppendArgs a = {};
  lacache_kv_pool pool;
  if (lacache_kv_get_pool(h, layer, &pool) != LACACHE_OK || n < 0 || !lc::known_dtype(dtype) ||
      !lc::device_table(table, &a.table))
    return LACACHE_ERR_INVALID_ARG;
  if (rope && (rope->rot_dim < 2 || rope->rot_dim % 2 || rope->rot_dim > h->cfg.head_dim)) return LACACHE_ERR_INVALID_ARG;
  if (n == 0) return LACACHE_OK;
  if (!seq_dev || !pos_dev || !lc::device_rows(k, dtype, &a.k) || !lc::device_rows(v, dtype, &a.v))
    return LACACHE_ERR_INVALID_ARG;
  if (q && (q_heads < 1 || !lc::device_rows(q, dtype, &a.q) || !lc::device_rows(q_out, dtype, &a.q_out)))
    return LACACHE_ERR_INVALID_ARG;
  lc::DeviceGuard guard(h->cfg.device);
  if (!guard.ok()) return LACACHE_ERR_CUDA;
  a.n = n;
  a.seq = seq_dev;
  a.pos = pos_dev;
  a.rope_pos = rope_pos_dev ? rope_pos_dev : pos_dev;
  a.q_heads = q ? q_heads : 0;
  a.kv_heads = h->cfg.kv_heads;
  a.chunks = h->cfg.head_dim / 8;
  a.lanes = lc::lanes_for(h->cfg.head_dim);
  a.page_size = h->cfg.page_size;
  a.pages = h->cfg.pages;
  a.rotate = rope ? 1 : 0;
  a.pk = pool.k;
  a.pv = pool.v;
  a.ks = pool.k_scale;
  a.vs = pool.v_scale;
  a.status = h->dev_status;
  static const lacache_rope none = {};
  const lacache_rope& plan = rope ? *rope : none;
  const unsigned grid = (unsigned)(n < 65536 ? n : 65536);
  const cudaStream_t st = (cudaStream_t)cuda_stream;
  if (dtype == LACACHE_BF16) lc::launch_append<__nv_bfloat16>(h->cfg.format, plan, a, grid, st);
  else if (dtype == LACACHE_F16) lc::launch_append<__half>(h->cfg.format, plan, a, grid, st);
  else lc::launch_append<float>(h->cfg.format, plan, a, grid, st);
  return lc::from_cuda(cudaGetLastError());
}

extern "C" lacache_status lacache_kv_read(lacache_kv_t* h, int32_t layer, const lacache_kv_table* table, int64_t n,
                                          const int32_t* seq_dev, const int32_t* pos_dev, int32_t dtype,
                                          const lacache_rows* k, const lacache_rows* v, void* cuda_stream) {
  lc::NvtxRange nvtx("lacache_kv_read");
  lc::ReadArgs a = {};
  lacache_kv_pool pool;
  if (lacache_kv_get_pool(h, layer, &pool) != LACACHE_OK || n < 0 || !lc::known_dtype(dtype) ||
      !lc::device_table(table, &a.table))
    return LACACHE_ERR_INVALID_ARG;
  if (n == 0 || (!k && !v)) return LACACHE_OK;
  if (!seq_dev || !pos_dev || (k && !lc::device_rows(k, dtype, &a.k)) || (v && !lc::device_rows(v, dtype, &a.v)))
    return LACACHE_ERR_INVALID_ARG;
  lc::DeviceGuard guard(h->cfg.device);
  if (!guard.ok()) return LACACHE_ERR_CUDA;
  a.n = n;
  a.seq = seq_dev;
  a.pos = pos_dev;
  a.kv_heads = h->cfg.kv_heads;
  a.chunks = h->cfg.head_dim / 8;
  a.lanes = lc::lanes_for(h->cfg.head_dim);
  a.page_size = h->cfg.page_size;
  a.pages = h->cfg.pages;
  a.pk = pool.k;
  a.pv = pool.v;
  a.ks = pool.k_scale;
  a.vs = pool.v_scale;
  a.status = h->dev_status;
  const unsigned grid = (unsigned)(n < 65536 ? n : 65536);
  const cudaStream_t st = (cudaStream_t)cuda_stream;
  if (dtype == LACACHE_BF16) lc::launch_read<__nv_bfloat16>(h->cfg.format, a, grid, st);
  else if (dtype == LACACHE_F16) lc::launch_read<__half>(h->cfg.format, a, grid, st);
  else lc::launch_read<float>(h->cfg.format, a, grid, st);
  return lc::from_cuda(cudaGetLastError());
}

extern "C" lacache_status lacache_kv_sync(lacache_kv_t* h) {
  lc::NvtxRange nvtx("lacache_kv_sync");
  if (!h) return LACACHE_ERR_INVALID_ARG;
  lc::DeviceGuard guard(h->cfg.device);
  unsigned int word = 0;
  if (!guard.ok() || cudaDeviceSynchronize() != cudaSuccess ||
      cudaMemcpy(&word, h->dev_status, 4, cudaMemcpyDeviceToHost) != cudaSuccess)
    return LACACHE_ERR_CUDA;
  if (!word) return LACACHE_OK;
  if (cudaMemset(h->dev_status, 0, 4) != cudaSuccess || cudaDeviceSynchronize() != cudaSuccess) return LACACHE_ERR_CUDA;
  return LACACHE_ERR_INVALID_ARG;
}
