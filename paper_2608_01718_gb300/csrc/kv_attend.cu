// Attention of new tokens over the paged cache.
#include <math.h>

#include "decode.cuh"

namespace lc {
namespace {

struct AttendArgs {
  Table table;
  int new_tokens, q_heads, kv_heads, head_dim, page_size, window;
  int64_t pages;
  float scale;
  const int32_t* lengths;
  const int32_t* starts;
  Rows q, out;
  float* lse;
  const void* pk;
  const void* pv;
  const float* ks;
  const float* vs;
  unsigned int* status;
};

template <int FMT>
__device__ __forceinline__ float cached(const void* pool, int64_t i) {
  if constexpr (FMT == LACACHE_KV_BF16) return __bfloat162float(static_cast<const __nv_bfloat16*>(pool)[i]);
  if constexpr (FMT == LACACHE_KV_F16) return __half2float(static_cast<const __half*>(pool)[i]);
  if constexpr (FMT == LACACHE_KV_E4M3)
    return __half2float(__half(__nv_cvt_fp8_to_halfraw(static_cast<const __nv_fp8_storage_t*>(pool)[i], __NV_E4M3)));
  return (float)static_cast<const int8_t*>(pool)[i];
}

// The first kernel: a warp per query head row, one key at a time, running maximum and sum.
template <typename T, int FMT>
__global__ void __launch_bounds__(128) attend_kernel(const __grid_constant__ AttendArgs a) {
  const int lane = threadIdx.x & 31;
  const int64_t r = blockIdx.x * 4ll + (threadIdx.x >> 5);
  if (r >= (int64_t)a.table.seqs * a.new_tokens * a.q_heads) return;
  const int64_t tok = r / a.q_heads;
  const int qh = (int)(r % a.q_heads), s = (int)(tok / a.new_tokens), t = (int)(tok % a.new_tokens);
  const int h = qh / (a.q_heads / a.kv_heads), D = a.head_dim;
  const int64_t room = (int64_t)a.table.width * a.page_size;
  int64_t len = a.lengths[s];
  if (len < 0 || len > room) {
    if (lane == 0) atomicOr(a.status, kBadIndex);
    len = len < 0 ? 0 : room;
  }
  const int64_t p = len - a.new_tokens + t;
  int64_t lo = a.starts ? a.starts[s] : 0;
  if (a.window > 0 && p - a.window + 1 > lo) lo = p - a.window + 1;
  if (lo < 0) lo = 0;
  const T* q = reinterpret_cast<const T*>(a.q.p + tok * a.q.token + qh * a.q.head);
  float qv[kMaxHeadDim / 32], o[kMaxHeadDim / 32] = {};
#pragma unroll
  for (int i = 0; i < kMaxHeadDim / 32; ++i) qv[i] = lane + 32 * i < D ? (float)q[lane + 32 * i] : 0.f;
  float m = -INFINITY, l = 0.f;
  for (int64_t j = lo; j <= p; ++j) {
    const int page = a.table.pages[s * a.table.stride + j / a.page_size];
    if (page < 0 || page >= a.pages) {
      if (lane == 0) atomicOr(a.status, kBadIndex);
      continue;
    }
    const int64_t row = ((int64_t)page * a.kv_heads + h) * a.page_size + j % a.page_size;
    float dot = 0.f;
#pragma unroll
    for (int i = 0; i < kMaxHeadDim / 32; ++i)
      if (lane + 32 * i < D) dot += qv[i] * cached<FMT>(a.pk, row * D + lane + 32 * i);
    for (int off = 16; off; off >>= 1) dot += __shfl_xor_sync(0xffffffffu, dot, off);
    const float x = dot * a.scale * (a.ks ? a.ks[row] : 1.f);
    const float top = fmaxf(m, x), shift = top == -INFINITY ? 0.f : top;
    const float f = expf(m - shift), w = expf(x - shift);
    l = l * f + w;
    const float wv = a.vs ? w * a.vs[row] : w;
#pragma unroll
    for (int i = 0; i < kMaxHeadDim / 32; ++i)
      if (lane + 32 * i < D) o[i] = o[i] * f + wv * cached<FMT>(a.pv, row * D + lane + 32 * i);
    m = top;
  }
  T* out = reinterpret_cast<T*>(a.out.p + tok * a.out.token + qh * a.out.head);
#pragma unroll
  for (int i = 0; i < kMaxHeadDim / 32; ++i)
    if (lane + 32 * i < D) out[lane + 32 * i] = (T)(l == 0.f ? 0.f : o[i] / l);
  if (a.lse && lane == 0) a.lse[r] = l == 0.f ? -INFINITY : m + logf(l);
}

template <typename T>
void launch_attend(int format, const AttendArgs& a, cudaStream_t st) {
  const int64_t rows = (int64_t)a.table.seqs * a.new_tokens * a.q_heads;
  const unsigned grid = (unsigned)((rows + 3) / 4);
  switch (format) {
    case LACACHE_KV_BF16: attend_kernel<T, LACACHE_KV_BF16><<<grid, 128, 0, st>>>(a); break;
    case LACACHE_KV_F16: attend_kernel<T, LACACHE_KV_F16><<<grid, 128, 0, st>>>(a); break;
    case LACACHE_KV_E4M3: attend_kernel<T, LACACHE_KV_E4M3><<<grid, 128, 0, st>>>(a); break;
    default: attend_kernel<T, LACACHE_KV_INT8><<<grid, 128, 0, st>>>(a); break;
  }
}

}  // namespace
}  // namespace lc

extern "C" lacache_status lacache_kv_attend(lacache_kv_t* h, int32_t layer, const lacache_kv_table* table,
                                            const lacache_attention* at, void* cuda_stream) {
  lc::NvtxRange nvtx("lacache_kv_attend");
  lc::AttendArgs a = {};
  lacache_kv_pool pool;
  if (lacache_kv_get_pool(h, layer, &pool) != LACACHE_OK || !at || !lc::device_table(table, &a.table))
    return LACACHE_ERR_INVALID_ARG;
  const lacache_kv_config& c = h->cfg;
  if (at->new_tokens < 1 || at->q_heads < 1 || at->q_heads % c.kv_heads || at->window < 0 || !isfinite(at->scale) ||
      (at->dtype != LACACHE_BF16 && at->dtype != LACACHE_F16))
    return LACACHE_ERR_INVALID_ARG;
  if (at->new_tokens > lc::kMaxNewTokens || (c.format == LACACHE_KV_BF16 && at->dtype != LACACHE_BF16) ||
      (c.format == LACACHE_KV_F16 && at->dtype != LACACHE_F16))
    return LACACHE_ERR_UNSUPPORTED;
  if (table->seqs == 0) return LACACHE_OK;
  if (!at->lengths_dev || !lc::device_rows(&at->q, at->dtype, &a.q) || !lc::device_rows(&at->out, at->dtype, &a.out))
    return LACACHE_ERR_INVALID_ARG;
  lc::DeviceGuard guard(c.device);
  if (!guard.ok()) return LACACHE_ERR_CUDA;
  a.new_tokens = at->new_tokens;
  a.q_heads = at->q_heads;
  a.kv_heads = c.kv_heads;
  a.head_dim = c.head_dim;
  a.page_size = c.page_size;
  a.window = at->window;
  a.pages = c.pages;
  a.scale = at->scale;
  a.lengths = at->lengths_dev;
  a.starts = at->starts_dev;
  a.lse = at->lse_dev;
  a.pk = pool.k;
  a.pv = pool.v;
  a.ks = pool.k_scale;
  a.vs = pool.v_scale;
  a.status = h->dev_status;
  const cudaStream_t st = (cudaStream_t)cuda_stream;
  if (at->dtype == LACACHE_BF16) lc::launch_attend<__nv_bfloat16>(c.format, a, st);
  else lc::launch_attend<__half>(c.format, a, st);
  return lc::from_cuda(cudaGetLastError());
}
