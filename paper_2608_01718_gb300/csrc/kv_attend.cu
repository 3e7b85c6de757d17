// Attention of new tokens over the paged cache: the C entry.
#include <algorithm>

#include "kv_attend.cuh"

namespace lc {

// What every pass of new tokens over the cache takes: checked, and as the kernels want it (out, lse and scratch excepted).
lacache_status attend_args(lacache_kv_t* h, int layer, const lacache_kv_table* table, int new_tokens, int q_heads, int window,
                           int dtype, float scale, const int32_t* lengths, const int32_t* starts, const lacache_rows* q,
                           AttendArgs* out) {
  AttendArgs& a = *out;
  lacache_kv_pool pool;
  if (lacache_kv_get_pool(h, layer, &pool) != LACACHE_OK || !device_table(table, &a.table)) return LACACHE_ERR_INVALID_ARG;
  const lacache_kv_config& c = h->cfg;
  if (new_tokens < 1 || q_heads < 1 || q_heads % c.kv_heads || window < 0 || !isfinite(scale) ||
      (dtype != LACACHE_BF16 && dtype != LACACHE_F16))
    return LACACHE_ERR_INVALID_ARG;
  if (new_tokens > kMaxNewTokens || q_heads > kMaxQHeads || (c.format == LACACHE_KV_BF16 && dtype != LACACHE_BF16) ||
      (c.format == LACACHE_KV_F16 && dtype != LACACHE_F16))
    return LACACHE_ERR_UNSUPPORTED;
  if (table->seqs == 0) return LACACHE_OK;
  if (!lengths || !device_rows(q, dtype, &a.q)) return LACACHE_ERR_INVALID_ARG;
  a.new_tokens = new_tokens;
  a.q_heads = q_heads;
  a.kv_heads = c.kv_heads;
  a.head_dim = c.head_dim;
  a.page_size = c.page_size;
  a.window = window < kMaxPositions ? window : 0;   // no position lies further back
  a.group = q_heads / c.kv_heads;
  a.rows = a.group * new_tokens;
  a.q_f16 = dtype == LACACHE_F16;
  a.max_len = (int)std::min<int64_t>((int64_t)table->width * c.page_size, kMaxPositions);
  a.device = c.device;
  a.pages = c.pages;
  a.page_rows = (int64_t)c.kv_heads * c.page_size;
  a.page_bytes = a.page_rows * c.head_dim * (is_quantised(c.format) ? 1 : 2);
  // n / d = n * ceil(2^(26 + s) / d) >> (26 + s) for n < 2^26 and d <= 2^s
  const uint32_t d = (uint32_t)c.page_size / 16;
  a.page_shift = 26;
  while ((1u << (a.page_shift - 26)) < d) ++a.page_shift;
  a.page_mul = (uint32_t)((((uint64_t)1 << a.page_shift) + d - 1) / d);
  a.scale = scale;
  a.lengths = lengths;
  a.starts = starts;
  a.pk = static_cast<const unsigned char*>(pool.k);
  a.pv = static_cast<const unsigned char*>(pool.v);
  a.ks = pool.k_scale;
  a.vs = pool.v_scale;
  a.partial = h->partial;
  a.arrived = h->arrived;
  a.status = h->dev_status;
  return LACACHE_OK;
}

// An attention with its outputs, by the kernel that its sizes call for.
lacache_status launch_whole(lacache_kv_t* h, AttendArgs& a, cudaStream_t st) {
  const lacache_kv_config& c = h->cfg;
  cudaError_t e;
  if (takes_tc(a.rows, a.group, c.head_dim, is_quantised(c.format))) {
    if (h->inject_stall > 0) {
      a.inject_stall = 1;
      --h->inject_stall;
    }
    e = launch_attend_tc(a, c.format, h->num_sms, st);
  } else switch (c.format) {
    case LACACHE_KV_BF16: e = launch_attend_bf16(a, h->num_sms, st); break;
    case LACACHE_KV_F16: e = launch_attend_f16(a, h->num_sms, st); break;
    case LACACHE_KV_E4M3: e = launch_attend_e4m3(a, h->num_sms, st); break;
    default: e = launch_attend_int8(a, h->num_sms, st); break;
  }
  return e == cudaErrorNotSupported ? LACACHE_ERR_UNSUPPORTED : from_cuda(e);
}

}  // namespace lc

extern "C" lacache_status lacache_kv_attend(lacache_kv_t* h, int32_t layer, const lacache_kv_table* table,
                                            const lacache_attention* at, void* cuda_stream) {
  lc::NvtxRange nvtx("lacache_kv_attend");
  lc::AttendArgs a = {};
  if (!at) return LACACHE_ERR_INVALID_ARG;
  const lacache_status status = lc::attend_args(h, layer, table, at->new_tokens, at->q_heads, at->window, at->dtype, at->scale,
                                                at->lengths_dev, at->starts_dev, &at->q, &a);
  if (status != LACACHE_OK || table->seqs == 0) return status;
  if (!lc::device_rows(&at->out, at->dtype, &a.out) || at->out.data == at->q.data) return LACACHE_ERR_INVALID_ARG;
  const lacache_kv_config& c = h->cfg;
  lc::DeviceGuard guard(c.device);
  if (!guard.ok()) return LACACHE_ERR_CUDA;
  a.lse = at->lse_dev;
  return lc::launch_whole(h, a, (cudaStream_t)cuda_stream);
}
