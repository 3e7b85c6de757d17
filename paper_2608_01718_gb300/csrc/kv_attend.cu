// Attention of new tokens over the paged cache: the C entry.
#include <algorithm>

#include "kv_attend.cuh"

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
  if (at->new_tokens > lc::kMaxNewTokens || at->q_heads > lc::kMaxQHeads || (c.format == LACACHE_KV_BF16 && at->dtype != LACACHE_BF16) ||
      (c.format == LACACHE_KV_F16 && at->dtype != LACACHE_F16))
    return LACACHE_ERR_UNSUPPORTED;
  if (table->seqs == 0) return LACACHE_OK;
  if (!at->lengths_dev || !lc::device_rows(&at->q, at->dtype, &a.q) || !lc::device_rows(&at->out, at->dtype, &a.out) ||
      at->out.data == at->q.data)
    return LACACHE_ERR_INVALID_ARG;
  lc::DeviceGuard guard(c.device);
  if (!guard.ok()) return LACACHE_ERR_CUDA;
  a.new_tokens = at->new_tokens;
  a.q_heads = at->q_heads;
  a.kv_heads = c.kv_heads;
  a.head_dim = c.head_dim;
  a.page_size = c.page_size;
  a.window = at->window < lc::kMaxPositions ? at->window : 0;   // no position lies further back
  a.group = at->q_heads / c.kv_heads;
  a.rows = a.group * at->new_tokens;
  a.q_f16 = at->dtype == LACACHE_F16;
  a.max_len = (int)std::min<int64_t>((int64_t)table->width * c.page_size, lc::kMaxPositions);
  a.device = c.device;
  a.pages = c.pages;
  a.page_rows = (int64_t)c.kv_heads * c.page_size;
  a.page_bytes = a.page_rows * c.head_dim * (lc::is_quantised(c.format) ? 1 : 2);
  // n / d = n * ceil(2^(26 + s) / d) >> (26 + s) for n < 2^26 and d <= 2^s
  const uint32_t d = (uint32_t)c.page_size / 16;
  a.page_shift = 26;
  while ((1u << (a.page_shift - 26)) < d) ++a.page_shift;
  a.page_mul = (uint32_t)((((uint64_t)1 << a.page_shift) + d - 1) / d);
  a.scale = at->scale;
  a.lengths = at->lengths_dev;
  a.starts = at->starts_dev;
  a.lse = at->lse_dev;
  a.pk = static_cast<const unsigned char*>(pool.k);
  a.pv = static_cast<const unsigned char*>(pool.v);
  a.ks = pool.k_scale;
  a.vs = pool.v_scale;
  a.partial = h->partial;
  a.arrived = h->arrived;
  a.status = h->dev_status;
  const cudaStream_t st = (cudaStream_t)cuda_stream;
  cudaError_t e;
  if (lc::takes_tc(a.rows, a.group, c.head_dim, lc::is_quantised(c.format))) {
    if (h->inject_stall > 0) {
      a.inject_stall = 1;
      --h->inject_stall;
    }
    e = lc::launch_attend_tc(a, c.format, h->num_sms, st);
  } else switch (c.format) {
    case LACACHE_KV_BF16: e = lc::launch_attend_bf16(a, h->num_sms, st); break;
    case LACACHE_KV_F16: e = lc::launch_attend_f16(a, h->num_sms, st); break;
    case LACACHE_KV_E4M3: e = lc::launch_attend_e4m3(a, h->num_sms, st); break;
    default: e = lc::launch_attend_int8(a, h->num_sms, st); break;
  }
  return e == cudaErrorNotSupported ? LACACHE_ERR_UNSUPPORTED : lc::from_cuda(e);
}
