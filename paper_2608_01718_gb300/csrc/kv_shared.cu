// Attention for batches of sequences that have their first positions in common (a system prompt, a document), which are read and
// multiplied once for all sequences of a group. With a row's scores s_j, split at its group's common length P:
//
//   (o_1, L_1) over j < P,  (o_2, L_2) over j >= P,  L = log(e^L_1 + e^L_2),  out = e^(L_1 - L) o_1 + e^(L_2 - L) o_2,
//
// where o is a part's output and L its lse. Three kernels: what each group's rows see of the common positions, and where each
// sequence's own begin; the common part, in which a group stands for a sequence and the new tokens of all of its sequences are
// its rows (so that K and V are read for up to 128 rows at a time, and products run at the tensor cores' rate instead of HBM's);
// the own part, which ends each row by joining it with the other. The common part's outputs and lse stay fp32 in the workspace.
// The kernels are those of kv_attend.cuh and kv_attend_tc.cu, in their forms kCommon and kOwn.
#include <algorithm>

#include "kv_attend.cuh"

namespace lc {
namespace {

struct Groups {
  int groups, seqs, new_tokens, window, max_len;
  const int32_t* bounds;    // nullptr: one group of all
  const int32_t* common;
  const int32_t* lengths;
  const int32_t* starts;
  int4* spans;
  int32_t* own_starts;
  int32_t* joined;
  unsigned int* status;
};
constexpr int kGroupThreads = 128;

// A block a group. Bounds that do not rise within [0, seqs] leave no group: every sequence is then read for itself.
__global__ void __launch_bounds__(kGroupThreads) group_kernel(const __grid_constant__ Groups a) {
  const int g = blockIdx.x;
  int bad = 0;
  if (a.bounds) {
    for (int i = threadIdx.x; i <= a.groups; i += kGroupThreads) {
      const int x = a.bounds[i];
      bad |= x < 0 || x > a.seqs || (i > 0 && a.bounds[i - 1] > x);
    }
  }
  bad = __syncthreads_or(bad);
  const int all_first = bad ? 0 : a.bounds ? a.bounds[0] : 0, all_end = bad ? 0 : a.bounds ? a.bounds[a.groups] : a.seqs;
  if (g == 0) {   // sequences of no group
    for (int s = threadIdx.x; s < a.seqs; s += kGroupThreads) {
      if (s >= all_first && s < all_end) continue;
      a.own_starts[s] = a.starts ? a.starts[s] : 0;
      a.joined[s] = 0;
    }
    if (bad && threadIdx.x == 0) atomicOr(a.status, kBadIndex);
  }
  const int first = bad ? 0 : a.bounds ? a.bounds[g] : 0, end = bad ? 0 : a.bounds ? a.bounds[g + 1] : a.seqs;
  const int raw = a.common[g], common = raw < 0 ? 0 : raw > a.max_len ? a.max_len : raw;
  if (raw != common && threadIdx.x == 0) atomicOr(a.status, kBadIndex);
  int lo = INT_MAX, hi = 0;
  for (int s = first + threadIdx.x; s < end; s += kGroupThreads) {
    const int len = min(max(a.lengths[s], 0), a.max_len), start = a.starts ? a.starts[s] : 0;
    int seen = max(start, 0);
    if (a.window > 0) seen = max(seen, len - a.new_tokens - a.window + 1);   // (window < 2^30: no overflow)
    lo = min(lo, seen);
    hi = max(hi, min(len, common));
    a.own_starts[s] = max(start, common);
    a.joined[s] = common > 0;
  }
  __shared__ int s_lo, s_hi;
  if (threadIdx.x == 0) s_lo = INT_MAX, s_hi = 0;
  __syncthreads();
  lo = __reduce_min_sync(0xffffffffu, lo);
  hi = __reduce_max_sync(0xffffffffu, hi);
  if ((threadIdx.x & 31) == 0) {
    atomicMin(&s_lo, lo);
    atomicMax(&s_hi, hi);
  }
  __syncthreads();
  // (without common positions: no rows either)
  if (threadIdx.x == 0) a.spans[g] = make_int4(min(s_lo, s_hi), s_hi, first, common > 0 ? end - first : 0);
}

struct Workspace {
  size_t spans, own_starts, joined, lse, common, bytes;   // offsets
};
inline size_t round16(size_t n) { return (n + 15) / 16 * 16; }
Workspace workspace_of(int64_t seqs, int groups, int new_tokens, int q_heads, int head_dim) {
  Workspace w;
  const size_t rows = (size_t)seqs * new_tokens * q_heads;
  w.spans = 0;
  w.own_starts = (size_t)groups * sizeof(int4);
  w.joined = w.own_starts + round16((size_t)seqs * 4);
  w.lse = w.joined + round16((size_t)seqs * 4);
  w.common = w.lse + round16(rows * 4);
  w.bytes = w.common + rows * head_dim * 4;
  return w;
}

cudaError_t launch_common(const AttendArgs& a, int format, int num_sms, cudaStream_t st) {
  switch (format) {
    case LACACHE_KV_BF16: return launch_common_bf16(a, num_sms, st);
    case LACACHE_KV_F16: return launch_common_f16(a, num_sms, st);
    case LACACHE_KV_E4M3: return launch_common_e4m3(a, num_sms, st);
    default: return launch_common_int8(a, num_sms, st);
  }
}
cudaError_t launch_own(const AttendArgs& a, int format, int num_sms, cudaStream_t st) {
  switch (format) {
    case LACACHE_KV_BF16: return launch_own_bf16(a, num_sms, st);
    case LACACHE_KV_F16: return launch_own_f16(a, num_sms, st);
    case LACACHE_KV_E4M3: return launch_own_e4m3(a, num_sms, st);
    default: return launch_own_int8(a, num_sms, st);
  }
}

}  // namespace
}  // namespace lc

extern "C" size_t lacache_kv_attend_shared_workspace_bytes(const lacache_kv_t* h, int32_t seqs, int32_t groups,
                                                           int32_t new_tokens, int32_t q_heads) {
  if (!h || seqs < 0 || groups < 0 || new_tokens < 1 || q_heads < 1) return 0;
  return lc::workspace_of(seqs, groups, new_tokens, q_heads, h->cfg.head_dim).bytes;
}

extern "C" lacache_status lacache_kv_attend_shared(lacache_kv_t* h, int32_t layer, const lacache_kv_table* table,
                                                   const lacache_attention* at, const lacache_shared* shared,
                                                   void* workspace_dev, size_t workspace_bytes, void* cuda_stream) {
  lc::NvtxRange nvtx("lacache_kv_attend_shared");
  lc::AttendArgs a = {};
  if (!at || !shared || shared->groups < 1 || (!shared->bounds_dev && shared->groups != 1)) return LACACHE_ERR_INVALID_ARG;
  const lacache_status status = lc::attend_args(h, layer, table, at->new_tokens, at->q_heads, at->window, at->dtype, at->scale,
                                                at->lengths_dev, at->starts_dev, &at->q, &a);
  if (status != LACACHE_OK || table->seqs == 0) return status;
  const lacache_kv_config& c = h->cfg;
  const lc::Workspace w = lc::workspace_of(table->seqs, shared->groups, at->new_tokens, at->q_heads, c.head_dim);
  if (!lc::device_rows(&at->out, at->dtype, &a.out) || at->out.data == at->q.data || !shared->lengths_dev || !workspace_dev ||
      !lc::aligned16(workspace_dev) || workspace_bytes < w.bytes)
    return LACACHE_ERR_INVALID_ARG;
  if ((double)table->seqs * a.rows >= 2147483648.0) return LACACHE_ERR_UNSUPPORTED;   // a group's rows are counted in 32 bits
  lc::DeviceGuard guard(c.device);
  if (!guard.ok()) return LACACHE_ERR_CUDA;
  const cudaStream_t st = (cudaStream_t)cuda_stream;
  unsigned char* ws = static_cast<unsigned char*>(workspace_dev);
  a.lse = at->lse_dev;
  a.groups = shared->groups;
  a.spans = reinterpret_cast<const int4*>(ws + w.spans);
  a.joined = reinterpret_cast<const int32_t*>(ws + w.joined);
  a.common_lse = reinterpret_cast<float*>(ws + w.lse);
  a.common = reinterpret_cast<float*>(ws + w.common);
  lc::Groups g = {};
  g.groups = shared->groups;
  g.seqs = table->seqs;
  g.new_tokens = a.new_tokens;
  g.window = a.window;
  g.max_len = a.max_len;
  g.bounds = shared->bounds_dev;
  g.common = shared->lengths_dev;
  g.lengths = a.lengths;
  g.starts = a.starts;
  g.spans = reinterpret_cast<int4*>(ws + w.spans);
  g.own_starts = reinterpret_cast<int32_t*>(ws + w.own_starts);
  g.joined = reinterpret_cast<int32_t*>(ws + w.joined);
  g.status = a.status;
  const bool eight = lc::is_quantised(c.format);
  const int64_t group_rows = (int64_t)a.rows * table->seqs / shared->groups;   // on average
  const bool common_tc = c.head_dim <= 128 && group_rows > (eight && c.head_dim <= 64 ? 32 : 16);
  const bool own_tc = lc::takes_tc(a.rows, a.group, c.head_dim, eight);
  lc::AttendArgs own = a;
  own.starts = g.own_starts;
  lc::group_kernel<<<shared->groups, lc::kGroupThreads, 0, st>>>(g);
  cudaError_t e = cudaGetLastError();
  if (e == cudaSuccess) {
    if (common_tc && h->inject_stall > 0) {
      a.inject_stall = 1;
      --h->inject_stall;
    }
    e = common_tc ? lc::launch_common_tc(a, c.format, h->num_sms, st) : lc::launch_common(a, c.format, h->num_sms, st);
  }
  if (e == cudaSuccess) e = own_tc ? lc::launch_own_tc(own, c.format, h->num_sms, st) : lc::launch_own(own, c.format, h->num_sms, st);
  return e == cudaErrorNotSupported ? LACACHE_ERR_UNSUPPORTED : lc::from_cuda(e);
}
