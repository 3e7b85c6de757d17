// Attention for batches of sequences that have their first positions in common (a system prompt, a document), which are read and
// multiplied once for all sequences of a group. With a row's scores s_j, split at its group's common length P:
//
//   (o_1, L_1) over j < P,  (o_2, L_2) over j >= P,  L = log(e^L_1 + e^L_2),  out = e^(L_1 - L) o_1 + e^(L_2 - L) o_2,
//
// where o is a part's output and L its lse. Four kernels: what each group's rows see of the common positions, and where each
// sequence's own begin; the own part, by the kernels of kv_attend.cuh and kv_attend_tc.cu; the common part, in which a group
// stands for a sequence and the new tokens of all of its sequences are its rows, by kv_shared_tc_common.cu (or, few rows or wide
// heads, kv_attend.cuh); the join. Parts stay fp32 in the workspace. Each kernel is launched while the one before runs.
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
  int32_t* group_of;        // of a sequence, plus 1; 0: none, or nothing in common
  unsigned int* status;
};
constexpr int kGroupThreads = 128;

// A block a group. Bounds that do not rise within [0, seqs] leave no group: every sequence is then read for itself.
__global__ void __launch_bounds__(kGroupThreads) group_kernel(const __grid_constant__ Groups a) {
  asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
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
      a.group_of[s] = 0;
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
    a.group_of[s] = common > 0 ? g + 1 : 0;
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

// ---- the join: a warp a row ----
struct Join {
  int64_t rows;             // tokens x q heads
  int new_tokens, q_heads, group, head_dim, q_f16;
  int cut;                  // the common part was cut into partial sums (by kv_shared_tc_common.cu)
  int slot_rows;
  const int32_t* group_of;
  const int4* spans;
  const int* line;
  const float* own;
  const float* own_lse;
  const float* common;
  const float* common_lse;
  const float* partial;
  Rows out;
  float* lse;
};
constexpr int kJoinThreads = 128;

__device__ __forceinline__ float4 scaled(float4 x, float f) { return make_float4(x.x * f, x.y * f, x.z * f, x.w * f); }
__device__ __forceinline__ void add_scaled(float4& x, float4 y, float f) {
  x.x += y.x * f, x.y += y.y * f, x.z += y.z * f, x.w += y.w * f;
}

// WIDE: heads past 128, two values of four a lane.
template <bool WIDE>
__global__ void __launch_bounds__(kJoinThreads) join_kernel(const __grid_constant__ Join a) {
  constexpr int kValues = WIDE ? 2 : 1;
  const int lane = threadIdx.x & 31, D = a.head_dim;
  const int64_t x = blockIdx.x * (int64_t)(kJoinThreads / 32) + (threadIdx.x >> 5);
  asm volatile("griddepcontrol.wait;" ::: "memory");
  if (x >= a.rows) return;
  const int64_t token = x / a.q_heads;
  const int qh = (int)(x - token * a.q_heads), seq = (int)(token / a.new_tokens);
  const int g = __ldcg(a.group_of + seq);
  auto four = [&](const float* row, int v) {
    const int d = lane * 4 + v * 128;
    return d < D ? __ldcg(reinterpret_cast<const float4*>(row + d)) : make_float4(0.f, 0.f, 0.f, 0.f);
  };
  float4 own[kValues], common[kValues];
#pragma unroll
  for (int v = 0; v < kValues; ++v) {
    own[v] = four(a.own + x * D, v);
    common[v] = make_float4(0.f, 0.f, 0.f, 0.f);
  }
  float l = __ldcg(a.own_lse + x);   // base 2
  if (g > 0) {
    // the common part: one row, or a block's partial sums each
    float other = -INFINITY;
    int c_first = 0, c_last = 0, r = 0;
    if (a.cut) {
      const int4 span = __ldcg(a.spans + g - 1);
      const int share = __ldcg(a.line), longer = __ldcg(a.line + 1), base = __ldcg(a.line + 1 + g);
      const int row = ((int)(token - (int64_t)span.z * a.new_tokens)) * a.group + qh % a.group;
      const int tiles = (span.w * a.new_tokens * a.group + kCommonRows - 1) / kCommonRows;
      const int keys = span.y - (span.x & ~15), units = keys <= 0 ? 1 : (keys + kCommonKeys - 1) / kCommonKeys;
      const int begin = base + (qh / a.group * tiles + row / kCommonRows) * (units + kCommonCost) + kCommonCost;
      const int in_longer = longer * (share + 1);
      auto block_of = [&](int cell) { return cell < in_longer ? cell / (share + 1) : longer + (cell - in_longer) / share; };
      c_first = block_of(begin);
      c_last = block_of(begin + units - 1);
      r = row % kCommonRows;
    }
    if (c_first == c_last) {
      other = __ldcg(a.common_lse + x);
#pragma unroll
      for (int v = 0; v < kValues; ++v) common[v] = four(a.common + x * D, v);
    } else {
      const int64_t slot = (int64_t)a.slot_rows * (D + 2);
      auto part = [&](int c) { return a.partial + ((int64_t)c * 2 + (c == c_first ? 1 : 0)) * slot; };
      auto end = [&](int c) { return __ldcg(reinterpret_cast<const float2*>(part(c) + (int64_t)a.slot_rows * D) + r); };   // (m, l)
      float top = -INFINITY, sum = 0.f;
      for (int c0 = c_first; c0 <= c_last; c0 += 32) {   // (at most an SM a block)
        const float2 y = c0 + lane <= c_last ? end(c0 + lane) : make_float2(-INFINITY, 0.f);
        float most = y.x;
#pragma unroll
        for (int o = 16; o; o >>= 1) most = fmaxf(most, __shfl_xor_sync(0xffffffffu, most, o));
        const float now = fmaxf(top, most), to = now == -INFINITY ? 0.f : now, was = exp2_fast(top - to), w = exp2_fast(y.x - to);
        float add = w * y.y;
#pragma unroll
        for (int o = 16; o; o >>= 1) add += __shfl_xor_sync(0xffffffffu, add, o);
        sum = sum * was + add;
#pragma unroll
        for (int v = 0; v < kValues; ++v) common[v] = scaled(common[v], was);
        const int n = min(c_last - c0 + 1, 32);
        for (int e0 = 0; e0 < n; e0 += 8) {   // eight loads in flight
          float4 z[8][kValues];
#pragma unroll
          for (int e = 0; e < 8; ++e) {
#pragma unroll
            for (int v = 0; v < kValues; ++v)
              z[e][v] = e0 + e < n ? four(part(c0 + e0 + e) + (int64_t)r * D, v) : make_float4(0.f, 0.f, 0.f, 0.f);
          }
#pragma unroll
          for (int e = 0; e < 8; ++e) {
            const float f = __shfl_sync(0xffffffffu, w, (e0 + e) & 31);
            if (e0 + e < n) {
#pragma unroll
              for (int v = 0; v < kValues; ++v) add_scaled(common[v], z[e][v], f);
            }
          }
        }
        top = now;
      }
      other = sum == 0.f ? -INFINITY : top + log2f(sum);
#pragma unroll
      for (int v = 0; v < kValues; ++v)
        common[v] = sum == 0.f ? make_float4(0.f, 0.f, 0.f, 0.f) : scaled(common[v], 1.f / sum);
    }
    // both: their shares of the sum of weights (NaN, where a row sees a score that is, stays)
    const float most = fmaxf(l, other);
    if (most > -INFINITY || l != l || other != other) {
      const float mine = exp2_fast(l - most), its = exp2_fast(other - most), both = mine + its;
#pragma unroll
      for (int v = 0; v < kValues; ++v) {
        own[v] = scaled(own[v], mine / both);
        add_scaled(own[v], common[v], its / both);
      }
      l = most + log2f(both);
    }
  }
  unsigned char* out = a.out.at(token, qh);
#pragma unroll
  for (int v = 0; v < kValues; ++v) {
    const int d = lane * 4 + v * 128;
    if (d < D)
      *reinterpret_cast<uint2*>(out + d * 2) = a.q_f16 ? make_uint2(pack2<false>(own[v].x, own[v].y), pack2<false>(own[v].z, own[v].w))
                                                       : make_uint2(pack2<true>(own[v].x, own[v].y), pack2<true>(own[v].z, own[v].w));
  }
  if (lane == 0 && a.lse) a.lse[x] = l * 0.6931471805599453f;
}

struct Workspace {
  size_t spans, line, own_starts, group_of, own_lse, common_lse, own, common, partial, bytes;   // offsets
  int slot_rows;
};
inline size_t round16(size_t n) { return (n + 15) / 16 * 16; }
// `blocks`: of the common part's kernel on tcgen05 (0: not for these heads).
Workspace workspace_of(int64_t seqs, int groups, int new_tokens, int q_heads, int kv_heads, int head_dim, int blocks) {
  Workspace w;
  const size_t rows = (size_t)seqs * new_tokens * q_heads;
  const size_t group_rows = (rows / kv_heads + 15) / 16 * 16;   // (a group's rows a kv head, at most)
  w.slot_rows = (int)std::min<size_t>(group_rows, kCommonRows);
  w.spans = 0;
  w.line = (size_t)groups * sizeof(int4);
  w.own_starts = w.line + round16((size_t)(groups + 2) * 4);
  w.group_of = w.own_starts + round16((size_t)seqs * 4);
  w.own_lse = w.group_of + round16((size_t)seqs * 4);
  w.common_lse = w.own_lse + round16(rows * 4);
  w.own = w.common_lse + round16(rows * 4);
  w.common = w.own + rows * head_dim * 4;
  w.partial = w.common + rows * head_dim * 4;
  w.bytes = w.partial + (size_t)blocks * 2 * w.slot_rows * (head_dim + 2) * 4;
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
  const lacache_kv_config& c = h->cfg;
  return lc::workspace_of(seqs, groups, new_tokens, q_heads, c.kv_heads, c.head_dim, c.head_dim <= 128 ? h->num_sms : 0).bytes;
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
  const lc::Workspace w = lc::workspace_of(table->seqs, shared->groups, at->new_tokens, at->q_heads, c.kv_heads, c.head_dim,
                                           c.head_dim <= 128 ? h->num_sms : 0);
  lc::Join j = {};
  if (!lc::device_rows(&at->out, at->dtype, &j.out) || at->out.data == at->q.data || !shared->lengths_dev || !workspace_dev ||
      !lc::aligned16(workspace_dev) || workspace_bytes < w.bytes)
    return LACACHE_ERR_INVALID_ARG;
  if ((double)table->seqs * a.rows >= 2147483648.0) return LACACHE_ERR_UNSUPPORTED;   // a group's rows are counted in 32 bits
  lc::DeviceGuard guard(c.device);
  if (!guard.ok()) return LACACHE_ERR_CUDA;
  const cudaStream_t st = (cudaStream_t)cuda_stream;
  unsigned char* ws = static_cast<unsigned char*>(workspace_dev);
  auto floats = [&](size_t at_byte) { return reinterpret_cast<float*>(ws + at_byte); };
  auto ints = [&](size_t at_byte) { return reinterpret_cast<int32_t*>(ws + at_byte); };
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
  g.own_starts = ints(w.own_starts);
  g.group_of = ints(w.group_of);
  g.status = a.status;
  lc::group_kernel<<<shared->groups, lc::kGroupThreads, 0, st>>>(g);
  cudaError_t e = cudaGetLastError();
  const bool eight = lc::is_quantised(c.format);
  // the sequences' own positions
  lc::AttendArgs own = a;
  own.starts = g.own_starts;
  own.part = floats(w.own);
  own.part_lse = floats(w.own_lse);
  if (e == cudaSuccess)
    e = lc::takes_tc(a.rows, a.group, c.head_dim, eight) ? lc::launch_own_tc(own, c.format, h->num_sms, st)
                                                         : lc::launch_own(own, c.format, h->num_sms, st);
  // the common ones
  a.groups = shared->groups;
  a.spans = g.spans;
  a.line = ints(w.line);
  a.slot_rows = w.slot_rows;
  a.part = floats(w.common);
  a.part_lse = floats(w.common_lse);
  const int64_t group_rows = (int64_t)a.rows * table->seqs / shared->groups;   // on average
  const bool cut = c.head_dim <= 128 && group_rows > 16;
  if (e == cudaSuccess && cut) {
    a.partial = floats(w.partial);
    if (h->inject_stall > 0) {
      a.inject_stall = 1;
      --h->inject_stall;
    }
    e = lc::launch_common_tc(a, c.format, h->num_sms, st);
  } else if (e == cudaSuccess) {
    e = lc::launch_common(a, c.format, h->num_sms, st);
  }
  if (e != cudaSuccess) return e == cudaErrorNotSupported ? LACACHE_ERR_UNSUPPORTED : LACACHE_ERR_CUDA;
  j.rows = (int64_t)table->seqs * a.new_tokens * a.q_heads;
  j.new_tokens = a.new_tokens;
  j.q_heads = a.q_heads;
  j.group = a.group;
  j.head_dim = c.head_dim;
  j.q_f16 = a.q_f16;
  j.cut = cut;
  j.slot_rows = w.slot_rows;
  j.group_of = g.group_of;
  j.spans = g.spans;
  j.line = a.line;
  j.own = own.part;
  j.own_lse = own.part_lse;
  j.common = a.part;
  j.common_lse = a.part_lse;
  j.partial = a.partial;
  j.lse = at->lse_dev;
  const int64_t blocks = (j.rows + lc::kJoinThreads / 32 - 1) / (lc::kJoinThreads / 32);
  if (blocks > INT32_MAX) return LACACHE_ERR_UNSUPPORTED;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3((unsigned)blocks);
  cfg.blockDim = dim3(lc::kJoinThreads);
  cfg.stream = st;
  cudaLaunchAttribute attr;
  attr.id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr.val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = &attr;
  cfg.numAttrs = 1;
  return lc::from_cuda(cudaLaunchKernelEx(&cfg, c.head_dim > 128 ? lc::join_kernel<true> : lc::join_kernel<false>, j));
}
