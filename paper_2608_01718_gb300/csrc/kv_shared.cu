// Attention for batches of sequences that have their first positions in common (a system prompt, a document), which are read and
// multiplied once for all sequences of a group. With a row's scores s_j, split at its group's common length P:
//
//   (o_1, L_1) over j < P,  (o_2, L_2) over j >= P,  L = log(e^L_1 + e^L_2),  out = e^(L_1 - L) o_1 + e^(L_2 - L) o_2,
//
// where o is a part's output and L its lse. Four kernels: what each group's rows see of the common positions, and where each
// sequence's own begin; the own part, by the kernels of kv_attend.cuh and kv_attend_tc.cu; the common part, in which a group
// stands for a sequence and the new tokens of all of its sequences are its rows, by kv_shared_tc_common.cu (or, few rows or wide
// heads, kv_attend.cuh); the join. Parts stay fp32 in the workspace. Each kernel is launched while the one before runs.
//
// 64 sequences of 1 to 700 tokens of their own behind 6,000 in common (32 heads on 8, d = 128, bf16) take 52 us: some 4 for the
// groups, 21 for the own parts (3.3 TB/s of them, as an attention of that size alone), 20 for the common part, 7.6 for the join. The
// same attention without groups reads the common positions 64 times.
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
    const int last = min(len, common);
    if (seen < last) lo = min(lo, seen), hi = max(hi, last);   // (an empty one, or one past its window, asks for no pages)
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
  // (without common positions: no rows either; none seen: [0, 0))
  if (threadIdx.x == 0) a.spans[g] = make_int4(min(s_lo, s_hi), s_hi, first, common > 0 ? end - first : 0);
}

// ---- the join ----
struct Join {
  int rows;                 // of a kv head: tokens x group
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
constexpr int kJoinWarps = 8;
constexpr double kSmall = 64e6;   // bytes of K and V

// 32 rows of a kv head a block, a row a lane; each warp four of the dimensions. The common part is one row, in
// the order of the outputs (not cut) or with four dimensions of neighbouring rows side by side, or partial sums, a block's each, in
// that order too, of which a lane loads LOADS at once.
//
// What bounds it is how many of those loads are in flight: the line of 152 blocks leaves 64 sequences of 32 heads 18 partial sums a
// row, 20 MB in all. With few blocks the registers are spent on loads (12 at once, two blocks an SM): there 7.6 us after the common
// part, 12 with six at once; with more than two blocks an SM on warps: 24 sequences of 17 tokens and 16 heads 10.2 us, 13.3 with 12.
template <int LOADS, int PER_SM>
__global__ void __launch_bounds__(kJoinWarps * 32, PER_SM) join_kernel(const __grid_constant__ Join a) {
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, D = a.head_dim, head = blockIdx.y;
  const int row = blockIdx.x * 32 + lane;                // of the kv head
  const bool mine = row < a.rows;
  const int token = mine ? row / a.group : 0, qh = head * a.group + (mine ? row - token * a.group : 0), seq = token / a.new_tokens;
  const int64_t x = (int64_t)token * a.q_heads + qh;     // in the outputs' order
  // (known before the parts are: each was launched after the groups were)
  const int g = mine ? __ldcg(a.group_of + seq) : 0;
  const int4 span = g > 0 && a.cut ? __ldcg(a.spans + g - 1) : make_int4(0, 0, 0, 0);
  asm volatile("griddepcontrol.wait;" ::: "memory");
  float l = mine ? __ldcg(a.own_lse + x) : -INFINITY;    // base 2
  // where the common part is
  int c_first = 0, c_last = 0, in_slot = 0;
  float other = -INFINITY, top = -INFINITY, sum = 0.f;
  if (g > 0 && a.cut) {
    const int share = __ldcg(a.line), longer = __ldcg(a.line + 1), base = __ldcg(a.line + 1 + g);
    const int in_group = row - span.z * a.new_tokens * a.group, tiles = (span.w * a.new_tokens * a.group + kCommonRows - 1) / kCommonRows;
    const int keys = span.y - (span.x & ~15), units = keys <= 0 ? 1 : (keys + kCommonKeys - 1) / kCommonKeys;
    const int begin = base + (head * tiles + in_group / kCommonRows) * (units + kCommonCost) + kCommonCost;
    const int in_longer = longer * (share + 1);
    auto block_of = [&](int cell) { return cell < in_longer ? cell / (share + 1) : longer + (cell - in_longer) / share; };
    c_first = block_of(begin);
    c_last = block_of(begin + units - 1);
    in_slot = in_group % kCommonRows;
  }
  const int slot = a.slot_rows * (D + 2);
  const bool parts = c_first < c_last;
  const int d = (blockIdx.z * kJoinWarps + warp) * 4, d_in = d < D ? d : 0;   // (warps past the row's end compute, and write nothing)
  const float4 y = mine ? __ldcg(reinterpret_cast<const float4*>(a.own + x * D + d_in)) : make_float4(0.f, 0.f, 0.f, 0.f);
  float4 z = make_float4(0.f, 0.f, 0.f, 0.f);
  auto add = [](float4& to, float4 v, float f) { to.x += v.x * f, to.y += v.y * f, to.z += v.z * f, to.w += v.w * f; };
  if (parts) {
    for (int c0 = c_first; c0 <= c_last; c0 += LOADS) {
      float2 ml[LOADS];
      float4 v[LOADS];
#pragma unroll
      for (int e = 0; e < LOADS; ++e) {
        const int c = min(c0 + e, c_last);
        const float* from = a.partial + (int64_t)(2 * c + (c == c_first ? 1 : 0)) * slot;   // (a block's first triple, its last)
        ml[e] = __ldcg(reinterpret_cast<const float2*>(from + D * a.slot_rows) + in_slot);
        v[e] = __ldcg(reinterpret_cast<const float4*>(from + d_in * a.slot_rows) + in_slot);
      }
      float now = top;
#pragma unroll
      for (int e = 0; e < LOADS; ++e) now = fmaxf(now, ml[e].x);
      const float to = now == -INFINITY ? 0.f : now, f = exp2_fast(top - to);
      sum *= f;
      z = make_float4(z.x * f, z.y * f, z.z * f, z.w * f);
#pragma unroll
      for (int e = 0; e < LOADS; ++e) {
        if (c0 + e > c_last) continue;
        const float w = exp2_fast(ml[e].x - to);
        sum += w * ml[e].y;
        add(z, v[e], w);
      }
      top = now;
    }
    other = sum == 0.f ? -INFINITY : top + log2f(sum);
  } else if (g > 0) {
    other = __ldcg(a.common_lse + x);
    z = a.cut ? __ldcg(reinterpret_cast<const float4*>(a.common) + ((int64_t)head * (D / 4) + d_in / 4) * a.rows + row)
              : __ldcg(reinterpret_cast<const float4*>(a.common + x * D + d_in));
  }
  if (!mine) return;
  // both: their shares of the sum of weights (NaN, where a row sees a score that is, stays)
  float4 out4 = y;
  if (g > 0) {
    const float most = fmaxf(l, other);
    if (most > -INFINITY || l != l || other != other) {
      const float own = exp2_fast(l - most), its = exp2_fast(other - most), both = own + its, f = own / both;
      out4 = make_float4(y.x * f, y.y * f, y.z * f, y.w * f);
      if (!parts || sum != 0.f) add(out4, z, parts ? its / both / sum : its / both);
      l = most + log2f(both);
    }
  }
  if (d < D)
    *reinterpret_cast<uint2*>(a.out.at(token, qh) + d * 2) =
        a.q_f16 ? make_uint2(pack2<false>(out4.x, out4.y), pack2<false>(out4.z, out4.w))
                : make_uint2(pack2<true>(out4.x, out4.y), pack2<true>(out4.z, out4.w));
  if (d == 0 && a.lse) a.lse[x] = l * 0.6931471805599453f;
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

namespace lc {
namespace {
// What the table can name at most, read for every sequence, against four kernels. us with L2 flushed, so / in parts, of 4, 16 and 64
// sequences with nine tenths in common (8 kv heads; lengths that fill the table):
//   bf16, d = 128, 4 q heads a kv head   16 MB 18 / 36, 16 / 30, 17 / 34     64 MB 25 / 56, 22 / 32, 22 / 34
//                                       128 MB 30 / 54, 28 / 36, 26 / 36    256 MB 43 / 66, 36 / 44, 36 / 42
//   bf16, d = 64, 1 q head               16 MB 18 / 30, 16 / 32, 16 / 26     64 MB 24 / 38, 22 / 36, 24 / 28
//                                       128 MB 30 / 44, 28 / 40, 28 / 30    256 MB 44 / 54, 38 / 50, 38 / 40
//   e4m3, d = 128, 4 q heads             16 MB 20 / 44, 18 / 34, 20 / 44     64 MB 28 / 63, 26 / 40, 30 / 40
//                                       128 MB 37 / 61, 36 / 46, 37 / 42    256 MB 52 / 73, 50 / 54, 54 / 54
// (what is in common is read from L2 after the first time). Parts win beyond some 250 MB: 118 / 52 with 64 sequences of 6,400 tokens,
// 984 / 150 with 128 of 30,300 over e4m3. In between this takes the slower way; lengths, which would say more than the table's width, are on the device.
bool is_small(const lacache_kv_config& c, const lacache_kv_table& t) {
  const double reach = std::min<double>((double)t.width * c.page_size, kMaxPositions);
  return 2.0 * t.seqs * reach * c.kv_heads * c.head_dim * (is_quantised(c.format) ? 1 : 2) <= kSmall;
}
}  // namespace
}  // namespace lc

extern "C" size_t lacache_kv_attend_shared_workspace_bytes(const lacache_kv_t* h, const lacache_kv_table* table, int32_t groups,
                                                           int32_t new_tokens, int32_t q_heads) {
  if (!h || !table || table->seqs < 0 || table->width < 1 || groups < 1 || new_tokens < 1 || q_heads < 1) return 0;
  const lacache_kv_config& c = h->cfg;
  if (new_tokens > lc::kMaxNewTokens || q_heads > lc::kMaxQHeads || q_heads % c.kv_heads || lc::is_small(c, *table)) return 0;
  return lc::workspace_of(table->seqs, groups, new_tokens, q_heads, c.kv_heads, c.head_dim, c.head_dim <= 128 ? h->num_sms : 0).bytes;
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
  const bool small = lc::is_small(c, *table);
  lc::Join j = {};
  if (!lc::device_rows(&at->out, at->dtype, &j.out) || at->out.data == at->q.data || !shared->lengths_dev ||
      (!small && (!workspace_dev || !lc::aligned16(workspace_dev) || workspace_bytes < w.bytes)))
    return LACACHE_ERR_INVALID_ARG;
  if ((double)table->seqs * a.rows >= 2147483648.0) return LACACHE_ERR_UNSUPPORTED;   // a group's rows are counted in 32 bits
  lc::DeviceGuard guard(c.device);
  if (!guard.ok()) return LACACHE_ERR_CUDA;
  const cudaStream_t st = (cudaStream_t)cuda_stream;
  if (small) {
    a.out = j.out;
    a.lse = at->lse_dev;
    return lc::launch_whole(h, a, st);
  }
  const bool eight = lc::is_quantised(c.format);
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
  // The common part by tcgen05 or by the warp-level kernel, by the rows of a group on average (bounds are on the device). us of the
  // call, warp-level / tcgen05, one group behind 2,000 and 30,000 common positions (8 kv heads):
  //   bf16, d = 128   20 rows 28 / 26, 59 / 55     32 rows 32 / 28, 69 / 54     64 rows 33 / 28, 90 / 54     256 rows 52 / 37, 281 / 68
  //   bf16, d = 64    20 rows 22 / 23, 39 / 44     32 rows 25 / 24, 47 / 46     64 rows 27 / 25, 60 / 46     256 rows 38 / 34, 160 / 58
  //   e4m3, d = 128   20 rows 27 / 30, 52 / 70     32 rows 33 / 31, 69 / 71     64 rows 35 / 33, 85 / 72     256 rows 51 / 43, 229 / 93
  //   e4m3, d = 64    20 rows 25 / 26, 43 / 52     32 rows 29 / 27, 52 / 53     64 rows 30 / 28, 67 / 53     256 rows 43 / 37, 193 / 68
  // Below 32 rows tcgen05 is the slower one but over bf16 at d = 128; a large group among many small ones goes by their average. (9 to
  // 16 rows take 36 and 71 over bf16 at d = 128 in tiles of 16, and 29 and 54 in two of 8, which a smaller average gives them.)
  const int64_t group_rows = (int64_t)a.rows * table->seqs / shared->groups;
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
  j.rows = table->seqs * a.rows;
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
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3((unsigned)((j.rows + 31) / 32), (unsigned)c.kv_heads, (unsigned)((c.head_dim / 4 + lc::kJoinWarps - 1) / lc::kJoinWarps));
  cfg.blockDim = dim3(lc::kJoinWarps * 32);
  cfg.stream = st;
  cudaLaunchAttribute attr;
  attr.id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr.val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = &attr;
  cfg.numAttrs = 1;
  const int64_t blocks = (int64_t)cfg.gridDim.x * cfg.gridDim.y * cfg.gridDim.z;
  return lc::from_cuda(blocks <= 2 * h->num_sms ? cudaLaunchKernelEx(&cfg, lc::join_kernel<12, 2>, j)
                                                : cudaLaunchKernelEx(&cfg, lc::join_kernel<6, 4>, j));
}
