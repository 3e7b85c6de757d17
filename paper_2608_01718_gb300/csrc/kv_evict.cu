// Eviction from the paged cache by weight: which tokens of every sequence and kv head are kept (the last `recent`, and of the
// others those of the largest weight), and their copy to other pages.
#include <cooperative_groups.h>

#include <algorithm>

#include "kv_attend.cuh"

namespace lc {
namespace {

struct EvictArgs {
  Table table, to;
  const int32_t* lengths;
  const int32_t* starts;
  const float* weights;
  int64_t w_seq, w_head;
  int kv_heads, keep, recent, max_len, page_size;
  int64_t pages;
  int32_t* kept;
  int32_t* new_lengths;
  float* new_weights;
  int64_t nw_seq, nw_head;
  // the copy
  int units, lanes;     // 16-byte units of a row; lanes a row (a power of two)
  unsigned char* pk;
  unsigned char* pv;
  float* ks;
  float* vs;
  unsigned int* status;
};

struct Held {
  int start, len;   // positions that are there: [start, len)
  __device__ __forceinline__ int count() const { return len - start; }
};
__device__ __forceinline__ Held held_of(const EvictArgs& a, int seq) {
  Held x;
  const int len = a.lengths[seq], start = a.starts ? a.starts[seq] : 0;
  x.len = len < 0 ? 0 : len > a.max_len ? a.max_len : len;
  x.start = start < 0 ? 0 : start > x.len ? x.len : start;
  return x;
}

// ---- which tokens ----
// A weight's order as an unsigned number: NaN below everything, -0 and 0 equal.
__device__ __forceinline__ uint32_t order_of(float w) {
  if (!(w == w)) return 0u;
  const uint32_t u = __float_as_uint(w + 0.f);
  return u & 0x80000000u ? ~u : u | 0x80000000u;
}

// Bound by instructions, some 60 for 32 weights, and by the cluster's round trips: 43 us of the 110 that 24 sequences of 3,000 to 40,000
// tokens take with 8 heads (4,096 kept); 5 of the 9.5 for one of 500 (one block a head: three digits, each a sum over all threads).
//
// A cluster of 1 to 8 blocks a sequence and head, each with an equal run of the positions, whose orders stay in shared memory.
// The least kept weight is found digit by digit (11, 11 and 10 bits, from the top): each block counts its digits, and all blocks
// read all counts through the cluster's shared memory. Of the weights that equal it the first `want` are kept: a position's
// place is the number of larger weights before it plus that of equal ones, at most `want`.
constexpr int kSelectThreads = 512, kSelectWarps = kSelectThreads / 32, kMaxCluster = 8, kDigits = 2048;

struct SelectArgs {
  EvictArgs e;
  int blocks, cached;   // a cluster's blocks; orders that a block holds in shared memory
};

__global__ void __launch_bounds__(kSelectThreads) select_kernel(const __grid_constant__ SelectArgs s) {
  namespace cg = cooperative_groups;
  cg::cluster_group cluster = cg::this_cluster();
  extern __shared__ __align__(16) uint32_t orders[];
  __shared__ __align__(16) unsigned int hist[3][kDigits];
  __shared__ unsigned int warp_sum[2][kSelectWarps], s_digit, s_above, s_own[2];   // s_own: this block's larger weights, and equal ones
  const EvictArgs& a = s.e;
  asm volatile("griddepcontrol.launch_dependents;" ::: "memory");   // (the copy starts, and waits, as soon as it has room)
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const int pair = blockIdx.x / s.blocks, rank = blockIdx.x - pair * s.blocks;
  const int seq = pair / a.kv_heads, head = pair - seq * a.kv_heads;
  const Held held = held_of(a, seq);
  const int count = min(held.count(), a.keep);
  if (head == 0 && rank == 0 && threadIdx.x == 0) {
    if (a.lengths[seq] != held.len) atomicOr(a.status, kBadIndex);
    a.new_lengths[seq] = count;
  }
  const float* w = a.weights + seq * a.w_seq + head * a.w_head;
  int32_t* kept = a.kept + (int64_t)pair * a.keep;
  const int thread = rank * kSelectThreads + threadIdx.x, threads = s.blocks * kSelectThreads;
  for (int i = count + thread; i < a.keep; i += threads) kept[i] = -1;
  if (held.count() <= a.keep) {
    for (int i = thread; i < count; i += threads) kept[i] = held.start + i;
    return;
  }
  const int must = held.len - a.recent, of_others = a.keep - a.recent;   // positions from `must` on are kept in any case
  for (int i = thread; i < a.recent; i += threads) kept[of_others + i] = must + i;
  if (of_others == 0) return;
  // this block's run of the others
  const int run = (must - held.start + s.blocks - 1) / s.blocks;
  const int first = (int)min((int64_t)held.start + (int64_t)rank * run, (int64_t)must), n = min(run, must - first);
  w += first;
  auto order_at = [&](int i) { return i < s.cached ? orders[i] : order_of(w[i]); };
  for (int i = threadIdx.x; i < 3 * kDigits / 4; i += kSelectThreads) reinterpret_cast<uint4*>(&hist[0][0])[i] = make_uint4(0, 0, 0, 0);
  if (threadIdx.x < 2) s_own[threadIdx.x] = 0;
  __syncthreads();
  constexpr int kLoads = 8;
  for (int i0 = threadIdx.x; i0 < n; i0 += kLoads * kSelectThreads) {
    float x[kLoads];
#pragma unroll
    for (int e = 0; e < kLoads; ++e) x[e] = i0 + e * kSelectThreads < n ? w[i0 + e * kSelectThreads] : 0.f;
#pragma unroll
    for (int e = 0; e < kLoads; ++e) {
      const int i = i0 + e * kSelectThreads;
      if (i >= n) break;
      const uint32_t o = order_of(x[e]);
      if (i < s.cached) orders[i] = o;
      atomicAdd(&hist[0][o >> 21], 1u);
    }
  }
  unsigned int want = of_others;
  uint32_t least = 0;
  for (int pass = 0; pass < 3; ++pass) {
    const int shift = pass == 0 ? 21 : pass == 1 ? 10 : 0, bits = pass == 2 ? 10 : 11;
    if (pass > 0) {
      auto count = [&](uint32_t o) {
        if (o >> (shift + bits) == least) atomicAdd(&hist[pass][o >> shift & ((1u << bits) - 1)], 1u);
      };
      const int whole = min(n, s.cached) / 4;
      for (int i = threadIdx.x; i < whole; i += kSelectThreads) {
        const uint4 o = reinterpret_cast<const uint4*>(orders)[i];
        count(o.x), count(o.y), count(o.z), count(o.w);
      }
      for (int i = whole * 4 + threadIdx.x; i < n; i += kSelectThreads) count(order_at(i));
    }
    cluster.sync();
    // the digit that the want-th largest lies in: four digits a thread, from the top
    const int d0 = kDigits - 4 - 4 * (int)threadIdx.x;
    uint4 sum = make_uint4(0, 0, 0, 0), x[kMaxCluster];
#pragma unroll
    for (int r = 0; r < kMaxCluster; ++r)
      if (r < s.blocks) x[r] = *reinterpret_cast<const uint4*>(cluster.map_shared_rank(&hist[pass][d0], r));
#pragma unroll
    for (int r = 0; r < kMaxCluster; ++r)
      if (r < s.blocks) sum.x += x[r].x, sum.y += x[r].y, sum.z += x[r].z, sum.w += x[r].w;
    const unsigned int mine = sum.x + sum.y + sum.z + sum.w;
    unsigned int upto = mine;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const unsigned int y = __shfl_up_sync(0xffffffffu, upto, o);
      if (lane >= o) upto += y;
    }
    if (lane == 31) warp_sum[0][warp] = upto;
    __syncthreads();
    upto += __reduce_add_sync(0xffffffffu, lane < warp ? warp_sum[0][lane] : 0u);
    unsigned int above = upto - mine;
    if (above < want && upto >= want) {
      const unsigned int c[4] = {sum.w, sum.z, sum.y, sum.x};
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        if (above < want && above + c[e] >= want) {
          s_digit = d0 + 3 - e;
          s_above = above;
          above = want;   // (done)
        } else {
          above += c[e];
        }
      }
    }
    __syncthreads();
    const unsigned int digit = s_digit;
    want -= s_above;
    least = least << bits | digit;
    // this block's share of what lies above (its own digits)
    unsigned int own = 0;
#pragma unroll
    for (int e = 0; e < 4; ++e)
      if (d0 + e > (int)digit) own += hist[pass][d0 + e];
    own = __reduce_add_sync(0xffffffffu, own);
    if (lane == 0 && own) atomicAdd(&s_own[0], own);
    if (pass == 2 && threadIdx.x == 0) s_own[1] = hist[2][digit];
    __syncthreads();
  }
  cluster.sync();
  unsigned int larger = 0, equal = 0;   // before this block's run
  for (int r = 0; r < rank; ++r) {
    const unsigned int* x = cluster.map_shared_rank(s_own, r);
    larger += x[0], equal += x[1];
  }
  cluster.sync();   // the other blocks' shared memory has been read
  // ---- positions in order: a warp a run of its own, four consecutive a lane ----
  const int each = (n + kSelectWarps * 128 - 1) / (kSelectWarps * 128) * 128;
  const int begin = min(warp * each, n), end = min(begin + each, n);
  auto four = [&](int i) {   // (0 past the run's end: counted as neither, or as what is never kept)
    if (i + 4 <= min(end, s.cached)) return *reinterpret_cast<const uint4*>(orders + i);
    return make_uint4(i < end ? order_at(i) : 0u, i + 1 < end ? order_at(i + 1) : 0u, i + 2 < end ? order_at(i + 2) : 0u,
                      i + 3 < end ? order_at(i + 3) : 0u);
  };
  auto classes = [&](uint32_t o) { return (o > least ? 1u : 0u) + (o == least ? 0x10000u : 0u); };   // larger, and equal ones above
  unsigned int own_larger = 0, own_equal = 0;
  for (int i = begin + 4 * lane; i < end; i += 128) {
    const uint4 o = four(i);
    const unsigned int mine = classes(o.x) + classes(o.y) + classes(o.z) + classes(o.w);
    own_larger += mine & 0xffffu, own_equal += mine >> 16;
  }
  own_larger = __reduce_add_sync(0xffffffffu, own_larger);
  own_equal = __reduce_add_sync(0xffffffffu, own_equal);
  if (lane == 0) warp_sum[0][warp] = own_larger, warp_sum[1][warp] = own_equal;
  __syncthreads();
  larger += __reduce_add_sync(0xffffffffu, lane < warp ? warp_sum[0][lane] : 0u);
  equal += __reduce_add_sync(0xffffffffu, lane < warp ? warp_sum[1][lane] : 0u);
  for (int i0 = begin; i0 < end; i0 += 128) {
    const int i = i0 + 4 * lane;
    const uint4 o4 = i < end ? four(i) : make_uint4(0, 0, 0, 0);
    const uint32_t o[4] = {o4.x, o4.y, o4.z, o4.w};
    const unsigned int mine = classes(o[0]) + classes(o[1]) + classes(o[2]) + classes(o[3]);
    unsigned int upto = mine;
#pragma unroll
    for (int x = 1; x < 32; x <<= 1) {
      const unsigned int y = __shfl_up_sync(0xffffffffu, upto, x);
      if (lane >= x) upto += y;
    }
    const unsigned int all = __shfl_sync(0xffffffffu, upto, 31), before = upto - mine;
    unsigned int l = larger + (before & 0xffffu), q = equal + (before >> 16);
    if (mine) {
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const bool is_larger = o[e] > least, is_equal = o[e] == least && i + e < end;
        if (is_larger || (is_equal && q < want)) kept[l + min(q, want)] = first + i + e;
        l += is_larger;
        q += is_equal;
      }
    }
    larger += all & 0xffffu;
    equal += all >> 16;
  }
}

// ---- their copy: `batch` kept tokens a warp, whose places its lanes look up at once ----
// Bound by memory, at random rows: many warps with one row of K and one of V in flight a lane group each (24 x 3,000 to 40,000 tokens
// of e4m3, d = 128, 8 heads, 4,096 kept: 66.5 us; two rows 72, four 75, eight 110, and fewer tokens a warp than 16 more too).
constexpr int kCopyThreads = 128, kCopyBlocks = 16;
constexpr int kMaxCached = 48 * 1024;   // orders in shared memory: 192 KB beside the counts

__global__ void __launch_bounds__(kCopyThreads, kCopyBlocks) evict_copy_kernel(const __grid_constant__ EvictArgs a, int64_t tasks,
                                                                               int per_head, int batch) {
  const int lane = threadIdx.x & 31;
  const int64_t task = blockIdx.x * (int64_t)(kCopyThreads / 32) + (threadIdx.x >> 5);
  asm volatile("griddepcontrol.wait;" ::: "memory");   // for the kept positions
  if (task >= tasks) return;
  const int pair = (int)(task / per_head);
  const int i0 = (int)(task - (int64_t)pair * per_head) * batch, seq = pair / a.kv_heads, head = pair - seq * a.kv_heads;
  const int n = min(a.new_lengths[seq] - i0, batch);
  if (n <= 0) return;
  int64_t from = -1, to = -1;   // rows of the pool
  if (lane < n) {
    const int i = i0 + lane, pos = a.kept[(int64_t)pair * a.keep + i];
    from = slot_row(a.table, seq, pos, a.kv_heads, a.page_size, a.pages, a.status);
    to = slot_row(a.to, seq, i, a.kv_heads, a.page_size, a.pages, a.status);
    if (a.new_weights) a.new_weights[seq * a.nw_seq + head * a.nw_head + i] = a.weights[seq * a.w_seq + head * a.w_head + pos];
    if (from < 0) to = -1;
    if (to >= 0) from += (int64_t)head * a.page_size, to += (int64_t)head * a.page_size;
    if (a.ks && to >= 0) {
      a.ks[to] = a.ks[from];
      a.vs[to] = a.vs[from];
    }
  }
  const int pass = 32 / a.lanes, sub = lane / a.lanes, unit = lane & (a.lanes - 1);
  const int64_t row_bytes = (int64_t)a.units * 16;
  for (int r0 = 0; r0 < n; r0 += pass) {
    const int r = r0 + sub;
    const int64_t f = __shfl_sync(0xffffffffu, from, r & 31), t = __shfl_sync(0xffffffffu, to, r & 31);
    if (r < n && unit < a.units && t >= 0) {
      const uint4 k = __ldcs(reinterpret_cast<const uint4*>(a.pk + f * row_bytes + unit * 16));
      const uint4 v = __ldcs(reinterpret_cast<const uint4*>(a.pv + f * row_bytes + unit * 16));
      *reinterpret_cast<uint4*>(a.pk + t * row_bytes + unit * 16) = k;
      *reinterpret_cast<uint4*>(a.pv + t * row_bytes + unit * 16) = v;
    }
  }
}

}  // namespace
}  // namespace lc

extern "C" lacache_status lacache_kv_evict(lacache_kv_t* h, int32_t layer, const lacache_kv_table* table,
                                           const int32_t* lengths_dev, const int32_t* starts_dev, const lacache_weights* weights,
                                           int32_t keep, int32_t recent, const lacache_kv_table* to, int32_t* kept_dev,
                                           int32_t* new_lengths_dev, const lacache_weights* new_weights, void* cuda_stream) {
  lc::NvtxRange nvtx("lacache_kv_evict");
  lc::EvictArgs a = {};
  lacache_kv_pool pool;
  if (lacache_kv_get_pool(h, layer, &pool) != LACACHE_OK || !lc::device_table(table, &a.table) || !lc::device_table(to, &a.to) ||
      keep < 1 || recent < 0 || recent > keep || to->seqs != table->seqs ||
      (int64_t)to->width * h->cfg.page_size < keep)
    return LACACHE_ERR_INVALID_ARG;
  if (table->seqs == 0) return LACACHE_OK;
  if (!lengths_dev || !weights || !weights->data_dev || weights->width < 1 || !kept_dev || !new_lengths_dev ||
      to->pages_dev == table->pages_dev)
    return LACACHE_ERR_INVALID_ARG;
  // (a sequence's heads read its length while another block writes what is left of it)
  const int64_t seq_bytes = (int64_t)table->seqs * 4;
  if (lc::overlap(new_lengths_dev, seq_bytes, lengths_dev, seq_bytes) || lc::overlap(new_lengths_dev, seq_bytes, starts_dev, seq_bytes))
    return LACACHE_ERR_INVALID_ARG;
  if (new_weights && new_weights->data_dev &&   // (rows of its own: tokens are copied in no order)
      (new_weights->width < keep || new_weights->data_dev == weights->data_dev || (table->seqs > 1 && new_weights->seq_stride == 0) ||
       (h->cfg.kv_heads > 1 && new_weights->head_stride == 0)))
    return LACACHE_ERR_INVALID_ARG;
  lc::DeviceGuard guard(h->cfg.device);
  if (!guard.ok()) return LACACHE_ERR_CUDA;
  const lacache_kv_config& c = h->cfg;
  a.lengths = lengths_dev;
  a.starts = starts_dev;
  a.weights = weights->data_dev;
  a.w_seq = weights->seq_stride;
  a.w_head = weights->head_stride;
  a.kv_heads = c.kv_heads;
  a.keep = keep;
  a.recent = recent;
  a.max_len = (int)std::min<int64_t>(std::min<int64_t>((int64_t)table->width * c.page_size, lc::kMaxPositions), weights->width);
  a.page_size = c.page_size;
  a.pages = c.pages;
  a.kept = kept_dev;
  a.new_lengths = new_lengths_dev;
  if (new_weights && new_weights->data_dev) {
    a.new_weights = new_weights->data_dev;
    a.nw_seq = new_weights->seq_stride;
    a.nw_head = new_weights->head_stride;
  }
  a.units = c.head_dim * (lc::is_quantised(c.format) ? 1 : 2) / 16;
  a.lanes = 1;
  while (a.lanes < a.units) a.lanes *= 2;
  a.pk = static_cast<unsigned char*>(pool.k);
  a.pv = static_cast<unsigned char*>(pool.v);
  a.ks = pool.k_scale;
  a.vs = pool.v_scale;
  a.status = h->dev_status;
  const int64_t pairs = (int64_t)table->seqs * c.kv_heads;
  if (pairs > INT32_MAX) return LACACHE_ERR_UNSUPPORTED;
  const cudaStream_t st = (cudaStream_t)cuda_stream;
  // as many blocks a pair as leave each 2,048 positions of the longest sequence, about two a SM in all; more if its orders would
  // not fit in shared memory otherwise
  lc::SelectArgs s = {a, 1, 0};
  while (s.blocks < lc::kMaxCluster &&
         ((a.max_len / (2 * s.blocks) >= 2048 && pairs * s.blocks < 2 * h->num_sms) || a.max_len / s.blocks > lc::kMaxCached))
    s.blocks *= 2;
  s.cached = std::min((a.max_len + s.blocks - 1) / s.blocks, lc::kMaxCached);
  if (pairs * s.blocks > INT32_MAX) return LACACHE_ERR_UNSUPPORTED;
  static std::atomic<bool> ready[lc::kMaxDevices];
  if (c.device >= lc::kMaxDevices || !ready[c.device].load(std::memory_order_relaxed)) {
    if (cudaFuncSetAttribute(lc::select_kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, lc::kMaxCached * 4) != cudaSuccess)
      return LACACHE_ERR_CUDA;
    if (c.device < lc::kMaxDevices) ready[c.device].store(true, std::memory_order_relaxed);
  }
  cudaLaunchAttribute attrs[1];
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3((unsigned)(pairs * s.blocks));
  cfg.blockDim = dim3(lc::kSelectThreads);
  cfg.dynamicSmemBytes = (size_t)s.cached * 4;
  cfg.stream = st;
  attrs[0].id = cudaLaunchAttributeClusterDimension;
  attrs[0].val.clusterDim.x = (unsigned)s.blocks;
  attrs[0].val.clusterDim.y = attrs[0].val.clusterDim.z = 1;
  cfg.attrs = attrs;
  cfg.numAttrs = 1;
  cudaError_t e = cudaLaunchKernelEx(&cfg, lc::select_kernel, s);
  if (e != cudaSuccess) return lc::from_cuda(e);
  const int most = std::min(keep, a.max_len);   // (no sequence keeps more)
  int batch = 32;   // (small calls: more warps)
  while (batch > 4 && pairs * ((most + batch - 1) / batch) < 32 * h->num_sms) batch /= 2;
  const int per_head = (most + batch - 1) / batch;
  const int64_t tasks = pairs * per_head, blocks = (tasks + 3) / 4;
  if (blocks > INT32_MAX) return LACACHE_ERR_UNSUPPORTED;
  cfg.gridDim = dim3((unsigned)blocks);
  cfg.blockDim = dim3(lc::kCopyThreads);
  cfg.dynamicSmemBytes = 0;
  attrs[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  // (its blocks wait beside the first kernel's; where those do not all fit at once, that costs more than it hides: 130 us for 110 at
  // 24 x 3,000 to 40,000 tokens, and 9.5 for 11.1 at one sequence of 500)
  attrs[0].val.programmaticStreamSerializationAllowed = pairs * s.blocks <= h->num_sms;
  return lc::from_cuda(cudaLaunchKernelEx(&cfg, lc::evict_copy_kernel, a, tasks, per_head, batch));
}
