// Eviction from the paged cache by weight: which tokens of every sequence and kv head are kept (the last `recent`, and of the
// others those of the largest weight), and their copy to other pages.
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

constexpr int kSelectThreads = 512, kSelectWarps = kSelectThreads / 32, kEach = 4;

// A block a sequence and head: the least kept weight by its digits of 8 bits, from the top, then the positions in order.
__global__ void __launch_bounds__(kSelectThreads) select_kernel(const __grid_constant__ EvictArgs a) {
  __shared__ unsigned int hist[kSelectWarps][256];
  __shared__ unsigned int s_digit, s_above;
  __shared__ unsigned int warp_equal[kSelectWarps], warp_kept[kSelectWarps];
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const int seq = blockIdx.x / a.kv_heads, head = blockIdx.x - seq * a.kv_heads;
  const Held held = held_of(a, seq);
  const int count = min(held.count(), a.keep);
  if (head == 0 && threadIdx.x == 0) {
    if (a.lengths[seq] != held.len) atomicOr(a.status, kBadIndex);
    a.new_lengths[seq] = count;
  }
  const float* w = a.weights + seq * a.w_seq + head * a.w_head;
  int32_t* kept = a.kept + (int64_t)blockIdx.x * a.keep;
  float* new_w = a.new_weights ? a.new_weights + seq * a.nw_seq + head * a.nw_head : nullptr;
  for (int i = count + threadIdx.x; i < a.keep; i += kSelectThreads) kept[i] = -1;
  if (held.count() <= a.keep) {
    for (int i = threadIdx.x; i < count; i += kSelectThreads) {
      kept[i] = held.start + i;
      if (new_w) new_w[i] = w[held.start + i];
    }
    return;
  }
  const int must = held.len - a.recent;   // positions from here on are kept in any case
  unsigned int want = a.keep - a.recent;  // of the others
  uint32_t least = 0xffffffffu;           // the least kept weight: none, if want is 0
  if (want > 0) {
    uint32_t prefix = 0;
    for (int shift = 24; shift >= 0; shift -= 8) {
      for (int i = threadIdx.x; i < kSelectWarps * 256; i += kSelectThreads) (&hist[0][0])[i] = 0;
      __syncthreads();
      for (int j = held.start + threadIdx.x; j < must; j += kSelectThreads) {
        const uint32_t x = order_of(w[j]);
        if (shift == 24 || (x >> (shift + 8)) == prefix) atomicAdd(&hist[warp][x >> shift & 255u], 1u);
      }
      __syncthreads();
      if (threadIdx.x < 256) {
        unsigned int n = 0;
        for (int i = 0; i < kSelectWarps; ++i) n += hist[i][threadIdx.x];
        hist[0][threadIdx.x] = n;
      }
      __syncthreads();
      if (warp == 0) {   // the digit that the want-th largest lies in: eight digits a lane, from the top
        unsigned int own[8], sum = 0;
#pragma unroll
        for (int i = 0; i < 8; ++i) sum += own[i] = hist[0][255 - (lane * 8 + i)];
        unsigned int upto = sum;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
          const unsigned int y = __shfl_up_sync(0xffffffffu, upto, o);
          if (lane >= o) upto += y;
        }
        unsigned int above = upto - sum;
        if (above < want && upto >= want) {
#pragma unroll
          for (int i = 0; i < 8; ++i) {
            if (above < want && above + own[i] >= want) {
              s_digit = 255 - (lane * 8 + i);
              s_above = above;
              break;
            }
            above += own[i];
          }
        }
      }
      __syncthreads();
      prefix = prefix << 8 | s_digit;
      want -= s_above;
    }
    least = prefix;   // and `want` of the weights that equal it, the earliest
  }
  // ---- positions in order ----
  unsigned int equal_before = 0, kept_before = 0;
  const bool some = a.keep > a.recent;
  for (int j0 = held.start; j0 < held.len; j0 += kSelectThreads * kEach) {
    const int j = j0 + (int)threadIdx.x * kEach;
    float x[kEach];
    bool more[kEach], equal[kEach];
    unsigned int equals = 0;
#pragma unroll
    for (int e = 0; e < kEach; ++e) {
      x[e] = j + e < held.len ? w[j + e] : 0.f;
      const uint32_t o = order_of(x[e]);
      more[e] = j + e < held.len && (j + e >= must || (some && o > least));
      equal[e] = j + e < must && some && o == least;
      equals += equal[e];
    }
    // equals before this thread's
    unsigned int upto = equals;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const unsigned int y = __shfl_up_sync(0xffffffffu, upto, o);
      if (lane >= o) upto += y;
    }
    if (lane == 31) warp_equal[warp] = upto;
    __syncthreads();
    unsigned int rank = equal_before + upto - equals, equal_all = 0;
    for (int i = 0; i < kSelectWarps; ++i) {
      if (i < warp) rank += warp_equal[i];
      equal_all += warp_equal[i];
    }
    unsigned int own = 0;
#pragma unroll
    for (int e = 0; e < kEach; ++e) {
      more[e] = more[e] || (equal[e] && rank < want);
      rank += equal[e];
      own += more[e];
    }
    upto = own;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const unsigned int y = __shfl_up_sync(0xffffffffu, upto, o);
      if (lane >= o) upto += y;
    }
    if (lane == 31) warp_kept[warp] = upto;
    __syncthreads();
    unsigned int at = kept_before + upto - own, kept_all = 0;
    for (int i = 0; i < kSelectWarps; ++i) {
      if (i < warp) at += warp_kept[i];
      kept_all += warp_kept[i];
    }
#pragma unroll
    for (int e = 0; e < kEach; ++e) {
      if (more[e]) {
        kept[at] = j + e;
        if (new_w) new_w[at] = x[e];
        ++at;
      }
    }
    equal_before += equal_all;
    kept_before += kept_all;
  }
}

// ---- their copy: 32 kept tokens a warp, whose places its lanes look up at once ----
constexpr int kCopyThreads = 128, kCopyUnroll = 4;

__global__ void __launch_bounds__(kCopyThreads) evict_copy_kernel(const __grid_constant__ EvictArgs a, int64_t tasks, int per_head) {
  const int lane = threadIdx.x & 31;
  const int pass = 32 / a.lanes, sub = lane / a.lanes, unit = lane & (a.lanes - 1);
  const int64_t step = (int64_t)gridDim.x * (kCopyThreads / 32);
  for (int64_t task = blockIdx.x * (int64_t)(kCopyThreads / 32) + (threadIdx.x >> 5); task < tasks; task += step) {
    const int64_t pair = task / per_head;
    const int i0 = (int)(task - pair * per_head) * 32, seq = (int)(pair / a.kv_heads), head = (int)(pair - (int64_t)seq * a.kv_heads);
    const int count = min(held_of(a, seq).count(), a.keep);
    if (i0 >= count) continue;
    const int n = min(count - i0, 32);
    int64_t from = -1, dst = -1;   // rows of the pool
    if (lane < n) {
      const int pos = a.kept[pair * a.keep + i0 + lane];
      from = slot_row(a.table, seq, pos, a.kv_heads, a.page_size, a.pages, a.status);
      dst = slot_row(a.to, seq, i0 + lane, a.kv_heads, a.page_size, a.pages, a.status);
      if (from < 0) dst = -1;
      from += (int64_t)head * a.page_size;
      if (dst >= 0) dst += (int64_t)head * a.page_size;
    }
    if (a.ks && dst >= 0) {
      a.ks[dst] = a.ks[from];
      a.vs[dst] = a.vs[from];
    }
    const int64_t row_bytes = (int64_t)a.units * 16;
    for (int r0 = 0; r0 < n; r0 += pass * kCopyUnroll) {
      uint4 k[kCopyUnroll], v[kCopyUnroll];
      int64_t to[kCopyUnroll];
#pragma unroll
      for (int e = 0; e < kCopyUnroll; ++e) {
        const int r = r0 + e * pass + sub;
        const int64_t f = __shfl_sync(0xffffffffu, from, r & 31);
        to[e] = __shfl_sync(0xffffffffu, dst, r & 31);
        if (r >= n || unit >= a.units) to[e] = -1;
        if (to[e] >= 0) {
          k[e] = *reinterpret_cast<const uint4*>(a.pk + f * row_bytes + unit * 16);
          v[e] = *reinterpret_cast<const uint4*>(a.pv + f * row_bytes + unit * 16);
        }
      }
#pragma unroll
      for (int e = 0; e < kCopyUnroll; ++e) {
        if (to[e] >= 0) {
          *reinterpret_cast<uint4*>(a.pk + to[e] * row_bytes + unit * 16) = k[e];
          *reinterpret_cast<uint4*>(a.pv + to[e] * row_bytes + unit * 16) = v[e];
        }
      }
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
      (new_weights && new_weights->data_dev && new_weights->width < keep))
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
  lc::select_kernel<<<(unsigned)pairs, lc::kSelectThreads, 0, st>>>(a);
  const int most = std::min(keep, a.max_len);   // (no sequence keeps more)
  const int per_head = (most + 31) / 32;
  const int64_t tasks = pairs * per_head, blocks = std::min<int64_t>((tasks + 3) / 4, 1 << 30);
  lc::evict_copy_kernel<<<(unsigned)blocks, lc::kCopyThreads, 0, st>>>(a, tasks, per_head);
  return lc::from_cuda(cudaGetLastError());
}
