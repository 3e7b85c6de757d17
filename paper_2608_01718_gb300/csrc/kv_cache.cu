// The paged key-value cache: the handle, the write of new tokens (rotation, quantisation and placement in one pass), and
// reading cached tokens back.
//
// Both kernels are bound by memory: every input row is read once and every cached row written once (or the reverse). For each
// of its tokens a warp finds the place and the angles once, and runs over the rows.
//
// Measured (bf16 rows, 32 q heads, 8 of k and v, d = 128): 12,001 tokens written to an e4m3 cache, half of each head rotated,
// interleaved, 52 us, 5.2 TB/s; all rotated, in the half layout 57 and interleaved 54; the same to an int8 cache; to a bf16 cache
// 54 (half layout, all rotated), 5.4 TB/s. A loop for q's rows of its own is 6% faster for the e4m3 cache than one for all rows
// (3% slower for the bf16 one). Of 16-bit rows, the rotated kernels of whole chunks spill 36 to 48 bytes a thread (half layout)
// and 16 to 20 (interleaved) at the cap of 96 registers; with four rows in flight instead of two 150 to 580. 60,000 tokens of
// int8 read as f16: 64 us, 5.9 TB/s. Of 32 tokens written and 333 read: 4.3 and 2.9 us, a launch and two dependent loads.
#include <new>
#include <type_traits>

#include "kv_attend.cuh"

namespace lc {
namespace {

// Blocks an SM (append_kernel's angles and quotients take more registers: at 6 and 7 it is 17 to 23% slower).
constexpr int kAppendBlocks = 5, kReadBlocks = 8;

struct AppendArgs {
  RowPlan plan;
  const int32_t* seq;
  const int32_t* pos;
  const int32_t* rope_pos;
  Table table;
  int q_heads, kv_heads, chunks, lanes, page_size;
  int64_t head_bytes;   // a head's rows of a page
  int64_t pages;
  Rows k, v, q, q_out;
  unsigned char* pk;
  unsigned char* pv;
  float* ks;
  float* vs;
  unsigned int* status;
};

// The place of cached row `row`, in bytes from the pool's start.
template <int FMT>
__device__ __forceinline__ int64_t cached_at(int64_t row, int chunks) {
  return row * chunks * (FMT == LACACHE_KV_E4M3 || FMT == LACACHE_KV_INT8 ? 8 : 16);
}

// A token's rows: q, then k, then v. The tokens' places are looked up by the warp's lanes at once.
template <typename T, int FMT, int MODE>
__global__ void __launch_bounds__(kRowThreads, kAppendBlocks)
    append_kernel(const __grid_constant__ lacache_rope rope, const __grid_constant__ AppendArgs a) {
  using Stored = typename std::conditional<FMT == LACACHE_KV_F16, __half, __nv_bfloat16>::type;
  constexpr bool kEight = FMT == LACACHE_KV_E4M3 || FMT == LACACHE_KV_INT8;
  __shared__ float2 cs[kRowThreads / 32][kMaxHeadDim / 2];
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const int pass = 32 / a.lanes, sub = lane / a.lanes, kv = a.q_heads + a.kv_heads;
  const Chunks m = chunks_of<MODE>(lane & (a.lanes - 1), a.chunks, rope.rot_dim);
  const int64_t step = (int64_t)gridDim.x * (kRowThreads / 32);
  for (int64_t task = blockIdx.x * (int64_t)(kRowThreads / 32) + warp; task < a.plan.tasks; task += step) {
    const int64_t first_token = task / a.plan.slabs * a.plan.group;
    const int first = (int)(task % a.plan.slabs) * a.plan.slab;
    const int end = first + a.plan.slab < a.plan.rows ? first + a.plan.slab : a.plan.rows;
    const int tokens = a.plan.n - first_token < a.plan.group ? (int)(a.plan.n - first_token) : a.plan.group;
    int64_t own_place = -1;
    int own_pos = 0;
    if (lane < tokens) {
      const int64_t t = first_token + lane;
      if (MODE != kRopeNone) own_pos = a.rope_pos[t];
      own_place = slot_row(a.table, a.seq[t], a.pos[t], a.kv_heads, a.page_size, a.pages, a.status);
    }
    for (int g = 0; g < tokens; ++g) {
      const int64_t t = first_token + g, place = __shfl_sync(0xffffffffu, own_place, g);
      if (place < 0) continue;
      float2 angle[8];
      if (MODE != kRopeNone) warp_angles<MODE>(rope, __shfl_sync(0xffffffffu, own_pos, g), 1.f, m, cs[warp], angle);
      // q's rows: rotated
      const int q_end = end < a.q_heads ? end : a.q_heads;
      const unsigned char* from_q = a.q.at(t, first + sub);
      unsigned char* to_q = a.q_out.at(t, first + sub);
      const int64_t q_step = (int64_t)pass * a.q.head16 * 16, out_step = (int64_t)pass * a.q_out.head16 * 16;
      for (int r = first + sub; r - sub < q_end; r += kRowUnroll * pass, from_q += kRowUnroll * q_step, to_q += kRowUnroll * out_step) {
        typename Chunk<T>::raw raw[kRowUnroll][2];
#pragma unroll
        for (int i = 0; i < kRowUnroll; ++i) {
#pragma unroll
          for (int k = 0; k < 2; ++k)
            if (r + i * pass < q_end && m.live[k]) raw[i][k] = Chunk<T>::load(from_q + i * q_step + m.c[k] * (8 * (int)sizeof(T)));
        }
#pragma unroll
        for (int i = 0; i < kRowUnroll; ++i) {
          const bool live = r + i * pass < q_end;
          float x0[8], x1[8];
          Chunk<T>::widen(raw[i][0], x0);
          Chunk<T>::widen(raw[i][1], x1);
          if (MODE != kRopeNone)
            rotate<MODE>(x0, x1, m, rope.rot_dim, rope.layout, angle, cs[warp],
                         live ? reinterpret_cast<const T*>(from_q + i * q_step) : nullptr);
          if (MODE == kRopeOdd) __syncwarp();
          T* to = reinterpret_cast<T*>(to_q + i * out_step);
          if (live && m.live[0]) store8(to + m.c[0] * 8, x0);
          if (live && m.live[1]) store8(to + m.c[1] * 8, x1);
        }
      }
      // k's and v's: k rotated, both in the cache's format; where row r would lie if k and v each began at row 0
      const unsigned char* from_k = a.k.at(t, -a.q_heads);
      const unsigned char* from_v = a.v.at(t, -kv);
      const int64_t at_k = cached_at<FMT>(place, a.chunks);
      for (int r0 = first > a.q_heads ? first : a.q_heads; r0 < end; r0 += kRowUnroll * pass) {
        typename Chunk<T>::raw raw[kRowUnroll][2];
        const unsigned char* src[kRowUnroll];
#pragma unroll
        for (int i = 0; i < kRowUnroll; ++i) {
          const int r = r0 + i * pass + sub;
          src[i] = (r < kv ? from_k : from_v) + (int64_t)r * (r < kv ? a.k.head16 : a.v.head16) * 16;
#pragma unroll
          for (int k = 0; k < 2; ++k) {
            raw[i][k] = {};
            if (r < end && m.live[k]) raw[i][k] = Chunk<T>::load(src[i] + m.c[k] * (8 * (int)sizeof(T)));
          }
        }
#pragma unroll
        for (int i = 0; i < kRowUnroll; ++i) {
          const int at = r0 + i * pass, r = at + sub;
          if (at >= end) break;
          float x0[8], x1[8];
          Chunk<T>::widen(raw[i][0], x0);
          Chunk<T>::widen(raw[i][1], x1);
          if (MODE != kRopeNone && r < kv)
            rotate<MODE>(x0, x1, m, rope.rot_dim, rope.layout, angle, cs[warp],
                         r < end ? reinterpret_cast<const T*>(src[i]) : nullptr);
          const bool live[2] = {r < end && m.live[0], r < end && m.live[1]}, is_v = r >= kv;
          const int h = is_v ? r - kv : r - a.q_heads;
          unsigned char* to = (is_v ? a.pv : a.pk) + at_k + h * a.head_bytes;
          if constexpr (kEight) {
            const float scale = row_scale<FMT>(x0, x1, a.lanes), inv = __frcp_rn(scale);
            if (live[0]) reinterpret_cast<uint2*>(to)[m.c[0]] = quantise8<FMT>(x0, scale, inv);
            if (live[1]) reinterpret_cast<uint2*>(to)[m.c[1]] = quantise8<FMT>(x1, scale, inv);
            if (live[0] && m.c[0] == 0) (is_v ? a.vs : a.ks)[place + (int64_t)h * a.page_size] = scale;
          } else {
            if (live[0]) store8(reinterpret_cast<Stored*>(to) + m.c[0] * 8, x0);
            if (live[1]) store8(reinterpret_cast<Stored*>(to) + m.c[1] * 8, x1);
          }
        }
      }
    }
  }
}

struct ReadArgs {
  RowPlan plan;
  const int32_t* seq;
  const int32_t* pos;
  Table table;
  int kv_heads, chunks, lanes, page_size;
  int64_t pages;
  Rows k, v;   // p == nullptr: not wanted
  const unsigned char* pk;
  const unsigned char* pv;
  const float* ks;
  const float* vs;
  unsigned int* status;
};

// A token's rows: k, then v.
template <typename T, int FMT>
__global__ void __launch_bounds__(kRowThreads, kReadBlocks) read_kernel(const __grid_constant__ ReadArgs a) {
  using Stored = typename std::conditional<FMT == LACACHE_KV_F16, __half, __nv_bfloat16>::type;
  constexpr bool kEight = FMT == LACACHE_KV_E4M3 || FMT == LACACHE_KV_INT8;
  using Raw = typename std::conditional<kEight, uint2, uint4>::type;
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const int pass = 32 / a.lanes, sub = lane / a.lanes;
  const Chunks m = chunks_of<kRopeNone>(lane & (a.lanes - 1), a.chunks, 0);
  const int64_t step = (int64_t)gridDim.x * (kRowThreads / 32);
  for (int64_t task = blockIdx.x * (int64_t)(kRowThreads / 32) + warp; task < a.plan.tasks; task += step) {
    const int64_t first_token = task / a.plan.slabs * a.plan.group;
    const int first = (int)(task % a.plan.slabs) * a.plan.slab;
    const int end = first + a.plan.slab < a.plan.rows ? first + a.plan.slab : a.plan.rows;
    const int tokens = a.plan.n - first_token < a.plan.group ? (int)(a.plan.n - first_token) : a.plan.group;
    int64_t own_place = -1;
    if (lane < tokens)
      own_place = slot_row(a.table, a.seq[first_token + lane], a.pos[first_token + lane], a.kv_heads, a.page_size, a.pages,
                           a.status);
    for (int g = 0; g < tokens; ++g) {
      const int64_t t = first_token + g, place = __shfl_sync(0xffffffffu, own_place, g);
      if (place < 0) continue;
      for (int r0 = first; r0 < end; r0 += kRowUnroll * pass) {
        Raw raw[kRowUnroll][2];
        float scale[kRowUnroll];
#pragma unroll
        for (int i = 0; i < kRowUnroll; ++i) {
          const int r = r0 + i * pass + sub;
          const bool is_v = r >= a.kv_heads;
          if (r >= end || !m.live[0] || !(is_v ? a.v.p : a.k.p)) continue;
          const int64_t at = place + (int64_t)(is_v ? r - a.kv_heads : r) * a.page_size;
          const Raw* from = reinterpret_cast<const Raw*>((is_v ? a.pv : a.pk) + cached_at<FMT>(at, a.chunks));
          raw[i][0] = from[m.c[0]];
          if (m.live[1]) raw[i][1] = from[m.c[1]];
          if constexpr (kEight) scale[i] = (is_v ? a.vs : a.ks)[at];
        }
#pragma unroll
        for (int i = 0; i < kRowUnroll; ++i) {
          const int r = r0 + i * pass + sub;
          const bool is_v = r >= a.kv_heads;
          if (r >= end || !(is_v ? a.v.p : a.k.p)) continue;
          T* to = reinterpret_cast<T*>(is_v ? a.v.at(t, r - a.kv_heads) : a.k.at(t, r));
#pragma unroll
          for (int k = 0; k < 2; ++k) {
            if (!m.live[k]) continue;
            float x[8];
            if constexpr (kEight) dequantise8<FMT>(raw[i][k], scale[i], x);
            else widen8(raw[i][k], x, Stored());
            store8(to + m.c[k] * 8, x);
          }
        }
      }
    }
  }
}

template <typename T, int FMT>
void launch_append_mode(int mode, const lacache_rope& rope, const AppendArgs& a, unsigned grid, cudaStream_t st) {
  auto* kernel = mode == kRopeNone   ? append_kernel<T, FMT, kRopeNone>
                 : mode == kRopeHalf ? append_kernel<T, FMT, kRopeHalf>
                 : mode == kRopeNear ? append_kernel<T, FMT, kRopeNear>
                                     : append_kernel<T, FMT, kRopeOdd>;
  kernel<<<grid, kRowThreads, 0, st>>>(rope, a);
}
template <typename T>
void launch_append(int format, int mode, const lacache_rope& rope, const AppendArgs& a, unsigned grid, cudaStream_t st) {
  switch (format) {
    case LACACHE_KV_BF16: launch_append_mode<T, LACACHE_KV_BF16>(mode, rope, a, grid, st); break;
    case LACACHE_KV_F16: launch_append_mode<T, LACACHE_KV_F16>(mode, rope, a, grid, st); break;
    case LACACHE_KV_E4M3: launch_append_mode<T, LACACHE_KV_E4M3>(mode, rope, a, grid, st); break;
    default: launch_append_mode<T, LACACHE_KV_INT8>(mode, rope, a, grid, st); break;
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
  if (q && q_heads > lc::kMaxRowHeads) return LACACHE_ERR_UNSUPPORTED;
  if (n == 0) return LACACHE_OK;
  if (!seq_dev || !pos_dev || !lc::device_rows(k, dtype, &a.k) || !lc::device_rows(v, dtype, &a.v))
    return LACACHE_ERR_INVALID_ARG;
  if (q && (q_heads < 1 || !lc::device_rows(q, dtype, &a.q) || !lc::device_rows(q_out, dtype, &a.q_out)))
    return LACACHE_ERR_INVALID_ARG;
  lc::DeviceGuard guard(h->cfg.device);
  if (!guard.ok()) return LACACHE_ERR_CUDA;
  a.seq = seq_dev;
  a.pos = pos_dev;
  a.rope_pos = rope_pos_dev ? rope_pos_dev : pos_dev;
  a.q_heads = q ? q_heads : 0;
  a.kv_heads = h->cfg.kv_heads;
  a.chunks = h->cfg.head_dim / 8;
  a.page_size = h->cfg.page_size;
  a.pages = h->cfg.pages;
  a.head_bytes = (int64_t)h->cfg.page_size * h->cfg.head_dim * (lc::is_quantised(h->cfg.format) ? 1 : 2);
  const int mode = lc::rope_mode(rope);
  a.lanes = lc::lanes_for(h->cfg.head_dim, rope ? rope->rot_dim : 0, mode);
  a.pk = static_cast<unsigned char*>(pool.k);
  a.pv = static_cast<unsigned char*>(pool.v);
  a.ks = pool.k_scale;
  a.vs = pool.v_scale;
  a.status = h->dev_status;
  static const lacache_rope none = {};
  const lacache_rope& plan = rope ? *rope : none;
  unsigned grid;
  a.plan = lc::plan_rows(n, a.q_heads + 2 * a.kv_heads, a.lanes, lc::kAppendBlocks, lc::kRowGroup, &grid);
  const cudaStream_t st = (cudaStream_t)cuda_stream;
  if (dtype == LACACHE_BF16) lc::launch_append<__nv_bfloat16>(h->cfg.format, mode, plan, a, grid, st);
  else if (dtype == LACACHE_F16) lc::launch_append<__half>(h->cfg.format, mode, plan, a, grid, st);
  else lc::launch_append<float>(h->cfg.format, mode, plan, a, grid, st);
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
  a.seq = seq_dev;
  a.pos = pos_dev;
  a.kv_heads = h->cfg.kv_heads;
  a.chunks = h->cfg.head_dim / 8;
  a.lanes = lc::lanes_for(h->cfg.head_dim, 0, lc::kRopeNone);
  a.page_size = h->cfg.page_size;
  a.pages = h->cfg.pages;
  a.pk = static_cast<unsigned char*>(pool.k);
  a.pv = static_cast<unsigned char*>(pool.v);
  a.ks = pool.k_scale;
  a.vs = pool.v_scale;
  a.status = h->dev_status;
  unsigned grid;
  a.plan = lc::plan_rows(n, 2 * a.kv_heads, a.lanes, lc::kReadBlocks, lc::kRowGroup, &grid);
  const cudaStream_t st = (cudaStream_t)cuda_stream;
  if (dtype == LACACHE_BF16) lc::launch_read<__nv_bfloat16>(h->cfg.format, a, grid, st);
  else if (dtype == LACACHE_F16) lc::launch_read<__half>(h->cfg.format, a, grid, st);
  else lc::launch_read<float>(h->cfg.format, a, grid, st);
  return lc::from_cuda(cudaGetLastError());
}

extern "C" lacache_status lacache_kv_inject_stall(lacache_kv_t* h, int32_t attends) {
  if (!h || attends < 0) return LACACHE_ERR_INVALID_ARG;
  h->inject_stall = attends;
  return LACACHE_OK;
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
  return word & lc::kAttendTimeout ? LACACHE_ERR_DEVICE_TIMEOUT : LACACHE_ERR_INVALID_ARG;
}
