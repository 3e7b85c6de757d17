// The attention weight that cached tokens get from new ones, added to what they got before:
//
//   w_j <- decay w_j + sum over the rows r that see j of e^(s_rj - lse_r),   s_rj = scale <q_r, k_j>
//
// for every kv head, over the rows that share it (its group of q heads times the new tokens), from the lse that the attention of
// the same rows wrote. K is read once. Each key belongs to one warp, which adds its rows in order: no atomics, no joins.
//
// Products are the warp-level tensor instruction's, S^T [16 keys x 8 rows] = K Q^T, with the naming of a row's dimensions chosen
// so that a lane's share of K is 16 contiguous bytes (as in kv_attend.cuh). K goes from memory straight into the registers that
// the products read, 64 contiguous bytes of each row an instruction, and stays there for all rows, whose q is staged in shared
// memory, kChunk rows at a time. 8-bit codes are widened to f16 exactly; q of bf16 over an 8-bit cache is scaled to f16 by a power of
// two a row (exact for elements within 2^-14 of the row's largest). Scores, weights and sums are fp32.
#include <algorithm>

#include "kv_attend.cuh"

namespace lc {
namespace {

struct WeighArgs {
  AttendArgs a;   // (lse is read; out, the partial sums and the counters are not used)
  float decay;
  const float* past;
  int64_t past_seq, past_head;
  float* out;
  int64_t out_seq, out_head;
};

constexpr int kWeighWarps = 8, kWeighThreads = kWeighWarps * 32;
constexpr int kChunk = 64;   // rows of q staged at a time

template <int FMT, int DP>
struct WeighConfig {
  static constexpr bool kEight = FMT == LACACHE_KV_E4M3 || FMT == LACACHE_KV_INT8;
  static constexpr int kTiles = DP <= 128 ? 2 : 1;             // tiles of 16 keys a warp: 64 registers of operands
  static constexpr int kKeys = 16 * kTiles;
  static constexpr int kUnit = kWeighWarps * kKeys;
  static constexpr int kPieces = DP * (kEight ? 1 : 2) / 64;   // of a lane, 16 bytes each, in a row of K
  static constexpr int kSteps = DP / 16;
  static constexpr int kQStride = DP * 2 + (kEight ? 16 : 64); // of a row of q: what eight lanes read lies in eight bank groups
};

__device__ __forceinline__ int weigh_length(const AttendArgs& a, int seq) {
  const int len = a.lengths[seq];
  return len < 0 ? 0 : len > a.max_len ? a.max_len : len;
}

template <int FMT, int DP>
__global__ void __launch_bounds__(kWeighThreads, 2) weigh_kernel(const __grid_constant__ WeighArgs w) {
  using C = WeighConfig<FMT, DP>;
  constexpr bool kBf16 = FMT == LACACHE_KV_BF16;
  const AttendArgs& a = w.a;
  __shared__ __align__(16) unsigned char q_smem[kChunk * C::kQStride];
  __shared__ __align__(8) float row_lse[kChunk], row_factor[kChunk];   // lse log2(e), and scale log2(e) times what q was divided by
  __shared__ int row_pos[kChunk], row_lo[kChunk];                      // a row's last and first visible position
  __shared__ int4 tile_span[kChunk / 8];                               // of eight rows: least and largest last, least and largest first
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, g = lane >> 2, t = lane & 3;
  const int D = a.head_dim, row_bytes = D * (C::kEight ? 1 : 2);

  // ---- this block's part of the line of units: sequences, their heads, their keys ----
  int total = 0;
  for (int s = lane; s < a.table.seqs; s += 32) total += (weigh_length(a, s) + C::kUnit - 1) / C::kUnit;
  total = __reduce_add_sync(0xffffffffu, total) * a.kv_heads;
  const int share = total / gridDim.x, longer = total - share * gridDim.x, block = blockIdx.x;
  int left = share + (block < longer ? 1 : 0);
  const int u = block * share + min(block, longer);
  if (threadIdx.x == 0) {
    for (int s = block; s < a.table.seqs; s += gridDim.x)
      if (a.lengths[s] < 0 || a.lengths[s] > a.max_len) atomicOr(a.status, kBadIndex);
  }
  if (left == 0) return;
  int seq = 0, seq_base = 0;
  for (int s0 = 0; s0 < a.table.seqs; s0 += 32) {
    const int own = s0 + lane < a.table.seqs ? (weigh_length(a, s0 + lane) + C::kUnit - 1) / C::kUnit * a.kv_heads : 0;
    int upto = own;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const int y = __shfl_up_sync(0xffffffffu, upto, o);
      if (lane >= o) upto += y;
    }
    const unsigned past = __ballot_sync(0xffffffffu, seq_base + upto > u);
    if (past) {
      const int l0 = __ffs(past) - 1;
      seq = s0 + l0;
      seq_base += __shfl_sync(0xffffffffu, upto - own, l0);
      break;
    }
    seq_base += __shfl_sync(0xffffffffu, upto, 31);
  }
  int len = weigh_length(a, seq), units = (len + C::kUnit - 1) / C::kUnit;
  int head = (u - seq_base) / units, unit = (u - seq_base) - head * units;

  // q of rows [row0, row0 + kChunk) of this sequence and head; by the whole block, between barriers
  auto stage = [&](int row0) {
#pragma unroll 1
    for (int r = warp; r < kChunk; r += kWeighWarps) {
      const int row = row0 + r, d0 = lane * 8;
      const bool live = row < a.rows;
      if (!live && row - r % 8 >= a.rows) break;   // a tile without a row is not looked at
      const int tok = live ? row / a.group : 0, qh = head * a.group + row - tok * a.group;
      const int64_t token = (int64_t)seq * a.new_tokens + tok;
      uint4 raw = make_uint4(0, 0, 0, 0);
      if (live && d0 < D) raw = *reinterpret_cast<const uint4*>(a.q.at(token, qh) + d0 * 2);
      float back = 1.f;
      if (C::kEight && !a.q_f16) {
        float x[8], top = 0.f;
        widen8(raw, x, __nv_bfloat16());
#pragma unroll
        for (int i = 0; i < 8; ++i) top = fmaxf(top, fabsf(x[i]));
#pragma unroll
        for (int o = 16; o; o >>= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, o));
        // the power of two below top (1 for zeros, infinities and subnormals)
        uint32_t e = __float_as_uint(top) & 0x7f800000u;
        if (e != 0 && e != 0x7f800000u) {
          e = e < 0x7e800000u ? e : 0x7e800000u;
          back = __uint_as_float(e);
          const float down = __uint_as_float(0x7f000000u - e);
#pragma unroll
          for (int i = 0; i < 8; ++i) x[i] *= down;
        }
        raw = pack8(x, __half());
      }
      if (d0 < DP) *reinterpret_cast<uint4*>(q_smem + r * C::kQStride + d0 * 2) = raw;
      if (lane == 0) {
        const float lse = live ? w.a.lse[token * a.q_heads + qh] : -INFINITY;
        int p = live ? len - a.new_tokens + tok : -1, lo = a.starts ? a.starts[seq] : 0;
        if (a.window > 0 && p - a.window + 1 > lo) lo = p - a.window + 1;
        if (lse == -INFINITY) p = -1;   // a row that sees nothing (and those past the last)
        row_lse[r] = lse * 1.4426950408889634f;
        row_factor[r] = a.scale * 1.4426950408889634f * back;
        row_pos[r] = p;
        row_lo[r] = lo;
      }
    }
    __syncthreads();
    if (threadIdx.x < kChunk / 8 && row0 + (int)threadIdx.x * 8 < a.rows) {
      int4 x = make_int4(INT_MAX, -1, INT_MAX, INT_MIN);
      for (int r = threadIdx.x * 8; r < (int)threadIdx.x * 8 + 8; ++r) {
        x.x = min(x.x, row_pos[r]), x.y = max(x.y, row_pos[r]);
        x.z = min(x.z, row_lo[r]), x.w = max(x.w, row_lo[r]);
      }
      tile_span[threadIdx.x] = x;
    }
    __syncthreads();
  };

  bool staged = false;
  for (; left > 0; --left) {
    const int key0 = unit * C::kUnit + warp * C::kKeys;
    const int64_t head_row = (int64_t)head * a.page_size;
    // ---- K: from memory into the products' operands ----
    uint32_t x[C::kTiles][C::kSteps][4];
    float kscale[C::kTiles][2];
    bool there[C::kTiles];
#pragma unroll
    for (int b = 0; b < C::kTiles; ++b) {
      const int k0 = key0 + 16 * b;
      const int index = (int)(((uint64_t)(uint32_t)(k0 >> 4) * a.page_mul) >> a.page_shift);
      const int page = k0 < len ? __ldg(a.table.pages + seq * a.table.stride + index) : -1;
      there[b] = (unsigned)page < (unsigned)a.pages;
      if (k0 < len && !there[b] && lane == 0) atomicOr(a.status, kBadIndex);
      const int64_t row = there[b] ? page * a.page_rows + head_row + (k0 - index * a.page_size) : 0;
      const unsigned char* from = a.pk + (row + g) * row_bytes + t * 16;
#pragma unroll
      for (int c = 0; c < C::kPieces; ++c) {
        const bool in = there[b] && 64 * c + 16 * t < row_bytes;
        const uint4 y = in ? __ldg(reinterpret_cast<const uint4*>(from + 64 * c)) : make_uint4(0, 0, 0, 0);
        const uint4 z = in ? __ldg(reinterpret_cast<const uint4*>(from + 8 * row_bytes + 64 * c)) : make_uint4(0, 0, 0, 0);
        if constexpr (C::kEight) {
          const uint32_t yw[4] = {y.x, y.y, y.z, y.w}, zw[4] = {z.x, z.y, z.z, z.w};
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            widen4<FMT>(yw[i], x[b][4 * c + i][0], x[b][4 * c + i][2]);
            widen4<FMT>(zw[i], x[b][4 * c + i][1], x[b][4 * c + i][3]);
          }
        } else {
          x[b][2 * c][0] = y.x, x[b][2 * c][1] = z.x, x[b][2 * c][2] = y.y, x[b][2 * c][3] = z.y;
          x[b][2 * c + 1][0] = y.z, x[b][2 * c + 1][1] = z.z, x[b][2 * c + 1][2] = y.w, x[b][2 * c + 1][3] = z.w;
        }
      }
      kscale[b][0] = kscale[b][1] = 1.f;
      if (C::kEight && there[b]) kscale[b][0] = a.ks[row + g], kscale[b][1] = a.ks[row + g + 8];
    }
    // the key that this lane writes, and its weight so far
    const int own = key0 + (C::kTiles == 2 ? 8 * t : 8 * (t & 1)) + g;
    const bool writes = own < len && (C::kTiles == 2 || t < 2);
    float before = 0.f;
    if (writes && w.past && own < len - a.new_tokens) before = w.decay * w.past[seq * w.past_seq + head * w.past_head + own];

    float sum[C::kTiles][2] = {};
    for (int row0 = 0; row0 < a.rows; row0 += kChunk) {
      if (!staged || a.rows > kChunk) {
        __syncthreads();   // everyone is done with the last chunk
        stage(row0);
        staged = true;
      }
      const int tiles = (min(a.rows - row0, kChunk) + 7) / 8;
      for (int n = 0; n < tiles; ++n) {
        const int4 span = tile_span[n];
        if (key0 > span.y || key0 + C::kKeys - 1 < span.z) continue;   // keys that none of these rows sees
        float s[C::kTiles][4];
#pragma unroll
        for (int j = 0; j < C::kSteps / 2; ++j) {
          const uint4 q = *reinterpret_cast<const uint4*>(
              q_smem + (n * 8 + g) * C::kQStride + (C::kEight ? 128 * (j >> 1) + 32 * t + 16 * (j & 1) : 64 * j + 16 * t));
#pragma unroll
          for (int b = 0; b < C::kTiles; ++b) {
            const uint32_t(&y)[4] = x[b][2 * j], (&z)[4] = x[b][2 * j + 1];
            if (j == 0) mma16816_first<kBf16>(s[b], y[0], y[1], y[2], y[3], q.x, q.y);
            else mma16816<kBf16>(s[b], y[0], y[1], y[2], y[3], q.x, q.y);
            mma16816<kBf16>(s[b], z[0], z[1], z[2], z[3], q.z, q.w);
          }
        }
        const int r = n * 8 + 2 * t;
        const float2 lse = *reinterpret_cast<const float2*>(row_lse + r), f = *reinterpret_cast<const float2*>(row_factor + r);
#pragma unroll
        for (int b = 0; b < C::kTiles; ++b) {
          float p[4];
#pragma unroll
          for (int e = 0; e < 4; ++e)
            p[e] = exp2_fast(fmaf(s[b][e], (e & 1 ? f.y : f.x) * kscale[b][e >> 1], e & 1 ? -lse.y : -lse.x));
          const int k0 = key0 + 16 * b;
          if (!there[b] || k0 < span.w || k0 + 15 > span.x) {
#pragma unroll
            for (int e = 0; e < 4; ++e) {
              const int j = k0 + g + 8 * (e >> 1), rr = r + (e & 1);
              if (!there[b] || j > row_pos[rr] || j < row_lo[rr]) p[e] = 0.f;
            }
          }
          sum[b][0] += p[0] + p[1];
          sum[b][1] += p[2] + p[3];
        }
      }
    }
    // over the lanes that hold the other rows; then a key a lane
#pragma unroll
    for (int b = 0; b < C::kTiles; ++b) {
#pragma unroll
      for (int e = 0; e < 2; ++e) {
        sum[b][e] += __shfl_xor_sync(0xffffffffu, sum[b][e], 1);
        sum[b][e] += __shfl_xor_sync(0xffffffffu, sum[b][e], 2);
      }
    }
    const float low = t & 1 ? sum[0][1] : sum[0][0], high = t & 1 ? sum[C::kTiles - 1][1] : sum[C::kTiles - 1][0];
    const float got = t & 2 ? high : low;
    if (writes) w.out[seq * w.out_seq + head * w.out_head + own] = before + got;

    if (++unit == units && left > 1) {
      unit = 0;
      staged = false;
      if (++head == a.kv_heads) {
        head = 0;
        do len = weigh_length(a, ++seq);
        while (len == 0 && seq + 1 < a.table.seqs);
        units = (len + C::kUnit - 1) / C::kUnit;
      }
    }
  }
}

template <int FMT, int DP>
cudaError_t launch_weigh_one(const WeighArgs& w, int num_sms, cudaStream_t st) {
  using C = WeighConfig<FMT, DP>;
  const int64_t units = ((int64_t)w.a.max_len + C::kUnit - 1) / C::kUnit;
  const double most = (double)w.a.table.seqs * w.a.kv_heads * (double)units;
  if (most >= 2147483648.0) return cudaErrorNotSupported;   // units are counted in 32 bits
  const int blocks = most < 2.0 * num_sms ? (int)most : 2 * num_sms;
  weigh_kernel<FMT, DP><<<blocks, kWeighThreads, 0, st>>>(w);
  return cudaGetLastError();
}
template <int FMT>
cudaError_t launch_weigh(const WeighArgs& w, int num_sms, cudaStream_t st) {
  switch (padded_dim(w.a.head_dim)) {
    case 64: return launch_weigh_one<FMT, 64>(w, num_sms, st);
    case 128: return launch_weigh_one<FMT, 128>(w, num_sms, st);
    default: return launch_weigh_one<FMT, 256>(w, num_sms, st);
  }
}

}  // namespace
}  // namespace lc

extern "C" lacache_status lacache_kv_weigh(lacache_kv_t* h, int32_t layer, const lacache_kv_table* table,
                                           const lacache_weighing* in, void* cuda_stream) {
  lc::NvtxRange nvtx("lacache_kv_weigh");
  lc::WeighArgs w = {};
  if (!in || !isfinite(in->decay)) return LACACHE_ERR_INVALID_ARG;
  const lacache_status status = lc::attend_args(h, layer, table, in->new_tokens, in->q_heads, in->window, in->dtype, in->scale,
                                                in->lengths_dev, in->starts_dev, &in->q, &w.a);
  if (status != LACACHE_OK || table->seqs == 0) return status;
  if (!in->lse_dev || !in->out.data_dev || in->out.width < 1 || (in->past.data_dev && in->past.width < in->out.width))
    return LACACHE_ERR_INVALID_ARG;
  lc::DeviceGuard guard(h->cfg.device);
  if (!guard.ok()) return LACACHE_ERR_CUDA;
  w.a.lse = const_cast<float*>(in->lse_dev);
  w.a.max_len = std::min(w.a.max_len, in->out.width);
  w.decay = in->decay;
  w.past = in->past.data_dev;
  w.past_seq = in->past.seq_stride;
  w.past_head = in->past.head_stride;
  w.out = in->out.data_dev;
  w.out_seq = in->out.seq_stride;
  w.out_head = in->out.head_stride;
  const cudaStream_t st = (cudaStream_t)cuda_stream;
  cudaError_t e;
  switch (h->cfg.format) {
    case LACACHE_KV_BF16: e = lc::launch_weigh<LACACHE_KV_BF16>(w, h->num_sms, st); break;
    case LACACHE_KV_F16: e = lc::launch_weigh<LACACHE_KV_F16>(w, h->num_sms, st); break;
    case LACACHE_KV_E4M3: e = lc::launch_weigh<LACACHE_KV_E4M3>(w, h->num_sms, st); break;
    default: e = lc::launch_weigh<LACACHE_KV_INT8>(w, h->num_sms, st); break;
  }
  return e == cudaErrorNotSupported ? LACACHE_ERR_UNSUPPORTED : lc::from_cuda(e);
}
