// The attention weight of cached tokens: the kernel for few rows a kv head, and the C entry.
//
// Products are the warp-level tensor instruction's, S^T [16 keys x 8 rows] = K Q^T, with the naming of a row's dimensions chosen
// so that a lane's share of K is 16 contiguous bytes, as in kv_attend.cuh. 8-bit codes are widened to f16 exactly; q of bf16 over
// an 8-bit cache is scaled to f16 by a power of two a row (exact for elements within 2^-14 of the row's largest).
//
// Bound by reading K: every warp, for itself, has a ring of its own tiles of 16 or 32 keys in shared memory, filled by cp.async
// whole lines at a time (with the keys' scales and past weights), and takes an equal part of the line of units (sequences, their
// heads, their keys), whatever the lengths. q stays in registers; nothing is shared between warps. 64 sequences of 500 to 16,384
// tokens of e4m3 (32 heads on 8, d = 128) take 114 us, 5.3 TB/s of the 606 MB (155 with tiles loaded and multiplied in turns by a
// block); one of 700 in bf16 (8 heads, d = 64) 4.3, its launch and three dependent loads.
#include <algorithm>

#include "kv_weigh.cuh"

namespace lc {
namespace {

constexpr int kFewRows = 16;   // a kv head
constexpr int kWeighWarps = 4, kWeighThreads = kWeighWarps * 32;

template <int FMT, int DP, int NT>
struct WeighConfig {
  using C = AttendConfig<FMT, DP, NT>;
  static constexpr bool kEight = C::kEight;
  static constexpr int kSub = C::kSub, kKeys = C::kKeys, kTileBytes = C::kTileBytes, kRowBytes = C::kRowBytes;
  static constexpr int kPieces = C::kKPieces;                         // 16-byte pieces of a lane in a row of K
  static constexpr int kSteps = DP / 16;
  static constexpr int kScales = kSub * kTileBytes;                   // offsets in a stage
  static constexpr int kPast = kScales + (kEight ? kKeys * 4 : 0);
  static constexpr int kStageBytes = kPast + kKeys * 4;
  static constexpr int kStages = kSub * kTileBytes > 4096 ? 2 : kSub * kTileBytes > 2048 ? 4 : 7;
  static constexpr int kRing = kStages * kStageBytes;                 // of a warp
  static constexpr int kSmem = kWeighWarps * kRing;
  static constexpr int kBlocks = 3;                                   // an SM holds
};

template <int FMT, int DP, int NT>
__global__ void __launch_bounds__(kWeighThreads, WeighConfig<FMT, DP, NT>::kBlocks) weigh_kernel(const __grid_constant__ WeighArgs w) {
  using W = WeighConfig<FMT, DP, NT>;
  using C = typename W::C;
  constexpr bool kBf16 = FMT == LACACHE_KV_BF16;
  extern __shared__ __align__(128) unsigned char smem[];
  const AttendArgs& a = w.a;
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, g = lane >> 2, t = lane & 3;
  const int D = a.head_dim, row_bytes = D * C::kItem;

  weigh_check(a);
  // where the products are, and where the copies are, kStages - 1 units ahead
  WeighPlace<W::kKeys> at;
  const int mine = weigh_start<W::kKeys>(a, blockIdx.x + warp * gridDim.x, gridDim.x * kWeighWarps, at);
  if (mine == 0) return;
  WeighPlace<W::kKeys> ahead = at;

  unsigned char* ring = smem + warp * W::kRing;
  const uint32_t ring_addr = shared_addr(ring);
  auto page_of = [&](int k) { return (int)(((uint64_t)(uint32_t)(k >> 4) * a.page_mul) >> a.page_shift); };
  int ids[W::kSub], next_ids[W::kSub], in_batch = 0;   // lane i: page ids of the batch's unit i, and of the next batch's
  int ahead_left = mine, ahead_slot = 0, first_seen = 0;
  const int32_t* table_row;
  const unsigned char* head_k;
  const float* past;
  int64_t head_row;
  uint32_t bad_slots = 0;   // bit slot * kSub + s: that tile has no page
  auto look_up = [&](int from, int (&to)[W::kSub]) {
#pragma unroll
    for (int s = 0; s < W::kSub; ++s) {
      const int64_t k = (int64_t)from + lane * W::kKeys + 16 * s;
      to[s] = k < ahead.len ? __ldg(table_row + page_of((int)k)) : -1;
    }
  };
  auto enter = [&] {
    table_row = a.table.pages + ahead.seq * a.table.stride;
    head_row = (int64_t)ahead.head * a.page_size;
    head_k = a.pk + head_row * row_bytes;
    past = w.past ? w.past + ahead.seq * w.past_seq + ahead.head * w.past_head : nullptr;
    first_seen = weigh_first(a, ahead.seq);
    in_batch = 0;
    look_up(ahead.unit * W::kKeys, ids);
  };
  enter();
  auto issue = [&] {
    if (ahead_left > 0) {
      const uint32_t to = ring_addr + ahead_slot * W::kStageBytes;
      const int key = ahead.unit * W::kKeys;
#pragma unroll
      for (int s = 0; s < W::kSub; ++s) {
        const int k0 = key + 16 * s;
        const int page = __shfl_sync(0xffffffffu, ids[s], in_batch);
        const bool there = (unsigned)page < (unsigned)a.pages;
        if (!there && k0 < ahead.len && k0 + 15 >= first_seen && lane == 0) atomicOr(a.status, kBadIndex);
        const uint32_t bit = 1u << (ahead_slot * W::kSub + s);
        bad_slots = there ? bad_slots & ~bit : bad_slots | bit;
        if (!there || k0 + 15 < first_seen) continue;   // (not seen by any row: what the stage holds is not looked at)
        const int slot = k0 - page_of(k0) * a.page_size;
        const unsigned char* from = head_k + page * a.page_bytes + (int64_t)slot * row_bytes;
        const uint32_t kd = to + s * W::kTileBytes;
        const int unit = lane % C::kUnits, first = lane / C::kUnits;
        if (D == DP) {
#pragma unroll
          for (int i = 0; i < C::kCopies; ++i)
            copy_async<16>(kd + k_unit<W::kRowBytes>(i * C::kCopyRows + first, unit), from + i * 512 + lane * 16, true);
        } else {
          const bool live = unit * 16 < row_bytes;   // (past the row's end: zeros)
#pragma unroll
          for (int i = 0; i < C::kCopies; ++i) {
            const int j = i * C::kCopyRows + first;
            copy_async<16>(kd + k_unit<W::kRowBytes>(j, unit), from + (live ? j * row_bytes + unit * 16 : 0), live);
          }
        }
        if constexpr (W::kEight) {   // four scales a lane
          if (lane >> 2 == s)
            copy_async<16>(to + W::kScales + lane * 16, a.ks + page * a.page_rows + head_row + slot + (lane & 3) * 4, true);
        }
      }
      const int own = key + lane;
      if (past && lane < W::kKeys) {
        const bool live = own < ahead.len - a.new_tokens;
        copy_async<4>(to + W::kPast + lane * 4, live ? past + own : past, live);
      }
      --ahead_left;
      ahead_slot = ahead_slot + 1 == W::kStages ? 0 : ahead_slot + 1;
      if (++in_batch == 16) look_up((ahead.unit + 1 + 16) * W::kKeys, next_ids);
      if (in_batch == 32) {
        in_batch = 0;
#pragma unroll
        for (int s = 0; s < W::kSub; ++s) ids[s] = next_ids[s];
      }
      if (ahead_left > 0 && ahead.next(a)) enter();
    }
    copy_commit();
  };

  // ---- a triple's rows ----
  uint4 q[NT][W::kSteps / 2];
  float lse[NT][2], factor[NT][2];    // of rows 8 n + 2 t and the next: times log2(e); scale log2(e) times what q was divided by
  int pos[NT][2], lo[NT][2];          // their last and first visible position
  int min_pos = 0, max_lo = 0, max_pos = -1;
  auto load_rows = [&] {
    const int64_t token0 = (int64_t)at.seq * a.new_tokens;
    int least = INT_MAX, most = -1, latest = INT_MIN;
#pragma unroll
    for (int n = 0; n < NT; ++n) {
      {
        const int row = n * 8 + g, tok = row / a.group;
        const bool live = row < a.rows;
        const unsigned char* from = live ? a.q.at(token0 + tok, at.head * a.group + row - tok * a.group) : nullptr;
#pragma unroll
        for (int j = 0; j < W::kSteps / 2; ++j) {
          const int byte = W::kEight ? 128 * (j >> 1) + 32 * t + 16 * (j & 1) : 64 * j + 16 * t;
          q[n][j] = live && byte < D * 2 ? *reinterpret_cast<const uint4*>(from + byte) : make_uint4(0, 0, 0, 0);
        }
      }
      float back = 1.f;
      if (W::kEight && !a.q_f16) {
        float top = 0.f;
#pragma unroll
        for (int j = 0; j < W::kSteps / 2; ++j) {
          float x[8];
          widen8(q[n][j], x, __nv_bfloat16());
#pragma unroll
          for (int i = 0; i < 8; ++i) top = fmaxf(top, fabsf(x[i]));
        }
        top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 1));
        top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 2));
        // the power of two below top (1 for zeros, infinities and subnormals)
        uint32_t e = __float_as_uint(top) & 0x7f800000u;
        float down = 1.f;
        if (e != 0 && e != 0x7f800000u) {
          e = e < 0x7e800000u ? e : 0x7e800000u;
          back = __uint_as_float(e);
          down = __uint_as_float(0x7f000000u - e);
        }
#pragma unroll
        for (int j = 0; j < W::kSteps / 2; ++j) {
          float x[8];
          widen8(q[n][j], x, __nv_bfloat16());
#pragma unroll
          for (int i = 0; i < 8; ++i) x[i] *= down;
          q[n][j] = pack8(x, __half());
        }
      }
#pragma unroll
      for (int e = 0; e < 2; ++e) {
        const int r = 2 * t + e, row = n * 8 + r, tok = row / a.group;
        const bool live = row < a.rows;
        const float x = live ? w.a.lse[(token0 + tok) * a.q_heads + at.head * a.group + row - tok * a.group] : -INFINITY;
        int p = at.len - a.new_tokens + tok, first = a.starts ? a.starts[at.seq] : 0;
        if (a.window > 0 && p - a.window + 1 > first) first = p - a.window + 1;
        if (x == -INFINITY) p = -1;   // a row that sees nothing (and those past the last)
        lse[n][e] = x * 1.4426950408889634f;
        factor[n][e] = a.scale * 1.4426950408889634f * __shfl_sync(0xffffffffu, back, r * 4);
        pos[n][e] = p;
        lo[n][e] = first;
        least = min(least, p), most = max(most, p), latest = max(latest, first);
      }
    }
    min_pos = __reduce_min_sync(0xffffffffu, least);
    max_pos = __reduce_max_sync(0xffffffffu, most);
    max_lo = __reduce_max_sync(0xffffffffu, latest);
  };

  int slot = 0;
  bool fresh = true;
  int seen_from = 0;
  for (int i = 1 - W::kStages; i < mine; ++i) {
    issue();
    if (i < 0) continue;   // the copies' head start
    if (fresh) {
      load_rows();
      seen_from = weigh_first(a, at.seq);
      fresh = false;
    }
    copy_wait<W::kStages - 1>();
    __syncwarp();
    const unsigned char* st = ring + slot * W::kStageBytes;
    const int key = at.unit * W::kKeys;
    float got = 0.f;
#pragma unroll
    for (int b = 0; b < W::kSub; ++b) {
      const int k0 = key + 16 * b;
      float sum0 = 0.f, sum1 = 0.f;
      if (k0 <= max_pos && k0 + 15 >= seen_from && !(bad_slots >> (slot * W::kSub + b) & 1)) {
        const unsigned char* kt = st + b * W::kTileBytes;
        float s[NT][4];
#pragma unroll
        for (int c = 0; c < W::kPieces; ++c) {
          const uint4 x = *reinterpret_cast<const uint4*>(kt + k_unit<W::kRowBytes>(g, 4 * c + t));
          const uint4 y = *reinterpret_cast<const uint4*>(kt + k_unit<W::kRowBytes>(g + 8, 4 * c + t));
          if constexpr (W::kEight) {
            const uint32_t xw[4] = {x.x, x.y, x.z, x.w}, yw[4] = {y.x, y.y, y.z, y.w};
            uint32_t xa[8], ya[8];
#pragma unroll
            for (int e = 0; e < 4; ++e) {
              widen4<FMT>(xw[e], xa[2 * e], xa[2 * e + 1]);
              widen4<FMT>(yw[e], ya[2 * e], ya[2 * e + 1]);
            }
#pragma unroll
            for (int n = 0; n < NT; ++n) {
              const uint4 q0 = q[n][2 * c], q1 = q[n][2 * c + 1];
              if (c == 0) mma16816_first<false>(s[n], xa[0], ya[0], xa[1], ya[1], q0.x, q0.y);
              else mma16816<false>(s[n], xa[0], ya[0], xa[1], ya[1], q0.x, q0.y);
              mma16816<false>(s[n], xa[2], ya[2], xa[3], ya[3], q0.z, q0.w);
              mma16816<false>(s[n], xa[4], ya[4], xa[5], ya[5], q1.x, q1.y);
              mma16816<false>(s[n], xa[6], ya[6], xa[7], ya[7], q1.z, q1.w);
            }
          } else {
#pragma unroll
            for (int n = 0; n < NT; ++n) {
              const uint4 qn = q[n][c];
              if (c == 0) mma16816_first<kBf16>(s[n], x.x, y.x, x.y, y.y, qn.x, qn.y);
              else mma16816<kBf16>(s[n], x.x, y.x, x.y, y.y, qn.x, qn.y);
              mma16816<kBf16>(s[n], x.z, y.z, x.w, y.w, qn.z, qn.w);
            }
          }
        }
        float scale0 = 1.f, scale1 = 1.f;
        if constexpr (W::kEight) {
          const float* sc = reinterpret_cast<const float*>(st + W::kScales) + b * 16;
          scale0 = sc[g], scale1 = sc[g + 8];
        }
        const bool masked = k0 < max_lo || k0 + 15 > min_pos;
#pragma unroll
        for (int n = 0; n < NT; ++n) {
          float p[4];
#pragma unroll
          for (int e = 0; e < 4; ++e) p[e] = exp2_fast(fmaf(s[n][e], factor[n][e & 1] * (e < 2 ? scale0 : scale1), -lse[n][e & 1]));
          if (masked) {
#pragma unroll
            for (int e = 0; e < 4; ++e) {
              const int j = k0 + g + 8 * (e >> 1);
              if (j > pos[n][e & 1] || j < lo[n][e & 1]) p[e] = 0.f;
            }
          }
          sum0 += p[0] + p[1];
          sum1 += p[2] + p[3];
        }
      }
      // over the lanes that hold the other rows; then a key a lane: lane l the unit's key l
      sum0 += __shfl_xor_sync(0xffffffffu, sum0, 1);
      sum1 += __shfl_xor_sync(0xffffffffu, sum1, 1);
      sum0 += __shfl_xor_sync(0xffffffffu, sum0, 2);
      sum1 += __shfl_xor_sync(0xffffffffu, sum1, 2);
      const float from0 = __shfl_sync(0xffffffffu, sum0, (lane & 7) * 4), from1 = __shfl_sync(0xffffffffu, sum1, (lane & 7) * 4);
      if (lane >> 4 == b) got = lane & 8 ? from1 : from0;
    }
    const int own = key + lane;
    if (lane < W::kKeys && own < at.len) {
      const float before = w.past ? w.decay * reinterpret_cast<const float*>(st + W::kPast)[lane] : 0.f;
      w.out[at.seq * w.out_seq + at.head * w.out_head + own] = own < at.len - a.new_tokens ? before + got : got;
    }
    __syncwarp();   // the slot is free again
    slot = slot + 1 == W::kStages ? 0 : slot + 1;
    if (i + 1 < mine && at.next(a)) fresh = true;
  }
}

template <int FMT, int DP, int NT>
cudaError_t launch_weigh_one(const WeighArgs& w, int num_sms, cudaStream_t st) {
  using W = WeighConfig<FMT, DP, NT>;
  static_assert(W::kSmem <= 227 * 1024 && W::kStages * W::kSub <= 32, "shared memory, and a bit a tile");
  auto* kernel = weigh_kernel<FMT, DP, NT>;
  static std::atomic<int> resident[kMaxDevices];   // blocks an SM holds, by device; 0: not asked yet
  int per_sm = w.a.device < kMaxDevices ? resident[w.a.device].load(std::memory_order_relaxed) : 0;
  if (per_sm == 0) {
    cudaError_t e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, W::kSmem);
    if (e == cudaSuccess) e = cudaOccupancyMaxActiveBlocksPerMultiprocessor(&per_sm, kernel, kWeighThreads, W::kSmem);
    if (e != cudaSuccess) return e;
    per_sm = per_sm < 1 ? 1 : per_sm;
    if (w.a.device < kMaxDevices) resident[w.a.device].store(per_sm, std::memory_order_relaxed);
  }
  const int64_t units = ((int64_t)w.a.max_len + W::kKeys - 1) / W::kKeys;
  const double most = (double)w.a.table.seqs * w.a.kv_heads * (double)units;
  if (most >= 2147483648.0) return cudaErrorNotSupported;   // units are counted in 32 bits
  const int blocks = most < (double)per_sm * num_sms ? (int)most : per_sm * num_sms;
  kernel<<<blocks, kWeighThreads, W::kSmem, st>>>(w);
  return cudaGetLastError();
}
template <int FMT, int NT>
cudaError_t launch_weigh_rows(const WeighArgs& w, int num_sms, cudaStream_t st) {
  switch (padded_dim(w.a.head_dim)) {
    case 64: return launch_weigh_one<FMT, 64, NT>(w, num_sms, st);
    case 128: return launch_weigh_one<FMT, 128, NT>(w, num_sms, st);
    default: return launch_weigh_one<FMT, 256, NT>(w, num_sms, st);
  }
}
template <int FMT>
cudaError_t launch_weigh(const WeighArgs& w, int num_sms, cudaStream_t st) {
  return w.a.rows <= 8 ? launch_weigh_rows<FMT, 1>(w, num_sms, st) : launch_weigh_rows<FMT, 2>(w, num_sms, st);
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
  if (!in->lse_dev || !in->out.data_dev || in->out.width < 1 || (in->past.data_dev && in->past.width < in->out.width) ||
      (table->seqs > 1 && in->out.seq_stride == 0) || (h->cfg.kv_heads > 1 && in->out.head_stride == 0) ||
      (in->past.data_dev == in->out.data_dev &&
       ((table->seqs > 1 && in->past.seq_stride != in->out.seq_stride) ||
        (h->cfg.kv_heads > 1 && in->past.head_stride != in->out.head_stride))))
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
  if (w.a.rows > lc::kFewRows) {
    if (h->inject_stall > 0) {
      w.a.inject_stall = 1;
      --h->inject_stall;
    }
    e = lc::launch_weigh_tc(w, h->cfg.format, h->num_sms, st);
  } else switch (h->cfg.format) {
    case LACACHE_KV_BF16: e = lc::launch_weigh<LACACHE_KV_BF16>(w, h->num_sms, st); break;
    case LACACHE_KV_F16: e = lc::launch_weigh<LACACHE_KV_F16>(w, h->num_sms, st); break;
    case LACACHE_KV_E4M3: e = lc::launch_weigh<LACACHE_KV_E4M3>(w, h->num_sms, st); break;
    default: e = lc::launch_weigh<LACACHE_KV_INT8>(w, h->num_sms, st); break;
  }
  return e == cudaErrorNotSupported ? LACACHE_ERR_UNSUPPORTED : lc::from_cuda(e);
}
