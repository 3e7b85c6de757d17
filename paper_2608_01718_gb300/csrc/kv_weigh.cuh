// The attention weight that cached tokens get from new ones, added to what they got before:
//
//   w_j <- decay w_j + sum over the rows r that see j of e^(s_rj - lse_r),   s_rj = scale <q_r, k_j>
//
// for every kv head, over the rows that share it (its group of q heads times the new tokens), from the lse that the attention of
// the same rows wrote. K is read once. Each key belongs to one thread or warp, which adds its rows in order: no atomics, no
// joins. Scores, weights and sums are fp32. kv_weigh.cu has the kernel for few rows and the C entry, kv_weigh_tc.cu the kernel
// for many.
#pragma once

#include "kv_attend.cuh"

namespace lc {

struct WeighArgs {
  AttendArgs a;   // (lse is read; out, the partial sums and the counters are not used)
  float decay;
  const float* past;
  int64_t past_seq, past_head;
  float* out;
  int64_t out_seq, out_head;
};
cudaError_t launch_weigh_tc(const WeighArgs& w, int format, int num_sms, cudaStream_t st);

namespace {

__device__ __forceinline__ int weigh_length(const AttendArgs& a, int seq) {
  const int len = a.lengths[seq];
  return len < 0 ? 0 : len > a.max_len ? a.max_len : len;
}

// A place on the line of units (sequences, their heads, their keys by KEYS), and the next.
template <int KEYS>
struct WeighPlace {
  int seq, head, unit, units, len;
  __device__ __forceinline__ bool next(const AttendArgs& a) {   // true: another sequence or head
    if (++unit < units) return false;
    unit = 0;
    if (++head == a.kv_heads) {
      head = 0;
      do len = weigh_length(a, ++seq);
      while (len == 0 && seq + 1 < a.table.seqs);
      units = (len + KEYS - 1) / KEYS;
    }
    return true;
  }
};
// By a whole warp: where part `part` of `parts` equal parts of the line begins, and its units (0: none).
template <int KEYS>
__device__ __forceinline__ int weigh_start(const AttendArgs& a, int part, int parts, WeighPlace<KEYS>& at) {
  const int lane = threadIdx.x & 31;
  auto units_of = [&](int s) { return s < a.table.seqs ? (weigh_length(a, s) + KEYS - 1) / KEYS : 0; };
  int total = 0;
  for (int s = lane; s < a.table.seqs; s += 32) total += units_of(s);
  total = __reduce_add_sync(0xffffffffu, total) * a.kv_heads;
  const int share = total / parts, longer = total - share * parts;
  const int u = part * share + min(part, longer), mine = share + (part < longer ? 1 : 0);
  if (mine == 0) return 0;
  int base = 0;
  at.seq = 0;
  for (int s0 = 0; s0 < a.table.seqs; s0 += 32) {
    const int own = units_of(s0 + lane) * a.kv_heads;
    int upto = own;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const int y = __shfl_up_sync(0xffffffffu, upto, o);
      if (lane >= o) upto += y;
    }
    const unsigned past = __ballot_sync(0xffffffffu, base + upto > u);
    if (past) {
      const int l0 = __ffs(past) - 1;
      at.seq = s0 + l0;
      base += __shfl_sync(0xffffffffu, upto - own, l0);
      break;
    }
    base += __shfl_sync(0xffffffffu, upto, 31);
  }
  at.len = weigh_length(a, at.seq);
  at.units = (at.len + KEYS - 1) / KEYS;
  at.head = (u - base) / at.units;
  at.unit = (u - base) - at.head * at.units;
  return mine;
}
// The first position that any of a sequence's rows sees (INT_MAX: none is). Pages before it are not looked at.
__device__ __forceinline__ int weigh_first(const AttendArgs& a, int seq) {
  const Span sp = span_of(a, seq, 1);
  return sp.lo < sp.hi ? sp.lo : INT_MAX;
}
// Lengths outside their range, once a launch.
__device__ __forceinline__ void weigh_check(const AttendArgs& a) {
  if (blockIdx.x == 0) {
    for (int s = threadIdx.x; s < a.table.seqs; s += blockDim.x)
      if (a.lengths[s] < 0 || a.lengths[s] > a.max_len) atomicOr(a.status, kBadIndex);
  }
}

}  // namespace
}  // namespace lc
