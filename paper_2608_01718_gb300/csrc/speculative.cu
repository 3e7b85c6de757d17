// Draft verification for reusing the lookahead prefix on a miss (section 3.3, "Speculative Decoding"), by comparing the
// models' probabilities, and by given random numbers, which draw the next token too.
#include <cooperative_groups.h>

#include "internal.cuh"

namespace lc {

// By comparison: the number of leading draft tokens with P_f(t) >= P_g(t) for every query that is not served from the cache.
//
// One warp per query: each pass of 32 positions ballots the rejections (P_f < P_g); the first set bit, if any,
// ends the accepted prefix.

constexpr int kVerifyWarps = 8;

__global__ void __launch_bounds__(kVerifyWarps * 32)
    verify_draft_kernel(int B, int k, const float* __restrict__ pf, const float* __restrict__ pg,
                        const uint8_t* __restrict__ status, int32_t* __restrict__ accepted) {
  const int lane = threadIdx.x & 31;
  const int q = blockIdx.x * kVerifyWarps + (threadIdx.x >> 5);
  if (q >= B) return;
  if (status && status[q] == LACACHE_HIT) {
    if (lane == 0) accepted[q] = -1;
    return;
  }
  int n = k;
  for (int base = 0; base < k; base += 32) {
    const int i = base + lane;
    const bool reject = i < k && pf[(int64_t)q * k + i] < pg[(int64_t)q * k + i];
    const unsigned r = __ballot_sync(0xffffffffu, reject);
    if (r) {
      n = base + __ffs(r) - 1;
      break;
    }
  }
  if (lane == 0) accepted[q] = n;
}

// By given random numbers. With p and q the target's and the draft model's probabilities, draft t is accepted while
// u_t q_t(x_t) < p_t(x_t). Where the window ends, the next token is drawn with the weights
//   w_i = max(p_i - q_i, 0)  of the position that refused its draft,   w_i = p_i  where no draft was refused,
// as the first i whose cumulative weight C_i exceeds u_k C. Accepted drafts and the drawn token are then distributed as the
// target's own tokens.
//
// Both decisions are those of the real numbers but for the last bits of C: u q is a product of 24-bit numbers, exact in fp64; a
// difference of two fp32 is held exactly as two (the rounded difference and its rounding error; D. Knuth, "The Art of Computer
// Programming", vol. 2, 4.2.2), sums of them as a leading sum and the sum of its rounding errors, and C_i near the border in fp64.
// That sum of errors is rounded too, the more the longer it gets, so it is kept short: eight terms, then eight such sums, whose
// errors go back into a leading sum each time, then fp64. With u = 2^-24 the bounds, in u^2 = 2^-48 of the sum, are 43 for eight
// terms (their errors reach k u of it after k terms; each is rounded in itself and in its addition), 70 for eight sums, 40 for the
// five steps over a warp's lanes, 1 for a long sum's way back from fp64: 2^-40.7. fp64 adds 2^-67 for every token of the
// vocabulary: 2^-40 in all up to 2^25 tokens, 2^-36 at 2^30. (One running sum and its errors, without those steps, lost 2^-33 of
// rows with one large and 10^5 equal small numbers.) In fp32 alone, sums over 10^5 tokens would draw a
// neighbour of the token in some percent of the calls; in fp64 alone, the differences and sums of a row of 10^5 take longer than reading it.
//
// A cluster of 1 to 8 blocks a query, each warp a run of consecutive tokens, with sixteen loads in flight a lane. The runs'
// sums are exchanged through the cluster's shared memory; the block that holds the border adds its run again, a part a warp, and
// one warp looks for the token in that part. fp64 takes 16 cycles of an SM an instruction, so one warp a block takes those steps:
// by all warps they were a third of the time. 64 queries of 16 drafts and 100,003 tokens, two rows of one position read: 17.3 us
// (3.0 TB/s); one query of 32,000 tokens 7.8 us, the latency of the chain from the drafts to the token. What bounds both is that
// chain: with twice or half the loads in flight the times are the same.
constexpr int kSampleThreads = 256, kSampleWarps = kSampleThreads / 32, kMaxCluster = 8;
constexpr int kSampleUnroll = 8, kSampleTurns = 8;   // terms of a sum, and sums, before their errors are settled
constexpr int kSampleWalk = 64;   // of a part, walked 32 tokens at a time; a longer one is cut further first (196 tokens: 8% faster so)
constexpr int kMaxVocab = 1 << 30, kSampleResident = 152 * 8;

struct Probs {
  const float* data;
  int64_t seq, token;
};
struct SampleArgs {
  int k, vocab, blocks;   // blocks a query: the cluster
  int run;                // tokens a warp
  Probs target, draft;    // draft.data == nullptr: drafts of probability 1
  const int32_t* drafts;
  const float* u;
  const uint8_t* status;
  int32_t* accepted;
  int32_t* token;
};

// sum + rest
struct Twofold {
  float sum, rest;
};
// x - y, exactly
__device__ __forceinline__ Twofold difference(float x, float y) {
  const float d = __fsub_rn(x, y), b = __fsub_rn(d, x);
  return Twofold{d, __fsub_rn(__fsub_rn(x, __fsub_rn(d, b)), __fadd_rn(y, b))};
}
__device__ __forceinline__ Twofold plus(Twofold a, Twofold b) {
  const float s = __fadd_rn(a.sum, b.sum), c = __fsub_rn(s, a.sum);
  const float s_err = __fadd_rn(__fsub_rn(a.sum, __fsub_rn(s, c)), __fsub_rn(b.sum, c));
  return Twofold{s, __fadd_rn(__fadd_rn(a.rest, b.rest), s_err)};
}
// a + d where d.rest is at most half a last bit of d.sum: the errors of this addition first
__device__ __forceinline__ void add(Twofold& a, Twofold d) {
  const float s = __fadd_rn(a.sum, d.sum), c = __fsub_rn(s, a.sum);
  const float s_err = __fadd_rn(__fsub_rn(a.sum, __fsub_rn(s, c)), __fsub_rn(d.sum, c));
  a.sum = s;
  a.rest = __fadd_rn(a.rest, __fadd_rn(s_err, d.rest));
}
// The same sum with rest at most half a last bit of the leading one (exact: rest is smaller than it).
__device__ __forceinline__ Twofold settled(Twofold a) {
  const float s = __fadd_rn(a.sum, a.rest);
  return Twofold{s, __fsub_rn(a.rest, __fsub_rn(s, a.sum))};
}
__device__ __forceinline__ Twofold warp_sum(Twofold x) {
#pragma unroll
  for (int o = 16; o > 0; o >>= 1)
    x = plus(x, Twofold{__shfl_xor_sync(0xffffffffu, x.sum, o), __shfl_xor_sync(0xffffffffu, x.rest, o)});
  return x;
}
__device__ __forceinline__ double inclusive_sum(double x) {   // over the warp's lanes
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const double y = __shfl_up_sync(0xffffffffu, x, o);
    if ((threadIdx.x & 31) >= o) x += y;
  }
  return x;
}
// Of the warp's lanes, in order: the first that the cumulative weight `upto` exceeds `target` in, else (u at or above 1, sums that
// are not finite, or that end below those of the level above by their last bits) the last that has any weight, else -1. `base`: the
// weight before the first lane, then before that one.
__device__ __forceinline__ int border_lane(double own, double upto, double target, double& base) {
  const unsigned past = __ballot_sync(0xffffffffu, own > 0.0 && upto > target), some = __ballot_sync(0xffffffffu, own > 0.0);
  const int at = past ? __ffs(past) - 1 : 31 - __clz(some);
  const double before = __shfl_sync(0xffffffffu, upto, at > 0 ? at - 1 : 0);
  if (at > 0) base = before;
  return at;
}

__global__ void __launch_bounds__(kSampleThreads) verify_sample_kernel(const __grid_constant__ SampleArgs a) {
  namespace cg = cooperative_groups;
  cg::cluster_group cluster = cg::this_cluster();
  __shared__ alignas(16) Twofold run_sum[kSampleWarps];
  __shared__ Twofold part_sum[kSampleWarps];
  __shared__ int s_n, s_refused, s_run;
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const int64_t b = blockIdx.x / a.blocks;
  const int rank = blockIdx.x - (int)b * a.blocks, runs = a.blocks * kSampleWarps;
  if (a.status && a.status[b] == LACACHE_HIT) {
    if (rank == 0 && threadIdx.x == 0) a.accepted[b] = a.token[b] = -1;
    return;
  }
  const double u = a.u[b * (a.k + 1) + a.k];
  // how many drafts are accepted, and which one, if any, was refused
  if (warp == 0) {
    int n = a.k, refused = -1;
    for (int base = 0; base < a.k; base += 32) {
      const int t = base + lane;
      int x = -1;
      bool go = false;
      if (t < a.k) {
        x = a.drafts[b * a.k + t];
        if (x < 0 || x >= a.vocab) {
          x = -1;
        } else {
          const float p = a.target.data[b * a.target.seq + t * a.target.token + x];
          const float q = a.draft.data ? a.draft.data[b * a.draft.seq + t * a.draft.token + x] : 1.f;
          go = (double)a.u[b * (a.k + 1) + t] * (double)q < (double)p;
        }
      }
      const unsigned stop = __ballot_sync(0xffffffffu, t < a.k && !go);
      if (stop) {
        n = base + __ffs(stop) - 1;
        refused = __shfl_sync(0xffffffffu, x, __ffs(stop) - 1);
        break;
      }
    }
    if (lane == 0) s_n = n, s_refused = refused;
  }
  __syncthreads();
  const int n = s_n, refused = s_refused;
  const float* p = a.target.data + b * a.target.seq + n * a.target.token;
  // a second time with p alone where p - q leaves no weight
  for (int attempt = refused >= 0 ? 0 : 1; attempt < 2; ++attempt) {
    const float* q = attempt == 0 && a.draft.data ? a.draft.data + b * a.draft.seq + n * a.draft.token : nullptr;
    const int one = attempt == 0 && !a.draft.data ? refused : -1;   // where q is 1, if it has no row
    auto less = [&](int i) { return q ? q[i] : i == one ? 1.f : 0.f; };
    // tokens i, i + step, ... before `end`
    auto add_up = [&](int i, int end, int step) {
      auto short_sum = [&](int i0, int end) {   // of kSampleUnroll x kSampleTurns terms at most
        Twofold all = {0.f, 0.f};
#pragma unroll 1
        for (; i0 < end; i0 += step * kSampleUnroll) {
          float x[kSampleUnroll], y[kSampleUnroll];
#pragma unroll
          for (int e = 0; e < kSampleUnroll; ++e) {
            const int64_t i = i0 + (int64_t)step * e;
            x[e] = i < end ? p[i] : 0.f;
            y[e] = i < end ? less((int)i) : 0.f;
          }
          Twofold sum;
#pragma unroll
          for (int e = 0; e < kSampleUnroll; ++e) {
            const bool some = x[e] > y[e];
            const Twofold d = difference(some ? x[e] : 0.f, some ? y[e] : 0.f);
            if (e == 0) sum = d;
            else add(sum, d);
          }
          add(all, settled(sum));
        }
        return settled(all);
      };
      const int64_t each = (int64_t)step * kSampleUnroll * kSampleTurns;
      Twofold all = short_sum(i, (int)min((int64_t)end, i + each));
      if (i + each < end) {   // (a loop of its own: fp64 in the short sums' loop, even if it is not reached, was 5 us of 22 on 64 queries)
        double whole = (double)all.sum + (double)all.rest;
#pragma unroll 1
        for (int64_t at = i + each; at < end; at += each) {
          all = short_sum((int)at, (int)min((int64_t)end, at + each));
          whole += (double)all.sum + (double)all.rest;
        }
        all.sum = (float)whole;
        all.rest = (float)(whole - (double)all.sum);
      }
      return all;
    };
    const int first = (int)min((int64_t)(rank * kSampleWarps + warp) * a.run, (int64_t)a.vocab);
    const Twofold sum = warp_sum(add_up(first + lane, (int)min((int64_t)first + a.run, (int64_t)a.vocab), 32));
    if (lane == 0) run_sum[warp] = sum;
    cluster.sync();
    // the run that the border lies in: two runs a lane
    double base = 0.0, target = 0.0;
    if (warp == 0) {
      double s0 = 0.0, s1 = 0.0;
      if (2 * lane < runs) {
        const float4 x = *reinterpret_cast<const float4*>(cluster.map_shared_rank(&run_sum[2 * lane % kSampleWarps], 2 * lane / kSampleWarps));
        s0 = (double)x.x + (double)x.y;
        s1 = (double)x.z + (double)x.w;
        if (!(s0 > 0.0)) s0 = 0.0;   // (a sum that is NaN too)
        if (!(s1 > 0.0)) s1 = 0.0;
      }
      const double both = s0 + s1, upto = inclusive_sum(both);
      target = u * __shfl_sync(0xffffffffu, upto, 31);
      if (!(u < 1.0)) target = INFINITY;   // none qualifies, however the sums of the levels below round
      const int at = border_lane(both, upto, target, base);
      int run = -1;
      if (at >= 0) {
        const double of_first = __shfl_sync(0xffffffffu, s0, at), of_second = __shfl_sync(0xffffffffu, s1, at);
        const bool second = !(of_first > 0.0 && base + of_first > target) && of_second > 0.0;
        run = 2 * at + second;
        if (second) base += of_first;
      }
      if (lane == 0) s_run = run;
    }
    cluster.barrier_arrive();   // the sums have been read
    __syncthreads();
    const int run = s_run;
    if (run >= 0 && run / kSampleWarps == rank) {
      // its tokens again: a part of them a warp, then a few consecutive ones a lane of one warp, then a token a lane
      const int begin = run * a.run, end = (int)min((int64_t)begin + a.run, (int64_t)a.vocab);
      const int part = (a.run + kSampleWarps - 1) / kSampleWarps;
      auto past = [&](int64_t i) { return (int)min(i, (int64_t)end); };
      const int mine = past((int64_t)begin + warp * part);
      const Twofold of_warp = warp_sum(add_up(mine + lane, past((int64_t)mine + part), 32));
      if (lane == 0) part_sum[warp] = of_warp;
      __syncthreads();
      if (warp == 0) {
        const Twofold x = lane < kSampleWarps ? part_sum[lane] : Twofold{0.f, 0.f};
        auto border = [&](Twofold sum) {
          const double own = (double)sum.sum + (double)sum.rest;
          return max(border_lane(own, base + inclusive_sum(own), target, base), 0);
        };
        int from = past((int64_t)begin + border(x) * part), upto = past((int64_t)from + part);
        if (part > kSampleWalk) {
          const int each = (part + 31) / 32;
          auto of_lane = [&](int l) { return (int)min((int64_t)from + (int64_t)l * each, (int64_t)upto); };
          const int l = border(add_up(of_lane(lane), of_lane(lane + 1), 1)), lane_end = of_lane(l + 1);
          from = of_lane(l);
          upto = lane_end;
        }
        int token = -1;
        for (int i0 = from; i0 < upto; i0 += 32) {
          const int i = i0 + lane;
          const float x = i < upto ? p[i] : 0.f, y = i < upto ? less(i) : 0.f;
          const double own = x > y ? (double)x - (double)y : 0.0, sum = base + inclusive_sum(own);
          const unsigned over = __ballot_sync(0xffffffffu, own > 0.0 && sum > target), some = __ballot_sync(0xffffffffu, own > 0.0);
          if (over | some) token = i0 + (over ? __ffs(over) - 1 : 31 - __clz(some));
          if (over) break;
          base = __shfl_sync(0xffffffffu, sum, 31);
        }
        if (lane == 0) {
          a.accepted[b] = n;
          a.token[b] = token;
        }
      }
    }
    cluster.barrier_wait();
    if (run >= 0) return;
  }
  if (rank == 0 && threadIdx.x == 0) {   // a row without any weight
    a.accepted[b] = n;
    a.token[b] = -1;
  }
}

}  // namespace lc

extern "C" lacache_status lacache_verify_draft(int32_t B, int32_t k, const float* p_target_dev,
                                               const float* p_draft_dev, const uint8_t* status_dev,
                                               int32_t* accepted_dev, void* cuda_stream) {
  lc::NvtxRange nvtx("lacache_verify_draft");
  if (B < 1 || k < 1 || k > lc::kMaxK || !p_target_dev || !p_draft_dev || !accepted_dev)
    return LACACHE_ERR_INVALID_ARG;
  const int blocks = (B + lc::kVerifyWarps - 1) / lc::kVerifyWarps;
  const cudaStream_t st = (cudaStream_t)cuda_stream;
  lc::verify_draft_kernel<<<blocks, lc::kVerifyWarps * 32, 0, st>>>(B, k, p_target_dev, p_draft_dev, status_dev,
                                                                   accepted_dev);
  return cudaGetLastError() == cudaSuccess ? LACACHE_OK : LACACHE_ERR_CUDA;
}

extern "C" lacache_status lacache_verify_sample(int32_t B, int32_t k, int32_t vocab, const lacache_probs* p_target,
                                                const lacache_probs* p_draft, const int32_t* drafts_dev, const float* u_dev,
                                                const uint8_t* status_dev, int32_t* accepted_dev, int32_t* token_dev,
                                                void* cuda_stream) {
  lc::NvtxRange nvtx("lacache_verify_sample");
  if (B < 1 || k < 0 || k > lc::kMaxK || vocab < 1 || !p_target || !p_target->data_dev || (k > 0 && !drafts_dev) || !u_dev ||
      !accepted_dev || !token_dev || (p_draft && k > 0 && !p_draft->data_dev))
    return LACACHE_ERR_INVALID_ARG;
  if (vocab > lc::kMaxVocab) return LACACHE_ERR_UNSUPPORTED;
  // (queries are done in no order)
  const int64_t out_bytes = (int64_t)B * 4, draft_bytes = out_bytes * k;
  if (lc::overlap(accepted_dev, out_bytes, token_dev, out_bytes)) return LACACHE_ERR_INVALID_ARG;
  for (const int32_t* out : {accepted_dev, token_dev})
    if (lc::overlap(out, out_bytes, drafts_dev, draft_bytes) || lc::overlap(out, out_bytes, u_dev, draft_bytes + out_bytes) ||
        lc::overlap(out, out_bytes, status_dev, B))
      return LACACHE_ERR_INVALID_ARG;
  lc::SampleArgs a = {};
  a.k = k;
  a.vocab = vocab;
  a.target = lc::Probs{p_target->data_dev, p_target->seq_stride, p_target->token_stride};
  if (p_draft && k > 0) a.draft = lc::Probs{p_draft->data_dev, p_draft->seq_stride, p_draft->token_stride};
  a.drafts = drafts_dev;
  a.u = u_dev;
  a.status = status_dev;
  a.accepted = accepted_dev;
  a.token = token_dev;
  // as many blocks a query as leave each 1,024 tokens, eight an SM at most
  a.blocks = 1;
  while (a.blocks < lc::kMaxCluster && vocab / (2 * a.blocks) >= 1024 && (int64_t)B * 2 * a.blocks <= lc::kSampleResident)
    a.blocks *= 2;
  const int warps = a.blocks * lc::kSampleWarps;
  a.run = (vocab + warps - 1) / warps;
  if ((int64_t)B * a.blocks > INT32_MAX) return LACACHE_ERR_UNSUPPORTED;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3((unsigned)(B * a.blocks));
  cfg.blockDim = dim3(lc::kSampleThreads);
  cfg.stream = (cudaStream_t)cuda_stream;
  cudaLaunchAttribute attr;
  attr.id = cudaLaunchAttributeClusterDimension;
  attr.val.clusterDim.x = (unsigned)a.blocks;
  attr.val.clusterDim.y = attr.val.clusterDim.z = 1;
  cfg.attrs = &attr;
  cfg.numAttrs = 1;
  return lc::from_cuda(cudaLaunchKernelEx(&cfg, lc::verify_sample_kernel, a));
}
