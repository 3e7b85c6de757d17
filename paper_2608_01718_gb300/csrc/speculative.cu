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
// Programming", vol. 2, 4.2.2), sums of them as a leading sum and the sum of its rounding errors (some 2^-45 of the whole),
// and C_i near the border in fp64. In fp32 alone, sums over 10^5 tokens would draw a neighbour of the token in some percent
// of the calls; in fp64 alone, the differences and sums of a row of 10^5 take longer than reading it.
//
// A cluster of 1 to 8 blocks a query, each warp a run of consecutive tokens, with sixteen loads in flight a lane. The runs'
// sums are exchanged through the cluster's shared memory; the block that holds the border adds its run again in fp64, a few
// consecutive tokens a thread.
constexpr int kSampleThreads = 256, kSampleWarps = kSampleThreads / 32, kMaxCluster = 8;
constexpr int kSampleUnroll = 8;
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
// a + x - y for x > y >= 0
__device__ __forceinline__ void add_difference(Twofold& a, float x, float y) {
  const float d = __fsub_rn(x, y), b = __fsub_rn(d, x);
  const float d_err = __fsub_rn(__fsub_rn(x, __fsub_rn(d, b)), __fadd_rn(y, b));
  const float s = __fadd_rn(a.sum, d), c = __fsub_rn(s, a.sum);
  const float s_err = __fadd_rn(__fsub_rn(a.sum, __fsub_rn(s, c)), __fsub_rn(d, c));
  a.sum = s;
  a.rest = __fadd_rn(a.rest, __fadd_rn(s_err, d_err));
}
__device__ __forceinline__ double inclusive_sum(double x) {   // over the warp's lanes
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const double y = __shfl_up_sync(0xffffffffu, x, o);
    if ((threadIdx.x & 31) >= o) x += y;
  }
  return x;
}

__global__ void __launch_bounds__(kSampleThreads) verify_sample_kernel(const __grid_constant__ SampleArgs a) {
  namespace cg = cooperative_groups;
  cg::cluster_group cluster = cg::this_cluster();
  __shared__ double run_sum[kSampleWarps], all_sum[kSampleWarps * kMaxCluster], warp_sum[kSampleWarps];
  __shared__ int first_past, last_some;
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const int64_t b = blockIdx.x / a.blocks;
  const int rank = blockIdx.x - (int)b * a.blocks, runs = a.blocks * kSampleWarps;
  if (a.status && a.status[b] == LACACHE_HIT) {
    if (rank == 0 && threadIdx.x == 0) a.accepted[b] = a.token[b] = -1;
    return;
  }
  // how many drafts are accepted, and which one, if any, was refused: every warp for itself
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
  const float* p = a.target.data + b * a.target.seq + n * a.target.token;
  const double u = a.u[b * (a.k + 1) + a.k];
  int token = -1;
  // a second time with p alone where p - q leaves no weight
  for (int attempt = refused >= 0 ? 0 : 1; attempt < 2; ++attempt) {
    const float* q = attempt == 0 && a.draft.data ? a.draft.data + b * a.draft.seq + n * a.draft.token : nullptr;
    const int one = attempt == 0 && !a.draft.data ? refused : -1;   // where q is 1, if it has no row
    auto less = [&](int i) { return q ? q[i] : i == one ? 1.f : 0.f; };
    const int first = (int)min((int64_t)(rank * kSampleWarps + warp) * a.run, (int64_t)a.vocab);
    const int end = (int)min((int64_t)first + a.run, (int64_t)a.vocab);
    Twofold sum = {0.f, 0.f};
    for (int i0 = first + lane; i0 < end; i0 += 32 * kSampleUnroll) {
      float x[kSampleUnroll], y[kSampleUnroll];
#pragma unroll
      for (int e = 0; e < kSampleUnroll; ++e) {
        const int i = i0 + 32 * e;
        x[e] = i < end ? p[i] : 0.f;
        y[e] = i < end ? less(i) : 0.f;
      }
#pragma unroll
      for (int e = 0; e < kSampleUnroll; ++e)
        if (x[e] > y[e]) add_difference(sum, x[e], y[e]);
    }
    const double mine = inclusive_sum((double)sum.sum + (double)sum.rest);
    if (lane == 31) run_sum[warp] = mine;
    cluster.sync();
    if (threadIdx.x < runs)
      all_sum[threadIdx.x] = *cluster.map_shared_rank(&run_sum[threadIdx.x % kSampleWarps], threadIdx.x / kSampleWarps);
    if (threadIdx.x == 0) {
      first_past = kSampleThreads;
      last_some = -1;
    }
    __syncthreads();
    // the run that the border lies in: two runs a lane
    const double s0 = 2 * lane < runs ? all_sum[2 * lane] : 0.0, s1 = 2 * lane + 1 < runs ? all_sum[2 * lane + 1] : 0.0;
    const double upto = inclusive_sum(s0 + s1), total = __shfl_sync(0xffffffffu, upto, 31);
    const double before_lane = __shfl_up_sync(0xffffffffu, upto, 1);
    const double c0 = lane ? before_lane : 0.0, c1 = c0 + s0;
    const double target = u * total;
    const unsigned past0 = __ballot_sync(0xffffffffu, s0 > 0.0 && c1 > target), past1 = __ballot_sync(0xffffffffu, s1 > 0.0 && upto > target);
    const unsigned some0 = __ballot_sync(0xffffffffu, s0 > 0.0), some1 = __ballot_sync(0xffffffffu, s1 > 0.0);
    int run;
    if (past0 | past1) {
      const int l = __ffs(past0 | past1) - 1;
      run = 2 * l + (past0 >> l & 1 ? 0 : 1);
    } else {   // (u at or above 1, or sums that are not finite): the last that has any weight
      const int l = 31 - __clz(some0 | some1);
      run = some0 | some1 ? 2 * l + (some1 >> l & 1 ? 1 : 0) : -1;
    }
    const double base = __shfl_sync(0xffffffffu, run & 1 ? c1 : c0, run < 0 ? 0 : run >> 1);
    if (run >= 0 && run / kSampleWarps == rank) {
      // its tokens again, a few consecutive ones a thread
      const int from = run * a.run, upto_token = (int)min((int64_t)from + a.run, (int64_t)a.vocab);
      const int each = (a.run + kSampleThreads - 1) / kSampleThreads;
      const int i0 = (int)min((int64_t)from + threadIdx.x * each, (int64_t)upto_token), i1 = min(i0 + each, upto_token);
      double own = 0.0;
      for (int i = i0; i < i1; ++i) {
        const float x = p[i], y = less(i);
        if (x > y) own += (double)x - (double)y;
      }
      const double in_warp = inclusive_sum(own);
      if (lane == 31) warp_sum[warp] = in_warp;
      __syncthreads();
      double before = base;
      for (int w = 0; w < warp; ++w) before += warp_sum[w];
      const double prior = __shfl_up_sync(0xffffffffu, in_warp, 1);
      double c = before + (lane ? prior : 0.0);
      if (own > 0.0) {
        atomicMax(&last_some, (int)threadIdx.x);
        if (before + in_warp > target) atomicMin(&first_past, (int)threadIdx.x);
      }
      __syncthreads();
      if ((int)threadIdx.x == (first_past < kSampleThreads ? first_past : last_some)) {
        for (int i = i0; i < i1; ++i) {
          const float x = p[i], y = less(i);
          if (!(x > y)) continue;
          token = i;
          c += (double)x - (double)y;
          if (c > target) break;
        }
        a.accepted[b] = n;
        a.token[b] = token;
      }
    }
    cluster.sync();   // the sums have been read
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
  // as many blocks a query as leave each 1,024 tokens, and all of them resident at once
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
