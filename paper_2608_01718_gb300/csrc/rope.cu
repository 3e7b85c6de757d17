// Rotary positions of rows of heads, and their gradient (the rotation by the negated angles).
//
// Bound by memory: each element is read and written once. A token's angles are computed once, into shared memory, and serve
// all its heads. The plan (rotations as fractions of 2^64 a position) is a kernel argument.
#include <math.h>

#include "decode.cuh"

namespace lc {
namespace {

constexpr int kRopeThreads = 256;

template <typename T>
__global__ void __launch_bounds__(kRopeThreads)
    rope_kernel(const __grid_constant__ lacache_rope rope, int64_t n, int heads, int chunks, int lanes, Rows x,
                const int32_t* __restrict__ pos, float sign, Rows y) {
  __shared__ float2 cs[kMaxHeadDim / 2];
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const int rows_warp = 32 / lanes, c = lane & (lanes - 1), sub = lane / lanes;
  for (int64_t t = blockIdx.x; t < n; t += gridDim.x) {
    __syncthreads();
    if (threadIdx.x < rope.rot_dim / 2) cs[threadIdx.x] = rope_angle(rope, threadIdx.x, pos[t], sign);
    __syncthreads();
    for (int h0 = warp * rows_warp; h0 < heads; h0 += (kRopeThreads / 32) * rows_warp) {
      const int h = h0 + sub;
      const bool live = h < heads && c < chunks;
      const T* row = reinterpret_cast<const T*>(x.p + t * x.token + (h < heads ? h : 0) * x.head);
      float v[8] = {};
      if (live) load8(row + c * 8, v);
      rotate8(v, c, lanes, rope.rot_dim, rope.layout, cs, row);
      __syncwarp();
      if (live) store8(reinterpret_cast<T*>(y.p + t * y.token + h * y.head) + c * 8, v);
    }
  }
}

}  // namespace
}  // namespace lc

extern "C" lacache_status lacache_rope_init(int32_t rot_dim, int32_t layout, double base, int32_t scaling, double factor,
                                            double original_len, double low_turns, double high_turns, float amplitude,
                                            lacache_rope* out) {
  if (!out || rot_dim < 2 || rot_dim % 2 || rot_dim > lc::kMaxHeadDim) return LACACHE_ERR_INVALID_ARG;
  if (layout != LACACHE_ROPE_HALF && layout != LACACHE_ROPE_INTERLEAVED) return LACACHE_ERR_INVALID_ARG;
  if (scaling < LACACHE_ROPE_PLAIN || scaling > LACACHE_ROPE_BANDED) return LACACHE_ERR_INVALID_ARG;
  if (!(base > 1.0) || !isfinite(base) || !isfinite(amplitude)) return LACACHE_ERR_INVALID_ARG;
  if (scaling != LACACHE_ROPE_PLAIN && (!(factor > 0.0) || !isfinite(factor))) return LACACHE_ERR_INVALID_ARG;
  if (scaling == LACACHE_ROPE_BASE && rot_dim < 4) return LACACHE_ERR_INVALID_ARG;
  if (scaling == LACACHE_ROPE_BANDED &&
      (!(original_len > 0.0) || !isfinite(original_len) || !(low_turns < high_turns) || !isfinite(low_turns) ||
       !isfinite(high_turns)))
    return LACACHE_ERR_INVALID_ARG;
  lacache_rope r = {};
  r.rot_dim = rot_dim;
  r.layout = layout;
  r.amplitude = amplitude;
  if (scaling == LACACHE_ROPE_BASE) base *= pow(factor, (double)rot_dim / (rot_dim - 2));
  if (!isfinite(base)) return LACACHE_ERR_INVALID_ARG;
  const double two_pi = 6.283185307179586476925;
  for (int i = 0; i < rot_dim / 2; ++i) {
    double turns = pow(base, -2.0 * i / rot_dim) / two_pi;   // a position
    if (scaling == LACACHE_ROPE_LINEAR) turns /= factor;
    if (scaling == LACACHE_ROPE_BANDED) {
      double g = (original_len * turns - low_turns) / (high_turns - low_turns);
      g = g < 0.0 ? 0.0 : g > 1.0 ? 1.0 : g;
      turns = (1.0 - g) * turns / factor + g * turns;
    }
    const double phase = ldexp(turns - floor(turns), 64);   // in [0, 2^64]
    r.turn[i] = phase >= 18446744073709551616.0 ? 0u : (uint64_t)phase;
  }
  *out = r;
  return LACACHE_OK;
}

extern "C" lacache_status lacache_rope_apply(const lacache_rope* rope, int64_t n, int32_t heads, int32_t head_dim,
                                             int32_t dtype, const lacache_rows* x, const int32_t* pos_dev,
                                             int32_t inverse, const lacache_rows* y, void* cuda_stream) {
  lc::NvtxRange nvtx("lacache_rope_apply");
  lc::Rows xr, yr;
  if (!rope || n < 0 || heads < 1 || head_dim < 1 || !lc::known_dtype(dtype)) return LACACHE_ERR_INVALID_ARG;
  if (rope->rot_dim < 2 || rope->rot_dim % 2 || rope->rot_dim > head_dim) return LACACHE_ERR_INVALID_ARG;
  if (head_dim % 8 || head_dim > lc::kMaxHeadDim) return LACACHE_ERR_UNSUPPORTED;
  if (n == 0) return LACACHE_OK;
  if (!pos_dev || !lc::device_rows(x, dtype, &xr) || !lc::device_rows(y, dtype, &yr)) return LACACHE_ERR_INVALID_ARG;
  const unsigned grid = (unsigned)(n < 65536 ? n : 65536);
  const int lanes = lc::lanes_for(head_dim);
  const float sign = inverse ? -1.f : 1.f;
  const cudaStream_t st = (cudaStream_t)cuda_stream;
  if (dtype == LACACHE_BF16)
    lc::rope_kernel<__nv_bfloat16><<<grid, lc::kRopeThreads, 0, st>>>(*rope, n, heads, head_dim / 8, lanes, xr, pos_dev,
                                                                     sign, yr);
  else if (dtype == LACACHE_F16)
    lc::rope_kernel<__half><<<grid, lc::kRopeThreads, 0, st>>>(*rope, n, heads, head_dim / 8, lanes, xr, pos_dev, sign, yr);
  else
    lc::rope_kernel<float><<<grid, lc::kRopeThreads, 0, st>>>(*rope, n, heads, head_dim / 8, lanes, xr, pos_dev, sign, yr);
  return lc::from_cuda(cudaGetLastError());
}
