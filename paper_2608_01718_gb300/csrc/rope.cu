// Rotary positions of rows of heads, and their gradient (the rotation by the negated angles).
//
// Bound by memory: each element is read and written once. For each of its tokens a warp computes the angles once, holds those
// of its lanes' chunks in registers, and runs over the heads. The plan (rotations as fractions of 2^64 a position) is a kernel
// argument. Measured: 16,384 tokens of 32 heads, d = 128, bf16, 43.6 us, 6.2 TB/s; one token 2.8 us.
#include <math.h>

#include "decode.cuh"

namespace lc {
namespace {

// Blocks an SM, and passes in flight: four of 16-bit rows (16,384 x 32 x 128 of bf16: two, at eight blocks an SM, 48 us; four
// 43.6); two where a lane's rows or partners take twice the registers.
constexpr int kRopeBlocks = 5;

template <typename T, int MODE>
__global__ void __launch_bounds__(kRowThreads, kRopeBlocks)
    rope_kernel(const __grid_constant__ lacache_rope rope, const __grid_constant__ RowPlan plan, int chunks, int lanes,
                const __grid_constant__ Rows x, const int32_t* __restrict__ pos, float sign, const __grid_constant__ Rows y) {
  constexpr int kUnroll = sizeof(T) == 4 || MODE == kRopeOdd ? 2 : 4;
  __shared__ float2 cs[kRowThreads / 32][kMaxHeadDim / 2];
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const int pass = 32 / lanes, sub = lane / lanes;
  const Chunks m = chunks_of<MODE>(lane & (lanes - 1), chunks, rope.rot_dim);
  const int64_t step = (int64_t)gridDim.x * (kRowThreads / 32);
  for (int64_t task = blockIdx.x * (int64_t)(kRowThreads / 32) + warp; task < plan.tasks; task += step) {
    const int64_t t = task / plan.slabs;
    const int first = (int)(task - t * plan.slabs) * plan.slab;
    const int end = first + plan.slab < plan.rows ? first + plan.slab : plan.rows;
    const unsigned char* src = x.at(t, first + sub);
    unsigned char* dst = y.at(t, first + sub);
    const int64_t src_step = (int64_t)pass * x.head16 * 16, dst_step = (int64_t)pass * y.head16 * 16;
    float2 a[8];
    warp_angles<MODE>(rope, pos[t], sign, m, cs[warp], a);
    for (int h = first + sub; h - sub < end; h += kUnroll * pass) {
      typename Chunk<T>::raw raw[kUnroll][2];
#pragma unroll
      for (int i = 0; i < kUnroll; ++i) {
#pragma unroll
        for (int k = 0; k < 2; ++k)
          if (h + i * pass < end && m.live[k])
            raw[i][k] = Chunk<T>::load(src + i * src_step + m.c[k] * (8 * (int)sizeof(T)));
      }
#pragma unroll
      for (int i = 0; i < kUnroll; ++i) {
        const bool live = h + i * pass < end;
        float v0[8], v1[8];
        Chunk<T>::widen(raw[i][0], v0);
        Chunk<T>::widen(raw[i][1], v1);
        rotate<MODE>(v0, v1, m, rope.rot_dim, rope.layout, a, cs[warp],
                     live ? reinterpret_cast<const T*>(src + i * src_step) : nullptr);
        if (MODE == kRopeOdd) __syncwarp();
        T* to = reinterpret_cast<T*>(dst + i * dst_step);
        if (live && m.live[0]) store8(to + m.c[0] * 8, v0);
        if (live && m.live[1]) store8(to + m.c[1] * 8, v1);
      }
      src += kUnroll * src_step;
      dst += kUnroll * dst_step;
    }
  }
}

template <typename T>
void launch_rope(int mode, const lacache_rope& rope, int64_t n, int heads, int head_dim, const Rows& x, const int32_t* pos,
                 float sign, const Rows& y, cudaStream_t st) {
  const int lanes = lanes_for(head_dim, rope.rot_dim, mode);
  unsigned grid;
  const RowPlan plan = plan_rows(n, heads, lanes, kRopeBlocks, 1, &grid);
  auto* kernel = mode == kRopeHalf   ? rope_kernel<T, kRopeHalf>
                 : mode == kRopeNear ? rope_kernel<T, kRopeNear>
                                     : rope_kernel<T, kRopeOdd>;
  kernel<<<grid, kRowThreads, 0, st>>>(rope, plan, head_dim / 8, lanes, x, pos, sign, y);
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
       !isfinite(high_turns) || !isfinite(high_turns - low_turns)))
    return LACACHE_ERR_INVALID_ARG;
  lacache_rope r = {};
  r.rot_dim = rot_dim;
  r.layout = layout;
  r.amplitude = amplitude;
  if (scaling == LACACHE_ROPE_BASE) base *= pow(factor, (double)rot_dim / (rot_dim - 2));
  if (!(base > 0.0) || !isfinite(base)) return LACACHE_ERR_INVALID_ARG;
  const double two_pi = 6.283185307179586476925;
  for (int i = 0; i < rot_dim / 2; ++i) {
    double turns = pow(base, -2.0 * i / rot_dim) / two_pi;   // a position
    if (scaling == LACACHE_ROPE_LINEAR) turns /= factor;
    if (scaling == LACACHE_ROPE_BANDED) {
      double g = (original_len * turns - low_turns) / (high_turns - low_turns);
      g = g < 0.0 ? 0.0 : g > 1.0 ? 1.0 : g;
      turns = (1.0 - g) * turns / factor + g * turns;
    }
    if (!isfinite(turns)) return LACACHE_ERR_INVALID_ARG;
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
  if (head_dim % 8 || head_dim > lc::kMaxHeadDim || heads > lc::kMaxRowHeads) return LACACHE_ERR_UNSUPPORTED;
  if (n == 0) return LACACHE_OK;
  if (!pos_dev || !lc::device_rows(x, dtype, &xr) || !lc::device_rows(y, dtype, &yr)) return LACACHE_ERR_INVALID_ARG;
  const float sign = inverse ? -1.f : 1.f;
  const int mode = lc::rope_mode(rope);
  const cudaStream_t st = (cudaStream_t)cuda_stream;
  if (dtype == LACACHE_BF16) lc::launch_rope<__nv_bfloat16>(mode, *rope, n, heads, head_dim, xr, pos_dev, sign, yr, st);
  else if (dtype == LACACHE_F16) lc::launch_rope<__half>(mode, *rope, n, heads, head_dim, xr, pos_dev, sign, yr, st);
  else lc::launch_rope<float>(mode, *rope, n, heads, head_dim, xr, pos_dev, sign, yr, st);
  return lc::from_cuda(cudaGetLastError());
}
