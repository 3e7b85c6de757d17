// Shared by the decoding operators (rope.cu, kv_cache.cu, kv_attend.cu): rows of heads in 16-byte chunks, the rotation of a
// chunk, the cache's formats, and the handle.
//
// A row of head_dim elements is held by a group of lanes, eight consecutive elements (a chunk) a lane. Groups have a power
// of two of lanes, so that a row's maximum is a butterfly within the group; lanes past head_dim / 8 idle.
#pragma once

#include <cuda_fp16.h>
#include <cuda_fp8.h>

#include "internal.cuh"

struct lacache_kv {
  lacache_kv_config cfg;
  int num_sms;
  unsigned char* arena;      // one device allocation: pools, scales, the attention's scratch, status word
  size_t layer_bytes;        // K (or V) pages of one layer
  size_t layer_scales;       // scales of K (or V) of one layer, in floats (0 in 16-bit formats)
  unsigned char* k;          // [layers] pools
  unsigned char* v;
  float* ks;                 // [layers] scales, or nullptr
  float* vs;
  float* partial;            // the attention's partial sums, two slots a block
  unsigned int* arrived;     // its counters, one a block (each launch leaves them zero)
  unsigned int* dev_status;  // kBadIndex once a kernel met an index outside its range
};

namespace lc {

constexpr unsigned int kBadIndex = 1u;
constexpr int kMaxHeadDim = LACACHE_MAX_HEAD_DIM;
constexpr int kMaxNewTokens = 512;

struct Rows {   // lacache_rows on the device
  unsigned char* p;
  int64_t token;   // bytes
  int64_t head;
};

inline int dtype_bytes(int dtype) { return dtype == LACACHE_F32 ? 4 : 2; }
inline bool known_dtype(int dtype) { return dtype == LACACHE_BF16 || dtype == LACACHE_F32 || dtype == LACACHE_F16; }
inline bool is_quantised(int format) { return format == LACACHE_KV_E4M3 || format == LACACHE_KV_INT8; }

// *r as device rows; false if its address or strides are not multiples of 16 bytes.
inline bool device_rows(const lacache_rows* r, int dtype, Rows* out) {
  const int64_t b = dtype_bytes(dtype);
  if (!r || !r->data || !aligned16(r->data) || (r->token_stride * b) % 16 || (r->head_stride * b) % 16) return false;
  *out = Rows{static_cast<unsigned char*>(r->data), r->token_stride * b, r->head_stride * b};
  return true;
}

struct Table {
  const int32_t* pages;
  int64_t stride;
  int seqs, width;
};
inline bool device_table(const lacache_kv_table* t, Table* out) {
  if (!t || t->seqs < 0 || t->width < 1 || (t->seqs > 0 && !t->pages_dev)) return false;
  *out = Table{t->pages_dev, t->row_stride, t->seqs, t->width};
  return true;
}

// The row kernels give a warp one token and a slab of its rows, kRowUnroll passes of 32 / lanes rows in flight. A slab is all
// of a token's rows when the tokens alone fill the GPU; fewer tokens are cut into slabs of at least one pass.
constexpr int kRowThreads = 128;
constexpr int kRowUnroll = 4;
constexpr int64_t kRowWarps = 4096;   // about 27 warps an SM
struct RowPlan {
  int slab;          // rows
  int64_t tasks;     // tokens x slabs, one a warp
  unsigned blocks;
};
inline RowPlan plan_rows(int64_t n, int rows, int lanes) {
  const int pass = 32 / lanes, passes = (rows + pass - 1) / pass;
  int64_t slabs = (kRowWarps + n - 1) / n;
  if (slabs > passes) slabs = passes;
  RowPlan p;
  p.slab = (int)((passes + slabs - 1) / slabs) * pass;
  p.tasks = n * ((rows + p.slab - 1) / p.slab);
  const int64_t blocks = (p.tasks + kRowThreads / 32 - 1) / (kRowThreads / 32);
  p.blocks = (unsigned)(blocks < (1 << 30) ? blocks : 1 << 30);
  return p;
}

// Lanes of a group: the power of two that holds head_dim / 8 chunks.
inline int lanes_for(int head_dim) {
  int n = 1;
  while (n * 8 < head_dim) n *= 2;
  return n;
}

namespace {

// Eight elements of a row, as loaded and as fp32, and back.
__device__ __forceinline__ void widen8(uint4 u, float (&x)[8], __nv_bfloat16) {
  const uint32_t w[4] = {u.x, u.y, u.z, u.w};
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    x[2 * i] = __uint_as_float(w[i] << 16);
    x[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u);
  }
}
__device__ __forceinline__ void widen8(uint4 u, float (&x)[8], __half) {
  const uint32_t w[4] = {u.x, u.y, u.z, u.w};
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const float2 f = __half22float2(*reinterpret_cast<const __half2*>(&w[i]));
    x[2 * i] = f.x;
    x[2 * i + 1] = f.y;
  }
}
template <typename T>
struct Chunk {
  typedef uint4 raw;
  static __device__ __forceinline__ raw load(const unsigned char* p) { return *reinterpret_cast<const uint4*>(p); }
  static __device__ __forceinline__ void widen(raw u, float (&x)[8]) { widen8(u, x, T()); }
};
template <>
struct Chunk<float> {
  struct raw {
    float4 a, b;
  };
  static __device__ __forceinline__ raw load(const unsigned char* p) {
    return raw{reinterpret_cast<const float4*>(p)[0], reinterpret_cast<const float4*>(p)[1]};
  }
  static __device__ __forceinline__ void widen(const raw& u, float (&x)[8]) {
    x[0] = u.a.x, x[1] = u.a.y, x[2] = u.a.z, x[3] = u.a.w, x[4] = u.b.x, x[5] = u.b.y, x[6] = u.b.z, x[7] = u.b.w;
  }
};
__device__ __forceinline__ uint4 pack8(const float (&x)[8], __nv_bfloat16) {
  uint32_t w[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const __nv_bfloat162 h = __floats2bfloat162_rn(x[2 * i], x[2 * i + 1]);
    w[i] = *reinterpret_cast<const uint32_t*>(&h);
  }
  return make_uint4(w[0], w[1], w[2], w[3]);
}
__device__ __forceinline__ uint4 pack8(const float (&x)[8], __half) {
  uint32_t w[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const __half2 h = __floats2half2_rn(x[2 * i], x[2 * i + 1]);
    w[i] = *reinterpret_cast<const uint32_t*>(&h);
  }
  return make_uint4(w[0], w[1], w[2], w[3]);
}
__device__ __forceinline__ void store8(__nv_bfloat16* p, const float (&x)[8]) {
  *reinterpret_cast<uint4*>(p) = pack8(x, __nv_bfloat16());
}
__device__ __forceinline__ void store8(__half* p, const float (&x)[8]) {
  *reinterpret_cast<uint4*>(p) = pack8(x, __half());
}
__device__ __forceinline__ void store8(float* p, const float (&x)[8]) {
  reinterpret_cast<float4*>(p)[0] = make_float4(x[0], x[1], x[2], x[3]);
  reinterpret_cast<float4*>(p)[1] = make_float4(x[4], x[5], x[6], x[7]);
}

// cos and sin, times the amplitude, of pair i at `pos`, the sine times `sign` (-1 for the inverse). The phase position * turn is exact modulo a turn; its upper 32 bits
// are the fraction of a turn in [-1/2, 1/2), to 2^-33, at every position.
__device__ __forceinline__ float2 rope_angle(const lacache_rope& r, int i, int pos, float sign) {
  const uint64_t phase = r.turn[i] * (uint64_t)(int64_t)pos;
  const float half_turns = (float)(int32_t)(uint32_t)(phase >> 32) * 4.656612873077393e-10f;   // 2^-31: in half turns
  float s, c;
  sincospif(half_turns, &s, &c);
  return make_float2(c * r.amplitude, s * r.amplitude * sign);
}

// One rotated element: x cos -+ y sin, with the roundings fixed, so that every kernel gives the same bits.
__device__ __forceinline__ float turn_first(float x, float y, float2 a) { return __fmaf_rn(x, a.x, -__fmul_rn(y, a.y)); }
__device__ __forceinline__ float turn_second(float x, float y, float2 a) { return __fmaf_rn(x, a.x, __fmul_rn(y, a.y)); }

// A warp's angles of one token: every pair once, through shared memory, then those of this lane's chunk c into registers,
// where they serve all heads. a[i] belongs to element 8c + i in the half layout, to pair 4c + i (i < 4) in the other.
__device__ __forceinline__ void warp_angles(const lacache_rope& r, int pos, float sign, int c, float2* cs, float2 (&a)[8]) {
  const int lane = threadIdx.x & 31, h = r.rot_dim >> 1;
  __syncwarp();
  for (int i = lane; i < h; i += 32) cs[i] = rope_angle(r, i, pos, sign);
  __syncwarp();
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const int d = c * 8 + i;
    const int at = r.layout == LACACHE_ROPE_INTERLEAVED ? c * 4 + i : d < h ? d : d - h;
    a[i] = at < h ? cs[at] : make_float2(1.f, 0.f);
  }
}

// Rotates chunk c (elements 8c .. 8c+7) of the row whose chunk this lane holds in x, by the angles of warp_angles. All lanes
// of the warp call it. In the half layout the partner of a chunk is a whole chunk of another lane of the group (`lanes`
// wide) when rot_dim / 2 is a multiple of 8; `row` serves the other sizes, whose partners lie across chunks: the row's
// elements in memory, still unrotated (the caller stores only after __syncwarp).
template <typename T>
__device__ __forceinline__ void rotate8(float (&x)[8], int c, int lanes, int rot, int layout, const float2 (&a)[8],
                                        const T* row) {
  const int d0 = c * 8;
  if (layout == LACACHE_ROPE_INTERLEAVED) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      if (d0 + 2 * i < rot) {
        const float u = x[2 * i], v = x[2 * i + 1];
        x[2 * i] = turn_first(u, v, a[i]);
        x[2 * i + 1] = turn_second(v, u, a[i]);
      }
    }
    return;
  }
  const int h = rot >> 1;
  float y[8];
  if ((h & 7) == 0) {
    const bool first = d0 < h;
    const int src = (threadIdx.x & 31 & ~(lanes - 1)) | ((first ? c + (h >> 3) : c - (h >> 3)) & (lanes - 1));
#pragma unroll
    for (int i = 0; i < 8; ++i) y[i] = __shfl_sync(0xffffffffu, x[i], src);
    if (d0 < rot) {
#pragma unroll
      for (int i = 0; i < 8; ++i) x[i] = first ? turn_first(x[i], y[i], a[i]) : turn_second(x[i], y[i], a[i]);
    }
    return;
  }
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const int d = d0 + i;
    y[i] = row && d < rot ? (float)row[d < h ? d + h : d - h] : 0.f;
  }
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const int d = d0 + i;
    if (d < rot) x[i] = d < h ? turn_first(x[i], y[i], a[i]) : turn_second(x[i], y[i], a[i]);
  }
}

// The row's scale in an 8-bit format and its codes: scale = amax / top, code = x / scale to nearest even, both IEEE
// divisions. NaN for a row that holds an infinity or a NaN (its codes are 0).
template <int FMT>
__device__ __forceinline__ float row_scale(const float (&x)[8], int lanes) {
  float m = 0.f;
  bool bad = false;
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    m = fmaxf(m, fabsf(x[i]));
    bad |= !(fabsf(x[i]) <= 3.402823466e+38f);
  }
  if (bad) m = __int_as_float(0x7f800000);
  for (int o = lanes >> 1; o; o >>= 1) m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, o));
  if (m == __int_as_float(0x7f800000)) return __int_as_float(0x7fc00000);
  return __fdiv_rn(m, FMT == LACACHE_KV_E4M3 ? 448.f : 127.f);
}
template <int FMT>
__device__ __forceinline__ uint2 quantise8(const float (&x)[8], float scale) {
  uint32_t w[2] = {0, 0};
  if (scale > 0.f) {
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const float u = __fdiv_rn(x[i], scale);
      uint32_t code;
      if (FMT == LACACHE_KV_E4M3) {
        code = __nv_cvt_float_to_fp8(u, __NV_SATFINITE, __NV_E4M3);
      } else {
        code = (uint32_t)(int)fminf(fmaxf(rintf(u), -127.f), 127.f) & 0xffu;
      }
      w[i >> 2] |= code << (8 * (i & 3));
    }
  }
  return make_uint2(w[0], w[1]);
}
template <int FMT>
__device__ __forceinline__ void dequantise8(uint2 u, float scale, float (&x)[8]) {
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const uint32_t code = ((i < 4 ? u.x : u.y) >> (8 * (i & 3))) & 0xffu;
    if (FMT == LACACHE_KV_E4M3)
      x[i] = __half2float(__half(__nv_cvt_fp8_to_halfraw((__nv_fp8_storage_t)code, __NV_E4M3))) * scale;
    else
      x[i] = (float)(int)(int8_t)code * scale;
  }
}

// The cache row index (page * heads + head) * page_size + slot of a token, without the head: page * heads * page_size + slot,
// or -1 where an index is outside its range (and then *status, if given, says so) or seq is -1.
__device__ __forceinline__ int64_t slot_row(const Table& t, int seq, int pos, int heads, int page_size, int64_t pages,
                                            unsigned int* status) {
  if (seq == -1) return -1;
  if (seq >= 0 && seq < t.seqs && pos >= 0 && pos / page_size < t.width) {
    const int page = t.pages[seq * t.stride + pos / page_size];
    if (page >= 0 && page < pages) return (int64_t)page * heads * page_size + pos % page_size;
  }
  if (status) atomicOr(status, kBadIndex);
  return -1;
}

}  // namespace
}  // namespace lc
