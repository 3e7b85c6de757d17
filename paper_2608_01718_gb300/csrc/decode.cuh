// Shared by the decoding operators (rope.cu, kv_cache.cu, kv_attend.cu): rows of heads in 16-byte chunks, the rotation of a
// chunk, the cache's formats, and the handle.
//
// The row kernels hold a row of head_dim elements in a group of lanes, two chunks of eight consecutive elements a lane: the
// two halves of its pairs in the half layout, so that a rotation needs no exchange. Groups have a power of two of lanes, so
// that a row's maximum is a butterfly within the group; lanes past the row's chunks idle.
#pragma once

#include <cuda_fp16.h>
#include <cuda_fp8.h>

#include <type_traits>

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
  int inject_stall;          // attentions of many rows left that withhold a load (failure-detection tests)
  unsigned int* dev_status;  // kBadIndex: a kernel met an index outside its range; kAttendTimeout: a bounded wait ran out
};

namespace lc {

// Bits of a cache's status word.
constexpr unsigned int kBadIndex = 1u, kAttendTimeout = 2u;
constexpr int kMaxHeadDim = LACACHE_MAX_HEAD_DIM;
constexpr int kMaxNewTokens = 512;
constexpr int kMaxQHeads = 1 << 16;
constexpr int kMaxRowHeads = 1 << 30;   // of a rotation or a write: a token's rows, and some passes more, are counted in 32 bits

struct Rows {   // lacache_rows on the device
  unsigned char* p;
  int64_t token;   // bytes
  int head16;      // 16-byte units
  __device__ __forceinline__ unsigned char* at(int64_t t, int h) const { return p + t * token + (int64_t)h * head16 * 16; }
};

inline int dtype_bytes(int dtype) { return dtype == LACACHE_F32 ? 4 : 2; }
inline bool known_dtype(int dtype) { return dtype == LACACHE_BF16 || dtype == LACACHE_F32 || dtype == LACACHE_F16; }
inline bool is_quantised(int format) { return format == LACACHE_KV_E4M3 || format == LACACHE_KV_INT8; }

// *r as device rows; false if its address or strides are not multiples of 16 bytes (or its heads lie 32 GB apart).
inline bool device_rows(const lacache_rows* r, int dtype, Rows* out) {
  const int64_t b = dtype_bytes(dtype);
  if (!r || !r->data || !aligned16(r->data) || (r->token_stride * b) % 16 || (r->head_stride * b) % 16) return false;
  const int64_t head16 = r->head_stride * b / 16;
  if (head16 > INT32_MAX || head16 < INT32_MIN) return false;
  *out = Rows{static_cast<unsigned char*>(r->data), r->token_stride * b, (int)head16};
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

// The row kernels give a warp a group of tokens and a slab of their rows, kRowUnroll passes of 32 / lanes rows in flight. Few
// tokens are cut into slabs of at least one pass, until the warps fill the GPU; of many, a warp of the cache's kernels takes
// up to kRowGroup, whose places its lanes look up at once (write of 12,001 tokens of 48 rows: one 57.1 us, two 54.4, four
// 52.4; read of 60,000 of 16 rows: one 69.7, two 65.1, four 63.9, eight 72.8). Beyond that there are more blocks than the GPU holds.
constexpr int kRowThreads = 128;
constexpr int kRowUnroll = 2;
constexpr int kRowGroup = 4;
constexpr int kSms = 152;
struct RowPlan {
  int64_t n;         // tokens
  int rows, slab;    // of a token, and of a task
  int slabs, group;  // slabs of a token, tokens of a task
  int64_t tasks;
};
// `blocks`: blocks of the kernel an SM holds. `most`: tokens of a group. *grid: the launch's blocks.
inline RowPlan plan_rows(int64_t n, int rows, int lanes, int blocks, int most, unsigned* grid) {
  const int64_t resident = (int64_t)kSms * blocks * (kRowThreads / 32);
  const int pass = 32 / lanes, passes = (rows + pass - 1) / pass;
  int64_t slabs = resident / n, group = (n + resident - 1) / resident;
  slabs = slabs < 1 ? 1 : slabs > passes ? passes : slabs;
  group = group > most ? most : group;
  RowPlan p;
  p.n = n;
  p.rows = rows;
  p.slab = (int)((passes + slabs - 1) / slabs) * pass;
  p.slabs = (rows + p.slab - 1) / p.slab;
  p.group = (int)group;
  p.tasks = (n + group - 1) / group * p.slabs;
  const int64_t want = (p.tasks + kRowThreads / 32 - 1) / (kRowThreads / 32);
  *grid = (unsigned)(want < (1 << 30) ? want : 1 << 30);
  return p;
}

// How a rotation finds its pairs.
enum RopeMode {
  kRopeNone = 0,
  kRopeHalf = 1,    // pairs (i, i + rot_dim / 2), rot_dim / 2 a multiple of 8: whole chunks pair up
  kRopeNear = 2,    // pairs (2i, 2i + 1), rot_dim a multiple of 8
  kRopeOdd = 3      // either, of other sizes: partners are read from memory
};
inline int rope_mode(const lacache_rope* r) {
  if (!r) return kRopeNone;
  if (r->layout == LACACHE_ROPE_INTERLEAVED) return r->rot_dim % 8 ? kRopeOdd : kRopeNear;
  return r->rot_dim % 16 ? kRopeOdd : kRopeHalf;
}
// Lanes of a group.
inline int lanes_for(int head_dim, int rot_dim, int mode) {
  const int used = mode == kRopeHalf ? rot_dim / 16 + ((head_dim - rot_dim) / 8 + 1) / 2 : (head_dim / 8 + 1) / 2;
  int n = 1;
  while (n < used) n *= 2;
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

// cos and sin, times the amplitude, of pair i at `pos`, the sine times `sign` (-1 for the inverse). position * turn is exact
// modulo a turn, so the phase is as good as the turn that is stored (a double's 53 bits: position * 2^-55 of a turn or so, 2^-35
// at position 10^6 and 2^-24 at 2^31). Its upper 32 bits are the fraction of a turn in [-1/2, 1/2), cut to 2^-32.
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

// The chunks of lane p of a row's group: elements 8 c .. 8 c + 7.
struct Chunks {
  int c[2];
  bool live[2];
};
template <int MODE>
__device__ __forceinline__ Chunks chunks_of(int p, int chunks, int rot) {
  Chunks m;
  if (MODE == kRopeHalf) {
    const int pairs = rot / 16;
    m.c[0] = p < pairs ? p : 2 * p;   // past the rotated ones: rot / 8 + 2 (p - pairs)
    m.c[1] = p < pairs ? p + pairs : 2 * p + 1;
  } else {
    m.c[0] = p;
    m.c[1] = p + (chunks + 1) / 2;
  }
  m.live[0] = MODE == kRopeHalf ? m.c[0] < chunks : p < (chunks + 1) / 2;
  m.live[1] = m.live[0] && m.c[1] < chunks;
  return m;
}

// A warp's angles of one token: every pair once, through shared memory (which kRopeOdd keeps using), then this lane's into
// registers, where they serve all heads: those of the elements of chunk 0 in the half layout, of the four pairs of each
// chunk in the other.
template <int MODE>
__device__ __forceinline__ void warp_angles(const lacache_rope& r, int pos, float sign, const Chunks& m, float2* cs,
                                            float2 (&a)[8]) {
  const int lane = threadIdx.x & 31, h = r.rot_dim >> 1;
  __syncwarp();
  for (int i = lane; i < h; i += 32) cs[i] = rope_angle(r, i, pos, sign);
  __syncwarp();
  if constexpr (MODE != kRopeOdd) {
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const int at = MODE == kRopeHalf ? m.c[0] * 8 + i : m.c[i >> 2] * 4 + (i & 3);
      a[i] = at < h ? cs[at] : make_float2(1.f, 0.f);
    }
  }
}

// Rotates this lane's two chunks x0 and x1 of a row by the angles of warp_angles. kRopeOdd reads the partners from `row`, the
// row's elements in memory, still unrotated (nullptr: no row; the caller stores only after __syncwarp).
template <int MODE, typename T>
__device__ __forceinline__ void rotate(float (&x0)[8], float (&x1)[8], const Chunks& m, int rot, int layout,
                                       const float2 (&a)[8], const float2* cs, const T* row) {
  if (MODE == kRopeHalf) {
    if (m.c[0] * 8 >= rot) return;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const float u = x0[i], v = x1[i];
      x0[i] = turn_first(u, v, a[i]);
      x1[i] = turn_second(v, u, a[i]);
    }
  } else if (MODE == kRopeNear) {
#pragma unroll
    for (int k = 0; k < 2; ++k) {
      float(&x)[8] = k ? x1 : x0;
      if (m.c[k] * 8 < rot) {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const float u = x[2 * i], v = x[2 * i + 1];
          x[2 * i] = turn_first(u, v, a[4 * k + i]);
          x[2 * i + 1] = turn_second(v, u, a[4 * k + i]);
        }
      }
    }
  } else if (MODE == kRopeOdd) {
    const int h = rot >> 1;
    const bool near = layout == LACACHE_ROPE_INTERLEAVED;
    if (!row) return;
#pragma unroll
    for (int k = 0; k < 2; ++k) {
      float(&x)[8] = k ? x1 : x0;
      if (!m.live[k]) continue;
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const int d = m.c[k] * 8 + i;
        if (d >= rot) continue;
        const bool first = near ? !(d & 1) : d < h;
        const float y = (float)row[near ? d ^ 1 : first ? d + h : d - h];
        const float2 angle = cs[near ? d >> 1 : first ? d : d - h];
        x[i] = first ? turn_first(x[i], y, angle) : turn_second(x[i], y, angle);
      }
    }
  }
}

// Two fp32 at a time (kernels here that wait for memory least are bound by their instructions' issue), and the largest
// magnitude of three (NaN if one is).
__device__ __forceinline__ uint64_t bits_of(float2 x) { return (uint64_t)__float_as_uint(x.y) << 32 | __float_as_uint(x.x); }
__device__ __forceinline__ float2 pair_of(uint64_t u) {
  return make_float2(__uint_as_float((uint32_t)u), __uint_as_float((uint32_t)(u >> 32)));
}
__device__ __forceinline__ float2 fma_two(float2 x, float2 y, float2 z) {
  uint64_t d;
  asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(d) : "l"(bits_of(x)), "l"(bits_of(y)), "l"(bits_of(z)));
  return pair_of(d);
}
__device__ __forceinline__ float2 mul_two(float2 x, float2 y) {
  uint64_t d;
  asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(d) : "l"(bits_of(x)), "l"(bits_of(y)));
  return pair_of(d);
}
__device__ __forceinline__ float2 add_two(float2 x, float2 y) {
  uint64_t d;
  asm("add.rn.f32x2 %0, %1, %2;" : "=l"(d) : "l"(bits_of(x)), "l"(bits_of(y)));
  return pair_of(d);
}
__device__ __forceinline__ float largest(float x, float y, float z) {
  float d;
  asm("max.NaN.abs.f32 %0, %1, %2, %3;" : "=f"(d) : "f"(x), "f"(y), "f"(z));
  return d;
}

// The row's scale in an 8-bit format, amax / top by an IEEE division; NaN for a row that holds an infinity or a NaN (its codes
// are 0).
template <int FMT>
__device__ __forceinline__ float row_scale(const float (&x0)[8], const float (&x1)[8], int lanes) {
  float m = 0.f;
#pragma unroll
  for (int i = 0; i < 8; ++i) m = largest(m, x0[i], x1[i]);
  for (int o = lanes >> 1; o; o >>= 1) {
    const float y = __shfl_xor_sync(0xffffffffu, m, o);
    m = largest(m, y, y);
  }
  return m < INFINITY ? __fdiv_rn(m, FMT == LACACHE_KV_E4M3 ? 448.f : 127.f) : __int_as_float(0x7fc00000);
}
// x / scale correctly rounded, from r = 1 / scale correctly rounded: two of Markstein's corrections (P. Markstein,
// "Computation of elementary functions on the IBM RISC System/6000 processor", 1990): the first makes the quotient faithful,
// the second, from an exact remainder, correctly rounded. For scales within 2^+-100, where nothing under- or overflows
// (remainders below that belong to quotients whose code is 0).
__device__ __forceinline__ float2 quotients(float2 x, float scale, float r) {
  const float2 s = make_float2(-scale, -scale), t = make_float2(r, r);
  float2 q = mul_two(x, t);
  q = fma_two(fma_two(q, s, x), t, q);
  return fma_two(fma_two(q, s, x), t, q);
}
// The same for other scales. (A quotient of a plain scale is at most top, but for a rounding; a subnormal scale may be too
// small for its row.)
template <int FMT>
__device__ __noinline__ void far_quotients(float (&u)[8], float scale) {
#pragma unroll 1
  for (int i = 0; i < 8; ++i) {
    u[i] = __fdiv_rn(u[i], scale);
    if (FMT == LACACHE_KV_INT8) u[i] = fminf(fmaxf(u[i], -127.f), 127.f);
  }
}
// Codes of eight elements: x / scale (IEEE) to nearest, ties to even.
template <int FMT>
__device__ __forceinline__ uint2 quantise8(const float (&x)[8], float scale, float r) {
  if (!(scale > 0.f)) return make_uint2(0, 0);
  float2 u[4];
  if (scale > 0x1p-100f && scale < 0x1p100f) {
#pragma unroll
    for (int i = 0; i < 4; ++i) u[i] = quotients(make_float2(x[2 * i], x[2 * i + 1]), scale, r);
  } else {
    float y[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) y[i] = x[i];
    far_quotients<FMT>(y, scale);
#pragma unroll
    for (int i = 0; i < 4; ++i) u[i] = make_float2(y[2 * i], y[2 * i + 1]);
  }
  uint32_t w[2];
#pragma unroll
  for (int k = 0; k < 2; ++k) {
    if (FMT == LACACHE_KV_E4M3) {
      const uint32_t lo = __nv_cvt_float2_to_fp8x2(u[2 * k], __NV_SATFINITE, __NV_E4M3);
      const uint32_t hi = __nv_cvt_float2_to_fp8x2(u[2 * k + 1], __NV_SATFINITE, __NV_E4M3);
      w[k] = lo | hi << 16;
    } else {
      // adding 1.5 x 2^23 rounds to an integer in the low bits of the sum
      const float2 big = make_float2(12582912.f, 12582912.f), a = add_two(u[2 * k], big), b = add_two(u[2 * k + 1], big);
      w[k] = __byte_perm(__byte_perm(__float_as_uint(a.x), __float_as_uint(a.y), 0x0040),
                         __byte_perm(__float_as_uint(b.x), __float_as_uint(b.y), 0x0040), 0x5410);
    }
  }
  return make_uint2(w[0], w[1]);
}
// Four codes as f16 pairs: elements 0, 1 and 2, 3. Exact.
template <int FMT>
__device__ __forceinline__ void widen4(uint32_t u, uint32_t& lo, uint32_t& hi) {
  if constexpr (FMT == LACACHE_KV_E4M3) {
    asm("{\n\t.reg .b16 a, b;\n\tmov.b32 {a, b}, %2;\n\tcvt.rn.f16x2.e4m3x2 %0, a;\n\tcvt.rn.f16x2.e4m3x2 %1, b;\n\t}"
        : "=r"(lo), "=r"(hi)
        : "r"(u));
  } else {
    // 0x6400 | (code + 128) is 1024 + code + 128 as f16
    const uint32_t x = u ^ 0x80808080u;
    const uint32_t a = __byte_perm(x, 0x64646464u, 0x4140), b = __byte_perm(x, 0x64646464u, 0x4342);
    const __half2 bias = __float2half2_rn(1152.f);
    const __half2 p = __hsub2(*reinterpret_cast<const __half2*>(&a), bias), q = __hsub2(*reinterpret_cast<const __half2*>(&b), bias);
    lo = *reinterpret_cast<const uint32_t*>(&p);
    hi = *reinterpret_cast<const uint32_t*>(&q);
  }
}
template <int FMT>
__device__ __forceinline__ void dequantise8(uint2 u, float scale, float (&x)[8]) {
  uint32_t w[4];
  widen4<FMT>(u.x, w[0], w[1]);
  widen4<FMT>(u.y, w[2], w[3]);
  widen8(make_uint4(w[0], w[1], w[2], w[3]), x, __half());
#pragma unroll
  for (int i = 0; i < 8; ++i) x[i] *= scale;
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
