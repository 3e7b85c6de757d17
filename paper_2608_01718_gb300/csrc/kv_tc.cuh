// Shared by the attention kernels on tcgen05 (kv_attend_tc.cu, kv_shared_tc_common.cu) and the one of gathered weights
// (kv_weigh_tc.cu): the layout of tiles in shared memory, a block's part of the line of work, and a row key by key.
#pragma once

#include "kv_attend.cuh"
#include "tcgen05.cuh"

namespace lc {
namespace {

constexpr int kTile = 128;                   // keys of a tile, and the lanes of TMEM
constexpr int kBlockBytes = kTile * 128;     // 64 elements of 128 rows

// Where 16-byte unit u of row r lies in a tile of 128 rows: blocks of 64 elements, 128-byte swizzle.
__device__ __forceinline__ uint32_t unit_at(int r, int u) {
  return (uint32_t)((u >> 3) * kBlockBytes + r * 128 + (((u & 7) ^ (r & 7)) << 4));
}

// An MN-major operand in the 128-byte swizzle layout: 64 elements a row of 128 B, 8 rows 1024 B apart along K (stride byte
// offset), blocks of 64 elements kBlockBytes apart along N (leading byte offset).
__device__ __forceinline__ uint64_t smem_desc_mn(uint32_t addr) {
  uint64_t desc = (uint64_t)((addr >> 4) & 0x3FFFu);
  desc |= (uint64_t)(kBlockBytes >> 4) << 16;
  desc |= (uint64_t)(1024 >> 4) << 32;
  desc |= (uint64_t)1 << 46;
  desc |= (uint64_t)2 << 61;
  return desc;
}
// D += A B with both in shared memory
__device__ __forceinline__ void mma_ss(uint32_t d, uint64_t a, uint64_t b, uint32_t idesc, uint32_t accumulate) {
  asm volatile(
      "{\n\t.reg .pred p;\n\tsetp.ne.b32 p, %4, 0;\n\t"
      "tcgen05.mma.cta_group::1.kind::f16 [%0], %1, %2, %3, p;\n\t}" ::"r"(d),
      "l"(a), "l"(b), "r"(idesc), "r"(accumulate)
      : "memory");
}
// D += A B with A in TMEM (lane = row, two elements a column).
__device__ __forceinline__ void mma_ts(uint32_t d, uint32_t a, uint64_t b, uint32_t idesc, uint32_t accumulate) {
  asm volatile(
      "{\n\t.reg .pred p;\n\tsetp.ne.b32 p, %4, 0;\n\t"
      "tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], %2, %3, p;\n\t}" ::"r"(d),
      "r"(a), "l"(b), "r"(idesc), "r"(accumulate)
      : "memory");
}

__device__ __forceinline__ void tmem_st16(uint32_t taddr, const uint32_t (&r)[16]) {
  asm volatile(
      "tcgen05.st.sync.aligned.32x32b.x16.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, %16};"
      ::"r"(taddr), "r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]),
        "r"(r[8]), "r"(r[9]), "r"(r[10]), "r"(r[11]), "r"(r[12]), "r"(r[13]), "r"(r[14]), "r"(r[15])
      : "memory");
}

__device__ __forceinline__ void tmem_st8(uint32_t taddr, const uint32_t (&r)[8]) {
  asm volatile("tcgen05.st.sync.aligned.32x32b.x8.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};" ::"r"(taddr), "r"(r[0]), "r"(r[1]),
               "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7])
               : "memory");
}
// 16 columns of this thread's lane, waited for.
__device__ __forceinline__ void tmem_ld16(uint32_t taddr, uint32_t (&r)[16]) {
  asm volatile(
      "tcgen05.ld.sync.aligned.32x32b.x16.b32 {%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15}, [%16];\n\t"
      "tcgen05.wait::ld.sync.aligned;"
      : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]), "=r"(r[8]), "=r"(r[9]),
        "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15])
      : "r"(taddr)
      : "memory");
}
__device__ __forceinline__ float max_three(float x, float y, float z) {
  float d;
  asm("max.f32 %0, %1, %2, %3;" : "=f"(d) : "f"(x), "f"(y), "f"(z));
  return d;
}
// An arrival of this thread's, once all of its copies so far have landed.
__device__ __forceinline__ void copies_arrive(uint64_t& bar) {
  asm volatile("cp.async.mbarrier.arrive.noinc.shared::cta.b64 [%0];" ::"r"(smem_u32(&bar)) : "memory");
}
// One arrival for a warp, after what all of its lanes did.
__device__ __forceinline__ void warp_arrive(uint64_t& bar) {
  __syncwarp();
  if ((threadIdx.x & 31) == 0) mbar_arrive(smem_u32(&bar));
}

// This block's part of the line of cells: triples in order, each with its first unit and how many units are the block's.
// (COST: a triple's start and end, in units; ROWS: of a tile, where sequences have different numbers of them)
template <int FORM, int COST, int ROWS>
struct Walk {
  int seq, seq_base, triple, first_unit, left;   // left: cells, this triple's units first
  int per_whole;
  Span sp;
  __device__ __forceinline__ int per_seq(const AttendArgs& a) const { return FORM == kCommon ? a.kv_heads * sp.tiles : per_whole; }
  __device__ __forceinline__ int units() const { return min(sp.units - first_unit, left); }
  __device__ __forceinline__ bool done() const { return left <= 0; }
  __device__ __forceinline__ void next(const AttendArgs& a) {
    const int n = units();
    left -= n;
    if (first_unit + n == sp.units) left -= COST;
    first_unit = 0;
    if (left > 0 && ++triple == per_seq(a)) {
      triple = 0;
      seq_base += (sp.units + COST) * per_seq(a);
      seq = min(seq + 1, seqs_of<FORM>(a) - 1);
      sp = span_of<FORM>(a, seq, kTile, ROWS);
    }
  }
};
struct Line {
  int share, longer;
  __device__ __forceinline__ int block_of(int cell) const {
    const int in_longer = longer * (share + 1);
    return cell < in_longer ? cell / (share + 1) : longer + (cell - in_longer) / share;
  }
};
// By a whole warp. false: this block has no part.
template <int FORM, int COST, int ROWS>
__device__ bool start_walk(const AttendArgs& a, Walk<FORM, COST, ROWS>& w, Line& line) {
  const int lane = threadIdx.x & 31, block = blockIdx.x, seqs = seqs_of<FORM>(a);
  w.per_whole = a.kv_heads * a.row_tiles;
  auto cells_of = [&](int s) {   // of one of the sequence's triples, or, where their number differs, of all
    const Span x = span_of<FORM>(a, s, kTile, ROWS);
    return (x.units + COST) * (FORM == kCommon ? a.kv_heads * x.tiles : 1);
  };
  const int times = FORM == kCommon ? 1 : w.per_whole;
  int total = 0;
  for (int s = lane; s < seqs; s += 32) total += cells_of(s);
  total = __reduce_add_sync(0xffffffffu, total) * times;
  const int parts = min(total, a.parts);
  if (block >= parts) return false;
  line.share = total / parts;
  line.longer = total - line.share * parts;
  const int u = block * line.share + min(block, line.longer);
  w.seq = w.seq_base = 0;
  for (int s0 = 0; s0 < seqs; s0 += 32) {
    const int own = s0 + lane < seqs ? cells_of(s0 + lane) * times : 0;
    int upto = own;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const int y = __shfl_up_sync(0xffffffffu, upto, o);
      if (lane >= o) upto += y;
    }
    const unsigned past = __ballot_sync(0xffffffffu, w.seq_base + upto > u);
    if (past) {
      const int l0 = __ffs(past) - 1;
      w.seq = s0 + l0;
      w.seq_base += __shfl_sync(0xffffffffu, upto - own, l0);
      break;
    }
    w.seq_base += __shfl_sync(0xffffffffu, upto, 31);
  }
  w.sp = span_of<FORM>(a, w.seq, kTile, ROWS);
  w.triple = (u - w.seq_base) / (w.sp.units + COST);
  w.first_unit = u - w.seq_base - w.triple * (w.sp.units + COST) - COST;
  w.left = line.share + (block < line.longer ? 1 : 0);
  if (w.first_unit < 0) {
    w.left += w.first_unit;
    w.first_unit = 0;
  }
  return true;
}

// One row of one block's keys [from, to), by a warp, four keys at a time: lane i holds dimensions 4 i .. 4 i + 3. It may take
// longer than a wait's bound, so it tells the waits that it goes on.
template <int FMT, bool QF16>
__device__ __noinline__ void slow_row(const AttendArgs& a, int first, int head, int tok, int qh, int from, int to,
                                      volatile long long* progress, float4* acc, float* top, float* sum) {
  constexpr bool kEight = FMT == LACACHE_KV_E4M3 || FMT == LACACHE_KV_INT8;
  const int lane = threadIdx.x & 31, D = a.head_dim;
  const bool has = lane * 4 < D;
  auto four = [](uint2 u, bool f16) {
    if (!f16)
      return make_float4(__uint_as_float(u.x << 16), __uint_as_float(u.x & 0xffff0000u), __uint_as_float(u.y << 16),
                         __uint_as_float(u.y & 0xffff0000u));
    const float2 x = __half22float2(*reinterpret_cast<const __half2*>(&u.x)), y = __half22float2(*reinterpret_cast<const __half2*>(&u.y));
    return make_float4(x.x, x.y, y.x, y.y);
  };
  auto cached4 = [&](const unsigned char* pool, const float* scales, int64_t row) {
    if constexpr (kEight) {
      uint2 u;
      widen4<FMT>(*reinterpret_cast<const uint32_t*>(pool + row * D + lane * 4), u.x, u.y);
      const float4 x = four(u, true);
      const float f = scales[row];
      return make_float4(x.x * f, x.y * f, x.z * f, x.w * f);
    } else {
      return four(*reinterpret_cast<const uint2*>(pool + row * D * 2 + lane * 8), FMT == LACACHE_KV_F16);
    }
  };
  const float4 zero = make_float4(0.f, 0.f, 0.f, 0.f);
  const unsigned char* q_row = a.q.at((int64_t)first * a.new_tokens + tok, qh);
  const float4 q = has ? four(*reinterpret_cast<const uint2*>(q_row + lane * 8), QF16) : zero;
  float m = -INFINITY, l = 0.f;
  float4 o = zero;
  for (int j = from & ~3; j < to; j += 4) {
    if (lane == 0) *progress = clock64();
    const int index = (int)(((uint64_t)(uint32_t)(j >> 4) * a.page_mul) >> a.page_shift);
    const int page = a.table.pages[first * a.table.stride + index];
    if ((unsigned)page >= (unsigned)a.pages) continue;
    const int64_t row = page * a.page_rows + (int64_t)head * a.page_size + (j - index * a.page_size);
    float4 k[4], v[4];
    float s[4];
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const bool in = has && j + e >= from && j + e < to;
      k[e] = in ? cached4(a.pk, a.ks, row + e) : zero;
      v[e] = in ? cached4(a.pv, a.vs, row + e) : zero;
    }
#pragma unroll
    for (int e = 0; e < 4; ++e) s[e] = has ? q.x * k[e].x + q.y * k[e].y + q.z * k[e].z + q.w * k[e].w : 0.f;
#pragma unroll
    for (int x = 16; x; x >>= 1) {
#pragma unroll
      for (int e = 0; e < 4; ++e) s[e] += __shfl_xor_sync(0xffffffffu, s[e], x);
    }
    float now = m;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      s[e] = j + e >= from && j + e < to ? s[e] * (a.scale * 1.4426950408889634f) : -INFINITY;
      now = fmaxf(now, s[e]);
    }
    const float base = now == -INFINITY ? 0.f : now, f = exp2_fast(m - base);
    l *= f, o.x *= f, o.y *= f, o.z *= f, o.w *= f;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const float p = exp2_fast(s[e] - base);
      l += p, o.x += p * v[e].x, o.y += p * v[e].y, o.z += p * v[e].z, o.w += p * v[e].w;
    }
    m = now;
  }
  *acc = o;
  *top = m;
  *sum = l;
}


}  // namespace
}  // namespace lc
