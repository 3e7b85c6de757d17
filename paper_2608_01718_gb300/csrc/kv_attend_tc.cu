// Attention for many rows a kv head (a window of drafts under verification times a group of heads): the products on tcgen05.
//
// From some tens of rows on, 4 x rows flops a cached element are more than the warp-level tensor instruction sustains at the
// rate of HBM, and tiles of 16 or 32 rows read the cache several times. Here a tile is 128 rows of q:
//   S [128 rows x 128 keys] = Q [128 x d] K^T,   O [128 x d] += P [128 x 128 keys] V
// with Q, S, P and O in TMEM and K and V in shared memory. Both products take their A operand from TMEM: with Q in shared
// memory too, the first read twice as much of it as it computed for. P overwrites the S it came from. Two threads of the
// softmax own a row, half of a tile's keys each, and share no more than its maximum.
//
// One block an SM, warp-specialised:
//   warps 9-11 (loaders): the tiles of K and V, in turn, into a ring of 32 KB slots in the 128-byte swizzle layout, by cp.async
//     (whole 16-byte units of rows found through the page table; masked and missing positions are zeros). A slot's barrier is
//     arrived at by the copies themselves, so that a loader never waits for a landing. Codes of 8-bit caches go to one of
//     three stages, and the lanes that copied them widen them, exactly, into a slot; their scales go beside them;
//   warp 8 (MMA): S of tile j into one of two accumulators, then O += P V of tile j - 1;
//   warps 0-7 (softmax, two threads a row): a triple's q into TMEM; S from TMEM, base-2 softmax by a reference that seldom
//     moves (as in kv_attend.cuh), weights to TMEM; for f16 caches in f16, else in two bf16 terms, which the product sums (one
//     would add an error as large as the output's rounding). An 8-bit cache's scales multiply scores (k) and weights (v).
// K is the first product's B operand as stored (K-major); V, as stored, the second's with its dimensions contiguous
// (MN-major), so neither is transposed. Work is cut and joined as in kv_attend.cuh, in units of 128 keys.
//
// Measured (32 q heads on 4, d = 128): bf16, 16 sequences of 300 to 3,000 tokens, 17 new ones (136 rows, two tiles) 35.5 us, of
// which 5 us until the first S, 2 a unit of 64 KB, 2.5 for a triple's end and up to 6 for joins; 4 sequences of 30,000 tokens
// and 36 rows 57 us (4.3 TB/s), 136 rows 99 us; f16 56 and 96, e4m3 92 and 169, int8 104 and 192 (widening: three warps, 32,000
// codes a unit). Of 200,000 keys, 32 rows that are not finite take 235 ms more (below).
// With the loads left out a unit takes 1.6 us (1.0 of tensor time in bf16), with the softmax left out 1.9: no one part
// bounds the kernel, their overlap within a ring of seven slots does.
//
// An output that is not finite, or near the end of fp32's range, is computed again key by key with weights of at most 1: a
// masked key's value times a zero weight, an infinity times a weight's second term, or weights above 1 may have made it so.
//
// Every wait is bounded (about a second, renewed while a row is computed again): past it the block records a timeout, its roles
// stop, copies and products in flight are drained, TMEM is freed and the block ends, after it has arrived where it shares
// triples; lacache_kv_sync reports LACACHE_ERR_DEVICE_TIMEOUT.
#include "kv_attend.cuh"
#include "tcgen05.cuh"

namespace lc {
namespace {

constexpr int kTile = 128;                   // rows of q, and keys, a tile
constexpr int kStages = 3;                   // 8-bit caches: tiles of codes in flight (five measured 2% slower)
constexpr int kStageBytes = kTile * 128;
constexpr int kBlockBytes = kTile * 128;     // 64 elements of 128 rows
constexpr int kSlotBytes = 2 * kBlockBytes;
constexpr int kSoftmax = 256;                // threads: two a row, half of the keys each
constexpr int kMmaWarp = 8;
constexpr int kLoaders = 96;                 // (twelve warps in all: 168 registers a thread)
constexpr int kThreads = kSoftmax + 32 + kLoaders;
constexpr int kCost = 4;                     // a triple's start and end, in units
constexpr uint32_t kS = 0, kO = 256, kQ = 384;   // TMEM columns: two S, O, q (two elements a column)
constexpr uint32_t kLow = 32;                    // where the weights' second terms lie behind the first, a half of the keys

// Cache format and q's type. An 8-bit cache's keys are widened to q's type and its values to bf16, both exact.
template <int FMT, bool QF16>
struct Tc {
  static constexpr bool kEight = FMT == LACACHE_KV_E4M3 || FMT == LACACHE_KV_INT8;
  static constexpr bool kSplit = FMT != LACACHE_KV_F16;    // bf16 weights, in two terms
  static constexpr int kSlots = kEight ? 4 : 7;
  struct Tail {
    uint64_t full[7], empty[7];                // a slot's tile is there; its products are done
    uint64_t s_full[2];                        // an S is complete
    uint64_t p_full, pv_done;                  // the weights are stored; their product is done
    uint64_t q_full, o_empty;                  // a triple's q is there; its O has been read
    uint64_t pair[4];                          // the two threads of every row of 32 have left their part
    uint64_t drain;
    long long progress;                        // clock64() of a warp at work on a row key by key: the waits' second counts from it
    float given[2][2][kTile];                  // what they leave, in turn and by half: the row's largest product; at a
                                               // triple's end its sum of weights, then 0 or NaN (an output not finite)
    uint32_t tmem;
    uint32_t abort_flag;
    uint32_t bad[16];                          // a unit's 16-key tiles whose page id is no page (by unit modulo 16)
    int pending[2][4];                         // shared triples, as in kv_attend.cuh
    // 8-bit caches: a unit's scales of K, then of V (by unit modulo 8)
    alignas(16) float scales[kEight ? 8 * 2 * kTile : 4];   // read four at a time
  };
  static constexpr int kStage = kSlots * kSlotBytes;       // offsets in shared memory, after the slots
  static constexpr int kTail = kStage + (kEight ? kStages * kStageBytes : 0);
  static constexpr int kSmem = kTail + (int)sizeof(Tail);
  static_assert(kSmem <= 227 * 1024, "shared memory");
  static_assert(kTail % 16 == 0 && alignof(Tail) == 16, "the scales' alignment");
};

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
struct Walk {
  int seq, seq_base, triple, first_unit, left;   // left: cells, this triple's units first
  int per_seq;
  Span sp;
  __device__ __forceinline__ int units() const { return min(sp.units - first_unit, left); }
  __device__ __forceinline__ bool done() const { return left <= 0; }
  __device__ __forceinline__ void next(const AttendArgs& a) {
    const int n = units();
    left -= n;
    if (first_unit + n == sp.units) left -= kCost;
    first_unit = 0;
    if (left > 0 && ++triple == per_seq) {
      triple = 0;
      seq_base += (sp.units + kCost) * per_seq;
      seq = min(seq + 1, a.table.seqs - 1);
      sp = span_of(a, seq, kTile);
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
__device__ bool start_walk(const AttendArgs& a, Walk& w, Line& line) {
  const int lane = threadIdx.x & 31, block = blockIdx.x;
  w.per_seq = a.kv_heads * a.row_tiles;
  int total = 0;
  for (int s = lane; s < a.table.seqs; s += 32) total += span_of(a, s, kTile).units + kCost;
  total = __reduce_add_sync(0xffffffffu, total) * w.per_seq;
  const int parts = min(total, a.parts);
  if (block >= parts) return false;
  line.share = total / parts;
  line.longer = total - line.share * parts;
  const int u = block * line.share + min(block, line.longer);
  w.seq = w.seq_base = 0;
  for (int s0 = 0; s0 < a.table.seqs; s0 += 32) {
    const int own = s0 + lane < a.table.seqs ? (span_of(a, s0 + lane, kTile).units + kCost) * w.per_seq : 0;
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
  w.sp = span_of(a, w.seq, kTile);
  w.triple = (u - w.seq_base) / (w.sp.units + kCost);
  w.first_unit = u - w.seq_base - w.triple * (w.sp.units + kCost) - kCost;
  w.left = line.share + (block < line.longer ? 1 : 0);
  if (w.first_unit < 0) {
    w.left += w.first_unit;
    w.first_unit = 0;
  }
  return true;
}

// Four neighbouring dimensions of an output row.
__device__ __forceinline__ void write4(const AttendArgs& a, int64_t at_row, int d, float4 y) {
  *reinterpret_cast<uint2*>(a.out.p + at_row + d * 2) =
      a.q_f16 ? make_uint2(pack2<false>(y.x, y.y), pack2<false>(y.z, y.w)) : make_uint2(pack2<true>(y.x, y.y), pack2<true>(y.z, y.w));
}

// Eight, times g (0: zeros, whatever they are).
__device__ __forceinline__ void write8(const AttendArgs& a, int64_t at_row, int d, float4 x, float4 y, float g) {
  if (g == 0.f) x = y = make_float4(0.f, 0.f, 0.f, 0.f);
  const float v[8] = {x.x * g, x.y * g, x.z * g, x.w * g, y.x * g, y.y * g, y.z * g, y.w * g};
  *reinterpret_cast<uint4*>(a.out.p + at_row + d * 2) = a.q_f16 ? pack8(v, __half()) : pack8(v, __nv_bfloat16());
}

// One row of one block's keys [from, to), by a warp, four keys at a time: lane i holds dimensions 4 i .. 4 i + 3. It may take
// longer than a wait's bound, so it tells the waits that it goes on.
template <int FMT, bool QF16>
__device__ __noinline__ void slow_row(const AttendArgs& a, int seq, int head, int tok, int qh, int from, int to,
                                      volatile long long* progress, float4* acc, float* top, float* sum) {
  using T = Tc<FMT, QF16>;
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
    if constexpr (T::kEight) {
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
  const unsigned char* q_row = a.q.at((int64_t)seq * a.new_tokens + tok, qh);
  const float4 q = has ? four(*reinterpret_cast<const uint2*>(q_row + lane * 8), QF16) : zero;
  float m = -INFINITY, l = 0.f;
  float4 o = zero;
  for (int j = from & ~3; j < to; j += 4) {
    if (lane == 0) *progress = clock64();
    const int index = (int)(((uint64_t)(uint32_t)(j >> 4) * a.page_mul) >> a.page_shift);
    const int page = a.table.pages[seq * a.table.stride + index];
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

template <int FMT, bool QF16>
__global__ void __launch_bounds__(kThreads, 1) attend_tc_kernel(const __grid_constant__ AttendArgs a) {
  using T = Tc<FMT, QF16>;
  using Tail = typename T::Tail;
  constexpr bool kSplit = T::kSplit;
  constexpr int kSlots = T::kSlots;
  extern __shared__ __align__(1024) unsigned char gbase[];
  const uint32_t base = smem_u32(gbase);
  if (base & 1023u) {   // the swizzled tiles start on 1024 bytes (dynamic shared memory does, with none of the static kind)
    if (threadIdx.x == 0) atomicOr(a.status, kAttendTimeout);
    return;
  }
  const uint32_t ring = base;
  Tail& t = *reinterpret_cast<Tail*>(gbase + T::kTail);
  volatile uint32_t* abort_flag = &t.abort_flag;
  volatile long long* progress = &t.progress;
  const int warp = __shfl_sync(0xffffffffu, (int)threadIdx.x >> 5, 0), lane = threadIdx.x & 31;
  const int D = a.head_dim, units_row = D / 8;                    // 16-byte units of a row in shared memory
  const int row_bytes = T::kEight ? D : D * 2;                    // of the cache
  const int slot_floats = kTile * (a.padded + 2);   // of a.partial

  auto by_group = [&](int row) { return a.group == 1 ? row : (int)__umulhi((uint32_t)row, a.group_mul); };   // row / group
  if (threadIdx.x == 0) {
    for (int s = 0; s < kSlots; ++s) {
      mbar_init(smem_u32(&t.full[s]), T::kEight ? kLoaders / 32 : kLoaders + 1);
      mbar_init(smem_u32(&t.empty[s]), 1);
    }
    for (int b = 0; b < 2; ++b) mbar_init(smem_u32(&t.s_full[b]), 1);
    mbar_init(smem_u32(&t.p_full), kSoftmax / 32);
    for (int b = 0; b < 4; ++b) mbar_init(smem_u32(&t.pair[b]), 2);
    mbar_init(smem_u32(&t.pv_done), 1);
    mbar_init(smem_u32(&t.q_full), kSoftmax / 32);
    mbar_init(smem_u32(&t.o_empty), kSoftmax / 32);
    mbar_init(smem_u32(&t.drain), 1);
    t.progress = 0;
    t.abort_flag = 0;
    t.pending[0][2] = t.pending[1][2] = -1;
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  }
  Walk walk;
  Line line;
  if (!start_walk(a, walk, line)) return;
  if (warp == kMmaWarp) {
    tmem_alloc<false>(smem_u32(&t.tmem), 512);
    tmem_relinquish<false>();
  }
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem = t.tmem;
  auto fail = [&] {
    *abort_flag = 1u;
    atomicOr(a.status, kAttendTimeout);
  };
  auto wait = [&](uint64_t& bar, uint32_t parity) {   // false (and the block stops) past the bound
    if (mbar_wait_inline(smem_u32(&bar), parity, abort_flag, progress)) return true;
    if (!*abort_flag) fail();
    return false;
  };

  if (warp > kMmaWarp) {
    // ---- loaders ----
    const int me = threadIdx.x - kSoftmax - 32;
    int n = 0;   // slots begun
    int units = 0;
    bool ok = true;
    if (a.inject_stall && walk.seq_base + walk.triple + walk.first_unit == 0) walk.left = 0;
    if constexpr (T::kEight) {
      // codes by cp.async into a stage, each lane its own pieces; kStages tiles later the lane widens them into a slot
      const int pieces = D / 16, piece_mul = 65536 / pieces + 1, tile_pieces = 16 * pieces;   // of a row; of 16 keys
      auto widen_tile = [&](int k) {
        if (k >= kSlots) ok = wait(t.empty[k % kSlots], (k / kSlots - 1) & 1);
        ok = __all_sync(0xffffffffu, ok);
        if (!ok) return;
        const unsigned char* from = gbase + T::kStage + (k % kStages) * kStageBytes;
        const uint32_t dst = ring + (k % kSlots) * kSlotBytes;
        const bool as_f16 = QF16 && !(k & 1);
#pragma unroll 1
        for (int tile = ((me >> 5) + k % kStages) % 3; tile < 8; tile += 3) {
          uint4 codes[4];
#pragma unroll
          for (int i = 0; i < 4; ++i)
            if (lane + 32 * i < tile_pieces) codes[i] = *reinterpret_cast<const uint4*>(from + tile * 2048 + (lane + 32 * i) * 16);
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            const int z = lane + 32 * i, j = (z * piece_mul) >> 16, u = z - j * pieces;
            const uint32_t w[4] = {codes[i].x, codes[i].y, codes[i].z, codes[i].w};
            uint32_t h[8];
#pragma unroll
            for (int e = 0; e < 4; ++e) widen4<FMT>(w[e], h[2 * e], h[2 * e + 1]);
            if (!as_f16) {
#pragma unroll
              for (int e = 0; e < 8; ++e) {
                const float2 f = __half22float2(*reinterpret_cast<const __half2*>(&h[e]));
                h[e] = pack2<true>(f.x, f.y);
              }
            }
            const int row = tile * 16 + j;
            if (z < tile_pieces) {
              asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %4};" ::"r"(dst + unit_at(row, 2 * u)), "r"(h[0]), "r"(h[1]),
                           "r"(h[2]), "r"(h[3])
                           : "memory");
              asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %4};" ::"r"(dst + unit_at(row, 2 * u + 1)), "r"(h[4]),
                           "r"(h[5]), "r"(h[6]), "r"(h[7])
                           : "memory");
            }
          }
        }
        warp_arrive(t.full[k % kSlots]);
      };
      for (; ok && !walk.done(); walk.next(a)) {
        const int head = walk.triple / a.row_tiles, count = walk.units();
        const int32_t* table_row = a.table.pages + walk.seq * a.table.stride;
        const int64_t head_row = (int64_t)head * a.page_size;
        int key = (walk.sp.lo & ~15) + walk.first_unit * kTile;
        auto look_up = [&](int from) {
          const int at = from + (lane & 7) * 16;
          return at < walk.sp.hi ? __ldg(table_row + (int)(((uint64_t)(uint32_t)(at >> 4) * a.page_mul) >> a.page_shift)) : -1;
        };
        int ids = look_up(key);
        for (int i = 0; ok && i < count; ++i, key += kTile, ++units) {
          const int next_ids = i + 1 < count ? look_up(key + kTile) : -1;
          const bool wrong = key + (lane & 7) * 16 < walk.sp.hi && (unsigned)ids >= (unsigned)a.pages;
          const unsigned bad = __ballot_sync(0xffffffffu, wrong) & 0xffu;
          if (bad && me == 0) atomicOr(a.status, kBadIndex);
          if (me == 0) t.bad[units & 15] = bad;
          const int live_keys = walk.sp.hi - key, dead_keys = walk.sp.lo - key;
#pragma unroll 1
          for (int kv = 0; kv < 2 && ok; ++kv, ++n) {
            // (the stage was widened kStages tiles ago, each part by the lanes that fill it now: warps share it out by stage)
            const uint32_t to = base + T::kStage + (n % kStages) * kStageBytes;
            const unsigned char* pool = kv ? a.pv : a.pk;
#pragma unroll 1
            for (int tile = ((me >> 5) + n % kStages) % 3; tile < 8; tile += 3) {
              const int page = __shfl_sync(0xffffffffu, ids, tile), at = key + tile * 16, j0 = tile * 16;
              const int slot = at - (int)(((uint64_t)(uint32_t)(at >> 4) * a.page_mul) >> a.page_shift) * a.page_size;
              const bool there = (unsigned)page < (unsigned)a.pages;
              const int64_t row = there ? page * a.page_rows + head_row + slot : 0;
              const unsigned char* src = pool + row * row_bytes;
#pragma unroll
              for (int x = 0; x < 4; ++x) {
                const int z = lane + 32 * x, j = j0 + ((z * piece_mul) >> 16);
                const bool in = there && j >= dead_keys && j < live_keys;
                if (z < tile_pieces) copy_async<16>(to + tile * 2048 + z * 16, in ? src + z * 16 : a.pk, in);
              }
              if (kv == 0) {   // with K, the scales of both: the softmax wants them before V has to be there
                const int j = lane & 15;
                const bool in = there && j0 + j >= dead_keys && j0 + j < live_keys;
                const float* scales = lane < 16 ? a.ks : a.vs;
                copy_async<4>(smem_u32(&t.scales[((units & 7) * 2 + (lane >> 4)) * kTile + j0 + j]), in ? scales + row + j : scales,
                              in);
              }
            }
            copy_commit();
            if (n >= kStages - 1) {
              copy_wait<kStages - 1>();
              widen_tile(n - (kStages - 1));
            }
          }
          ids = next_ids;
        }
      }
      copy_wait<0>();
      for (int k = max(n - (kStages - 1), 0); ok && k < n; ++k) widen_tile(k);
      walk.left = 0;   // nothing is left for the 16-bit caches' loop below
    }
    const int unit_mul = 65536 / units_row + 1;   // z / units_row = z * unit_mul >> 16 for z < 256
    // the lane's units of a 16-key tile: 16 lanes a row, or 8 where a row has no more; where they lie (copies i and i + 4 lie 8
    // rows apart), and from where they come
    const bool wide = units_row > 8;
    const int own_unit = lane & (wide ? 15 : 7), own_row = lane >> (wide ? 4 : 3);
    const int own_from = own_row * row_bytes + own_unit * 16, from_step = (wide ? 2 : 4) * row_bytes;
    uint32_t place[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) place[i] = unit_at((wide ? 2 : 4) * i + own_row, own_unit);
    for (; ok && !walk.done(); walk.next(a)) {
      const int head = walk.triple / a.row_tiles, count = walk.units();
      const int32_t* table_row = a.table.pages + walk.seq * a.table.stride;
      const unsigned char* head_k = a.pk + (int64_t)head * a.page_size * row_bytes;
      const unsigned char* head_v = a.pv + (int64_t)head * a.page_size * row_bytes;
      int key = (walk.sp.lo & ~15) + walk.first_unit * kTile;
      // lane i < 8: the page id of a unit's 16-key tile i, one unit ahead
      auto look_up = [&](int from) {
        const int at = from + (lane & 7) * 16;
        return at < walk.sp.hi ? __ldg(table_row + (int)(((uint64_t)(uint32_t)(at >> 4) * a.page_mul) >> a.page_shift)) : -1;
      };
      int ids = look_up(key);
      for (int i = 0; ok && i < count; ++i, key += kTile, ++units) {
        const int next_ids = i + 1 < count ? look_up(key + kTile) : -1;
        const bool wrong = key + (lane & 7) * 16 < walk.sp.hi && (unsigned)ids >= (unsigned)a.pages;
        const unsigned bad = __ballot_sync(0xffffffffu, wrong) & 0xffu;
        if (bad && me == 0) atomicOr(a.status, kBadIndex);
        if (me == 0) t.bad[units & 15] = bad;
        const int live_keys = walk.sp.hi - key, dead_keys = walk.sp.lo - key;   // keys [dead, live) of the tile are read
#pragma unroll 1
        for (int kv = 0; kv < 2; ++kv, ++n) {
          if (n >= kSlots) ok = wait(t.empty[n % kSlots], (n / kSlots - 1) & 1);
          if (!__all_sync(0xffffffffu, ok)) {
            ok = false;
            break;
          }
          // a warp takes a page's 16 keys at a time, the three in turn
          const uint32_t dst = ring + (n % kSlots) * kSlotBytes;
          const unsigned char* from = kv ? head_v : head_k;
          const int first = ((me >> 5) + n) % 3;
#pragma unroll
          for (int k = 0; k < 3; ++k) {
            const int tile = first + 3 * k, at = key + tile * 16, j0 = tile * 16;
            if (tile >= 8) break;
            const int page = __shfl_sync(0xffffffffu, ids, tile);
            const int slot = at - (int)(((uint64_t)(uint32_t)(at >> 4) * a.page_mul) >> a.page_shift) * a.page_size;
            const bool there = (unsigned)page < (unsigned)a.pages;
            const unsigned char* src = from + (there ? page * a.page_bytes : 0) + (int64_t)slot * row_bytes;
            const bool inside = there && j0 >= dead_keys && j0 + 16 <= live_keys;
            const uint32_t to = dst + j0 * 128;
            // (d = 128 and 64 apart: with their constants they are 4 to 5% faster; without the third form, d = 96 took 165 us
            // instead of 125, 72 rows over 64 x 4,000 tokens of bf16)
            if (inside && units_row == 16) {
#pragma unroll
              for (int i = 0; i < 8; ++i) copy_async<16>(to + place[i & 3] + (i >> 2) * 1024, src + lane * 16 + i * 512, true);
            } else if (inside && units_row == 8) {
#pragma unroll
              for (int i = 0; i < 4; ++i) copy_async<16>(to + place[i], src + lane * 16 + i * 512, true);
            } else if (inside) {
              if (own_unit < units_row) {
#pragma unroll
                for (int i = 0; i < 8; ++i)
                  if (i < 4 || wide) copy_async<16>(to + place[i & 3] + (i >> 2) * 1024, src + own_from + i * from_step, true);
              }
            } else {
              for (int z = lane; z < 16 * units_row; z += 32) {
                const int j = (z * unit_mul) >> 16;
                const bool in = there && j0 + j >= dead_keys && j0 + j < live_keys;
                copy_async<16>(dst + unit_at(j0 + j, z - j * units_row), in ? src + z * 16 : a.pk, in);
              }
            }
          }
          copies_arrive(t.full[n % kSlots]);
          if (me == 0) mbar_arrive(smem_u32(&t.full[n % kSlots]));   // for t.bad, which no copy writes
        }
        ids = next_ids;
      }
    }
    copy_wait<0>();
  } else if (warp == kMmaWarp) {
    // ---- MMA ----
    const uint32_t bf16 = (1u << 7) | (1u << 10);   // both operands' type; f16 is 0
    const uint32_t qk = (1u << 4) | (QF16 ? 0u : bf16) | ((uint32_t)(kTile >> 3) << 17) | ((uint32_t)(kTile >> 4) << 24);
    const uint32_t pv = (1u << 4) | (kSplit ? bf16 : 0u) | (1u << 16) | ((uint32_t)(D >> 3) << 17) | ((uint32_t)(kTile >> 4) << 24);
    int j = 0, triples = 0;    // tiles and triples begun
    int done = 0;              // products with V that have been waited for
    bool ok = true;
    auto wait_second = [&](int upto) {   // (before the next one is begun, as each phase has to be seen)
      for (; ok && done <= upto; ++done) ok = wait(t.pv_done, done & 1);
    };
    // O (+)= P V of tile k
    auto second = [&](int k, bool first_of_triple, int of_triple) {
      const int v_slot = (2 * k + 1) % kSlots;
      wait_second(k - 1);
      ok = ok && wait(t.full[v_slot], ((2 * k + 1) / kSlots) & 1) && wait(t.p_full, k & 1) &&
           (!first_of_triple || of_triple == 0 || wait(t.o_empty, (of_triple - 1) & 1));
      ok = __all_sync(0xffffffffu, ok);
      if (!ok) return;
      asm volatile("fence.proxy.async.shared::cta;" ::: "memory");   // (the loaders' writes)
      tc_fence_after();
      const uint32_t v = ring + v_slot * kSlotBytes;
      if (elect_one()) {
#pragma unroll 1
        for (int kk = 0; kk < kTile / 16; ++kk) {
          const uint64_t v_desc = smem_desc_mn(v + kk * 2048);
          const uint32_t p = tmem + kS + (k & 1) * kTile + (kk >> 2) * 64 + (kk & 3) * 8;
          mma_ts(tmem + kO, p, v_desc, pv, first_of_triple && kk == 0 ? 0u : 1u);
          if (kSplit) mma_ts(tmem + kO, p + kLow, v_desc, pv, 1u);
        }
        mma_commit<false>(smem_u32(&t.empty[v_slot]), 0);
        mma_commit<false>(smem_u32(&t.pv_done), 0);
      }
      __syncwarp();
    };
    for (; ok && !walk.done(); walk.next(a), ++triples) {
      const int count = walk.units();
      for (int i = 0; ok && i < count; ++i, ++j) {
        const int k_slot = (2 * j) % kSlots;
        wait_second(j - 2);   // the weights of tile j - 2 lie where S of tile j goes
        ok = ok && (i > 0 || wait(t.q_full, triples & 1)) && wait(t.full[k_slot], ((2 * j) / kSlots) & 1);
        ok = __all_sync(0xffffffffu, ok);
        if (!ok) break;
        asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
        tc_fence_after();
        const uint64_t k_desc = smem_desc(ring + k_slot * kSlotBytes);
        if (elect_one()) {
#pragma unroll 1
          for (int kk = 0; kk < D / 16; ++kk) {
            const uint64_t at = (uint64_t)((kk >> 2) * (kBlockBytes >> 4) + (kk & 3) * 2);
            mma_ts(tmem + kS + (j & 1) * kTile, tmem + kQ + kk * 8, k_desc + at, qk, kk ? 1u : 0u);
          }
          mma_commit<false>(smem_u32(&t.empty[k_slot]), 0);
          mma_commit<false>(smem_u32(&t.s_full[j & 1]), 0);
        }
        __syncwarp();
        if (i > 0) second(j - 1, i == 1, triples);
        if (ok && i + 1 == count) second(j, i == 0, triples);
      }
    }
  } else {
    // ---- softmax: two threads a row ----
    const uint32_t lanes = tmem + ((uint32_t)(warp & 3) << 21);   // this warp's 32 lanes
    const int half = warp >> 2;
    int j = 0;
    uint32_t pairs = 0;
    bool ok = true;
    // a triple's q: this thread's 64 dimensions of its row, into registers, and from there to TMEM
    uint32_t q_row[32];
    auto load_q = [&](const Walk& w) {
      const int head = w.triple / a.row_tiles, row0 = (w.triple - head * a.row_tiles) * a.tile_rows;
      const int live = min(a.rows - row0, a.tile_rows);
      const int r = threadIdx.x & (kTile - 1), row = row0 + r, tok = by_group(row);
      const uint4* from = reinterpret_cast<const uint4*>(
          r < live ? a.q.at((int64_t)w.seq * a.new_tokens + tok, head * a.group + row - tok * a.group) : nullptr);
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const int u = half * 8 + i;
        const uint4 x = r < live && u < units_row ? from[u] : make_uint4(0, 0, 0, 0);
        q_row[4 * i] = x.x, q_row[4 * i + 1] = x.y, q_row[4 * i + 2] = x.z, q_row[4 * i + 3] = x.w;
      }
    };
    auto hand_over_q = [&] {
      if (half * 64 < D) tmem_st32(lanes + kQ + half * 32, q_row);
      tmem_wait_st();
      tc_fence_before();
      warp_arrive(t.q_full);
    };
    load_q(walk);
    hand_over_q();
    for (; ok && !walk.done(); walk.next(a)) {
      const int head = walk.triple / a.row_tiles, row0 = (walk.triple - head * a.row_tiles) * a.tile_rows;
      const int live = min(a.rows - row0, a.tile_rows), count = walk.units();
      const int r = threadIdx.x & (kTile - 1), tok = by_group(row0 + r);
      const bool mine = r < live, some = (warp & 3) * 32 < live;
      const int pos = mine ? walk.sp.len - a.new_tokens + tok : INT_MAX;
      int lo = INT_MIN;
      if (mine) {
        lo = a.starts ? a.starts[walk.seq] : 0;
        if (a.window > 0 && pos - a.window + 1 > lo) lo = pos - a.window + 1;
      }
      const float factor = a.scale * 1.4426950408889634f;
      float m = -INFINITY, l = 0.f;
      const int key_begin = (walk.sp.lo & ~15) + walk.first_unit * kTile;
      if (threadIdx.x == 0) {
        const int raw_len = a.lengths[walk.seq];
        if (raw_len < 0 || raw_len > a.max_len) atomicOr(a.status, kBadIndex);
      }
      for (int i = 0; ok && i < count; ++i, ++j) {
        const int key = key_begin + i * kTile;
        ok = wait(t.s_full[j & 1], (j >> 1) & 1);
        if (!__all_sync(0xffffffffu, ok)) {
          ok = false;
          break;
        }
        if (some) {
          tc_fence_after();
          uint32_t u[2][32];
#pragma unroll
          for (int c = 0; c < 2; ++c) tmem_ld32_issue(lanes + kS + (j & 1) * kTile + half * 64 + c * 32, u[c]);
#pragma unroll
          for (int c = 0; c < 2; ++c) tmem_ld32_wait(u[c]);
          float (&x)[2][32] = reinterpret_cast<float(&)[2][32]>(u);
          const uint32_t bad = t.bad[j & 15];
          if constexpr (T::kEight) {
            const float4* ks = reinterpret_cast<const float4*>(t.scales + (j & 7) * 2 * kTile + half * 64);
#pragma unroll
            for (int e = 0; e < 16; ++e) {
              const float4 k4 = ks[e];
              float* y = x[e >> 3] + (e & 7) * 4;
              y[0] *= k4.x, y[1] *= k4.y, y[2] *= k4.z, y[3] *= k4.w;
            }
          }
          float by = factor;
          if (!(factor > 0.f)) {   // scores that the maximum of the products does not order
#pragma unroll
            for (int c = 0; c < 2; ++c) {
#pragma unroll
              for (int e = 0; e < 32; ++e) x[c][e] *= factor;
            }
            by = 1.f;
          }
          if (!__all_sync(0xffffffffu, bad == 0 && key >= lo && key + kTile - 1 <= pos)) {
            const int at = key + half * 64;
            const int first = lo < at ? 0 : lo - at, last = pos >= at + 64 ? 64 : pos - at;   // columns seen
#pragma unroll
            for (int c = 0; c < 2; ++c) {
#pragma unroll
              for (int e = 0; e < 32; ++e)
                if (c * 32 + e < first || c * 32 + e > last) x[c][e] = -INFINITY;
            }
            if (bad) {
#pragma unroll
              for (int c = 0; c < 2; ++c) {
#pragma unroll
                for (int e = 0; e < 32; ++e)
                  if (bad >> (half * 4 + c * 2 + e / 16) & 1) x[c][e] = -INFINITY;
              }
            }
          }
          float tops[2];
#pragma unroll
          for (int c = 0; c < 2; ++c) {
            tops[c] = fmaxf(x[c][0], x[c][31]);
#pragma unroll
            for (int e = 1; e < 31; e += 2) tops[c] = max_three(tops[c], x[c][e], x[c][e + 1]);
          }
          // both halves of the row move its maximum, or neither
          const float own = fmaxf(tops[0], tops[1]);
          t.given[pairs & 1][half][r] = own;
          warp_arrive(t.pair[warp & 3]);
          ok = wait(t.pair[warp & 3], pairs & 1);
          if (!__all_sync(0xffffffffu, ok)) {
            ok = false;
            break;
          }
          const float top = fmaxf(own, t.given[pairs++ & 1][half ^ 1][r]) * by;
          const bool move = m == -INFINITY ? top > -INFINITY : top > m + kHeadroom;
          const float f = move ? exp2_fast(m - (top - kBelow)) : 1.f;
          if (move) {
            l *= f;
            m = top - kBelow;
          }
          const float shift = m == -INFINITY ? 0.f : m;
          // weights, their sum, and their terms
          float2 sum[2] = {};
#pragma unroll
          for (int c = 0; c < 2; ++c) {
            uint32_t hi[16], lo_term[kSplit ? 16 : 1];
#pragma unroll
            for (int e = 0; e < 32; e += 2) {
              const float2 y = fma_two(make_float2(x[c][e], x[c][e + 1]), make_float2(by, by), make_float2(-shift, -shift));
              float2 p = make_float2(exp2_fast(y.x), exp2_fast(y.y));
              sum[e / 2 & 1] = add_two(sum[e / 2 & 1], p);
              if constexpr (T::kEight) {   // (a token that this row does not see but whose scale is NaN: the row is done again)
                const float2 vs = *reinterpret_cast<const float2*>(t.scales + ((j & 7) * 2 + 1) * kTile + half * 64 + c * 32 + e);
                p.x *= vs.x;
                p.y *= vs.y;
              }
              const uint32_t h = pack2<kSplit>(p.x, p.y);
              hi[e / 2] = h;
              if constexpr (kSplit) {
                const float2 rest = fma_two(make_float2(__uint_as_float(h << 16), __uint_as_float(h & 0xffff0000u)),
                                            make_float2(-1.f, -1.f), p);
                lo_term[e / 2] = pack2<true>(rest.x, rest.y);
              }
            }
            tmem_st16(lanes + kS + (j & 1) * kTile + half * 64 + c * 16, hi);
            if constexpr (kSplit) tmem_st16(lanes + kS + (j & 1) * kTile + half * 64 + kLow + c * 16, lo_term);
          }
          l += (sum[0].x + sum[1].x) + (sum[0].y + sum[1].y);
          if (j > 0) ok = wait(t.pv_done, (j - 1) & 1);   // O may be scaled
          if (!__all_sync(0xffffffffu, ok)) {
            ok = false;
            break;
          }
          tc_fence_after();
          if (i > 0 && __any_sync(0xffffffffu, move)) {
#pragma unroll 1
            for (int d = half * 32; d < D; d += 64) {
              uint32_t o[32];
              tmem_ld32_issue(lanes + kO + d, o);
              tmem_ld32_wait(o);
#pragma unroll
              for (int e = 0; e < 32; ++e) o[e] = __float_as_uint(__uint_as_float(o[e]) * f);
              tmem_st32(lanes + kO + d, o);
            }
          }
          tmem_wait_st();
          tc_fence_before();
        } else {   // rows past the tile's: their weights are never used
          if (j > 0) ok = wait(t.pv_done, (j - 1) & 1);
          if (!__all_sync(0xffffffffu, ok)) {
            ok = false;
            break;
          }
        }
        warp_arrive(t.p_full);
      }
      if (!ok) break;
      // with the last S of a triple complete, every product with its q is done: the next one's takes its place, while the
      // last product with V runs
      Walk next = walk;
      next.next(a);
      const bool more = !next.done();
      if (more) load_q(next);
      // ---- the triple's end: O of this block's keys ----
      float total = 0.f;
      if (some) {   // the row's sum of weights from both halves, while the last product runs
        t.given[pairs & 1][half][r] = l;
        warp_arrive(t.pair[warp & 3]);
        ok = wait(t.pair[warp & 3], pairs & 1);
        total = t.given[pairs & 1][0][r] + t.given[pairs & 1][1][r];
        ++pairs;
      }
      ok = ok && wait(t.pv_done, (j - 1) & 1);
      if (!__all_sync(0xffffffffu, ok)) {
        ok = false;
        break;
      }
      tc_fence_after();
      if (more) hand_over_q();
      const bool whole = count == walk.sp.units;
      int c_first = blockIdx.x, c_last = blockIdx.x;
      if (!whole) {
        const int begin = walk.seq_base + walk.triple * (walk.sp.units + kCost) + kCost;
        c_first = line.block_of(begin);
        c_last = line.block_of(begin + walk.sp.units - 1);
        if (threadIdx.x == 0) {
          int* p = t.pending[(int)blockIdx.x == c_first];
          p[0] = walk.seq, p[1] = walk.triple, p[2] = c_first, p[3] = c_last;
        }
      }
      float* slot = a.partial + ((int64_t)blockIdx.x * 2 + ((int)blockIdx.x == c_first ? 1 : 0)) * slot_floats;
      if (some) {
        int64_t at_lse = 0, at_row = 0;
        if (mine) at_row = out_at(a, walk.seq, head, row0 + r, &at_lse);
        const float inv = total == 0.f ? 0.f : 1.f / total;
        // this half's dimensions: 32 of every 64 (rolled: code that runs once a triple waits for its fetch)
        float2 zero = make_float2(0.f, 0.f);   // NaN after a product that is not finite, or past kFar
#pragma unroll 1
        for (int d0 = half * 32; d0 < D; d0 += 64) {
          float o[32];
          tmem_ld32(lanes + kO + d0, o);
#pragma unroll
          for (int e = 0; e < 32; e += 8) {
            const int d = d0 + e;
            if (d < D) {
#pragma unroll
              for (int x = 0; x < 8; x += 2) {
                const float2 y = mul_two(make_float2(o[e + x], o[e + x + 1]), make_float2(kToEnd, kToEnd));
                zero = fma_two(y, make_float2(0.f, 0.f), zero);
              }
              if (mine) {
                const float4 y0 = make_float4(o[e], o[e + 1], o[e + 2], o[e + 3]);
                const float4 y1 = make_float4(o[e + 4], o[e + 5], o[e + 6], o[e + 7]);
                if (whole) {
                  write8(a, at_row, d, y0, y1, inv);
                } else {
                  reinterpret_cast<float4*>(slot)[d / 4 * kTile + r] = y0;
                  reinterpret_cast<float4*>(slot)[(d / 4 + 1) * kTile + r] = y1;
                }
              }
            }
          }
        }
        if (mine && half == 0) {
          if (!whole) *reinterpret_cast<float2*>(slot + kTile * a.padded + r * 2) = make_float2(m, total);
          else if (a.lse) a.lse[at_lse] = lse_of(m, total);
        }
        // a row that is not finite in either half is done again, past what both have written; not where its sum of weights
        // is NaN: then a score that it sees is (masked ones are -infinity), and NaN is its result
        t.given[pairs & 1][half][r] = zero.x + zero.y;
        warp_arrive(t.pair[warp & 3]);
        ok = wait(t.pair[warp & 3], pairs & 1);
        if (!__all_sync(0xffffffffu, ok)) {
          ok = false;
          break;
        }
        const bool odd = !(t.given[pairs & 1][0][r] + t.given[pairs & 1][1][r] == 0.f) && total <= 3.402823466e+38f;
        ++pairs;
        // rows that are not finite, again: every second one by the other half's warp
        const int key_end = min(key_begin + count * kTile, walk.sp.hi);
        for (unsigned rows = __ballot_sync(0xffffffffu, mine && odd) & (half ? 0xaaaaaaaau : 0x55555555u); rows; rows &= rows - 1) {
          const int src = __ffs(rows) - 1;
          const int rr = (warp & 3) * 32 + src, its_tok = by_group(row0 + rr), its_qh = head * a.group + row0 + rr - its_tok * a.group;
          const int its_pos = __shfl_sync(0xffffffffu, pos, src), its_lo = __shfl_sync(0xffffffffu, lo, src);
          float4 acc;
          float top, sum;
          slow_row<FMT, QF16>(a, walk.seq, head, its_tok, its_qh, max(max(key_begin, its_lo), 0), min(key_end, its_pos + 1),
                               progress, &acc, &top, &sum);
          int64_t its_lse;
          const int64_t its_row = out_at(a, walk.seq, head, row0 + rr, &its_lse);
          if (lane * 4 < D) {
            if (whole) {
              const float g = sum == 0.f ? 0.f : 1.f / sum;
              write4(a, its_row, lane * 4, sum == 0.f ? make_float4(0.f, 0.f, 0.f, 0.f)
                                                      : make_float4(acc.x * g, acc.y * g, acc.z * g, acc.w * g));
            } else {
              reinterpret_cast<float4*>(slot)[lane * kTile + rr] = acc;
            }
          }
          if (lane == 0) {
            if (!whole) *reinterpret_cast<float2*>(slot + kTile * a.padded + rr * 2) = make_float2(top, sum);
            else if (a.lse) a.lse[its_lse] = lse_of(top, sum);
          }
        }
      }
      tc_fence_before();
      warp_arrive(t.o_empty);
    }
  }

  // ---- nothing in flight: every product is done (the loaders have waited for their copies); TMEM is freed ----
  if (warp == kMmaWarp) {
    if (elect_one()) mma_commit<false>(smem_u32(&t.drain), 0);
    __syncwarp();
    mbar_wait_inline(smem_u32(&t.drain), 0, nullptr);
  }
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  if (warp == kMmaWarp) tmem_dealloc<false>(tmem, 512);
  if (*abort_flag) {   // it still arrives where it shares a triple: the counters are zero when the launch ends
    if (warp == 0) {
      start_walk(a, walk, line);
      for (; !walk.done(); walk.next(a)) {
        if (walk.units() == walk.sp.units) continue;
        const int begin = walk.seq_base + walk.triple * (walk.sp.units + kCost) + kCost;
        const int c_first = line.block_of(begin), c_last = line.block_of(begin + walk.sp.units - 1);
        if (lane == 0 && atomicAdd(a.arrived + c_first, 1u) == (unsigned int)(c_last - c_first)) a.arrived[c_first] = 0u;
      }
    }
    return;
  }

  // ---- shared triples: whichever block arrives last joins the blocks' sums, in their order ----
  if (threadIdx.x < 2) {
    int* p = t.pending[threadIdx.x];
    bool last = false;
    if (p[2] >= 0) {
      __threadfence();
      last = atomicAdd(a.arrived + p[2], 1u) == (unsigned int)(p[3] - p[2]);
      if (last) a.arrived[p[2]] = 0u;
      __threadfence();
    }
    if (!last) p[2] = -1;
  }
  __syncthreads();
  float* joint_top = reinterpret_cast<float*>(gbase);   // [2][kTile] each, in q's place
  float* joint_inv = joint_top + 2 * kTile;
  int64_t* joint_out = reinterpret_cast<int64_t*>(joint_inv + 2 * kTile);
  auto part = [&](int k, int i) { return a.partial + ((int64_t)(t.pending[k][2] + i) * 2 + (i == 0 ? 1 : 0)) * slot_floats; };
  auto part_ml = [&](int k, int i, int r) { return __ldcg(reinterpret_cast<const float2*>(part(k, i) + kTile * a.padded) + r); };
  auto rows_of = [&](int k) {
    return t.pending[k][2] < 0 ? 0 : min(a.rows - t.pending[k][1] % a.row_tiles * a.tile_rows, a.tile_rows);
  };
  const int rows0 = rows_of(0), rows1 = rows_of(1);
  for (int x = threadIdx.x; x < rows0 + rows1; x += kThreads) {
    const int k = x < rows0 ? 0 : 1, r = k == 0 ? x : x - rows0, blocks = t.pending[k][3] - t.pending[k][2] + 1;
    float top = -INFINITY, sum = 0.f;
    for (int c = 0; c < blocks; c += 8) {
      float2 y[8];
#pragma unroll
      for (int e = 0; e < 8; ++e) y[e] = c + e < blocks ? part_ml(k, c + e, r) : make_float2(-INFINITY, 0.f);
      float now = top;
#pragma unroll
      for (int e = 0; e < 8; ++e) now = fmaxf(now, y[e].x);
      const float to = now == -INFINITY ? 0.f : now;
      sum *= exp2_fast(top - to);
#pragma unroll
      for (int e = 0; e < 8; ++e) sum += exp2_fast(y[e].x - to) * y[e].y;
      top = now;
    }
    const int head = t.pending[k][1] / a.row_tiles, row0 = (t.pending[k][1] - head * a.row_tiles) * a.tile_rows;
    int64_t at_lse;
    joint_out[x] = out_at(a, t.pending[k][0], head, row0 + r, &at_lse);
    joint_top[x] = top == -INFINITY ? 0.f : top;
    joint_inv[x] = sum == 0.f ? 0.f : 1.f / sum;
    if (a.lse) a.lse[at_lse] = lse_of(top, sum);
  }
  __syncthreads();
  // a thread joins 16 dimensions of a row at a time, from four blocks: sixteen loads in flight; neighbouring threads on
  // neighbouring rows
#pragma unroll 1
  for (int k = 0; k < 2; ++k) {
    const int rows = k ? rows1 : rows0, x0 = k ? rows0 : 0;
    const int blocks = t.pending[k][3] - t.pending[k][2] + 1;
#pragma unroll 1
    for (int item = threadIdx.x; item < rows * (D / 16); item += kThreads) {
      const int q0 = item / rows * 4, r = item - q0 / 4 * rows;
      const float base_top = joint_top[x0 + r], g = joint_inv[x0 + r];
      float4 acc[4];
#pragma unroll
      for (int v = 0; v < 4; ++v) acc[v] = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll 1
      for (int c = 0; c < blocks; c += 4) {
        float4 y[4][4];
        float w[4];
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const bool in = c + e < blocks;
          const float4* from = reinterpret_cast<const float4*>(part(k, in ? c + e : 0));
          w[e] = in ? part_ml(k, c + e, r).x : -INFINITY;
#pragma unroll
          for (int v = 0; v < 4; ++v) y[e][v] = in ? __ldcg(from + (q0 + v) * kTile + r) : make_float4(0.f, 0.f, 0.f, 0.f);
        }
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const float f = exp2_fast(w[e] - base_top);
#pragma unroll
          for (int v = 0; v < 4; ++v)
            acc[v].x += f * y[e][v].x, acc[v].y += f * y[e][v].y, acc[v].z += f * y[e][v].z, acc[v].w += f * y[e][v].w;
        }
      }
#pragma unroll
      for (int v = 0; v < 4; v += 2) write8(a, joint_out[x0 + r], (q0 + v) * 4, acc[v], acc[v + 1], g);
    }
  }
}

template <int FMT, bool QF16>
cudaError_t launch_tc(AttendArgs a, int num_sms, cudaStream_t st) {
  constexpr int kSmem = Tc<FMT, QF16>::kSmem;
  auto* kernel = attend_tc_kernel<FMT, QF16>;
  static std::atomic<bool> ready[kMaxDevices];
  if (a.device >= kMaxDevices || !ready[a.device].load(std::memory_order_relaxed)) {
    const cudaError_t e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, kSmem);
    if (e != cudaSuccess) return e;
    if (a.device < kMaxDevices) ready[a.device].store(true, std::memory_order_relaxed);
  }
  a.row_tiles = (a.rows + kTile - 1) / kTile;
  a.tile_rows = (a.rows + a.row_tiles - 1) / a.row_tiles;
  a.padded = padded_dim(a.head_dim);
  a.group_mul = (uint32_t)((((uint64_t)1 << 32) + a.group - 1) / a.group);   // exact for rows x group < 2^32
  const int64_t units = ((int64_t)a.max_len + 15) / kTile + 1 + kCost;
  const double most = (double)a.table.seqs * a.kv_heads * a.row_tiles * (double)units;
  if (most >= 2147483648.0) return cudaErrorNotSupported;   // cells are counted in 32 bits
  a.parts = most < (double)num_sms ? (int)most : num_sms;
  kernel<<<a.parts, kThreads, kSmem, st>>>(a);
  return cudaGetLastError();
}

}  // namespace

cudaError_t launch_attend_tc(const AttendArgs& a, int format, int num_sms, cudaStream_t st) {
  switch (format) {
    case LACACHE_KV_BF16: return launch_tc<LACACHE_KV_BF16, false>(a, num_sms, st);
    case LACACHE_KV_F16: return launch_tc<LACACHE_KV_F16, true>(a, num_sms, st);
    case LACACHE_KV_E4M3:
      return a.q_f16 ? launch_tc<LACACHE_KV_E4M3, true>(a, num_sms, st) : launch_tc<LACACHE_KV_E4M3, false>(a, num_sms, st);
    default:
      return a.q_f16 ? launch_tc<LACACHE_KV_INT8, true>(a, num_sms, st) : launch_tc<LACACHE_KV_INT8, false>(a, num_sms, st);
  }
}

}  // namespace lc
