// The attention weight of cached tokens from many rows a kv head (the tokens of a prompt times a group of heads): the products on
// tcgen05, with keys as the rows of the accumulator,
//   S^T [128 keys x rows] = K [128 x d] Q^T [d x rows],
// so that a thread of the sums owns a key: it takes its scores of all rows from TMEM, a tile of rows at a time, and adds
// e^(s - lse) in its registers. Nothing is exchanged, and no weight is ever stored.
//
// One block an SM, warp-specialised, over units of 256 keys (128 for heads past 128) that stay in shared memory while the rows
// of q pass by:
//   warps 9-12 (loaders): a unit's K into one of two sets, 16-bit rows by cp.async (found through the page table), 8-bit codes
//     widened on the way to q's type (exact), and with it the keys' scales and past weights; q's tiles into a ring, with each row's
//     lse and the positions that it sees. All in the 128-byte swizzle layout; a barrier is arrived at by the copies themselves;
//   warp 8 (MMA): for every tile of rows the unit's one or two blocks of 128 keys, into one of two accumulators each;
//   warps 0-7 (sums): two blocks of keys, four warps each (one block: half of the rows each).
// A tile of rows that sees none of a unit's keys is left out by all of them.
//
// Bound by the exponentials, one a score, beside the instructions that scale and add it: four prompts of 512 to 4,000 tokens whose
// last 512 are weighed (32 heads on 8, d = 128, bf16) take 52 us, 309 in the kernel for few rows, and the products alone would 16.
// Every wait is bounded (about a second): past it the block records a timeout, its roles
// stop, copies and products in flight are drained, TMEM is freed and the block ends; lacache_kv_sync reports
// LACACHE_ERR_DEVICE_TIMEOUT.
#include "kv_tc.cuh"
#include "kv_weigh.cuh"

namespace lc {
namespace {

constexpr int kSums = 256, kMmaWarp = 8, kLoaders = 128;
constexpr int kThreads = kSums + 32 + kLoaders;

// FMT: the cache's format; QF16: q's type, and that of the operands; DP: the padded head dimension.
template <int FMT, bool QF16, int DP>
struct Weigh {
  static constexpr bool kEight = FMT == LACACHE_KV_E4M3 || FMT == LACACHE_KV_INT8;
  static constexpr int kBlocks = DP == 256 ? 1 : 2;              // of 128 keys a unit
  static constexpr int kKeys = 128 * kBlocks;
  static constexpr int kRows = DP == 64 ? 128 : DP == 128 ? 96 : 64;   // of q a tile
  static constexpr int kSetBytes = kKeys * DP * 2;               // K of a unit
  static constexpr int kTileBytes = kRows * DP * 2;              // a tile of q
  static constexpr int kTiles = DP == 64 ? 6 : DP == 128 ? 3 : 2;      // in the ring
  struct Tail {
    uint64_t k_full[2], k_empty[2];      // a set is there; its products are done and its weights are written
    uint64_t q_full[kTiles], q_empty[kTiles];
    uint64_t s_full[2], s_empty[2];      // an accumulator is complete; it has been read
    uint64_t half_full, half_empty;      // one block of keys: the second half of the rows has left its sums; they have been added
    uint64_t drain;
    uint32_t tmem, abort_flag;
    uint32_t bad[2];                     // of a set: 16-key tiles without a page
    alignas(16) float scale[2][kKeys];   // of the keys
    alignas(16) float past[2][kKeys];
    alignas(16) float lse[kTiles][kRows];        // of the rows: -lse log2(e), and the last and first position that they see
    alignas(16) int pos[kTiles][kRows], lo[kTiles][kRows];
    int min_pos[kTiles][4], max_lo[kTiles][4];   // by the loader warps
    float half[128];                     // one block of keys: what the other half of the rows adds
  };
  static constexpr int kQ = 2 * kSetBytes, kTail = kQ + kTiles * kTileBytes;
  static constexpr int kSmem = kTail + (int)sizeof(Tail);
  static_assert(kSmem <= 227 * 1024, "shared memory");
  static constexpr uint32_t kColumns = DP == 256 ? 128 : 512;    // of TMEM, 2 x kBlocks x kRows of them used
};

// unit_at in an operand of ROWS rows.
template <int ROWS>
__device__ __forceinline__ uint32_t unit_of(int r, int u) {
  return (uint32_t)((u >> 3) * (ROWS * 128) + r * 128 + (((u & 7) ^ (r & 7)) << 4));
}

// The tiles of rows that see any of the keys [key, key + KEYS): [first, end).
template <int KEYS, int ROWS>
__device__ __forceinline__ int2 live_tiles(const AttendArgs& a, int len, int start, int key) {
  const int p0 = len - a.new_tokens;   // the first new token's position
  const int tiles = (a.rows + ROWS - 1) / ROWS;
  if (start >= key + KEYS) return make_int2(0, 0);
  const int64_t tok0 = max(max(key - p0, -p0), 0);                                     // the first token that sees so far
  int64_t tok1 = a.new_tokens;                                                         // one past the last that sees as late
  if (a.window > 0) tok1 = min(tok1, (int64_t)key + KEYS - 1 + a.window - p0);
  if (tok0 >= tok1) return make_int2(0, 0);
  return make_int2((int)(tok0 * a.group / ROWS), min(tiles, (int)((tok1 * a.group + ROWS - 1) / ROWS)));
}

template <int FMT, bool QF16, int DP>
__global__ void __launch_bounds__(kThreads, 1) weigh_tc_kernel(const __grid_constant__ WeighArgs w) {
  using W = Weigh<FMT, QF16, DP>;
  using Tail = typename W::Tail;
  using Place = WeighPlace<W::kKeys>;
  extern __shared__ __align__(1024) unsigned char gbase[];
  const uint32_t base = smem_u32(gbase);
  const AttendArgs& a = w.a;
  if (base & 1023u) {   // the swizzled operands start on 1024 bytes
    if (threadIdx.x == 0) atomicOr(a.status, kAttendTimeout);
    return;
  }
  Tail& t = *reinterpret_cast<Tail*>(gbase + W::kTail);
  volatile uint32_t* abort_flag = &t.abort_flag;
  const int warp = __shfl_sync(0xffffffffu, (int)threadIdx.x >> 5, 0), lane = threadIdx.x & 31;
  const int D = a.head_dim;
  weigh_check(a);
  if (threadIdx.x == 0) {
    for (int i = 0; i < 2; ++i) {
      mbar_init(smem_u32(&t.k_full[i]), kLoaders + kLoaders / 32);
      mbar_init(smem_u32(&t.k_empty[i]), 1 + kSums / 32);
      mbar_init(smem_u32(&t.s_full[i]), 1);
      mbar_init(smem_u32(&t.s_empty[i]), kSums / 32);
    }
    for (int i = 0; i < W::kTiles; ++i) {
      mbar_init(smem_u32(&t.q_full[i]), kLoaders + kLoaders / 32);
      mbar_init(smem_u32(&t.q_empty[i]), 1 + kSums / 32);
    }
    mbar_init(smem_u32(&t.half_full), kSums / 64);
    mbar_init(smem_u32(&t.half_empty), kSums / 64);
    mbar_init(smem_u32(&t.drain), 1);
    t.abort_flag = 0;
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  }
  Place at;
  int left = weigh_start<W::kKeys>(a, blockIdx.x, gridDim.x, at);
  if (left == 0) return;
  if (warp == kMmaWarp) {
    tmem_alloc<false>(smem_u32(&t.tmem), W::kColumns);
    tmem_relinquish<false>();
  }
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem = t.tmem;
  auto wait = [&](uint64_t& bar, uint32_t parity) {   // false (and the block stops) past the bound
    if (mbar_wait_inline(smem_u32(&bar), parity, abort_flag)) return true;
    if (!*abort_flag) {
      *abort_flag = 1u;
      atomicOr(a.status, kAttendTimeout);
    }
    return false;
  };
  auto tiles_of = [&](const Place& p) {
    return live_tiles<W::kKeys, W::kRows>(a, p.len, a.starts ? a.starts[p.seq] : 0, p.unit * W::kKeys);
  };

  if (warp > kMmaWarp) {
    // ---- loaders ----
    const int me = warp - kMmaWarp - 1;
    constexpr int kLanes = DP / 8, kEachCopy = 32 / kLanes;     // lanes a 16-bit row, rows a copy
    const int own_unit = lane % kLanes, own_row = lane / kLanes;
    const bool in_row = own_unit < D / 8;
    bool ok = true;
    int units = 0, tiles = 0;    // K and q tiles begun
    if (a.inject_stall && at.seq == 0 && at.head == 0 && at.unit == 0) left = 0;
    auto load_k = [&](const Place& p) {
      const int set = units & 1, key = p.unit * W::kKeys;
      if (units >= 2) ok = wait(t.k_empty[set], (units / 2 - 1) & 1);
      ok = __all_sync(0xffffffffu, ok);
      if (!ok) return;
      ++units;
      const int2 live = tiles_of(p);
      const int32_t* table_row = a.table.pages + p.seq * a.table.stride;
      const int64_t head_row = (int64_t)p.head * a.page_size;
      const int from = key + 16 * (lane & (W::kKeys / 16 - 1));   // lane i: the i-th 16 keys
      const int index = (int)(((uint64_t)(uint32_t)(from >> 4) * a.page_mul) >> a.page_shift);
      const int page = from < p.len ? __ldg(table_row + index) : -1;
      const bool there = (unsigned)page < (unsigned)a.pages;
      const int64_t row = there ? page * a.page_rows + head_row + (from - index * a.page_size) : -1;   // of the pool
      const unsigned wrong = __ballot_sync(0xffffffffu, !there && from < p.len && lane < W::kKeys / 16);
      if (me == 0 && lane == 0) t.bad[set] = wrong;
      if (live.x < live.y) {
        if constexpr (W::kEight) {
          // eight loads in flight, each sixteen codes of a row
          constexpr int kLanes8 = DP / 16, kRows8 = 32 / kLanes8, kPer = 16 / kRows8;   // lanes a row, rows a load, loads 16 keys
          const int unit8 = lane % kLanes8, row8 = lane / kLanes8;
          constexpr int kBatch = 8, kLoads = W::kKeys / 16 / (kLoaders / 32) * kPer;
#pragma unroll 1
          for (int x0 = 0; x0 < kLoads; x0 += kBatch) {
            uint4 codes[kBatch];
#pragma unroll
            for (int x = 0; x < kBatch; ++x) {
              const int tile = me + (x0 + x) / kPer * (kLoaders / 32), j = (x0 + x) % kPer * kRows8 + row8;
              const int64_t r = __shfl_sync(0xffffffffu, row, tile & 31);
              codes[x] = r >= 0 && unit8 < D / 16 ? *reinterpret_cast<const uint4*>(a.pk + (r + j) * D + unit8 * 16) : make_uint4(0, 0, 0, 0);
            }
#pragma unroll
            for (int x = 0; x < kBatch; ++x) {
              const int tile = me + (x0 + x) / kPer * (kLoaders / 32), j = (x0 + x) % kPer * kRows8 + row8;
              const uint32_t c[4] = {codes[x].x, codes[x].y, codes[x].z, codes[x].w};
              uint32_t h[8];
#pragma unroll
              for (int e = 0; e < 4; ++e) widen4<FMT>(c[e], h[2 * e], h[2 * e + 1]);
              if (!QF16) {
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                  const float2 f = __half22float2(*reinterpret_cast<const __half2*>(&h[e]));
                  h[e] = pack2<true>(f.x, f.y);
                }
              }
              const int r = tile * 16 + j;   // of the unit
              const uint32_t dst = base + set * W::kSetBytes + (r >> 7) * (128 * DP * 2);
              if (unit8 < D / 16) {
                asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %4};" ::"r"(dst + unit_of<128>(r & 127, 2 * unit8)), "r"(h[0]),
                             "r"(h[1]), "r"(h[2]), "r"(h[3])
                             : "memory");
                asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %4};" ::"r"(dst + unit_of<128>(r & 127, 2 * unit8 + 1)), "r"(h[4]),
                             "r"(h[5]), "r"(h[6]), "r"(h[7])
                             : "memory");
              }
            }
          }
        } else {
#pragma unroll 1
          for (int tile = me; tile < W::kKeys / 16; tile += kLoaders / 32) {
            const int64_t r = __shfl_sync(0xffffffffu, row, tile);
            if (r < 0) continue;
            const unsigned char* src = a.pk + (r + own_row) * (D * 2) + own_unit * 16;
            const uint32_t dst = base + set * W::kSetBytes + (tile >> 3) * (128 * DP * 2);
            const int j0 = (tile & 7) * 16 + own_row;
            if (in_row) {
#pragma unroll
              for (int i = 0; i < 16; i += kEachCopy) copy_async<16>(dst + unit_of<128>(j0 + i, own_unit), src + i * (D * 2), true);
            }
          }
        }
      }
      // the keys' scales and past weights
      for (int k = me * 32 + lane; k < W::kKeys; k += kLoaders) {
        const int64_t r = __shfl_sync(0xffffffffu, row, k >> 4);
        if (W::kEight) copy_async<4>(smem_u32(&t.scale[set][k]), r >= 0 ? a.ks + r + (k & 15) : a.ks, r >= 0);
        if (w.past) {
          const float* past = w.past + p.seq * w.past_seq + p.head * w.past_head;
          const bool old = key + k < p.len - a.new_tokens;
          copy_async<4>(smem_u32(&t.past[set][k]), old ? past + key + k : past, old);
        }
      }
      copies_arrive(t.k_full[set]);
      warp_arrive(t.k_full[set]);
    };
    // q of rows [row0, row0 + kRows) of p's sequence and head; this warp's share of them
    constexpr int kOwn = W::kRows / 4;
    auto load_q = [&](const Place& p, int tile) {
      const int slot = tiles % W::kTiles;
      const int row = tile * W::kRows + me * kOwn + lane, tok = row / a.group;
      const bool live = lane < kOwn && row < a.rows;
      const int64_t token = (int64_t)p.seq * a.new_tokens + tok;
      const int qh = p.head * a.group + row - tok * a.group;
      const float lse = live ? __ldg(w.a.lse + token * a.q_heads + qh) : -INFINITY;
      const unsigned char* from = live ? a.q.at(token, qh) : nullptr;
      if (tiles >= W::kTiles) ok = wait(t.q_empty[slot], (tiles / W::kTiles - 1) & 1);
      ok = __all_sync(0xffffffffu, ok);
      if (!ok) return;
      ++tiles;
      const uint32_t dst = base + W::kQ + slot * W::kTileBytes;
#pragma unroll
      for (int i = 0; i < kOwn; i += kEachCopy) {
        const unsigned char* src = reinterpret_cast<const unsigned char*>(
            __shfl_sync(0xffffffffu, reinterpret_cast<unsigned long long>(from), i + own_row));
        if (src && in_row) copy_async<16>(dst + unit_of<W::kRows>(me * kOwn + i + own_row, own_unit), src + own_unit * 16, true);
      }
      copies_arrive(t.q_full[slot]);
      int pos = p.len - a.new_tokens + tok, lo = a.starts ? a.starts[p.seq] : 0;
      if (a.window > 0 && pos - a.window + 1 > lo) lo = pos - a.window + 1;
      if (lse == -INFINITY) pos = -1;   // a row that sees nothing (and those past the last)
      if (lane < kOwn) {
        t.lse[slot][me * kOwn + lane] = -1.4426950408889634f * lse;
        t.pos[slot][me * kOwn + lane] = pos;
        t.lo[slot][me * kOwn + lane] = lo;
      }
      const int least = __reduce_min_sync(0xffffffffu, lane < kOwn ? pos : INT_MAX);
      const int most = __reduce_max_sync(0xffffffffu, lane < kOwn ? lo : INT_MIN);
      if (lane == 0) t.min_pos[slot][me] = least, t.max_lo[slot][me] = most;
      warp_arrive(t.q_full[slot]);
    };
    // K of the next unit goes behind the first tile of q of this one
    Place ahead = at;
    if (left > 0) load_k(at);
    for (; ok && left > 0; --left) {
      if (left > 1) ahead.next(a);
      const int2 live = tiles_of(at);
      bool next_k = left > 1;
      for (int i = live.x; ok && i < live.y; ++i) {
        load_q(at, i);
        if (ok && next_k) load_k(ahead);
        next_k = false;
      }
      if (ok && next_k) load_k(ahead);
      at = ahead;
    }
    copy_wait<0>();
  } else if (warp == kMmaWarp) {
    // ---- MMA ----
    bool ok = true;
    int units = 0, tiles = 0;
    for (; ok && left > 0; --left, ++units) {
      const int2 live = tiles_of(at);
      ok = wait(t.k_full[units & 1], (units >> 1) & 1);
      ok = __all_sync(0xffffffffu, ok);
      if (ok && lane == 0) {   // a page that is none: is the last of them seen? (here, where registers are left)
        const uint32_t bad = t.bad[units & 1];
        if (bad && at.unit * W::kKeys + (31 - __clz(bad)) * 16 + 15 >= weigh_first(a, at.seq)) atomicOr(a.status, kBadIndex);
      }
      for (int i = live.x; ok && i < live.y; ++i, ++tiles) {
        const int slot = tiles % W::kTiles, buffer = tiles & 1;
        ok = wait(t.q_full[slot], (tiles / W::kTiles) & 1) && (tiles < 2 || wait(t.s_empty[buffer], (tiles / 2 - 1) & 1));
        ok = __all_sync(0xffffffffu, ok);
        if (!ok) break;
        asm volatile("fence.proxy.async.shared::cta;" ::: "memory");   // (the loaders' writes)
        tc_fence_after();
        const int n = min(W::kRows, (a.rows - i * W::kRows + 15) / 16 * 16);
        const uint32_t type = QF16 ? 0u : (1u << 7) | (1u << 10);      // both operands'
        const uint32_t idesc = (1u << 4) | type | ((uint32_t)(n >> 3) << 17) | ((uint32_t)(128 >> 4) << 24);
        const uint64_t q_desc = smem_desc(base + W::kQ + slot * W::kTileBytes);
        const uint64_t k_desc = smem_desc(base + (units & 1) * W::kSetBytes);
        const uint32_t s_to = tmem + buffer * W::kBlocks * W::kRows;
        if (elect_one()) {
#pragma unroll
          for (int b = 0; b < W::kBlocks; ++b) {
#pragma unroll
            for (int kk = 0; kk < DP / 16; ++kk)
              if (kk < D / 16)
                mma_ss(s_to + b * W::kRows, k_desc + (uint64_t)((b * 128 * DP * 2 + (kk >> 2) * (128 * 128)) / 16 + (kk & 3) * 2),
                       q_desc + (uint64_t)((kk >> 2) * (W::kRows * 128) / 16 + (kk & 3) * 2), idesc, kk ? 1u : 0u);
          }
          mma_commit<false>(smem_u32(&t.q_empty[slot]), 0);
          mma_commit<false>(smem_u32(&t.s_full[buffer]), 0);
        }
        __syncwarp();
      }
      ok = __all_sync(0xffffffffu, ok);
      if (!ok) break;
      if (elect_one()) mma_commit<false>(smem_u32(&t.k_empty[units & 1]), 0);
      __syncwarp();
      if (left > 1) at.next(a);
    }
  } else {
    // ---- sums: a key a thread ----
    const int half = warp >> 2;
    const uint32_t lanes = tmem + ((uint32_t)(warp & 3) << 21);   // this warp's 32 lanes
    const int own = (W::kBlocks == 2 ? half * 128 : 0) + (warp & 3) * 32 + lane;   // the thread's key of a unit
    constexpr int kColumns = W::kBlocks == 2 ? W::kRows : W::kRows / 2;            // of a tile's rows, this thread's ...
    const int first_column = W::kBlocks == 2 ? 0 : half * kColumns;                // ... from here on
    bool ok = true;
    int units = 0, tiles = 0;
    for (; ok && left > 0; --left, ++units) {
      const int set = units & 1, key0 = at.unit * W::kKeys, key = key0 + own;
      const int2 live = tiles_of(at);
      ok = wait(t.k_full[set], (units >> 1) & 1);
      ok = __all_sync(0xffffffffu, ok);
      if (!ok) break;
      const float f = a.scale * 1.4426950408889634f * (W::kEight ? t.scale[set][own] : 1.f);
      const bool no_page = t.bad[set] >> (own >> 4) & 1;
      const int warp_key = key - lane;
      float2 sum[2] = {};
      for (int i = live.x; ok && i < live.y; ++i, ++tiles) {
        const int slot = tiles % W::kTiles, buffer = tiles & 1;
        ok = wait(t.q_full[slot], (tiles / W::kTiles) & 1) && wait(t.s_full[buffer], (tiles >> 1) & 1);
        ok = __all_sync(0xffffffffu, ok);
        if (!ok) break;
        tc_fence_after();
        const uint32_t s_at = lanes + (buffer * W::kBlocks + (W::kBlocks == 2 ? half : 0)) * W::kRows + first_column;
        const int rows = min(kColumns, a.rows - i * W::kRows - first_column);   // (0 or less: the other half has them all)
        const int4 min4 = *reinterpret_cast<const int4*>(t.min_pos[slot]), lo4 = *reinterpret_cast<const int4*>(t.max_lo[slot]);
        const int min_pos = min(min(min4.x, min4.y), min(min4.z, min4.w)), max_lo = max(max(lo4.x, lo4.y), max(lo4.z, lo4.w));
        const bool masked = warp_key < max_lo || warp_key + 31 > min_pos;
#pragma unroll 1
        for (int c = 0; c < rows; c += 32) {
          uint32_t u[32];
          tmem_ld32_issue(s_at + c, u);
          tmem_ld32_wait(u);
          const float4* lse = reinterpret_cast<const float4*>(t.lse[slot] + first_column + c);
          if (!masked) {
#pragma unroll
            for (int e = 0; e < 32; e += 4) {
              const float4 l = lse[e / 4];
              const float2 x = fma_two(make_float2(__uint_as_float(u[e]), __uint_as_float(u[e + 1])), make_float2(f, f), make_float2(l.x, l.y));
              const float2 y = fma_two(make_float2(__uint_as_float(u[e + 2]), __uint_as_float(u[e + 3])), make_float2(f, f), make_float2(l.z, l.w));
              sum[0] = add_two(sum[0], make_float2(exp2_fast(x.x), exp2_fast(x.y)));
              sum[1] = add_two(sum[1], make_float2(exp2_fast(y.x), exp2_fast(y.y)));
            }
          } else {
            const int4* pos = reinterpret_cast<const int4*>(t.pos[slot] + first_column + c);
            const int4* lo = reinterpret_cast<const int4*>(t.lo[slot] + first_column + c);
#pragma unroll
            for (int e = 0; e < 32; e += 4) {
              const float4 l = lse[e / 4];
              const int4 p = pos[e / 4], q = lo[e / 4];
              const float x[4] = {fmaf(__uint_as_float(u[e]), f, l.x), fmaf(__uint_as_float(u[e + 1]), f, l.y),
                                  fmaf(__uint_as_float(u[e + 2]), f, l.z), fmaf(__uint_as_float(u[e + 3]), f, l.w)};
              sum[0].x += key >= q.x && key <= p.x ? exp2_fast(x[0]) : 0.f;
              sum[0].y += key >= q.y && key <= p.y ? exp2_fast(x[1]) : 0.f;
              sum[1].x += key >= q.z && key <= p.z ? exp2_fast(x[2]) : 0.f;
              sum[1].y += key >= q.w && key <= p.w ? exp2_fast(x[3]) : 0.f;
            }
          }
        }
        tc_fence_before();
        warp_arrive(t.s_empty[buffer]);
        warp_arrive(t.q_empty[slot]);
      }
      if (!ok) break;
      float got = (sum[0].x + sum[1].x) + (sum[0].y + sum[1].y);
      if constexpr (W::kBlocks == 1) {
        if (half) {
          if (units > 0) ok = wait(t.half_empty, (units - 1) & 1);
          t.half[own] = got;
          warp_arrive(t.half_full);
        } else {
          ok = wait(t.half_full, units & 1);
          got += t.half[own];
          warp_arrive(t.half_empty);
        }
        ok = __all_sync(0xffffffffu, ok);
        if (!ok) break;
      }
      if ((W::kBlocks == 2 || !half) && key < at.len) {
        const bool is_new = key >= at.len - a.new_tokens;
        const float before = w.past && !is_new ? w.decay * t.past[set][own] : 0.f;
        w.out[at.seq * w.out_seq + at.head * w.out_head + key] = before + (no_page ? 0.f : got);
      }
      warp_arrive(t.k_empty[set]);
      if (left > 1) at.next(a);
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
  if (warp == kMmaWarp) tmem_dealloc<false>(tmem, W::kColumns);
}

template <int FMT, bool QF16, int DP>
cudaError_t launch_one(const WeighArgs& w, int num_sms, cudaStream_t st) {
  using W = Weigh<FMT, QF16, DP>;
  auto* kernel = weigh_tc_kernel<FMT, QF16, DP>;
  static std::atomic<bool> ready[kMaxDevices];
  if (w.a.device >= kMaxDevices || !ready[w.a.device].load(std::memory_order_relaxed)) {
    const cudaError_t e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, W::kSmem);
    if (e != cudaSuccess) return e;
    if (w.a.device < kMaxDevices) ready[w.a.device].store(true, std::memory_order_relaxed);
  }
  const int64_t units = ((int64_t)w.a.max_len + W::kKeys - 1) / W::kKeys;
  const double most = (double)w.a.table.seqs * w.a.kv_heads * (double)units;
  if (most >= 2147483648.0) return cudaErrorNotSupported;   // units are counted in 32 bits
  kernel<<<most < num_sms ? (int)most : num_sms, kThreads, W::kSmem, st>>>(w);
  return cudaGetLastError();
}
template <int FMT, bool QF16>
cudaError_t launch_tc(const WeighArgs& w, int num_sms, cudaStream_t st) {
  switch (padded_dim(w.a.head_dim)) {
    case 64: return launch_one<FMT, QF16, 64>(w, num_sms, st);
    case 128: return launch_one<FMT, QF16, 128>(w, num_sms, st);
    default: return launch_one<FMT, QF16, 256>(w, num_sms, st);
  }
}

}  // namespace

cudaError_t launch_weigh_tc(const WeighArgs& w, int format, int num_sms, cudaStream_t st) {
  switch (format) {
    case LACACHE_KV_BF16: return launch_tc<LACACHE_KV_BF16, false>(w, num_sms, st);
    case LACACHE_KV_F16: return launch_tc<LACACHE_KV_F16, true>(w, num_sms, st);
    case LACACHE_KV_E4M3:
      return w.a.q_f16 ? launch_tc<LACACHE_KV_E4M3, true>(w, num_sms, st) : launch_tc<LACACHE_KV_E4M3, false>(w, num_sms, st);
    default:
      return w.a.q_f16 ? launch_tc<LACACHE_KV_INT8, true>(w, num_sms, st) : launch_tc<LACACHE_KV_INT8, false>(w, num_sms, st);
  }
}

}  // namespace lc
