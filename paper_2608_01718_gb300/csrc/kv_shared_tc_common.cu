// Attention over what groups of sequences have in common, for many rows: the products on tcgen05, 256 rows of q a block.
//
//   S [128 rows x 128 keys] = Q [128 x d] K^T,   O [128 x d] += P [128 x 128 keys] V,   twice for each tile of K and V.
//
// A group's rows (the new tokens of all of its sequences times the heads of a kv head) see almost the same keys, so a tile of
// K and V, copied once, serves two tiles of rows whose products alternate: while the softmax of one tile of rows makes its
// weights, the tensor cores work on the other. Q and K are read from shared memory, P takes the place of its S in TMEM (two
// S of 128 columns and two O of up to 128 fill it).
//
// One block an SM, warp-specialised:
//   warps 10-15 (loaders): the tiles of K and V, in turn, into a ring of four slots (8-bit caches) to eight, in the 128-byte swizzle
//     layout: 16-bit rows by cp.async (found through the page table; positions past the common ones are zeros), 8-bit codes through
//     registers, a slot ahead, widened exactly (keys to q's type, values to bf16), with their scales beside them;
//   warps 8 and 9 (MMA), a tile of rows each: S of a unit, then O += P V as soon as its weights are there;
//   warps 0-7 (softmax, a thread a row, four warps a tile; the tiles take turns): a triple's q into shared memory; base-2 softmax by a
//     reference that seldom moves, the scores read from TMEM for the maximum (only where it is needed first) and for the weights,
//     which overwrite them 32 keys at a time; for f16 caches weights in f16, else in two bf16 terms, as in kv_attend_tc.cu, whose
//     treatment of values that are not finite is used too.
// Work is cut as in kv_attend.cuh, in units of 128 keys. A triple that one block does not finish is left as partial sums, which
// the join (kv_shared.cu) adds, instead of the last block for all.
//
// Bound by the softmax beside the tensor cores: a unit of 256 rows and 128 keys takes 4,550 cycles of a block at d = 128 over bf16,
// of which the products are 3,070 (two-term weights: three products a key), and 7,700 over 8-bit caches, whose scales cost the
// softmax 3,400 a tile of rows. 128 sequences of 32 heads on 8 behind 30,011 common positions of e4m3 take some 105 us of the call's
// 150 here; 223 in all with a tile of 128 rows a block, each joined by its last block, and 158 without turns. Rows that are done again
// (values that are not finite, or scores that rise by 100 powers of two after a block's first unit) are: 64 sequences behind 30,011
// positions whose every block has such a rise for every row take 16 ms over bf16 and 30 over e4m3, for 0.15 and 0.16.
//
// Every wait is bounded (about a second, renewed while a row is computed again): past it the block records a timeout, its roles
// stop, copies and products in flight are drained, TMEM is freed and the block ends; lacache_kv_sync reports
// LACACHE_ERR_DEVICE_TIMEOUT.
#include "kv_tc.cuh"

namespace lc {
namespace {

constexpr int kRows = kCommonRows;           // of q a block
static_assert(kRows == 2 * kTile && kCommonKeys == kTile, "two tiles of rows");
constexpr int kSoftmax = 256;                // threads: one a row
constexpr int kMmaWarp = 8;                  // and 9: one a tile of rows
constexpr float kFarScore = 100.f;           // above the reference, in powers of two: a row with one is done again
constexpr int kCost = kCommonCost;           // a triple's start and end, in units (24 x 17 tokens: 52.8 us so, 54.8 with 4, 55.6 with 9)

template <int FMT, bool QF16, int DP>
struct Common {
  static constexpr bool kEight = FMT == LACACHE_KV_E4M3 || FMT == LACACHE_KV_INT8;
  static constexpr bool kSplit = FMT != LACACHE_KV_F16;    // bf16 weights, in two terms
  static constexpr int kLoaders = 6;                       // warps
  static constexpr int kThreads = kSoftmax + 64 + 32 * kLoaders;
  static constexpr int kSlotBytes = kTile * DP * 2;
  static constexpr int kSlots = DP == 64 ? 8 : kEight ? 4 : 5;
  struct Tail {
    uint64_t full[8], empty[8];                // a slot's tile is there; its products are done
    uint64_t q_full[2], s_full[2], p_full[2];  // of each tile of rows: a triple's q is there; an S is complete; its weights are stored
    uint64_t pv_done[2], o_empty[2];           // their product is done; a triple's O has been read
    uint64_t turn[2];                          // a tile of rows may make its weights: the other has
    uint64_t drain;
    long long progress;                        // clock64() of a warp at work on a row key by key: the waits' second counts from it
    uint32_t tmem;
    uint32_t abort_flag;
    uint32_t bad[16];                          // a unit's 16-key tiles whose page id is no page (by unit modulo 16)
    alignas(16) float scales[kEight ? 8 * 2 * kTile : 4];   // 8-bit caches: a unit's scales of K times scale log2(e), then of V (by
                                                            // unit modulo 8)
  };
  static constexpr int kQ = kSlots * kSlotBytes;           // offsets in shared memory
  static constexpr int kTail = kQ + 2 * kSlotBytes;
  static constexpr int kSmem = kTail + (int)sizeof(Tail);
  static_assert(kSmem <= 227 * 1024, "shared memory");
  static constexpr uint32_t kS = 0, kO = 2 * kTile;        // TMEM columns: an S a tile of rows, then an O
};

template <int FMT, bool QF16, int DP>
__global__ void __launch_bounds__(Common<FMT, QF16, DP>::kThreads, 1) common_kernel(const __grid_constant__ AttendArgs a) {
  using T = Common<FMT, QF16, DP>;
  using Tail = typename T::Tail;
  using Place = Walk<kCommon, kCost, kRows>;
  constexpr bool kSplit = T::kSplit;
  constexpr int kSlots = T::kSlots, kLoaders = T::kLoaders;
  extern __shared__ __align__(1024) unsigned char gbase[];
  const uint32_t base = smem_u32(gbase);
  // (Launched beside the pass over the sequences' own positions, once each of that pass's blocks has waited for the groups: this
  // kernel reads the spans without a wait of its own, so that pass is in front of it in every call, and lets it go only after its wait.)
  asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
  if (base & 1023u) {   // the swizzled tiles start on 1024 bytes
    if (threadIdx.x == 0) atomicOr(a.status, kAttendTimeout);
    asm volatile("griddepcontrol.wait;" ::: "memory");
    return;
  }
  Tail& t = *reinterpret_cast<Tail*>(gbase + T::kTail);
  volatile uint32_t* abort_flag = &t.abort_flag;
  volatile long long* progress = &t.progress;
  const int warp = __shfl_sync(0xffffffffu, (int)threadIdx.x >> 5, 0), lane = threadIdx.x & 31;
  const int D = a.head_dim, units_row = D / 8;                    // 16-byte units of a row in shared memory
  if (threadIdx.x == 0) {
    for (int s = 0; s < kSlots; ++s) {
      mbar_init(smem_u32(&t.full[s]), T::kEight ? kLoaders : 32 * kLoaders + 1);
      mbar_init(smem_u32(&t.empty[s]), 2);
    }
    for (int b = 0; b < 2; ++b) {
      mbar_init(smem_u32(&t.q_full[b]), kSoftmax / 2);
      mbar_init(smem_u32(&t.s_full[b]), 1);
      mbar_init(smem_u32(&t.p_full[b]), 4);
      mbar_init(smem_u32(&t.pv_done[b]), 1);
      mbar_init(smem_u32(&t.o_empty[b]), 4);
      mbar_init(smem_u32(&t.turn[b]), 4);
    }
    mbar_init(smem_u32(&t.drain), 2);
    t.progress = 0;
    t.abort_flag = 0;
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  }
  Place walk;
  Line line;
  const bool some_part = start_walk(a, walk, line);
  if (blockIdx.x == 0 && warp == 0) {   // for the join
    int before = 0;
    for (int g0 = 0; g0 < a.groups; g0 += 32) {
      const Span x = g0 + lane < a.groups ? span_of<kCommon>(a, g0 + lane, kTile, kRows) : Span();
      const int own = g0 + lane < a.groups ? (x.units + kCost) * a.kv_heads * x.tiles : 0;
      int upto = own;
#pragma unroll
      for (int o = 1; o < 32; o <<= 1) {
        const int y = __shfl_up_sync(0xffffffffu, upto, o);
        if (lane >= o) upto += y;
      }
      if (g0 + lane < a.groups) a.line[2 + g0 + lane] = before + upto - own;
      before += __shfl_sync(0xffffffffu, upto, 31);
    }
    if (lane == 0) a.line[0] = line.share, a.line[1] = line.longer;
  }
  if (!some_part) {
    asm volatile("griddepcontrol.wait;" ::: "memory");
    return;
  }
  if (warp == kMmaWarp) {
    tmem_alloc<false>(smem_u32(&t.tmem), 512);
    tmem_relinquish<false>();
  }
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem = t.tmem;
  auto wait = [&](uint64_t& bar, uint32_t parity) {   // false (and the block stops) past the bound
    if (mbar_wait_inline(smem_u32(&bar), parity, abort_flag, progress)) return true;
    if (!*abort_flag) {
      *abort_flag = 1u;
      atomicOr(a.status, kAttendTimeout);
    }
    return false;
  };
  auto row0_of = [&](const Place& w) { return w.triple % w.sp.tiles * kRows; };
  auto has_two = [&](const Place& w) { return w.sp.rows - row0_of(w) > kTile; };
  auto page_index = [&](int at) { return (int)(((uint64_t)(uint32_t)(at >> 4) * a.page_mul) >> a.page_shift); };

  if (warp > kMmaWarp + 1) {
    // ---- loaders ----
    const int me = warp - kMmaWarp - 2;
    bool ok = true;
    if (a.inject_stall && walk.seq_base + walk.triple + walk.first_unit == 0) walk.left = 0;
    // the units of this block, one after another, with the page ids of each (lane i < 8: of its i-th 16 keys), and of the next
    struct Units {
      Place w;
      int i, count, key, ids, next_ids;
      bool done;
    };
    auto look_up = [&](const Place& w, int from) {
      const int at = from + (lane & 7) * 16;
      return at < w.sp.hi ? __ldg(a.table.pages + w.sp.first * a.table.stride + page_index(at)) : -1;
    };
    auto enter = [&](Units& u) {
      u.done = u.w.done();
      if (u.done) return;
      u.i = 0;
      u.count = u.w.units();
      u.key = (u.w.sp.lo & ~15) + u.w.first_unit * kTile;
      u.ids = look_up(u.w, u.key);
      u.next_ids = u.count > 1 ? look_up(u.w, u.key + kTile) : -1;
    };
    auto step = [&](Units& u) {
      if (++u.i < u.count) {
        u.key += kTile;
        u.ids = u.next_ids;
        u.next_ids = u.i + 1 < u.count ? look_up(u.w, u.key + kTile) : -1;
      } else {
        u.w.next(a);
        enter(u);
      }
    };
    Units at;
    at.w = walk;
    enter(at);
    auto note_bad = [&](int unit) {   // by the first loader warp
      const unsigned bad =
          __ballot_sync(0xffffffffu, at.key + (lane & 7) * 16 < at.w.sp.hi && (unsigned)at.ids >= (unsigned)a.pages) & 0xffu;
      if (lane == 0) {
        if (bad) atomicOr(a.status, kBadIndex);
        t.bad[unit & 15] = bad;
      }
    };
    if constexpr (T::kEight) {
      // a warp's one or two 16-key tiles of a slot (the n-th); their codes are loaded a slot ahead
      constexpr int kLanes = DP / 16, kRowsLoad = 32 / kLanes, kLoads = 16 / kRowsLoad;   // lanes a row; rows a load; loads a tile
      const int unit = lane % kLanes, row = lane / kLanes;
      struct Codes {
        uint4 x[2][kLoads];
        float scale[2];
      };
      auto load = [&](const Units& u, int n, Codes& c) {
        const bool is_v = n & 1;
        const unsigned char* pool = is_v ? a.pv : a.pk;
        const int64_t head_row = (int64_t)(u.w.triple / u.w.sp.tiles) * a.page_size;
#pragma unroll
        for (int e = 0; e < 2; ++e) {
          const int tile = (me + n) % kLoaders + kLoaders * e, first = u.key + tile * 16;
          const int page = __shfl_sync(0xffffffffu, u.ids, tile & 7);
          const bool there = tile < 8 && (unsigned)page < (unsigned)a.pages;
          const int64_t from = there ? page * a.page_rows + head_row + (first - page_index(first) * a.page_size) : 0;
#pragma unroll
          for (int i = 0; i < kLoads; ++i) {
            const int j = first + i * kRowsLoad + row;
            const bool in = there && unit < D / 16 && j >= u.w.sp.lo && j < u.w.sp.hi;
            c.x[e][i] = in ? __ldg(reinterpret_cast<const uint4*>(pool + (from + i * kRowsLoad + row) * D + unit * 16)) : make_uint4(0, 0, 0, 0);
          }
          const int j = first + (lane & 15);
          const bool in = there && !is_v && j >= u.w.sp.lo && j < u.w.sp.hi;
          c.scale[e] = in ? __ldg((lane < 16 ? a.ks : a.vs) + from + (lane & 15)) * (lane < 16 ? a.scale * 1.4426950408889634f : 1.f) : 0.f;
        }
      };
      auto store = [&](int n, const Codes& c) {
        const uint32_t dst = base + (n % kSlots) * T::kSlotBytes;
        const bool as_f16 = QF16 && !(n & 1);
#pragma unroll
        for (int e = 0; e < 2; ++e) {
          const int tile = (me + n) % kLoaders + kLoaders * e;
          if (tile >= 8) break;
          if (!(n & 1)) t.scales[((n / 2 & 7) * 2 + (lane >> 4)) * kTile + tile * 16 + (lane & 15)] = c.scale[e];
#pragma unroll
          for (int i = 0; i < kLoads; ++i) {
            const uint32_t w[4] = {c.x[e][i].x, c.x[e][i].y, c.x[e][i].z, c.x[e][i].w};
            uint32_t h[8];
#pragma unroll
            for (int x = 0; x < 4; ++x) widen4<FMT>(w[x], h[2 * x], h[2 * x + 1]);
            if (!as_f16) {
#pragma unroll
              for (int x = 0; x < 8; ++x) {
                const float2 f = __half22float2(*reinterpret_cast<const __half2*>(&h[x]));
                h[x] = pack2<true>(f.x, f.y);
              }
            }
            const int r = tile * 16 + i * kRowsLoad + row;
            if (unit < D / 16) {
              asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %4};" ::"r"(dst + unit_at(r, 2 * unit)), "r"(h[0]), "r"(h[1]),
                           "r"(h[2]), "r"(h[3])
                           : "memory");
              asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %4};" ::"r"(dst + unit_at(r, 2 * unit + 1)), "r"(h[4]),
                           "r"(h[5]), "r"(h[6]), "r"(h[7])
                           : "memory");
            }
          }
        }
      };
      auto finish = [&](int n, const Codes& c) {
        if (n >= kSlots) ok = wait(t.empty[n % kSlots], (n / kSlots - 1) & 1);
        ok = __all_sync(0xffffffffu, ok);
        if (!ok) return;
        store(n, c);
        warp_arrive(t.full[n % kSlots]);
      };
      Codes of_k, of_v;
      if (!at.done) load(at, 0, of_k);
      for (int n = 0; ok && !at.done; n += 2) {
        if (me == 0) note_bad(n / 2);
        load(at, n + 1, of_v);
        finish(n, of_k);
        step(at);
        if (!at.done) load(at, n + 2, of_k);
        if (ok) finish(n + 1, of_v);
      }
    } else {
      const int row_bytes = D * 2;
      constexpr int kLanes = DP / 8, kRowsCopy = 32 / kLanes;   // lanes a row; rows a copy
      const int unit = lane % kLanes, row = lane / kLanes;
      for (int n = 0; ok && !at.done; ++n) {
        if (n >= kSlots) ok = wait(t.empty[n % kSlots], (n / kSlots - 1) & 1);
        ok = __all_sync(0xffffffffu, ok);
        if (!ok) break;
        if (me == 0 && !(n & 1)) note_bad(n / 2);
        const uint32_t dst = base + (n % kSlots) * T::kSlotBytes;
        const unsigned char* pool = n & 1 ? a.pv : a.pk;
        const int64_t head_row = (int64_t)(at.w.triple / at.w.sp.tiles) * a.page_size;
        for (int tile = (me + n) % kLoaders; tile < 8; tile += kLoaders) {
          const int first = at.key + tile * 16, page = __shfl_sync(0xffffffffu, at.ids, tile);
          const bool there = (unsigned)page < (unsigned)a.pages;
          const int64_t from = there ? page * a.page_rows + head_row + (first - page_index(first) * a.page_size) : 0;
          const unsigned char* src = pool + (from + row) * row_bytes + unit * 16;
          if (there && first >= at.w.sp.lo && first + 16 <= at.w.sp.hi) {
            if (unit < units_row) {
#pragma unroll
              for (int i = 0; i < 16; i += kRowsCopy) copy_async<16>(dst + unit_at(tile * 16 + i + row, unit), src + i * row_bytes, true);
            }
          } else if (unit < units_row) {
#pragma unroll 1
            for (int i = 0; i < 16; i += kRowsCopy) {
              const int j = first + i + row;
              const bool in = there && j >= at.w.sp.lo && j < at.w.sp.hi;   // (else zeros)
              copy_async<16>(dst + unit_at(tile * 16 + i + row, unit), in ? src + i * row_bytes : a.pk, in);
            }
          }
        }
        copies_arrive(t.full[n % kSlots]);
        if (me == 0 && lane == 0) mbar_arrive(smem_u32(&t.full[n % kSlots]));   // for t.bad, which no copy writes
        if (n & 1) step(at);
      }
    }
    copy_wait<0>();
  } else if (warp >= kMmaWarp) {
    // ---- MMA: a warp a tile of rows ----
    const int b = warp - kMmaWarp;
    const uint32_t bf16 = (1u << 7) | (1u << 10);   // both operands' type; f16 is 0
    const uint32_t qk = (1u << 4) | (QF16 ? 0u : bf16) | ((uint32_t)(kTile >> 3) << 17) | ((uint32_t)(kTile >> 4) << 24);
    const uint32_t pv = (1u << 4) | (kSplit ? bf16 : 0u) | (1u << 16) | ((uint32_t)(D >> 3) << 17) | ((uint32_t)(kTile >> 4) << 24);
    const uint32_t s_to = tmem + T::kS + b * kTile, o_to = tmem + T::kO + b * kTile;
    bool ok = true;
    int j = 0, k = 0, triples = 0;   // units of the block, units and triples of this tile of rows
    for (; ok && !walk.done(); walk.next(a)) {
      const int count = walk.units();
      if (b == 1 && !has_two(walk)) {   // (one by one: a wait for a slot's later phase would take an earlier one of its parity for it)
        for (int i = 0; ok && i < 2 * count; ++i) {
          const int n = 2 * j + i, slot = n % kSlots;
          ok = wait(t.full[slot], (n / kSlots) & 1);
          ok = __all_sync(0xffffffffu, ok);
          if (ok) warp_arrive(t.empty[slot]);
        }
        j += count;
        continue;
      }
      for (int i = 0; ok && i < count; ++i, ++j, ++k) {
        // S, once the product with its last weights, which lie there, is done
        const int k_slot = (2 * j) % kSlots, v_slot = (2 * j + 1) % kSlots;
        ok = (k == 0 || wait(t.pv_done[b], (k - 1) & 1)) && (i > 0 || wait(t.q_full[b], triples & 1)) &&
             wait(t.full[k_slot], ((2 * j) / kSlots) & 1);
        ok = __all_sync(0xffffffffu, ok);
        if (!ok) break;
        asm volatile("fence.proxy.async.shared::cta;" ::: "memory");   // (the loaders' and the softmax's writes)
        tc_fence_after();
        const uint64_t q_desc = smem_desc(base + T::kQ + b * T::kSlotBytes), k_desc = smem_desc(base + k_slot * T::kSlotBytes);
        if (elect_one()) {
          // (unrolled, all under one election: 56 to 78 cycles a product of 128 x 128 x 16, 64 of them the tensor core's; rolled 92,
          // an election each 143)
#pragma unroll
          for (int kk = 0; kk < DP / 16; ++kk) {
            const uint64_t at = (uint64_t)((kk >> 2) * (kBlockBytes >> 4) + (kk & 3) * 2);
            if (kk < D / 16) mma_ss(s_to, q_desc + at, k_desc + at, qk, kk ? 1u : 0u);
          }
          mma_commit<false>(smem_u32(&t.s_full[b]), 0);
          mma_commit<false>(smem_u32(&t.empty[k_slot]), 0);
        }
        __syncwarp();
        // O (+)= P V
        ok = wait(t.full[v_slot], ((2 * j + 1) / kSlots) & 1) && (i > 0 || triples == 0 || wait(t.o_empty[b], (triples - 1) & 1)) &&
             wait(t.p_full[b], k & 1);
        ok = __all_sync(0xffffffffu, ok);
        if (!ok) break;
        asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
        tc_fence_after();
        const uint64_t v_desc = smem_desc_mn(base + v_slot * T::kSlotBytes);
        if (elect_one()) {
#pragma unroll
          for (int kk = 0; kk < kTile / 16; ++kk) {
            const uint32_t p = s_to + (kk >> 1) * 32 + (kk & 1) * 8;
            mma_ts(o_to, p, v_desc + kk * (2048 >> 4), pv, kk || i ? 1u : 0u);
            if (kSplit) mma_ts(o_to, p + 16, v_desc + kk * (2048 >> 4), pv, 1u);
          }
          mma_commit<false>(smem_u32(&t.pv_done[b]), 0);
          mma_commit<false>(smem_u32(&t.empty[v_slot]), 0);
        }
        __syncwarp();
      }
      ++triples;
    }
  } else {
    // ---- softmax: a thread a row ----
    const int b = warp >> 2, r = threadIdx.x & (kTile - 1);
    const uint32_t lanes = tmem + ((uint32_t)(warp & 3) << 21);   // this warp's 32 lanes
    const uint32_t s_at = lanes + T::kS + b * kTile, o_at = lanes + T::kO + b * kTile;
    int j = 0, k = 0, turns = 0;   // units of the block, of this tile of rows, and of those with two
    bool ok = true;
    // the triple's q: 32 rows a warp, whole rows at a time
    auto hand_over_q = [&](const Place& w) {
      constexpr int kLanes = DP / 8, kRowsCopy = 32 / kLanes;
      const int r0 = (warp & 3) * 32, its = row0_of(w) + b * kTile + r0 + lane, tok = its / a.group, head = w.triple / w.sp.tiles;
      const unsigned char* from =
          its < w.sp.rows ? a.q.at((int64_t)w.sp.first * a.new_tokens + tok, head * a.group + its - tok * a.group) : nullptr;
      const int unit = lane % kLanes;
      const uint32_t to = base + T::kQ + b * T::kSlotBytes;
#pragma unroll
      for (int i = 0; i < 32; i += kRowsCopy) {
        const int row = i + lane / kLanes;
        const unsigned char* src = reinterpret_cast<const unsigned char*>(
            __shfl_sync(0xffffffffu, reinterpret_cast<unsigned long long>(from), row));
        if (unit < units_row) copy_async<16>(to + unit_at(r0 + row, unit), src ? src + unit * 16 : a.pk, src != nullptr);   // (no row: zeros)
      }
      copies_arrive(t.q_full[b]);
    };
    auto takes_part = [&](const Place& w) { return b == 0 || has_two(w); };
    if (takes_part(walk)) hand_over_q(walk);
    bool handed = takes_part(walk);
    for (; ok && !walk.done(); walk.next(a)) {
      const int count = walk.units(), key_begin = (walk.sp.lo & ~15) + walk.first_unit * kTile;
      if (!takes_part(walk)) {
        j += count;
        handed = false;
        continue;
      }
      if (!handed) hand_over_q(walk);   // (the triple before had no rows here)
      const bool two = has_two(walk);
      const int head = walk.triple / walk.sp.tiles, row = row0_of(walk) + b * kTile + r, tok = row / a.group;
      const bool mine = row < walk.sp.rows, some = row - lane < walk.sp.rows;
      int pos = INT_MAX, lo = INT_MIN;
      if (mine) {
        const int2 seen = seen_by<kCommon>(a, walk.seq, walk.sp, tok);
        pos = seen.x, lo = seen.y;
      }
      const float factor = a.scale * 1.4426950408889634f;
      float m = -INFINITY, l = 0.f, seen_top = -INFINITY;   // (of the unit before)
      for (int i = 0; i < count; ++i, ++j, ++k) {
        const int key = key_begin + i * kTile;
        // the tiles make their weights in turn, so that the products of one run beside the other's softmax
        ok = wait(t.s_full[b], k & 1) && (!two || (b == 0 && turns == 0) || wait(t.turn[b], (b ? turns : turns - 1) & 1));
        ok = __all_sync(0xffffffffu, ok);
        if (!ok) break;
        if (some) {
          tc_fence_after();
          const uint32_t bad = t.bad[j & 15];
          const bool masked = !__all_sync(0xffffffffu, bad == 0 && key >= lo && key + kTile - 1 <= pos);
          const float* scales = t.scales + (j & 7) * 2 * kTile;
          // 32 scores less `shift`, -infinity where not seen
          auto scores = [&](int c, uint32_t (&u)[32], float shift) {
            float (&x)[32] = reinterpret_cast<float(&)[32]>(u);
            tmem_ld32_issue(s_at + c * 32, u);
            tmem_ld32_wait(u);
#pragma unroll
            for (int e = 0; e < 32; e += 4) {
              float4 by = make_float4(factor, factor, factor, factor);
              if constexpr (T::kEight) by = *reinterpret_cast<const float4*>(scales + c * 32 + e);   // (times the factor)
              const float2 less = make_float2(-shift, -shift);
              const float2 p = fma_two(make_float2(x[e], x[e + 1]), make_float2(by.x, by.y), less);
              const float2 q = fma_two(make_float2(x[e + 2], x[e + 3]), make_float2(by.z, by.w), less);
              x[e] = p.x, x[e + 1] = p.y, x[e + 2] = q.x, x[e + 3] = q.y;
            }
            if (masked) {
              const int at = key + c * 32;
              const int first = lo < at ? 0 : lo - at, last = pos >= at + 32 ? 32 : pos - at;   // columns seen
#pragma unroll
              for (int e = 0; e < 32; ++e)
                if (e < first || e > last || (bad >> (c * 2 + e / 16) & 1)) x[e] = -INFINITY;
            }
          };
          // The reference. bf16 weights have fp32's range, so only the first unit that a row sees needs its maximum before its
          // weights: a later one's moves the reference for the units after it. A row with a score further above it than kFarScore is
          // done again (an infinite reference says so, and nothing moves it): below that its weights, 2^107 a unit at most before
          // the reference follows, have a finite sum. f16 weights need each unit's maximum.
          auto move_to = [&](float top) {
            const bool move = m == -INFINITY ? top > -INFINITY : top > m + kHeadroom;
            if (i > 0 && __any_sync(0xffffffffu, move)) {
              const float f = move ? exp2_fast(m - (top - kBelow)) : 1.f;
              l *= f;
#pragma unroll 1
              for (int d = 0; d < D; d += 32) {   // (the last product into O is done: this S was begun after it)
                uint32_t o[32];
                tmem_ld32_issue(o_at + d, o);
                tmem_ld32_wait(o);
#pragma unroll
                for (int e = 0; e < 32; ++e) o[e] = __float_as_uint(__uint_as_float(o[e]) * f);
                tmem_st32(o_at + d, o);
              }
            }
            if (move) m = top - kBelow;
          };
          if (!kSplit || __any_sync(0xffffffffu, mine && m == -INFINITY && lo <= key + kTile - 1 && pos >= key)) {
            float top = -INFINITY;
#pragma unroll 1
            for (int c = 0; c < 4; ++c) {
              uint32_t u[32];
              scores(c, u, 0.f);
              const float (&x)[32] = reinterpret_cast<const float(&)[32]>(u);
#pragma unroll
              for (int e = 0; e < 32; e += 2) top = max_three(top, x[e], x[e + 1]);
            }
            move_to(top);
          } else if (i > 0) {
            move_to(seen_top);
          }
          const float shift = m == -INFINITY ? 0.f : m;
          float2 sum[2] = {};
          float tops[2] = {-INFINITY, -INFINITY};
#pragma unroll 1
          for (int c = 0; c < 4; ++c) {
            uint32_t u[32];
            scores(c, u, shift);
            const float (&y)[32] = reinterpret_cast<const float(&)[32]>(u);
            uint32_t hi[16], lo_term[kSplit ? 16 : 1];
#pragma unroll
            for (int e = 0; e < 32; e += 4) {
              float4 vs;
              if constexpr (T::kEight) vs = *reinterpret_cast<const float4*>(scales + kTile + c * 32 + e);
#pragma unroll
              for (int x = 0; x < 4; x += 2) {
                if (kSplit) tops[x / 2] = max_three(tops[x / 2], y[e + x], y[e + x + 1]);
                float2 p = make_float2(exp2_fast(y[e + x]), exp2_fast(y[e + x + 1]));
                sum[x / 2] = add_two(sum[x / 2], p);
                if constexpr (T::kEight)   // (a token that this row does not see but whose scale is NaN: the row is done again)
                  p = mul_two(p, x ? make_float2(vs.z, vs.w) : make_float2(vs.x, vs.y));
                const uint32_t h = pack2<kSplit>(p.x, p.y);
                hi[(e + x) / 2] = h;
                if constexpr (kSplit) {
                  const float2 rest = fma_two(make_float2(__uint_as_float(h << 16), __uint_as_float(h & 0xffff0000u)),
                                              make_float2(-1.f, -1.f), p);
                  lo_term[(e + x) / 2] = pack2<true>(rest.x, rest.y);
                }
              }
            }
            tmem_st16(s_at + c * 32, hi);
            if constexpr (kSplit) tmem_st16(s_at + c * 32 + 16, lo_term);
          }
          seen_top = fmaxf(tops[0], tops[1]) + shift;
          if (kSplit && fmaxf(tops[0], tops[1]) > kFarScore) m = INFINITY;
          l += (sum[0].x + sum[1].x) + (sum[0].y + sum[1].y);
          tmem_wait_st();
          tc_fence_before();
        }
        warp_arrive(t.p_full[b]);
        if (two) {
          warp_arrive(t.turn[b ^ 1]);
          ++turns;
        }
      }
      if (!ok) break;
      // with the last S of a triple complete every product with its q is done: the next one's takes its place, while the last
      // product with V runs
      Place next = walk;
      next.next(a);
      handed = !next.done() && takes_part(next);
      if (handed) hand_over_q(next);
      ok = wait(t.pv_done[b], (k - 1) & 1);
      ok = __all_sync(0xffffffffu, ok);
      if (!ok) break;
      // ---- the triple's end: O of this block's keys ----
      tc_fence_after();
      const bool whole = count == walk.sp.units;
      int c_first = blockIdx.x;
      if (!whole) c_first = line.block_of(walk.seq_base + walk.triple * (walk.sp.units + kCost) + kCost);
      float* slot = a.partial + ((int64_t)blockIdx.x * 2 + ((int)blockIdx.x == c_first ? 1 : 0)) * ((int64_t)a.slot_rows * (D + 2));
      if (some) {
        int64_t at_lse = 0;
        if (mine) out_at<kCommon>(a, walk.sp.first, head, row, &at_lse);
        // four dimensions of neighbouring rows side by side: of all rows of a kv head, or of the slot's
        const int64_t stride = whole ? (int64_t)a.table.seqs * a.rows : a.slot_rows;
        float4* to = whole ? reinterpret_cast<float4*>(a.part) + head * (D / 4) * stride + (int64_t)walk.sp.first * a.rows + row
                           : reinterpret_cast<float4*>(slot) + b * kTile + r;
        const float g = whole ? (l == 0.f ? 0.f : 1.f / l) : 1.f;
        float2 zero = make_float2(0.f, 0.f);   // NaN after a product that is not finite, or past kFar
#pragma unroll 1
        for (int d0 = 0; d0 < D; d0 += 32) {
          float o[32];
          tmem_ld32(o_at + d0, o);
#pragma unroll
          for (int e = 0; e < 32; e += 8) {
            if (d0 + e < D) {
              float v[8];
#pragma unroll
              for (int x = 0; x < 8; x += 2) {
                const float2 y = mul_two(make_float2(o[e + x], o[e + x + 1]), make_float2(kToEnd, kToEnd));
                zero = fma_two(y, make_float2(0.f, 0.f), zero);
                v[x] = g == 0.f ? 0.f : o[e + x] * g;
                v[x + 1] = g == 0.f ? 0.f : o[e + x + 1] * g;
              }
              if (mine) {
                to[(d0 + e) / 4 * stride] = make_float4(v[0], v[1], v[2], v[3]);
                to[((d0 + e) / 4 + 1) * stride] = make_float4(v[4], v[5], v[6], v[7]);
              }
            }
          }
        }
        auto write_end = [&](int at_row, int64_t at, float top, float sum) {
          if (!whole) *reinterpret_cast<float2*>(slot + (int64_t)a.slot_rows * D + at_row * 2) = make_float2(top, sum);
          else write_lse<kCommon>(a, at, top, sum);
        };
        if (mine) write_end(b * kTile + r, at_lse, m, l);
        // a row that is not finite is done again, past what was written; not where its sum of weights is NaN though no score was
        // far above the reference: then one that it sees is (masked ones are -infinity), and NaN is its result
        const bool odd = mine && (m == INFINITY || (!(zero.x + zero.y == 0.f) && l <= 3.402823466e+38f));
        const int key_end = min(key_begin + count * kTile, walk.sp.hi);
        for (unsigned rows = __ballot_sync(0xffffffffu, odd); rows; rows &= rows - 1) {
          const int src = __ffs(rows) - 1, its = row - lane + src, its_tok = its / a.group, its_qh = head * a.group + its - its_tok * a.group;
          const int its_pos = __shfl_sync(0xffffffffu, pos, src), its_lo = __shfl_sync(0xffffffffu, lo, src);
          const int64_t its_lse = __shfl_sync(0xffffffffu, at_lse, src);
          float4 acc;
          float top, sum;
          slow_row<FMT, QF16>(a, walk.sp.first, head, its_tok, its_qh, max(max(key_begin, its_lo), 0), min(key_end, its_pos + 1),
                              progress, &acc, &top, &sum);
          const int at_row = b * kTile + r - lane + src;
          const float s = whole ? (sum == 0.f ? 0.f : 1.f / sum) : 1.f;
          if (lane * 4 < D)
            to[src - lane + lane * stride] =
                s == 0.f ? make_float4(0.f, 0.f, 0.f, 0.f) : make_float4(acc.x * s, acc.y * s, acc.z * s, acc.w * s);
          if (lane == 0) write_end(at_row, its_lse, top, sum);
        }
      }
      tc_fence_before();
      warp_arrive(t.o_empty[b]);
    }
    copy_wait<0>();
  }

  // ---- nothing in flight: every product is done (the loaders have waited for their copies); TMEM is freed ----
  if (warp == kMmaWarp || warp == kMmaWarp + 1) {
    if (elect_one()) mma_commit<false>(smem_u32(&t.drain), 0);
    __syncwarp();
    mbar_wait_inline(smem_u32(&t.drain), 0, nullptr);
  }
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  if (warp == kMmaWarp) tmem_dealloc<false>(tmem, 512);
  asm volatile("griddepcontrol.wait;" ::: "memory");   // so that the end of this pass is the end of the one before it too
}

template <int FMT, bool QF16, int DP>
cudaError_t launch_heads(AttendArgs a, int num_sms, cudaStream_t st) {
  constexpr int kSmem = Common<FMT, QF16, DP>::kSmem;
  auto* kernel = common_kernel<FMT, QF16, DP>;
  static std::atomic<bool> ready[kMaxDevices];
  if (a.device >= kMaxDevices || !ready[a.device].load(std::memory_order_relaxed)) {
    const cudaError_t e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, kSmem);
    if (e != cudaSuccess) return e;
    if (a.device < kMaxDevices) ready[a.device].store(true, std::memory_order_relaxed);
  }
  const int64_t units = ((int64_t)a.max_len + 15) / kTile + 1 + kCost;
  const double tiles = (double)a.table.seqs * a.rows / kRows + a.groups, most = tiles * a.kv_heads * (double)units;
  if (most >= 2147483648.0) return cudaErrorNotSupported;   // cells are counted in 32 bits
  a.parts = most < (double)num_sms ? (int)most : num_sms;
  return launch_form<kCommon>(kernel, a.parts, Common<FMT, QF16, DP>::kThreads, kSmem, a, st);
}
template <int FMT, bool QF16>
cudaError_t launch_type(const AttendArgs& a, int num_sms, cudaStream_t st) {
  return a.head_dim <= 64 ? launch_heads<FMT, QF16, 64>(a, num_sms, st) : launch_heads<FMT, QF16, 128>(a, num_sms, st);
}

}  // namespace

cudaError_t launch_common_tc(const AttendArgs& a, int format, int num_sms, cudaStream_t st) {
  switch (format) {
    case LACACHE_KV_BF16: return launch_type<LACACHE_KV_BF16, false>(a, num_sms, st);
    case LACACHE_KV_F16: return launch_type<LACACHE_KV_F16, true>(a, num_sms, st);
    case LACACHE_KV_E4M3:
      return a.q_f16 ? launch_type<LACACHE_KV_E4M3, true>(a, num_sms, st) : launch_type<LACACHE_KV_E4M3, false>(a, num_sms, st);
    default:
      return a.q_f16 ? launch_type<LACACHE_KV_INT8, true>(a, num_sms, st) : launch_type<LACACHE_KV_INT8, false>(a, num_sms, st);
  }
}

}  // namespace lc
