// Attention of new tokens over the paged cache: the kernel, instantiated for one cache format a source file
// (kv_attend_*.cu) and dispatched by kv_attend.cu.
//
//   s_j = scale <q, k_j>,  out = sum_j e^(s_j - m) v_j / sum_j e^(s_j - m)   over the visible j
//
// A kv head's K and V are read once for all rows that share it: the q heads of its group times the new tokens. With up to
// 32 rows that is 4 x rows flops a cached element, so the kernel is bound by reading the cache, and every choice below is
// about keeping enough loads in flight with little work a byte.
//
// Products. Both run on the warp-level tensor instruction m16n8k16, with keys (or dimensions) as M and the rows of q as N:
// a tile of 8 rows wastes nothing at 8 rows, where the 64- or 128-row tiles of tcgen05 would take the scores through TMEM
// and shared memory for no gain in a kernel that waits for HBM.
//   S^T [16 keys x 8 rows] = K [16 x d] Q^T [d x 8],   O^T [16 dims x 8 rows] += V^T [16 dims x 16 keys] P^T [16 keys x 8]
// The order of a contraction is free, and so is the naming of V's dimensions, so each lane takes 16 contiguous bytes of a
// row of K or V as its share of several instructions' A operand: lane (g, t) = (lane / 4, lane % 4) owns bytes 16 t of every
// 64 of key rows g and g + 8 of K, and (8-bit formats) of V bytes 16 g of every 128 of the rows of keys 2t, 2t+1, 2t+8 and 2t+9. Those
// copies to shared memory (cp.async) are a deep register file with an asynchronous front: each lane reads back what it copied
// itself. A 16-bit V goes through shared memory in swizzled rows and comes back transposed (ldmatrix); 8-bit codes are
// widened first and paired by byte permutes. Nothing is shared between warps: no barriers in the loop. P^T is the transpose of the S^T accumulator, one movmatrix for 8 x 8.
//
// Softmax. Base 2, running maximum m a row, moved only when a score exceeds it by more than 8: weights then stay below 2^8,
// the sum is fp32, and most tiles need a vote instead of a maximum over the lanes. Weights: f16 for f16 and 8-bit caches (11
// bits); on a bf16 cache, whose products need bf16 weights of 8 bits, a weight is split in two bf16 terms (16 bits), as
// one alone would add an error as large as the output's own rounding.
//
// 8-bit rows. Codes become f16 exactly. q of a bf16 type is scaled to f16 by a power of two that brings its row's largest
// magnitude to [1, 2): exact for elements within 2^-14 of that. The scales multiply the scores (k) and the weights (v);
// the weights times scales are brought into f16's range by a factor a row, kept like the maximum.
//
// Work. All (sequence, kv head, tile of rows) triples, each of its length in units of 4 warps x KT keys, form one line of
// units; block i of P takes the i-th of P equal parts, whatever the lengths. Within a unit each warp has KT keys of its
// own, with its own maximum and sum; they join through shared memory at the end of a triple. A triple that several blocks
// share is joined by whichever of them comes last, in the order of the blocks, so results do not depend on it. Nothing
// waits for another block.
#pragma once

#include <math.h>

#include <atomic>

#include "decode.cuh"

namespace lc {

struct AttendArgs {
  Table table;
  int new_tokens, q_heads, kv_heads, group, head_dim, page_size, window, q_f16;
  int row_tiles;        // tiles of rows a kv head
  int rows;             // rows a kv head: group x new_tokens
  int parts;            // blocks the units may be split over (at most the grid)
  int max_len;          // positions the table can name
  int device;
  int64_t pages;
  float scale;
  const int32_t* lengths;
  const int32_t* starts;
  Rows q, out;
  float* lse;
  const unsigned char* pk;
  const unsigned char* pv;
  const float* ks;
  const float* vs;
  float* partial;       // two slots a block: [kMaxRowTile rows x DP] sums, then (m, l) a row
  unsigned int* arrived;   // blocks that have left their part of the triple that begins in this block; zero between launches
  unsigned int* status;
};

constexpr int kAttendWarps = 4;
constexpr int kAttendThreads = kAttendWarps * 32;
constexpr int kMinUnits = 1;                 // a block's least part
constexpr int kMaxRowTile = 32;
constexpr int kMaxPositions = 1 << 30;      // a table's reach is cut to this
constexpr int kMaxDevices = 64;

// Floats of one partial slot, for the largest row tile at a padded head dimension.
constexpr int64_t partial_floats(int padded) { return (int64_t)(padded == 256 ? 16 : 32) * (padded + 2); }
constexpr int padded_dim(int head_dim) { return head_dim <= 64 ? 64 : head_dim <= 128 ? 128 : 256; }

constexpr int kMaxBlocksPerSm = 4;           // sizes the scratch: two partial slots a block
cudaError_t launch_attend_bf16(const AttendArgs& a, int num_sms, cudaStream_t st);
cudaError_t launch_attend_f16(const AttendArgs& a, int num_sms, cudaStream_t st);
cudaError_t launch_attend_e4m3(const AttendArgs& a, int num_sms, cudaStream_t st);
cudaError_t launch_attend_int8(const AttendArgs& a, int num_sms, cudaStream_t st);

namespace {

template <int FMT, int DP, int NT>
struct AttendConfig {
  static constexpr bool kEight = FMT == LACACHE_KV_E4M3 || FMT == LACACHE_KV_INT8;
  static constexpr int kItem = kEight ? 1 : 2;
  static constexpr int kRows = 8 * NT;
  static constexpr int kSub = (kEight ? DP <= 128 : DP <= 64) ? 2 : 1;   // 16-key tiles a stage: 4 KB of K at most at 128
  static constexpr int kKeys = 16 * kSub;                                // keys a stage of a warp
  static constexpr int kUnit = kAttendWarps * kKeys;
  static constexpr int kKPieces = DP * kItem / 64;                       // 16-byte pieces of a lane in a row of K
  static constexpr int kVBytes = DP * kItem >= 128 ? 16 : 8;             // bytes of a piece of V
  static constexpr int kVPieces = DP * kItem / (8 * kVBytes);
  static constexpr int kUnits = DP / 8 < 32 ? DP / 8 : 32;               // 16-bit V: 16-byte units of a row
  static constexpr int kUnitRows = 32 / kUnits;                          // ... and rows that one copy of the warp covers
  static constexpr int kTileBytes = 16 * DP * kItem;                     // K (or V) of 16 keys
  static constexpr int kStageBytes = kSub * 2 * kTileBytes + (kEight ? kKeys * 8 : 0);
  static constexpr int kStages = DP == 256 && !kEight ? 3 : kStageBytes <= 4096 + 256 ? 6 : kStageBytes <= 8192 + 256 ? 3 : 3;
  static constexpr int kMTiles = DP / 16;
  static constexpr int kQStride = DP * 2 + 64;                           // bytes of a row of q in shared memory
  static constexpr int kRing = kAttendWarps * kStages * kStageBytes;
  static constexpr int kOStride = DP + 4;                                // floats of a row of sums in the join
  static constexpr int kJoin = kAttendWarps * kRows * kOStride * 4;
  static constexpr int kBody = kRing > kJoin ? kRing : kJoin;            // the join reuses the ring
  static constexpr int kSmem = kBody + kRows * kQStride;
};

__device__ __forceinline__ uint32_t shared_addr(const void* p) { return (uint32_t)__cvta_generic_to_shared(p); }
template <int BYTES>
__device__ __forceinline__ void copy_async(uint32_t dst, const void* src, bool live) {
  const int n = live ? BYTES : 0;   // 0: the destination is filled with zeros and src is not read
  if constexpr (BYTES == 16)
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst), "l"(src), "r"(n) : "memory");
  else
    asm volatile("cp.async.ca.shared.global [%0], [%1], %2, %3;" ::"r"(dst), "l"(src), "n"(BYTES), "r"(n) : "memory");
}
__device__ __forceinline__ void copy_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int N>
__device__ __forceinline__ void copy_wait() {
  asm volatile("cp.async.wait_group %0;" ::"n"(N) : "memory");
}

template <bool BF16>
__device__ __forceinline__ void mma16816(float (&c)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0,
                                         uint32_t b1) {
  if constexpr (BF16)
    asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
                 : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
                 : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
  else
    asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
                 : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
                 : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}
// 8 x 8 of 16-bit values, one row of four lanes' registers, transposed across the warp.
__device__ __forceinline__ uint32_t transpose8(uint32_t x) {
  uint32_t y;
  asm volatile("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(y) : "r"(x));
  return y;
}
__device__ __forceinline__ float exp2_fast(float x) {
  float y;
  asm("ex2.approx.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}

// Four 8 x 8 tiles of 16-bit values from shared memory, transposed: lane l names the 16-byte row l % 8 of tile l / 8.
__device__ __forceinline__ void load_transposed(uint32_t addr, uint32_t& a0, uint32_t& a1, uint32_t& a2, uint32_t& a3) {
  asm volatile("ldmatrix.sync.aligned.m8n8.x4.trans.shared.b16 {%0, %1, %2, %3}, [%4];"
               : "=r"(a0), "=r"(a1), "=r"(a2), "=r"(a3)
               : "r"(addr)
               : "memory");
}
// Where a 16-bit row of V (key j of its tile) keeps its 16-byte unit u: eight keys' units of one column lie in different
// banks.
template <int DP>
__device__ __forceinline__ int v_unit(int j, int u) {
  return j * (DP * 2) + ((u ^ (j & 7)) * 16);
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

template <bool BF16>
__device__ __forceinline__ uint32_t pack2(float x, float y) {
  if constexpr (BF16) {
    const __nv_bfloat162 h = __floats2bfloat162_rn(x, y);
    return *reinterpret_cast<const uint32_t*>(&h);
  } else {
    const __half2 h = __floats2half2_rn(x, y);
    return *reinterpret_cast<const uint32_t*>(&h);
  }
}

// One triple's view of a sequence: its length (clamped to what the table can name), the positions its rows of this tile
// see at most, [lo, hi), and its units.
struct Span {
  int len, lo, hi, units;
};
__device__ __forceinline__ Span span_of(const AttendArgs& a, int seq, int unit_keys) {
  Span s;
  int len = a.lengths[seq];
  len = len < 0 ? 0 : len > a.max_len ? a.max_len : len;
  const int first = len - a.new_tokens;   // the first row's position
  int lo = a.starts ? a.starts[seq] : 0;
  if (a.window > 0 && first - a.window + 1 > lo) lo = first - a.window + 1;   // window < 2^31, first >= -512: no overflow
  lo = lo < 0 ? 0 : lo > len ? len : lo;
  s.len = len;
  s.lo = lo;
  s.hi = len;
  const int keys = len - (lo & ~15);
  s.units = keys <= 0 ? 1 : (keys + unit_keys - 1) / unit_keys;   // an empty sequence has rows to write
  return s;
}

__device__ __forceinline__ int64_t warp_sum64(int64_t x) {
#pragma unroll
  for (int o = 16; o; o >>= 1) x += __shfl_xor_sync(0xffffffffu, x, o);
  return x;
}

template <int FMT, int DP, int NT>
__global__ void __launch_bounds__(kAttendThreads) attend_kernel(const __grid_constant__ AttendArgs a) {
  using C = AttendConfig<FMT, DP, NT>;
  constexpr bool kBf16 = FMT == LACACHE_KV_BF16;
  constexpr bool kQInRegs = NT * DP <= 128;   // more would spill: q is read from shared memory at its use
  extern __shared__ __align__(128) unsigned char smem[];
  __shared__ float stat_m[kAttendWarps][C::kRows], stat_l[kAttendWarps][C::kRows];
  __shared__ int row_pos[C::kRows], row_lo[C::kRows];   // a row's own last and first visible position
  __shared__ float row_factor[C::kRows];                // scale log2(e), and what the row's q was divided by
  __shared__ int page_ids[kAttendWarps][C::kStages][C::kSub];
  __shared__ unsigned int last_flag;
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, g = lane >> 2, t = lane & 3;
  const int D = a.head_dim;
  const int64_t per_seq = (int64_t)a.kv_heads * a.row_tiles;

  // ---- this block's part of the line of units (each warp for itself) ----
  int64_t total = 0;
  for (int s = lane; s < a.table.seqs; s += 32) total += span_of(a, s, C::kUnit).units;
  total = warp_sum64(total) * per_seq;
  int64_t parts = (total + kMinUnits - 1) / kMinUnits;
  if (parts > a.parts) parts = a.parts;
  const int64_t block = blockIdx.x;
  if (block >= parts) return;
  int64_t u = total * block / parts;
  const int64_t u_end = total * (block + 1) / parts;
  int seq = 0;
  int64_t seq_base = 0;   // units before sequence seq
  for (int s0 = 0; s0 < a.table.seqs; s0 += 32) {
    const int64_t own = s0 + lane < a.table.seqs ? span_of(a, s0 + lane, C::kUnit).units * per_seq : 0;
    int64_t upto = own;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const int64_t y = __shfl_up_sync(0xffffffffu, upto, o);
      if (lane >= o) upto += y;
    }
    const unsigned past = __ballot_sync(0xffffffffu, seq_base + upto > u);
    if (past) {
      const int l0 = __ffs(past) - 1;
      seq = s0 + l0;
      seq_base += __shfl_sync(0xffffffffu, upto - own, l0);
      break;
    }
    seq_base += __shfl_sync(0xffffffffu, upto, 31);
  }

  unsigned char* ring = smem + warp * C::kStages * C::kStageBytes;
  unsigned char* q_smem = smem + C::kBody;
  const uint32_t ring_addr = shared_addr(ring);

  while (u < u_end) {
    // ---- the triple that unit u belongs to ----
    Span sp = span_of(a, seq, C::kUnit);
    while (seq + 1 < a.table.seqs && u >= seq_base + sp.units * per_seq) {
      seq_base += sp.units * per_seq;
      sp = span_of(a, ++seq, C::kUnit);
    }
    const int64_t in_seq = u - seq_base;
    const int triple = (int)(in_seq / sp.units), first_unit = (int)(in_seq % sp.units);
    const int head = triple / a.row_tiles, tile = triple % a.row_tiles;
    const int64_t begin = u - first_unit;                         // the triple's units: [begin, begin + sp.units)
    const int64_t left = u_end - u;
    const int units = sp.units - first_unit < left ? sp.units - first_unit : (int)left;
    const int row0 = tile * C::kRows;
    const int live_rows = a.rows - row0 < C::kRows ? a.rows - row0 : C::kRows;
    if (threadIdx.x == 0) {
      const int raw = a.lengths[seq];
      if (raw < 0 || raw > a.max_len) atomicOr(a.status, kBadIndex);
    }

    __syncthreads();   // the previous triple's readers are done

    // ---- this warp's keys: KT from each unit ----
    const int key0 = (sp.lo & ~15) + first_unit * C::kUnit + warp * C::kKeys;
      const int32_t* table_row = a.table.pages + seq * a.table.stride;

    // page ids of the stage that is issued next, read one stage ahead of their use
    int next_page[C::kSub], next_slot[C::kSub];
    auto look_up = [&](int i) {
      const int key = key0 + i * C::kUnit;
#pragma unroll
      for (int s = 0; s < C::kSub; ++s) {
        const int at = key + 16 * s;
        next_page[s] = -1;
        next_slot[s] = 0;
        if (i < units && at < sp.hi) {
          const int index = at / a.page_size;
          next_slot[s] = at - index * a.page_size;
          next_page[s] = __ldg(table_row + index);
        }
      }
    };
    auto issue = [&](int i) {
      if (i < units) {
        const int stage = i % C::kStages;
        const uint32_t at = ring_addr + stage * C::kStageBytes;
        const int key = key0 + i * C::kUnit;
#pragma unroll
        for (int s = 0; s < C::kSub; ++s) {
          const int k0 = key + 16 * s;
          int page = next_page[s];
          if (page < 0 || page >= a.pages) {
            if (k0 < sp.hi && lane == 0) atomicOr(a.status, kBadIndex);
            page = -1;
          }
          if (lane == 0) page_ids[warp][stage][s] = page;
          const int64_t row = ((int64_t)(page < 0 ? 0 : page) * a.kv_heads + head) * a.page_size + next_slot[s];
          const unsigned char* kp = a.pk + row * (int64_t)(D * C::kItem);
          const unsigned char* vp = a.pv + row * (int64_t)(D * C::kItem);
          // a key outside [lo, hi) is not read: zeros take its place
          auto inside = [&](int j) { return page >= 0 && k0 + j >= sp.lo && k0 + j < sp.hi; };
          const uint32_t kd = at + s * 2 * C::kTileBytes, vd = kd + C::kTileBytes;
          const int row_bytes = D * C::kItem;
          const unsigned char* ksrc = kp + (int64_t)(g * row_bytes + t * 16);
          if (D == DP && page >= 0 && k0 >= sp.lo && k0 + 16 <= sp.hi) {   // nothing to leave out: most tiles
#pragma unroll
            for (int c = 0; c < C::kKPieces; ++c) {
              copy_async<16>(kd + c * 512 + lane * 16, ksrc + c * 64, true);
              copy_async<16>(kd + (C::kKPieces + c) * 512 + lane * 16, ksrc + 8 * DP * C::kItem + c * 64, true);
            }
            if constexpr (C::kEight) {
              const unsigned char* vsrc = vp + 2 * t * DP + g * C::kVBytes;
#pragma unroll
              for (int r = 0; r < 4; ++r) {
#pragma unroll
                for (int c = 0; c < C::kVPieces; ++c)
                  copy_async<C::kVBytes>(vd + (r * C::kVPieces + c) * (32 * C::kVBytes) + lane * C::kVBytes,
                                         vsrc + ((r & 1) + 8 * (r >> 1)) * DP + c * 8 * C::kVBytes, true);
              }
            } else {
              const unsigned char* vsrc = vp + (lane / C::kUnits) * (DP * 2) + (lane % C::kUnits) * 16;
#pragma unroll
              for (int i = 0; i < C::kUnits / 2; ++i)
                copy_async<16>(vd + v_unit<DP>(i * C::kUnitRows + lane / C::kUnits, lane % C::kUnits), vsrc + i * 512, true);
            }
          } else {
#pragma unroll
            for (int r = 0; r < 2; ++r) {
              const bool in = inside(g + 8 * r);
#pragma unroll
              for (int c = 0; c < C::kKPieces; ++c) {
                const bool live = in && (c * 64 + t * 16) < row_bytes;
                copy_async<16>(kd + (r * C::kKPieces + c) * 512 + lane * 16, live ? ksrc + 8 * r * row_bytes + c * 64 : a.pk,
                               live);
              }
            }
            if constexpr (C::kEight) {
#pragma unroll
              for (int r = 0; r < 4; ++r) {
                const int j = 2 * t + (r & 1) + 8 * (r >> 1);
                const bool in = inside(j);
#pragma unroll
                for (int c = 0; c < C::kVPieces; ++c) {
                  const int d = c * 8 * C::kVBytes + g * C::kVBytes;
                  const bool live = in && d < row_bytes;
                  copy_async<C::kVBytes>(vd + (r * C::kVPieces + c) * (32 * C::kVBytes) + lane * C::kVBytes,
                                         live ? vp + j * row_bytes + d : a.pv, live);
                }
              }
            } else {
#pragma unroll
              for (int i = 0; i < C::kUnits / 2; ++i) {
                const int j = i * C::kUnitRows + lane / C::kUnits, unit = lane % C::kUnits;
                const bool live = inside(j) && unit * 16 < row_bytes;
                copy_async<16>(vd + v_unit<DP>(j, unit), live ? vp + j * row_bytes + unit * 16 : a.pv, live);
              }
            }
          }
          if constexpr (C::kEight) {
            // scales: lanes 0-15 those of k, 16-31 those of v
            const int j = lane & 15;
            const bool in = inside(j);
            const float* src = (lane < 16 ? a.ks : a.vs) + (in ? row + j : 0);
            copy_async<4>(at + C::kSub * 2 * C::kTileBytes + (s * 32 + lane) * 4, src, in);
          }
        }
        look_up(i + 1);
      }
      copy_commit();
    };

    int all_hi, all_lo;   // positions that every live row sees: [all_lo, all_hi]
    const bool rows_differ = a.new_tokens > 1;
    float factor[NT][2];
    uint4 qreg[kQInRegs ? NT * C::kKPieces * (C::kEight ? 2 : 1) : 1];
    float o[C::kMTiles][NT][4];
    float m[NT][2], l[NT][2], inv[NT][2];
    bool split = kBf16, again = false;   // bf16 weights in two terms
    do {
      look_up(0);
#pragma unroll 1
      for (int i = 0; i < C::kStages - 1; ++i) issue(i);
      if (!again) {
    // ---- q into shared memory, in the order of the K pieces, while the first keys are on their way ----
    for (int r = warp; r < C::kRows; r += kAttendWarps) {
      const int row = row0 + r;
      const bool live = r < live_rows;
      const int tok = live ? row / a.group : 0, qh = head * a.group + (live ? row % a.group : 0);
      const unsigned char* src = a.q.p + ((int64_t)seq * a.new_tokens + tok) * a.q.token + qh * a.q.head;
      float x[8] = {};
      const int d0 = lane * 8;
      const bool has = live && d0 < D;
      uint4 raw = make_uint4(0, 0, 0, 0);
      if (has) {
        raw = *reinterpret_cast<const uint4*>(src + d0 * 2);
        widen8(raw, x, __nv_bfloat16());   // used for bf16 rows alone
      }
      float back = 1.f;
      if (C::kEight && !a.q_f16) {
        float top = 0.f;
#pragma unroll
        for (int i = 0; i < 8; ++i) top = fmaxf(top, fabsf(x[i]));
#pragma unroll
        for (int o = 16; o; o >>= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, o));
        // the power of two below top: its exponent bits alone, at most 2^126 (1 for zeros, infinities and subnormals)
        uint32_t e = __float_as_uint(top) & 0x7f800000u;
        if (e != 0 && e != 0x7f800000u) {
          e = e < 0x7e800000u ? e : 0x7e800000u;
          back = __uint_as_float(e);
          const float down = __uint_as_float(0x7f000000u - e);
#pragma unroll
          for (int i = 0; i < 8; ++i) x[i] *= down;
        }
        raw = pack8(x, __half());
      }
      if (d0 < DP) *reinterpret_cast<uint4*>(q_smem + r * C::kQStride + d0 * 2) = raw;
      if (lane == 0) {
        const int p = live ? sp.len - a.new_tokens + tok : -1;
        int lo = a.starts ? a.starts[seq] : 0;
        if (a.window > 0 && p - a.window + 1 > lo) lo = p - a.window + 1;
        row_pos[r] = p;
        row_lo[r] = lo;
        row_factor[r] = a.scale * 1.4426950408889634f * back;
      }
    }
    __syncthreads();

    all_hi = row_pos[0];
    all_lo = row_lo[live_rows - 1];
#pragma unroll
    for (int n = 0; n < NT; ++n) {
      factor[n][0] = row_factor[n * 8 + 2 * t];
      factor[n][1] = row_factor[n * 8 + 2 * t + 1];
    }
    if constexpr (kQInRegs) {
#pragma unroll
      for (int n = 0; n < NT; ++n) {
#pragma unroll
        for (int c = 0; c < C::kKPieces; ++c) {
          const unsigned char* q = q_smem + (n * 8 + g) * C::kQStride;
          if constexpr (C::kEight) {
            const uint4* p = reinterpret_cast<const uint4*>(q + (c * 64 + t * 16) * 2);
            qreg[(n * C::kKPieces + c) * 2] = p[0];
            qreg[(n * C::kKPieces + c) * 2 + 1] = p[1];
          } else {
            qreg[n * C::kKPieces + c] = *reinterpret_cast<const uint4*>(q + (c * 32 + t * 8) * 2);
          }
        }
      }
    }

      }
#pragma unroll
    for (int n = 0; n < NT; ++n) {
#pragma unroll
      for (int i = 0; i < C::kMTiles; ++i) o[i][n][0] = o[i][n][1] = o[i][n][2] = o[i][n][3] = 0.f;
      m[n][0] = m[n][1] = -INFINITY;
      l[n][0] = l[n][1] = 0.f;
      inv[n][0] = inv[n][1] = C::kEight ? 0x1p126f : 1.f;
    }
    for (int i = 0; i < units; ++i) {
      issue(i + C::kStages - 1);
      copy_wait<C::kStages - 1>();
      __syncwarp();
      const int stage = i % C::kStages;
      const unsigned char* st = ring + stage * C::kStageBytes;
      const int key = key0 + i * C::kUnit;

      // scores
      float s[C::kSub][NT][4];
#pragma unroll
      for (int b = 0; b < C::kSub; ++b) {
        const unsigned char* kt = st + b * 2 * C::kTileBytes;
#pragma unroll
        for (int n = 0; n < NT; ++n) s[b][n][0] = s[b][n][1] = s[b][n][2] = s[b][n][3] = 0.f;
#pragma unroll
        for (int c = 0; c < C::kKPieces; ++c) {
          const uint4 x = *reinterpret_cast<const uint4*>(kt + c * 512 + lane * 16);
          const uint4 y = *reinterpret_cast<const uint4*>(kt + (C::kKPieces + c) * 512 + lane * 16);
          if constexpr (C::kEight) {
            const uint32_t xw[4] = {x.x, x.y, x.z, x.w}, yw[4] = {y.x, y.y, y.z, y.w};
            uint32_t xa[8], ya[8];
#pragma unroll
            for (int w = 0; w < 4; ++w) {
              widen4<FMT>(xw[w], xa[2 * w], xa[2 * w + 1]);
              widen4<FMT>(yw[w], ya[2 * w], ya[2 * w + 1]);
            }
#pragma unroll
            for (int n = 0; n < NT; ++n) {
              uint4 q0, q1;
              if constexpr (kQInRegs) {
                q0 = qreg[(n * C::kKPieces + c) * 2], q1 = qreg[(n * C::kKPieces + c) * 2 + 1];
              } else {
                const uint4* p = reinterpret_cast<const uint4*>(q_smem + (n * 8 + g) * C::kQStride + (c * 64 + t * 16) * 2);
                q0 = p[0], q1 = p[1];
              }
              mma16816<false>(s[b][n], xa[0], ya[0], xa[1], ya[1], q0.x, q0.y);
              mma16816<false>(s[b][n], xa[2], ya[2], xa[3], ya[3], q0.z, q0.w);
              mma16816<false>(s[b][n], xa[4], ya[4], xa[5], ya[5], q1.x, q1.y);
              mma16816<false>(s[b][n], xa[6], ya[6], xa[7], ya[7], q1.z, q1.w);
            }
          } else {
#pragma unroll
            for (int n = 0; n < NT; ++n) {
              uint4 q;
              if constexpr (kQInRegs) q = qreg[n * C::kKPieces + c];
              else q = *reinterpret_cast<const uint4*>(q_smem + (n * 8 + g) * C::kQStride + (c * 32 + t * 8) * 2);
              mma16816<kBf16>(s[b][n], x.x, y.x, x.y, y.y, q.x, q.y);
              mma16816<kBf16>(s[b][n], x.z, y.z, x.w, y.w, q.z, q.w);
            }
          }
        }
      }

      // base-2 scores, masks, and whether a maximum has to move
      float vscale[C::kSub][2];
      bool move = false, some_masked = false;
#pragma unroll
      for (int b = 0; b < C::kSub; ++b) {
        const int k0 = key + 16 * b;
        float kscale[2] = {1.f, 1.f};
        if constexpr (C::kEight) {
          const float* sc = reinterpret_cast<const float*>(st + C::kSub * 2 * C::kTileBytes) + b * 32;
          kscale[0] = sc[g], kscale[1] = sc[g + 8];
          vscale[b][0] = sc[16 + g], vscale[b][1] = sc[24 + g];
        }
        const bool page_ok = page_ids[warp][stage][b] >= 0;
        const bool masked = !page_ok || k0 < all_lo || k0 + 15 > all_hi;
        some_masked |= masked;
#pragma unroll
        for (int n = 0; n < NT; ++n) {
#pragma unroll
          for (int e = 0; e < 4; ++e) s[b][n][e] *= factor[n][e & 1] * kscale[e >> 1];
          if (masked) {
#pragma unroll
            for (int e = 0; e < 4; ++e) {
              const int j = k0 + g + 8 * (e >> 1), r = n * 8 + 2 * t + (e & 1);
              if (!page_ok || j > row_pos[r] || j < row_lo[r]) s[b][n][e] = -INFINITY;
            }
          }
#pragma unroll
          for (int e = 0; e < 4; ++e) move |= s[b][n][e] > m[n][e & 1] + 8.f;
        }
      }
      if (__any_sync(0xffffffffu, move)) {
#pragma unroll
        for (int n = 0; n < NT; ++n) {
#pragma unroll
          for (int h = 0; h < 2; ++h) {
            float top = m[n][h];
#pragma unroll
            for (int b = 0; b < C::kSub; ++b) top = fmaxf(top, fmaxf(s[b][n][h], s[b][n][h + 2]));
            top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 4));
            top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 8));
            top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 16));
            const float f = m[n][h] == -INFINITY ? 0.f : exp2_fast(m[n][h] - top);
            m[n][h] = top;
            l[n][h] *= f;
#pragma unroll
            for (int d = 0; d < C::kMTiles; ++d) {
              o[d][n][h] *= f;
              o[d][n][h + 2] *= f;
            }
          }
        }
      }
      // weights; in 8-bit formats times v's scales, brought below 2^8 by the row's factor
      float big = 0.f;
#pragma unroll
      for (int n = 0; n < NT; ++n) {
        const float m0 = m[n][0] == -INFINITY ? 0.f : m[n][0], m1 = m[n][1] == -INFINITY ? 0.f : m[n][1];
#pragma unroll
        for (int b = 0; b < C::kSub; ++b) {
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            const bool out = s[b][n][e] == -INFINITY;
            const float p = exp2_fast(s[b][n][e] - ((e & 1) ? m1 : m0));
            l[n][e & 1] += p;
            if constexpr (C::kEight) {
              s[b][n][e] = out ? 0.f : p * vscale[b][e >> 1];   // a masked token's scale may be NaN
              big = fmaxf(big, s[b][n][e] * inv[n][e & 1]);
            } else {
              s[b][n][e] = p;
            }
          }
        }
      }
      if constexpr (C::kEight) {
        if (__any_sync(0xffffffffu, big > 256.f)) {
#pragma unroll
          for (int n = 0; n < NT; ++n) {
#pragma unroll
            for (int h = 0; h < 2; ++h) {
              float top = 0.f;
#pragma unroll
              for (int b = 0; b < C::kSub; ++b) top = fmaxf(top, fmaxf(s[b][n][h], s[b][n][h + 2]));
              top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 4));
              top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 8));
              top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 16));
              if (top * inv[n][h] > 1.f) {
                const float now = __frcp_rn(top), f = now / inv[n][h];
                inv[n][h] = now;
#pragma unroll
                for (int d = 0; d < C::kMTiles; ++d) {
                  o[d][n][h] *= f;
                  o[d][n][h + 2] *= f;
                }
              }
            }
          }
        }
      }

      // O^T += V^T P^T
#pragma unroll
      for (int b = 0; b < C::kSub; ++b) {
        uint32_t p0[NT], p1[NT], r0[NT], r1[NT];
#pragma unroll
        for (int n = 0; n < NT; ++n) {
          float w[4];
#pragma unroll
          for (int e = 0; e < 4; ++e) w[e] = C::kEight ? s[b][n][e] * inv[n][e & 1] : s[b][n][e];
          const uint32_t u0 = pack2<kBf16>(w[0], w[1]), u1 = pack2<kBf16>(w[2], w[3]);
          p0[n] = transpose8(u0);
          p1[n] = transpose8(u1);
          if constexpr (kBf16) {
            const float h0 = __uint_as_float(u0 << 16), h1 = __uint_as_float(u0 & 0xffff0000u);
            const float h2 = __uint_as_float(u1 << 16), h3 = __uint_as_float(u1 & 0xffff0000u);
            r0[n] = transpose8(pack2<true>(w[0] - h0, w[1] - h1));
            r1[n] = transpose8(pack2<true>(w[2] - h2, w[3] - h3));
          }
        }
        const unsigned char* vt = st + b * 2 * C::kTileBytes + C::kTileBytes;
        // a value that is not finite at a position that only some rows see: the product would put 0 x it into the others.
        // It is taken out of the product here and added for the rows that see it.
        constexpr uint32_t ones = kBf16 ? 0x7f80u : 0x7c00u;
        bool fix = false;
        if constexpr (!C::kEight) {
          if (some_masked && rows_differ) {
#pragma unroll
            for (int i = 0; i < C::kTileBytes / 512; ++i) {
              const uint4 x = *reinterpret_cast<const uint4*>(vt + i * 512 + lane * 16);
              const uint32_t xw[4] = {x.x, x.y, x.z, x.w};
#pragma unroll
              for (int w = 0; w < 4; ++w) fix |= (xw[w] & ones) == ones || ((xw[w] >> 16) & ones) == ones;
            }
            fix = __any_sync(0xffffffffu, fix);
          }
        }
        auto product = [&](int d, uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3) {
#pragma unroll
          for (int n = 0; n < NT; ++n) {
            mma16816<kBf16>(o[d][n], a0, a1, a2, a3, p0[n], p1[n]);
            if constexpr (kBf16) {
              if (split) mma16816<true>(o[d][n], a0, a1, a2, a3, r0[n], r1[n]);
            }
          }
        };
        if constexpr (C::kEight) {
#pragma unroll
          for (int c = 0; c < C::kVPieces; ++c) {
            uint32_t x[4][4];   // [key][word]
#pragma unroll
            for (int r = 0; r < 4; ++r) {
              if constexpr (C::kVBytes == 16) {
                const uint4 y = *reinterpret_cast<const uint4*>(vt + (r * C::kVPieces + c) * 512 + lane * 16);
                x[r][0] = y.x, x[r][1] = y.y, x[r][2] = y.z, x[r][3] = y.w;
              } else {
                const uint2 y = *reinterpret_cast<const uint2*>(vt + (r * C::kVPieces + c) * 256 + lane * 8);
                x[r][0] = y.x, x[r][1] = y.y;
              }
            }
#pragma unroll
            for (int w = 0; w < C::kVBytes / 4; ++w) {
              uint32_t lo[4], hi[4];
#pragma unroll
              for (int r = 0; r < 4; ++r) widen4<FMT>(x[r][w], lo[r], hi[r]);
              const int d = c * (C::kVBytes / 2) + 2 * w;
              product(d, __byte_perm(lo[0], lo[1], 0x5410), __byte_perm(lo[0], lo[1], 0x7632),
                      __byte_perm(lo[2], lo[3], 0x5410), __byte_perm(lo[2], lo[3], 0x7632));
              product(d + 1, __byte_perm(hi[0], hi[1], 0x5410), __byte_perm(hi[0], hi[1], 0x7632),
                      __byte_perm(hi[2], hi[3], 0x5410), __byte_perm(hi[2], hi[3], 0x7632));
            }
          }
        } else {
          // tiles of a fragment: dims 0-7 and 8-15 of keys 0-7, then of keys 8-15
          const uint32_t v_addr = shared_addr(vt);
          const int j = (lane & 7) + ((lane & 16) >> 1), half = (lane >> 3) & 1;
#pragma unroll
          for (int d = 0; d < C::kMTiles; ++d) {
            uint32_t a0, a1, a2, a3;
            load_transposed(v_addr + v_unit<DP>(j, 2 * d + half), a0, a1, a2, a3);
            if (fix) {
              auto clean = [](uint32_t x) {
                if ((x & ones) == ones) x &= 0xffff0000u;
                if (((x >> 16) & ones) == ones) x &= 0x0000ffffu;
                return x;
              };
              a0 = clean(a0), a1 = clean(a1), a2 = clean(a2), a3 = clean(a3);
            }
            product(d, a0, a1, a2, a3);
          }
          if (fix) {
            const int k0 = key + 16 * b;
            for (int j = 0; j < 16; ++j) {
#pragma unroll
              for (int n = 0; n < NT; ++n) {
                const float w0 = __shfl_sync(0xffffffffu, j < 8 ? s[b][n][0] : s[b][n][2], (j & 7) * 4 + t);
                const float w1 = __shfl_sync(0xffffffffu, j < 8 ? s[b][n][1] : s[b][n][3], (j & 7) * 4 + t);
                const int r = n * 8 + 2 * t;
                const bool see0 = k0 + j <= row_pos[r] && k0 + j >= row_lo[r];
                const bool see1 = k0 + j <= row_pos[r + 1] && k0 + j >= row_lo[r + 1];
#pragma unroll
                for (int d = 0; d < C::kMTiles; ++d) {
#pragma unroll
                  for (int half = 0; half < 2; ++half) {
                    const uint32_t bits =
                        *reinterpret_cast<const uint16_t*>(vt + v_unit<DP>(j, 2 * d + half) + g * 2);
                    if ((bits & ones) != ones) continue;
                    float v;
                    if constexpr (kBf16) v = __uint_as_float(bits << 16);
                    else v = __half2float(__ushort_as_half((unsigned short)bits));
                    if (see0) o[d][n][2 * half] += w0 * v;
                    if (see1) o[d][n][2 * half + 1] += w1 * v;
                  }
                }
              }
            }
          }
        }
      }
      __syncwarp();   // page_ids and the ring slot are free again
    }
    copy_wait<0>();

    if constexpr (kBf16) {
      // an infinity of V times a weight's second term, which may be zero, gives NaN: such a triple is done again with
      // weights of one term
      bool odd = false;
#pragma unroll
      for (int d = 0; d < C::kMTiles; ++d) {
#pragma unroll
        for (int n = 0; n < NT; ++n) {
#pragma unroll
          for (int e = 0; e < 4; ++e) odd |= !(fabsf(o[d][n][e]) <= 3.402823466e+38f);
        }
      }
      again = split && __any_sync(0xffffffffu, odd);
      split = false;
    }
    } while (again);

    // ---- join the warps ----
    __syncthreads();   // every warp is done with the ring
    float* red = reinterpret_cast<float*>(smem) + warp * C::kRows * C::kOStride;
#pragma unroll
    for (int n = 0; n < NT; ++n) {
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        float sum = l[n][h];
        sum += __shfl_xor_sync(0xffffffffu, sum, 4);
        sum += __shfl_xor_sync(0xffffffffu, sum, 8);
        sum += __shfl_xor_sync(0xffffffffu, sum, 16);
        const int r = n * 8 + 2 * t + h;
        if (g == 0) {
          stat_m[warp][r] = m[n][h];
          stat_l[warp][r] = sum;
        }
        const float back = C::kEight ? __frcp_rn(inv[n][h]) : 1.f;
#pragma unroll
        for (int d = 0; d < C::kMTiles; ++d) {
          if constexpr (C::kEight) {   // tile d of a lane: two neighbouring dimensions
            constexpr int kPer = C::kVBytes / 2;
            const int at = d / kPer * (8 * C::kVBytes) + g * C::kVBytes + 2 * (d % kPer);
            *reinterpret_cast<float2*>(red + r * C::kOStride + at) = make_float2(o[d][n][h] * back, o[d][n][h + 2] * back);
          } else {
            red[r * C::kOStride + d * 16 + g] = o[d][n][h];
            red[r * C::kOStride + d * 16 + 8 + g] = o[d][n][h + 2];
          }
        }
      }
    }
    __syncthreads();
    const bool whole = units == sp.units;
    // the blocks that share the triple: c_first .. c_last; block i holds units [total i / parts, total (i + 1) / parts)
    const int64_t c_first = ((begin + 1) * parts - 1) / total, c_last = ((begin + sp.units) * parts - 1) / total;
    const float* all = reinterpret_cast<const float*>(smem);
    constexpr int kQuads = DP / 4;
    float* slot = a.partial + (block * 2 + (block == c_first ? 1 : 0)) * partial_floats(DP);
    auto write_row = [&](int r, int quad, float4 acc, float sum, float top) {
      const int row = row0 + r;
      const int64_t tok = (int64_t)seq * a.new_tokens + row / a.group;
      const int qh = head * a.group + row % a.group;
      const float f = sum == 0.f ? 0.f : 1.f / sum;
      const float4 y = sum == 0.f ? make_float4(0.f, 0.f, 0.f, 0.f) : make_float4(acc.x * f, acc.y * f, acc.z * f, acc.w * f);
      unsigned char* dst = a.out.p + tok * a.out.token + qh * a.out.head;
      if (quad * 4 < D) {
        uint2 w;
        if (a.q_f16) w = make_uint2(pack2<false>(y.x, y.y), pack2<false>(y.z, y.w));
        else w = make_uint2(pack2<true>(y.x, y.y), pack2<true>(y.z, y.w));
        *reinterpret_cast<uint2*>(dst + quad * 8) = w;
      }
      if (quad == 0 && a.lse) a.lse[tok * a.q_heads + qh] = sum == 0.f ? -INFINITY : (top + log2f(sum)) * 0.6931471805599453f;
    };
    for (int i = threadIdx.x; i < live_rows * kQuads; i += kAttendThreads) {
      const int r = i / kQuads, quad = i % kQuads;
      float top = -INFINITY;
#pragma unroll
      for (int w = 0; w < kAttendWarps; ++w) top = fmaxf(top, stat_m[w][r]);
      float4 acc = make_float4(0.f, 0.f, 0.f, 0.f);
      float sum = 0.f;
      const float base = top == -INFINITY ? 0.f : top;
#pragma unroll
      for (int w = 0; w < kAttendWarps; ++w) {
        const float f = exp2_fast(stat_m[w][r] - base);
        const float4 x = *reinterpret_cast<const float4*>(all + (w * C::kRows + r) * C::kOStride + quad * 4);
        acc.x += f * x.x, acc.y += f * x.y, acc.z += f * x.z, acc.w += f * x.w;
        sum += f * stat_l[w][r];
      }
      if (whole) {
        write_row(r, quad, acc, sum, top);
      } else {
        *reinterpret_cast<float4*>(slot + r * DP + quad * 4) = acc;
        if (quad == 0) *reinterpret_cast<float2*>(slot + C::kRows * DP + r * 2) = make_float2(top, sum);
      }
    }
    if (!whole) {
      __threadfence();
      __syncthreads();
      if (threadIdx.x == 0) {
        const unsigned int before = atomicAdd(a.arrived + c_first, 1u);
        last_flag = before == (unsigned int)(c_last - c_first);
        if (last_flag) a.arrived[c_first] = 0u;
      }
      __syncthreads();
      if (last_flag) {
        __threadfence();
        // the blocks' maxima and sums first (the ring is free), then their sums of values with eight loads in flight
        const int n_blocks = (int)(c_last - c_first) + 1;
        float2* ml = reinterpret_cast<float2*>(smem);
        auto part = [&](int i) { return a.partial + ((c_first + i) * 2 + (i == 0 ? 1 : 0)) * partial_floats(DP); };
        for (int i = threadIdx.x; i < n_blocks * C::kRows; i += kAttendThreads)
          ml[i] = __ldcg(reinterpret_cast<const float2*>(part(i / C::kRows) + C::kRows * DP) + i % C::kRows);
        __syncthreads();
        for (int r = warp; r < live_rows; r += kAttendWarps) {
          float top = -INFINITY, sum = 0.f;
          for (int i = lane; i < n_blocks; i += 32) top = fmaxf(top, ml[i * C::kRows + r].x);
#pragma unroll
          for (int x = 16; x; x >>= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, x));
          const float base = top == -INFINITY ? 0.f : top;
          for (int i = lane; i < n_blocks; i += 32) {
            const float2 y = ml[i * C::kRows + r];
            const float f = exp2_fast(y.x - base);
            sum += f * y.y;
            ml[i * C::kRows + r].x = f;
          }
#pragma unroll
          for (int x = 16; x; x >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, x);
          if (lane == 0) {
            stat_m[0][r] = top;
            stat_l[0][r] = sum;
          }
        }
        __syncthreads();
        for (int i = threadIdx.x; i < live_rows * kQuads; i += kAttendThreads) {
          const int r = i / kQuads, quad = i % kQuads;
          float4 acc = make_float4(0.f, 0.f, 0.f, 0.f);
          int c = 0;
          for (; c + 8 <= n_blocks; c += 8) {
            float4 x[8];
#pragma unroll
            for (int e = 0; e < 8; ++e) x[e] = __ldcg(reinterpret_cast<const float4*>(part(c + e) + r * DP + quad * 4));
#pragma unroll
            for (int e = 0; e < 8; ++e) {
              const float f = ml[(c + e) * C::kRows + r].x;
              acc.x += f * x[e].x, acc.y += f * x[e].y, acc.z += f * x[e].z, acc.w += f * x[e].w;
            }
          }
#pragma unroll 4
          for (; c < n_blocks; ++c) {
            const float4 x = __ldcg(reinterpret_cast<const float4*>(part(c) + r * DP + quad * 4));
            const float f = ml[c * C::kRows + r].x;
            acc.x += f * x.x, acc.y += f * x.y, acc.z += f * x.z, acc.w += f * x.w;
          }
          write_row(r, quad, acc, stat_l[0][r], stat_m[0][r]);
        }
      }
    }
    u += units;
  }
}

template <int FMT, int DP, int NT>
cudaError_t launch_one(AttendArgs a, int num_sms, cudaStream_t st) {
  using C = AttendConfig<FMT, DP, NT>;
  static_assert(C::kSmem <= 227 * 1024, "shared memory");

  auto* kernel = attend_kernel<FMT, DP, NT>;
  static std::atomic<int> resident[kMaxDevices];   // blocks an SM holds, by device; 0: not asked yet
  int per_sm = a.device < kMaxDevices ? resident[a.device].load(std::memory_order_relaxed) : 0;
  if (per_sm == 0) {
    cudaError_t e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, C::kSmem);
    if (e == cudaSuccess) e = cudaOccupancyMaxActiveBlocksPerMultiprocessor(&per_sm, kernel, kAttendThreads, C::kSmem);
    if (e != cudaSuccess) return e;
    per_sm = per_sm < 1 ? 1 : per_sm > kMaxBlocksPerSm ? kMaxBlocksPerSm : per_sm;
    if (a.device < kMaxDevices) resident[a.device].store(per_sm, std::memory_order_relaxed);
  }
  a.row_tiles = (a.rows + C::kRows - 1) / C::kRows;
  // the most units the table allows, so that small calls launch few blocks
  const int64_t units = ((int64_t)a.max_len + 15) / C::kUnit + 1;
  const double most = (double)a.table.seqs * a.kv_heads * a.row_tiles * (double)units / kMinUnits + 1;
  a.parts = most < (double)per_sm * num_sms ? (int)most : per_sm * num_sms;
  const int joinable = C::kBody / (C::kRows * 8);   // a join holds every block's maxima and sums in the ring
  if (a.parts > joinable) a.parts = joinable;
  kernel<<<a.parts, kAttendThreads, C::kSmem, st>>>(a);
  return cudaGetLastError();
}

template <int FMT>
cudaError_t launch_format(const AttendArgs& a, int num_sms, cudaStream_t st) {
  const int dp = padded_dim(a.head_dim), nt = a.rows <= 8 ? 1 : a.rows <= 16 || dp == 256 ? 2 : 4;
  switch (dp * 8 + nt) {
    case 64 * 8 + 1: return launch_one<FMT, 64, 1>(a, num_sms, st);
    case 64 * 8 + 2: return launch_one<FMT, 64, 2>(a, num_sms, st);
    case 64 * 8 + 4: return launch_one<FMT, 64, 4>(a, num_sms, st);
    case 128 * 8 + 1: return launch_one<FMT, 128, 1>(a, num_sms, st);
    case 128 * 8 + 2: return launch_one<FMT, 128, 2>(a, num_sms, st);
    case 128 * 8 + 4: return launch_one<FMT, 128, 4>(a, num_sms, st);
    case 256 * 8 + 1: return launch_one<FMT, 256, 1>(a, num_sms, st);
    default: return launch_one<FMT, 256, 2>(a, num_sms, st);
  }
}

}  // namespace
}  // namespace lc
