// Attention of new tokens over the paged cache: the kernel, instantiated for one cache format a source file
// (kv_attend_*.cu) and dispatched by kv_attend.cu.
//
//   s_j = scale <q, k_j>,  out = sum_j e^(s_j - m) v_j / sum_j e^(s_j - m)   over the visible j
//
// A kv head's K and V are read once for all rows that share it: the q heads of its group times the new tokens. This kernel
// is for few rows (takes_tc below has the rule): 4 x rows flops a cached element, so it is bound by reading the cache, and
// every choice below is about keeping enough loads in flight with little work a byte.
//
// Measured (bf16 q, 32 q heads on 8, d = 128, lse written; 6.69 TB/s is a plain copy's rate here): 200,003 tokens of one
// sequence 131 us, 6.3 TB/s; 32 sequences of 0 to 4,096 50 us, 5.5 TB/s, of which some 8 us are start and joins; e4m3, 64 of 500
// to 16,384 185 us, 6.2 TB/s. One sequence of 100 tokens (8 heads, d = 64): 5.8 us, a launch, two dependent loads to the
// first K, and a join. d = 256 with 16 rows (int8, a window of 1,024, 48 sequences): 44 us, 2.3 TB/s: there 255 registers
// leave two warps a scheduler and widening and products are 26,000 instructions an SM quarter, issued in 34% of the cycles.
//
// Products. Both run on the warp-level tensor instruction m16n8k16, with keys (or dimensions) as M and the rows of q as N:
// a tile of 8 rows wastes nothing at 8 rows, where the 64- or 128-row tiles of tcgen05 would take the scores through TMEM
// and shared memory for no gain in a kernel that waits for HBM.
//   S^T [16 keys x 8 rows] = K [16 x d] Q^T [d x 8],   O^T [16 dims x 8 rows] += V^T [16 dims x 16 keys] P^T [16 keys x 8]
// The order of a contraction is free, and so is the naming of V's dimensions, so an operand's share of a lane is 16
// contiguous bytes of a row wherever it can be: lane (g, t) = (lane / 4, lane % 4) takes bytes 16 t of every 64 of key rows g
// and g + 8 of K, and (8-bit formats) bytes 16 g of every 128 of rows 2t, 2t+1, 2t+8 and 2t+9 of V, whose codes are paired
// by byte permutes and widened; a 16-bit V is transposed by ldmatrix. P^T is the transpose of the S^T accumulator, one
// movmatrix for 8 x 8.
//
// Copies. Each warp has a ring of its own tiles in shared memory, filled by cp.async whole lines at a time (rows of V taken
// 32 bytes at a time, straight into the lane that uses them, halved the bandwidth of 8-bit caches), and runs it ahead of the
// products from one triple into the next. Nothing is shared between warps: no barriers in the loop.
//
// Softmax. Base 2, with a reference m a row: 7 below the largest score so far when it is set, and moved only when a score
// exceeds it by more than 15. Weights then stay below 2^15, the sum is fp32, and most tiles need a vote instead of a maximum
// over the lanes. (f16 weights have their full 11 bits down to 2^-21 of the largest that way; with a reference at the
// maximum, keys of small weight and large values lost some of theirs.) Weights: f16 for f16 and 8-bit caches (11
// bits); on a bf16 cache, whose products need bf16 weights of 8 bits, a weight is split in two bf16 terms (16 bits), as
// one alone would add an error as large as the output's own rounding. An f16 weight below 2^-21 of the largest is off by up to
// 2^-32 of it (the largest is 2^7 or more, and 2^-25 half of f16's last step; 2^-25 in a part that is done again, as below): that
// shows where the keys that outweigh all others have values of 0.
//
// Sums that are not finite, or past 2^110. A warp that finds one at a triple's end does its part of it again with weights of at
// most 1, and with V's values that are no finite numbers taken out of the tiles and multiplied in fp32 for the rows that see
// them: so none reaches a row by a weight of zero, or meets a weight's term that was rounded to zero.
//
// 8-bit rows. Codes become f16 exactly. q of a bf16 type is scaled to f16 by a power of two that brings its row's largest
// magnitude to [1, 2): exact for elements within 2^-14 of that. The scales multiply the scores (k) and the weights (v);
// the weights times scales are brought into f16's range by a factor a row, kept like the maximum and raised when that moves.
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
  int inject_stall;     // test support: the tcgen05 kernel's block with the first unit withholds its loads: waits run out
  // the tcgen05 kernel: rows of a tile, floats of a row of a partial slot, and ceil(2^32 / group)
  int tile_rows, padded;
  uint32_t group_mul;
  int64_t pages;
  int64_t page_rows;    // rows of a page: kv_heads x page_size ...
  int64_t page_bytes;   // ... and their bytes
  uint32_t page_mul;    // tile / (page_size / 16) = tile * page_mul >> page_shift, for tiles below 2^26
  int page_shift;
  float scale;
  const int32_t* lengths;
  const int32_t* starts;
  Rows q, out;
  float* lse;
  const unsigned char* pk;
  const unsigned char* pv;
  const float* ks;
  const float* vs;
  float* partial;       // two slots a block: [rows of a tile x DP] sums, then (m, l) a row
  unsigned int* arrived;   // blocks that have left their part of the triple that begins in this block; zero between launches
  unsigned int* status;
  // a pass of a call over groups of sequences that have their first positions in common (kv_shared.cu)
  int groups;
  const int4* spans;      // of each group: the first common position that is seen, one past the last, first sequence, sequences
  int* line;              // kCommon on tcgen05: cells a block has, blocks that have one more, the cells before each group
  int slot_rows;          // ... and rows of a slot of partial sums
  float* part;            // the pass's outputs, [tokens x q_heads x head_dim] ...
  float* part_lse;        // ... and base-2 lse
};

// The kernels' forms: a whole attention; the pass over what groups of sequences have in common, where a group takes a sequence's
// place and has the rows of all of its sequences; and the pass over what each sequence has of its own. The passes leave their
// outputs in fp32, to be joined.
constexpr int kWhole = 0, kCommon = 1, kOwn = 2;
constexpr int kCommonRows = 256, kCommonKeys = 128, kCommonCost = 2;   // kCommon on tcgen05: a block's rows, and the line's units

constexpr int kAttendWarps = 4;
constexpr int kAttendThreads = kAttendWarps * 32;
constexpr float kBelow = 7.f, kHeadroom = 15.f;   // a row's reference below its maximum, and scores above it, in powers of two
constexpr float kFar = 0x1p110f, kToEnd = 0x1p18f;   // sums past kFar (times kToEnd: infinite) are done again, weights at most 1
constexpr int kMaxPositions = 1 << 30;      // a table's reach is cut to this
constexpr int kMaxDevices = 64;

// Floats of one partial slot, for the largest row tile at a padded head dimension. (kMaxBlocksPerSm x 2 slots an SM of up to
// 32 rows, or 2 of the tcgen05 kernel's 128.)
constexpr int64_t partial_floats(int padded) { return (int64_t)(padded == 256 ? 16 : 32) * (padded + 2); }
constexpr int padded_dim(int head_dim) { return head_dim <= 64 ? 64 : head_dim <= 128 ? 128 : 256; }

constexpr int kMaxBlocksPerSm = 4;           // sizes the scratch: two partial slots a block
cudaError_t launch_attend_bf16(const AttendArgs& a, int num_sms, cudaStream_t st);
cudaError_t launch_attend_f16(const AttendArgs& a, int num_sms, cudaStream_t st);
cudaError_t launch_attend_e4m3(const AttendArgs& a, int num_sms, cudaStream_t st);
cudaError_t launch_attend_int8(const AttendArgs& a, int num_sms, cudaStream_t st);
// The tcgen05 kernel for many rows (kv_attend_tc.cu): heads of up to 128.
// From how many rows: us of this kernel / tcgen05 over 32 x 2,000 tokens, 2 x 1,000, 4 x 30,000, 64 x 100
//   4 kv heads, bf16, d = 128   16 rows 34 / 37, 14 / 12, 64 / 55, 12 / 16     20 rows 43 / 37, 16 / 12, 86 / 56, 18 / 16
//               bf16, d = 64    16 rows 23 / 31, 12 / 11, 36 / 50, 9 / 14      20 rows 31 / 31, 11 / 11, 48 / 50, 14 / 14
//               e4m3, d = 128   16 rows 32 / 51, 16 / 14, 51 / 82, 12 / 18     20 rows 46 / 51, 15 / 14, 68 / 82, 20 / 18
//               e4m3, d = 64    20 rows 43 / 49, 18 / 13, 57 / 77, 15 / 17     32 rows 46 / 49, 20 / 13, 65 / 77, 16 / 17
//   8 kv heads, bf16, d = 128   16 rows 54 / 63, 16 / 13, 91 / 94, 19 / 26     20 rows 91 / 63, 15 / 13, 156 / 95, 31 / 26
//               bf16, d = 64    16 rows 34 / 58, 12 / 12, 52 / 86, 15 / 23     20 rows 53 / 58, 13 / 12, 81 / 87, 24 / 23
//               e4m3, d = 128   16 rows 48 / 92, 16 / 16, 73 / 149, 20 / 30    20 rows 79 / 92, 18 / 16, 115 / 149, 35 / 30
//               e4m3, d = 64    20 rows 66 / 87, 19 / 15, 85 / 143, 27 / 27    32 rows 69 / 87, 21 / 15, 90 / 143, 28 / 27
//   1 kv head,  bf16, d = 128   16 rows 17 / 18, 13 / 12, 58 / 26, 12 / 11     20 rows 23 / 18, 14 / 12, 36 / 27, 12 / 11
//               e4m3, d = 128   16 rows 19 / 24, 15 / 14, 35 / 34, 12 / 12     20 rows 22 / 24, 16 / 14, 38 / 35, 11 / 12
// f16 is as bf16, int8 as e4m3 with tcgen05 some 10% slower; 24 and 32 rows as 20, which are tiles of 16 twice (of 32 over
// 8-bit heads of 64). Where the rule takes the slower one: 17 to 32 rows over long 8-bit caches at d = 128 (by 10 to 30%, int8
// by up to 47%; short ones are faster so, and weights keep 16 bits instead of 11), 20 rows over 8 heads of 64 in bf16 (by 8%),
// and 16 rows over long caches of few heads at d = 128 in 16 bits (64 for 55, with one head 58 for 26).
inline bool takes_tc(int rows, int group, int head_dim, bool eight) {   // (group: its products with rows fit in 32 bits)
  return head_dim <= 128 && group <= 2048 && rows > (eight && head_dim <= 64 ? 32 : 16);
}
cudaError_t launch_attend_tc(const AttendArgs& a, int format, int num_sms, cudaStream_t st);
// The two kernels' passes over sequences that have their first positions in common (kv_shared*.cu).
cudaError_t launch_common_bf16(const AttendArgs& a, int num_sms, cudaStream_t st);
cudaError_t launch_common_f16(const AttendArgs& a, int num_sms, cudaStream_t st);
cudaError_t launch_common_e4m3(const AttendArgs& a, int num_sms, cudaStream_t st);
cudaError_t launch_common_int8(const AttendArgs& a, int num_sms, cudaStream_t st);
cudaError_t launch_common_tc(const AttendArgs& a, int format, int num_sms, cudaStream_t st);   // heads of up to 128
cudaError_t launch_own_bf16(const AttendArgs& a, int num_sms, cudaStream_t st);
cudaError_t launch_own_f16(const AttendArgs& a, int num_sms, cudaStream_t st);
cudaError_t launch_own_e4m3(const AttendArgs& a, int num_sms, cudaStream_t st);
cudaError_t launch_own_int8(const AttendArgs& a, int num_sms, cudaStream_t st);
cudaError_t launch_own_tc(const AttendArgs& a, int format, int num_sms, cudaStream_t st);
lacache_status launch_whole(lacache_kv_t* h, AttendArgs& a, cudaStream_t st);
lacache_status attend_args(lacache_kv_t* h, int layer, const lacache_kv_table* table, int new_tokens, int q_heads, int window,
                           int dtype, float scale, const int32_t* lengths, const int32_t* starts, const lacache_rows* q,
                           AttendArgs* out);

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
  static constexpr int kRowBytes = DP * kItem;
  static constexpr int kUnits = kRowBytes / 16;                          // 16-byte units of a row
  static constexpr int kCopyRows = 32 / kUnits;                          // rows that one copy of the warp covers
  static constexpr int kCopies = 16 / kCopyRows;
  static constexpr int kTileBytes = 16 * DP * kItem;                     // K (or V) of 16 keys
  static constexpr int kStageBytes = kSub * 2 * kTileBytes + (kEight ? kKeys * 8 : 0);
  static constexpr int kStages = kStageBytes > 16000 ? (NT == 1 ? 3 : 2) : kStageBytes > 8000 ? 2 : 4;
  static constexpr int kTripleCost = kStageBytes > 8000 ? NT : 2;         // a triple's start and join, in units
  static constexpr int kMTiles = DP / 16;
  static constexpr int kQStride = DP * 2 + 64;                           // bytes of a row of q in shared memory
  static constexpr int kRing = kAttendWarps * kStages * kStageBytes;
  static constexpr int kOStride = DP / 4 + 8;                            // floats of a row of sums in a pass of the join
  static constexpr int kSmem = kRing + kRows * kQStride + kAttendWarps * kRows * kOStride * 4;
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

// c (+)= A B; the first product of a sum takes zeros instead of c.
template <bool BF16>
__device__ __forceinline__ void mma16816(float (&c)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0,
                                         uint32_t b1) {
  if constexpr (BF16)
    asm("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
        : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
        : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
  else
    asm("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
        : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
        : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}
template <bool BF16>
__device__ __forceinline__ void mma16816_first(float (&c)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3,
                                               uint32_t b0, uint32_t b1) {
  if constexpr (BF16)
    asm("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%10,%10,%10,%10};"
        : "=f"(c[0]), "=f"(c[1]), "=f"(c[2]), "=f"(c[3])
        : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1), "f"(0.f));
  else
    asm("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%10,%10,%10,%10};"
        : "=f"(c[0]), "=f"(c[1]), "=f"(c[2]), "=f"(c[3])
        : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1), "f"(0.f));
}
// 8 x 8 of 16-bit values, one row of four lanes' registers, transposed across the warp.
__device__ __forceinline__ uint32_t transpose8(uint32_t x) {
  uint32_t y;
  asm volatile("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(y) : "r"(x));
  return y;
}
__device__ __forceinline__ float exp2_fast(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}

// Four 8 x 8 tiles of 16-bit values from shared memory, transposed: lane l names the 16-byte row l % 8 of tile l / 8.
__device__ __forceinline__ void load_transposed(uint32_t addr, uint32_t& a0, uint32_t& a1, uint32_t& a2, uint32_t& a3) {
  asm volatile("ldmatrix.sync.aligned.m8n8.x4.trans.shared.b16 {%0, %1, %2, %3}, [%4];"
               : "=r"(a0), "=r"(a1), "=r"(a2), "=r"(a3)
               : "r"(addr));
}
// Where a tile of 16 keys keeps the 16-byte unit u of key j, so that what eight lanes read at once lies in eight different
// bank groups: K, read as units 4c + t of keys g (lanes 4 (g & 1) + t together); a 16-bit V, read by ldmatrix as one unit of
// eight keys; an 8-bit V, read as units g of keys 2t. Rows of 64 bytes share a 128-byte line in pairs.
template <int ROW>
__device__ __forceinline__ int k_unit(int j, int u) {
  return ROW == 64 ? j * 64 + u * 16 : j * ROW + ((u ^ ((j & 1) << 2)) << 4);
}
template <int ROW, bool EIGHT>
__device__ __forceinline__ int v_unit(int j, int u) {
  if (!EIGHT) return j * ROW + ((u ^ (j & 7)) << 4);
  return ROW == 64 ? (j >> 1) * 128 + ((((j & 1) * 4 + u) ^ (j & 6)) << 4) : j * ROW + ((u ^ (j & 6)) << 4);
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
  int first, rows, tiles;   // kCommon: the group's first sequence, its rows a kv head, their tiles
};
template <int FORM = kWhole>
__device__ __forceinline__ int seqs_of(const AttendArgs& a) { return FORM == kCommon ? a.groups : a.table.seqs; }
template <int FORM>
__device__ __forceinline__ int rows_of(const AttendArgs& a, const Span& s) { return FORM == kCommon ? s.rows : a.rows; }
template <int FORM>
__device__ __forceinline__ int tiles_of(const AttendArgs& a, const Span& s) { return FORM == kCommon ? s.tiles : a.row_tiles; }
template <int FORM>   // the row of the table, and of which sequence the rows' first token is
__device__ __forceinline__ int first_of(int seq, const Span& s) { return FORM == kCommon ? s.first : seq; }
template <int FORM>   // (kOwn: written as the spans are)
__device__ __forceinline__ int start_of(const AttendArgs& a, int seq) {
  return !a.starts ? 0 : FORM == kOwn ? __ldcg(a.starts + seq) : a.starts[seq];
}
template <int FORM = kWhole>
__device__ __forceinline__ Span span_of(const AttendArgs& a, int seq, int unit_keys, int tile_rows = 0) {
  Span s;
  if constexpr (FORM == kCommon) {
    const int4 x = __ldcg(a.spans + seq);   // (written by a kernel that this one may have started beside)
    s.lo = x.x;
    s.len = s.hi = x.y;
    s.first = x.z;
    s.rows = x.w * a.rows;
    s.tiles = s.rows ? (s.rows + tile_rows - 1) / tile_rows : 1;
    const int common = s.hi - (s.lo & ~15);
    s.units = common <= 0 ? 1 : (common + unit_keys - 1) / unit_keys;
    return s;
  }
  int len = a.lengths[seq];
  len = len < 0 ? 0 : len > a.max_len ? a.max_len : len;
  const int first = len - a.new_tokens;   // the first row's position
  int lo = start_of<FORM>(a, seq);
  if (a.window > 0 && first - a.window + 1 > lo) lo = first - a.window + 1;   // window < 2^31, first >= -512: no overflow
  lo = lo < 0 ? 0 : lo > len ? len : lo;
  s.len = len;
  s.lo = lo;
  s.hi = len;
  if (FORM == kOwn && lo >= len) s.lo = s.hi = len & ~15;   // nothing of its own: no page is looked up
  const int keys = s.hi - (s.lo & ~15);
  s.units = keys <= 0 ? 1 : (keys + unit_keys - 1) / unit_keys;   // an empty sequence has rows to write
  return s;
}

// The last and the first position that token tok of a triple sees.
template <int FORM>
__device__ __forceinline__ int2 seen_by(const AttendArgs& a, int seq, const Span& sp, int tok) {
  int of = seq, pos;
  if constexpr (FORM == kCommon) {
    const int i = tok / a.new_tokens;
    of = sp.first + i;
    const int len = a.lengths[of];
    pos = (len < 0 ? 0 : len > a.max_len ? a.max_len : len) - a.new_tokens + (tok - i * a.new_tokens);
  } else {
    pos = sp.len - a.new_tokens + tok;
  }
  int lo = start_of<FORM>(a, of);
  if (a.window > 0 && pos - a.window + 1 > lo) lo = pos - a.window + 1;
  if (FORM == kCommon && pos > sp.hi - 1) pos = sp.hi - 1;
  return make_int2(pos, lo);
}

// Where row `row` of a kv head goes: bytes into out (of a pass: into part), and its index in lse.
template <int FORM = kWhole>
__device__ __forceinline__ int64_t out_at(const AttendArgs& a, int first, int head, int row, int64_t* lse) {
  const int tok = row / a.group, qh = head * a.group + row - tok * a.group;
  const int64_t token = (int64_t)first * a.new_tokens + tok;
  *lse = token * a.q_heads + qh;
  if (FORM != kWhole) return *lse * a.head_dim * 4;
  return a.out.at(token, qh) - a.out.p;
}
// Four values of an output row. Sums are kept in the order of the accumulators: quad 4 d + p holds tile d's two values of
// lane group g = 2p and its two of g + 1. f is 1 / the row's sum of weights, 0 if nothing was seen.
template <typename C, int FORM = kWhole>
__device__ __forceinline__ void write_quad(const AttendArgs& a, int64_t at_row, int quad, float4 acc, float f) {
  const float4 y = f == 0.f ? make_float4(0.f, 0.f, 0.f, 0.f) : make_float4(acc.x * f, acc.y * f, acc.z * f, acc.w * f);
  const int d = quad >> 2, g = (quad & 3) * 2;
  int at[2];        // the first dimensions of two pairs
  float2 pair[2];
  if constexpr (C::kEight) {   // a lane's pair: two neighbours of its kVBytes dimensions
    constexpr int kPer = C::kVBytes / 2;
    at[0] = d / kPer * (8 * C::kVBytes) + g * C::kVBytes + 2 * (d % kPer);
    at[1] = at[0] + C::kVBytes;
    pair[0] = make_float2(y.x, y.y);
    pair[1] = make_float2(y.z, y.w);
  } else {                     // a lane's pair: dimensions g and g + 8 of the tile
    at[0] = d * 16 + g;
    at[1] = at[0] + 8;
    pair[0] = make_float2(y.x, y.z);
    pair[1] = make_float2(y.y, y.w);
  }
  if constexpr (FORM != kWhole) {
    float* out = a.part + at_row / 4;
#pragma unroll
    for (int i = 0; i < 2; ++i)
      if (at[i] < a.head_dim) *reinterpret_cast<float2*>(out + at[i]) = pair[i];
    return;
  }
  unsigned char* out = a.out.p + at_row;
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    if (at[i] < a.head_dim)
      *reinterpret_cast<uint32_t*>(out + at[i] * 2) =
          a.q_f16 ? pack2<false>(pair[i].x, pair[i].y) : pack2<true>(pair[i].x, pair[i].y);
  }
}
__device__ __forceinline__ float lse_of(float top, float sum) {
  return sum == 0.f ? -INFINITY : (top + log2f(sum)) * 0.6931471805599453f;
}
template <int FORM>
__device__ __forceinline__ void write_lse(const AttendArgs& a, int64_t at, float top, float sum) {
  if (FORM != kWhole) a.part_lse[at] = sum == 0.f ? -INFINITY : top + log2f(sum);
  else if (a.lse) a.lse[at] = lse_of(top, sum);
}

// The kernels of a call over groups are launched as soon as the one before has begun (programmatic dependent launch), and wait for
// its end here, before they let the next one begin: that one, and the one after it, read what was written before this one without a
// wait (kv_shared_tc_common.cu, kv_shared.cu).
template <int FORM>
__device__ __forceinline__ void pass_begins() {
  if (FORM != kWhole) {
    asm volatile("griddepcontrol.wait;" ::: "memory");
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
  }
}

template <int FMT, int DP, int NT, int FORM = kWhole>
__global__ void __launch_bounds__(kAttendThreads, NT == 1 && DP <= 128 ? 3 : 1) attend_kernel(const __grid_constant__ AttendArgs a) {
  using C = AttendConfig<FMT, DP, NT>;
  constexpr bool kBf16 = FMT == LACACHE_KV_BF16;
  constexpr bool kQInRegs = NT * DP <= 128;   // more would spill: q is read from shared memory at its use
  extern __shared__ __align__(128) unsigned char smem[];
  __shared__ float stat_m[kAttendWarps][C::kRows], stat_l[kAttendWarps][C::kRows];
  __shared__ int row_pos[C::kRows], row_lo[C::kRows];   // a row's own last and first visible position
  __shared__ float row_factor[C::kRows];                // scale log2(e), and what the row's q was divided by
  __shared__ int64_t row_out[C::kRows];                 // where a row goes, and 1 / its sum of weights
  __shared__ float row_inv[C::kRows];
  __shared__ int page_ids[kAttendWarps][C::kStages][C::kSub];
  __shared__ int pending[2][6];   // shared triples: sequence, triple, first and last block (-1: none), rows and tiles (kCommon)
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, g = lane >> 2, t = lane & 3;
  pass_begins<FORM>();
  const int D = a.head_dim, row_bytes = D * C::kItem;
  const int per_whole = a.kv_heads * a.row_tiles;
  auto triples_of = [&](const Span& s) { return FORM == kCommon ? a.kv_heads * s.tiles : per_whole; };   // of a sequence
  const int seqs = seqs_of<FORM>(a);
  auto span = [&](int s) { return span_of<FORM>(a, s, C::kUnit, C::kRows); };

  // ---- this block's part of the line of cells (each warp for itself) ----
  // a triple's cells: kTripleCost for its q and its join, which hold no keys, then its units
  constexpr int kTripleCost = C::kTripleCost;
  // (a sequence's: of one of its triples, or, where their number differs, of all)
  auto cells_of = [&](int s) {
    if (s >= seqs) return 0;
    const Span x = span(s);
    return (x.units + kTripleCost) * (FORM == kCommon ? triples_of(x) : 1);
  };
  const int per_seq = FORM == kCommon ? 1 : per_whole;
  int held[4], total = 0;   // the first 128 sequences', their loads all at once
#pragma unroll
  for (int i = 0; i < 4; ++i) held[i] = cells_of(32 * i + lane);
#pragma unroll
  for (int i = 0; i < 4; ++i) total += held[i];
  for (int s = lane + 128; s < seqs; s += 32) total += cells_of(s);
  total = __reduce_add_sync(0xffffffffu, total) * per_seq;
  const int parts = total < a.parts ? total : a.parts, block = blockIdx.x;
  if (block >= parts) return;
  const int share = total / parts, longer = total - share * parts;   // the first `longer` blocks have one cell more
  const int u = block * share + (block < longer ? block : longer);
  auto block_of = [&](int cell) {
    const int in_longer = longer * (share + 1);
    return cell < in_longer ? cell / (share + 1) : longer + (cell - in_longer) / share;
  };
  int seq = 0, seq_base = 0;   // the sequence that cell u belongs to, and the cells before it
#pragma unroll 1
  for (int s0 = 0; s0 < seqs; s0 += 32) {
    const int mine = s0 == 0 ? held[0] : s0 == 32 ? held[1] : s0 == 64 ? held[2] : s0 == 96 ? held[3] : cells_of(s0 + lane);
    const int own = mine * per_seq;
    int upto = own;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const int y = __shfl_up_sync(0xffffffffu, upto, o);
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
  if (threadIdx.x < 2) pending[threadIdx.x][2] = -1;   // (the first triple's q, and a barrier, come before its use)
  constexpr int kQuads = DP / 4;
  Span sp = span(seq);
  int triple = (u - seq_base) / (sp.units + kTripleCost);
  int first_unit = u - seq_base - triple * (sp.units + kTripleCost) - kTripleCost;
  int left = share + (block < longer ? 1 : 0);   // cells of this block that are not done
  if (first_unit < 0) {
    left += first_unit;
    first_unit = 0;
  }

  unsigned char* ring = smem + warp * C::kStages * C::kStageBytes;
  unsigned char* q_smem = smem + C::kRing;
  float* join = reinterpret_cast<float*>(smem + C::kRing + C::kRows * C::kQStride);
  const uint32_t ring_addr = shared_addr(ring);

  // ---- the copies run ahead of the products by kStages - 1 units, from one triple into the next ----
  struct {
    int left, seq, triple, unit, slot;
    Span sp;
    int key;                      // this warp's first key of the unit
    const int32_t* table_row;
    const unsigned char *k, *v;   // head's part of page 0
    int64_t scale_row;
    int ids[C::kSub], next_ids[C::kSub];   // lane i: page ids of the batch's unit i, and of the next batch's
    int in_batch;
  } ahead;
  auto page_of = [&](int at) { return (int)(((uint64_t)(uint32_t)(at >> 4) * a.page_mul) >> a.page_shift); };
  auto look_up = [&](int from, int (&ids)[C::kSub]) {   // the page ids of 32 units, from the one whose first key is `from`
#pragma unroll
    for (int s = 0; s < C::kSub; ++s) {
      const int64_t at = (int64_t)from + lane * C::kUnit + 16 * s;
      ids[s] = at < ahead.sp.hi ? __ldg(ahead.table_row + page_of((int)at)) : -1;
    }
  };
  auto enter_triple = [&] {
    const int head = ahead.triple / tiles_of<FORM>(a, ahead.sp);
    ahead.key = (ahead.sp.lo & ~15) + ahead.unit * C::kUnit + warp * C::kKeys;
    ahead.table_row = a.table.pages + first_of<FORM>(ahead.seq, ahead.sp) * a.table.stride;
    const int64_t rows = (int64_t)head * a.page_size;
    ahead.k = a.pk + rows * row_bytes;
    ahead.v = a.pv + rows * row_bytes;
    ahead.scale_row = rows;
    ahead.in_batch = 0;
    look_up(ahead.key, ahead.ids);
  };
  auto issue = [&] {
    if (ahead.left > 0) {
      const uint32_t at = ring_addr + ahead.slot * C::kStageBytes;
#pragma unroll
      for (int s = 0; s < C::kSub; ++s) {
        const int k0 = ahead.key + 16 * s;
        int page = __shfl_sync(0xffffffffu, ahead.ids[s], ahead.in_batch);
        const int at_page = k0 - page_of(k0) * a.page_size;
        if ((unsigned)page >= (unsigned)a.pages) {
          if (k0 < ahead.sp.hi && lane == 0) atomicOr(a.status, kBadIndex);
          page = -1;
        }
        if (lane == 0) page_ids[warp][ahead.slot][s] = page;
        const int64_t offset = (page < 0 ? 0 : (int64_t)page * a.page_bytes) + (int64_t)at_page * row_bytes;
        const unsigned char* kp = ahead.k + offset;
        const unsigned char* vp = ahead.v + offset;
        // a key outside [lo, hi) is not read: zeros take its place
        auto inside = [&](int j) { return page >= 0 && k0 + j >= ahead.sp.lo && k0 + j < ahead.sp.hi; };
        // 32 units of 16 bytes a copy, neighbouring lanes on neighbouring units: rows are requested in whole lines
        const uint32_t kd = at + s * 2 * C::kTileBytes, vd = kd + C::kTileBytes;
        const int unit = lane % C::kUnits, first = lane / C::kUnits;
        // (most tiles: no key to leave out. With D == DP's constants apart d = 256 is 4% faster; without the second form, heads
        // of 192 were 176 us instead of 124 over 64 x 4,000 tokens, 4 rows, bf16)
        const bool full = page >= 0 && k0 >= ahead.sp.lo && k0 + 16 <= ahead.sp.hi;
        if (full && D == DP) {
#pragma unroll
          for (int i = 0; i < C::kCopies; ++i) {
            const int j = i * C::kCopyRows + first;
            copy_async<16>(kd + k_unit<C::kRowBytes>(j, unit), kp + i * 512 + lane * 16, true);
            copy_async<16>(vd + v_unit<C::kRowBytes, C::kEight>(j, unit), vp + i * 512 + lane * 16, true);
          }
        } else if (full) {
          const bool live = unit * 16 < row_bytes;                        // (past the row's end: zeros)
          const int from = first * row_bytes + unit * 16, step = C::kCopyRows * row_bytes;
#pragma unroll
          for (int i = 0; i < C::kCopies; ++i) {
            const int j = i * C::kCopyRows + first;
            copy_async<16>(kd + k_unit<C::kRowBytes>(j, unit), kp + from + i * step, live);
            copy_async<16>(vd + v_unit<C::kRowBytes, C::kEight>(j, unit), vp + from + i * step, live);
          }
        } else {
#pragma unroll 1
          for (int i = 0; i < C::kCopies; ++i) {
            const int j = i * C::kCopyRows + first;
            const bool live = inside(j) && unit * 16 < row_bytes;
            const int from = j * row_bytes + unit * 16;
            copy_async<16>(kd + k_unit<C::kRowBytes>(j, unit), live ? kp + from : a.pk, live);
            copy_async<16>(vd + v_unit<C::kRowBytes, C::kEight>(j, unit), live ? vp + from : a.pv, live);
          }
        }
        if constexpr (C::kEight) {
          // scales, four keys a lane: lanes 8s to 8s + 3 those of k, 8s + 4 to 8s + 7 those of v
          if (lane >> 3 == s) {
            const float* src = (lane & 4 ? a.vs : a.ks);
            copy_async<16>(at + C::kSub * 2 * C::kTileBytes + lane * 16,
                           page >= 0 ? src + (page * a.page_rows + ahead.scale_row + at_page + (lane & 3) * 4) : src, page >= 0);
          }
        }
      }
      --ahead.left;
      ahead.slot = ahead.slot + 1 == C::kStages ? 0 : ahead.slot + 1;
      ahead.key += C::kUnit;
      if (++ahead.in_batch == 16) look_up(ahead.key + 16 * C::kUnit, ahead.next_ids);
      if (ahead.in_batch == 32) {
        ahead.in_batch = 0;
#pragma unroll
        for (int s = 0; s < C::kSub; ++s) ahead.ids[s] = ahead.next_ids[s];
      }
      if (++ahead.unit == ahead.sp.units && (ahead.left -= kTripleCost) > 0) {
        ahead.unit = 0;
        if (++ahead.triple == triples_of(ahead.sp)) {
          ahead.triple = 0;
          ahead.seq = ahead.seq + 1 < seqs ? ahead.seq + 1 : ahead.seq;
          ahead.sp = span(ahead.seq);
        }
        enter_triple();
      }
    }
    copy_commit();
  };

  // a row of q (row r of the tile that starts at row0), eight elements a lane; zeros past the live rows and dimensions
  auto load_q = [&](int of_seq, int of_head, int of_row0, int r) {   // (of_seq: the sequence of the rows' first token)
    const int row = of_row0 + r, tok = row / a.group;
    uint4 x = make_uint4(0, 0, 0, 0);
    if (row < rows_of<FORM>(a, sp) && lane * 8 < D)
      x = *reinterpret_cast<const uint4*>(
          a.q.at((int64_t)of_seq * a.new_tokens + tok, of_head * a.group + row - tok * a.group) + lane * 16);
    return x;
  };
  // the next triple's q is read ahead of the join: into registers, or where more rows would spill, by cp.async into its place
  // in shared memory, once every warp is done with the last
  constexpr bool kQEarly = NT <= 2;
  uint4 q_raw[kQEarly ? C::kRows / kAttendWarps : 1];
  auto load_q_early = [&](int seq_now, int of_triple) {   // (sp is that sequence's)
    const int of_seq = first_of<FORM>(seq_now, sp), tiles = tiles_of<FORM>(a, sp);
    const int of_head = of_triple / tiles, of_row0 = (of_triple - of_head * tiles) * C::kRows;
    if constexpr (kQEarly) {
#pragma unroll
      for (int k = 0; k < C::kRows / kAttendWarps; ++k)
        q_raw[k] = load_q(of_seq, of_head, of_row0, warp + k * kAttendWarps);
    } else {
#pragma unroll
      for (int k = 0; k < C::kRows / kAttendWarps; ++k) {
        const int r = warp + k * kAttendWarps, row = of_row0 + r, tok = row / a.group;
        const bool in = row < rows_of<FORM>(a, sp) && lane * 8 < D;
        if (lane * 8 < DP)
          copy_async<16>(shared_addr(q_smem + r * C::kQStride + lane * 16),
                         in ? a.q.at((int64_t)of_seq * a.new_tokens + tok, of_head * a.group + row - tok * a.group) + lane * 16
                            : a.pk, in);
      }
      copy_commit();
    }
  };
  float factor[NT][2];
  uint4 qreg[kQInRegs ? NT * C::kKPieces * (C::kEight ? 2 : 1) : 1];
  int all_hi = 0, all_lo = 0;   // positions that every live row sees: [all_lo, all_hi]
  bool fresh = true;                 // the copies start here
  bool careful = false;              // the triple's products are done again, V's values that are not finite apart
  int slot = 0;                      // of the unit whose products are next
  while (left > 0) {
    const int head = triple / tiles_of<FORM>(a, sp), tile = triple % tiles_of<FORM>(a, sp);
    const int units = sp.units - first_unit < left ? sp.units - first_unit : (int)left;
    const int row0 = tile * C::kRows;
    const int all_rows = rows_of<FORM>(a, sp), live_rows = all_rows - row0 < C::kRows ? all_rows - row0 : C::kRows;
    if (fresh) {
      if (!careful) load_q_early(seq, triple);   // before the copies, which would keep it waiting
      copy_wait<0>();
      __syncwarp();
      ahead.left = left;
      ahead.seq = seq;
      ahead.triple = triple;
      ahead.unit = first_unit;
      ahead.slot = slot = 0;
      ahead.sp = sp;
      enter_triple();
    }

    float o[C::kMTiles][NT][4];
    float m[NT][2], l[NT][2], inv[NT][2];
#pragma unroll
    for (int n = 0; n < NT; ++n) {
#pragma unroll
      for (int i = 0; i < C::kMTiles; ++i) o[i][n][0] = o[i][n][1] = o[i][n][2] = o[i][n][3] = 0.f;
      m[n][0] = m[n][1] = -INFINITY;
      l[n][0] = l[n][1] = 0.f;
      inv[n][0] = inv[n][1] = C::kEight ? 0x1p120f : 1.f;
    }

    int key = (sp.lo & ~15) + first_unit * C::kUnit + warp * C::kKeys;
    for (int i = fresh ? 1 - C::kStages : 0; i < units; ++i) {
      issue();
      if (i < 0) continue;   // the copies' head start
      if (i == 0 && !careful) {
        // ---- q into shared memory, in the order of the K pieces ----
        if constexpr (!kQEarly) copy_wait<1>();   // all but the newest copies: q's lie before them
        if (FORM != kCommon && threadIdx.x == 0) {
          const int raw = a.lengths[seq];
          if (raw < 0 || raw > a.max_len) atomicOr(a.status, kBadIndex);
        }
#pragma unroll
        for (int k = 0; k < C::kRows / kAttendWarps; ++k) {
          const int r = warp + k * kAttendWarps, row = row0 + r, d0 = lane * 8;
          const bool live = r < live_rows;
          const int tok = live ? row / a.group : 0;
          uint4 raw = make_uint4(0, 0, 0, 0);
          if (kQEarly) raw = q_raw[k];
          else if (d0 < DP) raw = *reinterpret_cast<const uint4*>(q_smem + r * C::kQStride + d0 * 2);
          float back = 1.f;
          if (C::kEight && !a.q_f16) {
            float x[8], top = 0.f;
            widen8(raw, x, __nv_bfloat16());
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
            if constexpr (FORM == kCommon) {
              const int2 seen = live ? seen_by<FORM>(a, seq, sp, tok) : make_int2(-1, 0);
              row_pos[r] = seen.x;
              row_lo[r] = seen.y;
            } else {
              const int p = live ? sp.len - a.new_tokens + tok : -1;
              int lo = start_of<FORM>(a, seq);
              if (a.window > 0 && p - a.window + 1 > lo) lo = p - a.window + 1;
              row_pos[r] = p;
              row_lo[r] = lo;
            }
            row_factor[r] = a.scale * 1.4426950408889634f * back;
          }
        }
        __syncthreads();

        if constexpr (FORM == kCommon) {   // rows of several sequences: in no order
          all_hi = lane < live_rows ? row_pos[lane] : INT_MAX;
          all_lo = lane < live_rows ? row_lo[lane] : INT_MIN;
          all_hi = __reduce_min_sync(0xffffffffu, all_hi);
          all_lo = __reduce_max_sync(0xffffffffu, all_lo);
        } else {
          all_hi = row_pos[0];
          all_lo = row_lo[live_rows - 1];
        }
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
      copy_wait<C::kStages - 1>();
      __syncwarp();
      const unsigned char* st = ring + slot * C::kStageBytes;

      // scores
      float s[C::kSub][NT][4];
#pragma unroll
      for (int b = 0; b < C::kSub; ++b) {
        const unsigned char* kt = st + b * 2 * C::kTileBytes;
#pragma unroll
        for (int c = 0; c < C::kKPieces; ++c) {
          const uint4 x = *reinterpret_cast<const uint4*>(kt + k_unit<C::kRowBytes>(g, 4 * c + t));
          const uint4 y = *reinterpret_cast<const uint4*>(kt + k_unit<C::kRowBytes>(g + 8, 4 * c + t));
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
              if (c == 0) {
                mma16816_first<false>(s[b][n], xa[0], ya[0], xa[1], ya[1], q0.x, q0.y);
                mma16816<false>(s[b][n], xa[2], ya[2], xa[3], ya[3], q0.z, q0.w);
              } else {
                mma16816<false>(s[b][n], xa[0], ya[0], xa[1], ya[1], q0.x, q0.y);
                mma16816<false>(s[b][n], xa[2], ya[2], xa[3], ya[3], q0.z, q0.w);
              }
              mma16816<false>(s[b][n], xa[4], ya[4], xa[5], ya[5], q1.x, q1.y);
              mma16816<false>(s[b][n], xa[6], ya[6], xa[7], ya[7], q1.z, q1.w);
            }
          } else {
#pragma unroll
            for (int n = 0; n < NT; ++n) {
              uint4 q;
              if constexpr (kQInRegs) q = qreg[n * C::kKPieces + c];
              else q = *reinterpret_cast<const uint4*>(q_smem + (n * 8 + g) * C::kQStride + (c * 32 + t * 8) * 2);
              if (c == 0) {
                mma16816_first<kBf16>(s[b][n], x.x, y.x, x.y, y.y, q.x, q.y);
                mma16816<kBf16>(s[b][n], x.z, y.z, x.w, y.w, q.z, q.w);
              } else {
                mma16816<kBf16>(s[b][n], x.x, y.x, x.y, y.y, q.x, q.y);
                mma16816<kBf16>(s[b][n], x.z, y.z, x.w, y.w, q.z, q.w);
              }
            }
          }
        }
      }

      // exponents (base-2 scores less the row's maximum), masks, and whether a maximum has to move
      float x2[C::kSub][NT][4];
      float kscale[C::kSub][2], vscale[C::kSub][2];
      bool move = false, some_masked = false;
#pragma unroll
      for (int b = 0; b < C::kSub; ++b) {
        const int k0 = key + 16 * b;
        if constexpr (C::kEight) {
          const float* sc = reinterpret_cast<const float*>(st + C::kSub * 2 * C::kTileBytes) + b * 32;
          kscale[b][0] = sc[g], kscale[b][1] = sc[g + 8];
          vscale[b][0] = sc[16 + g], vscale[b][1] = sc[24 + g];
        } else {
          kscale[b][0] = kscale[b][1] = 1.f;
        }
        const bool page_ok = page_ids[warp][slot][b] >= 0;
        const bool masked = !page_ok || k0 < all_lo || k0 + 15 > all_hi;
        some_masked |= masked;
#pragma unroll
        for (int n = 0; n < NT; ++n) {
#pragma unroll
          for (int e = 0; e < 4; ++e)
            x2[b][n][e] = fmaf(s[b][n][e], factor[n][e & 1] * kscale[b][e >> 1], -m[n][e & 1]);
          if (masked) {
#pragma unroll
            for (int e = 0; e < 4; ++e) {
              const int j = k0 + g + 8 * (e >> 1), r = n * 8 + 2 * t + (e & 1);
              if (!page_ok || j > row_pos[r] || j < row_lo[r]) x2[b][n][e] = -INFINITY;
            }
          }
          // m = -inf (nothing seen yet) gives +inf here, and NaN goes the long way too
#pragma unroll
          for (int e = 0; e < 4; ++e) move |= !(x2[b][n][e] <= kHeadroom);
        }
      }
      if (__any_sync(0xffffffffu, move) || careful) {   // (careful: weights of at most 1, so that sums stay in range)
#pragma unroll
        for (int n = 0; n < NT; ++n) {
#pragma unroll
          for (int b = 0; b < C::kSub; ++b) {
#pragma unroll
            for (int e = 0; e < 4; ++e)
              if (x2[b][n][e] != -INFINITY) x2[b][n][e] = s[b][n][e] * (factor[n][e & 1] * kscale[b][e >> 1]);   // the score
          }
#pragma unroll
          for (int h = 0; h < 2; ++h) {
            float top = -INFINITY;
#pragma unroll
            for (int b = 0; b < C::kSub; ++b) top = fmaxf(top, fmaxf(x2[b][n][h], x2[b][n][h + 2]));
            top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 4));
            top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 8));
            top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 16));
            top = fmaxf(m[n][h], careful ? top : top - kBelow);
            float f = m[n][h] == -INFINITY ? 0.f : exp2_fast(m[n][h] - top);
            l[n][h] *= f;
            if constexpr (C::kEight) {
              // what the factor was made for counts f times as much from here on: the factor rises by 1 / f (to its first
              // value at most), which leaves the sums as they are, so that weights are held relative to what still counts
              const float up = fminf(inv[n][h] * exp2_fast(top - m[n][h]), 0x1p120f);   // (from -inf, or to NaN: that value)
              f = f == 0.f ? 0.f : fminf(f * __fdividef(up, inv[n][h]), 1.f);
              inv[n][h] = up;
            }
            m[n][h] = top;
            const float base = top == -INFINITY ? 0.f : top;
#pragma unroll
            for (int b = 0; b < C::kSub; ++b) {
              x2[b][n][h] -= base;
              x2[b][n][h + 2] -= base;
            }
#pragma unroll
            for (int d = 0; d < C::kMTiles; ++d) {
              o[d][n][h] *= f;
              o[d][n][h + 2] *= f;
            }
          }
        }
      }
      // weights; in 8-bit formats times v's scales, brought below 2^15 by the row's factor
#pragma unroll
      for (int n = 0; n < NT; ++n) {
#pragma unroll
        for (int b = 0; b < C::kSub; ++b) {
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            s[b][n][e] = exp2_fast(x2[b][n][e]);
            l[n][e & 1] += s[b][n][e];
          }
        }
      }
      if constexpr (C::kEight) {
        float big = 0.f;
#pragma unroll
        for (int n = 0; n < NT; ++n) {
#pragma unroll
          for (int b = 0; b < C::kSub; ++b) {
#pragma unroll
            for (int e = 0; e < 4; ++e) {
              const bool out = some_masked && x2[b][n][e] == -INFINITY;   // its scale may be NaN
              x2[b][n][e] = s[b][n][e];
              s[b][n][e] = out ? 0.f : s[b][n][e] * (vscale[b][e >> 1] * inv[n][e & 1]);
              big = fmaxf(big, s[b][n][e]);
            }
          }
        }
        if (__any_sync(0xffffffffu, big > 32768.f)) {
#pragma unroll
          for (int n = 0; n < NT; ++n) {
#pragma unroll
            for (int h = 0; h < 2; ++h) {
              float top = 0.f;
#pragma unroll
              for (int b = 0; b < C::kSub; ++b)
                top = fmaxf(top, fmaxf(x2[b][n][h] * vscale[b][0], x2[b][n][h + 2] * vscale[b][1]));
              top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 4));
              top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 8));
              top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 16));
              top = fminf(top, 3.402823466e+38f);
              if (top * inv[n][h] > 128.f) {
                const float now = 128.f * __frcp_rn(top), f = now / inv[n][h];
                inv[n][h] = now;
#pragma unroll
                for (int d = 0; d < C::kMTiles; ++d) {
                  o[d][n][h] *= f;
                  o[d][n][h + 2] *= f;
                }
              }
#pragma unroll
              for (int b = 0; b < C::kSub; ++b) {
                if (s[b][n][h] != 0.f) s[b][n][h] = x2[b][n][h] * (vscale[b][0] * inv[n][h]);
                if (s[b][n][h + 2] != 0.f) s[b][n][h + 2] = x2[b][n][h + 2] * (vscale[b][1] * inv[n][h]);
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
          for (int e = 0; e < 4; ++e) w[e] = s[b][n][e];
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
        if constexpr (!C::kEight) {
          if (careful) {
            // a value that is not finite: a product would put 0 x it into the rows that do not see it, and into those whose
            // weight has a term that is 0. It is added here for the rows that see it, and taken out of the tile.
            constexpr uint32_t ones = kBf16 ? 0x7f80u : 0x7c00u;
            bool fix = false;
#pragma unroll 1
            for (int i = 0; i < C::kTileBytes / 512; ++i) {
              const uint4 x = *reinterpret_cast<const uint4*>(vt + i * 512 + lane * 16);
              const uint32_t xw[4] = {x.x, x.y, x.z, x.w};
#pragma unroll
              for (int w = 0; w < 4; ++w) fix |= (xw[w] & ones) == ones || ((xw[w] >> 16) & ones) == ones;
            }
            if (__any_sync(0xffffffffu, fix)) {
              const int k0 = key + 16 * b;
#pragma unroll 1
              for (int j = 0; j < 16; ++j) {
#pragma unroll
                for (int n = 0; n < NT; ++n) {
                  const float w0 = __shfl_sync(0xffffffffu, j < 8 ? s[b][n][0] : s[b][n][2], (j & 7) * 4 + t);
                  const float w1 = __shfl_sync(0xffffffffu, j < 8 ? s[b][n][1] : s[b][n][3], (j & 7) * 4 + t);
                  const int r = n * 8 + 2 * t;
                  const bool see0 = k0 + j <= row_pos[r] && k0 + j >= row_lo[r];
                  const bool see1 = k0 + j <= row_pos[r + 1] && k0 + j >= row_lo[r + 1];
#pragma unroll
                  for (int d = 0; d < 2 * C::kMTiles; ++d) {
                    const uint32_t bits = *reinterpret_cast<const uint16_t*>(vt + v_unit<C::kRowBytes, false>(j, d) + g * 2);
                    if ((bits & ones) != ones) continue;
                    float v;
                    if constexpr (kBf16) v = __uint_as_float(bits << 16);
                    else v = __half2float(__ushort_as_half((unsigned short)bits));
                    if (see0) o[d >> 1][n][2 * (d & 1)] += w0 * v;
                    if (see1) o[d >> 1][n][2 * (d & 1) + 1] += w1 * v;
                  }
                }
              }
              __syncwarp();
#pragma unroll 1
              for (int i = 0; i < C::kTileBytes / 64; ++i) {
                uint16_t* x = reinterpret_cast<uint16_t*>(ring + slot * C::kStageBytes + b * 2 * C::kTileBytes + C::kTileBytes +
                                                          i * 64) + lane;
                if ((*x & ones) == ones) *x = 0;
              }
              __syncwarp();
            }
          }
        }
        if constexpr (FMT == LACACHE_KV_E4M3) {
          if (careful) {
            // the same for codes that are no numbers (the only ones of the format that are not finite)
            unsigned char* codes = ring + slot * C::kStageBytes + b * 2 * C::kTileBytes + C::kTileBytes;
            auto no_numbers = [](uint32_t x) { return __vcmpeq4(x & 0x7f7f7f7fu, 0x7f7f7f7fu); };
            bool fix = false;
#pragma unroll 1
            for (int i = 0; i < C::kTileBytes / 128; ++i)
              fix |= no_numbers(reinterpret_cast<const uint32_t*>(codes)[i * 32 + lane]) != 0;
            if (__any_sync(0xffffffffu, fix)) {
              const int k0 = key + 16 * b;
#pragma unroll 1
              for (int j = 0; j < 16; ++j) {
#pragma unroll
                for (int n = 0; n < NT; ++n) {
                  const int r = n * 8 + 2 * t;
                  const bool see0 = k0 + j <= row_pos[r] && k0 + j >= row_lo[r];
                  const bool see1 = k0 + j <= row_pos[r + 1] && k0 + j >= row_lo[r + 1];
#pragma unroll
                  for (int d = 0; d < C::kMTiles; ++d) {   // as write_quad: tile d's two codes of this lane group's bytes
                    constexpr int kPer = C::kVBytes / 2;
                    const int at = C::kVBytes == 16 ? v_unit<C::kRowBytes, true>(j, 8 * (d / kPer) + g) + 2 * (d % kPer)
                                                    : v_unit<C::kRowBytes, true>(j, g >> 1) + (g & 1) * 8 + 2 * d;
#pragma unroll
                    for (int x = 0; x < 2; ++x) {
                      if ((codes[at + x] & 0x7f) != 0x7f) continue;
                      if (see0) o[d][n][2 * x] = NAN;
                      if (see1) o[d][n][2 * x + 1] = NAN;
                    }
                  }
                }
              }
              __syncwarp();
#pragma unroll 1
              for (int i = 0; i < C::kTileBytes / 128; ++i) {
                uint32_t& x = reinterpret_cast<uint32_t*>(codes)[i * 32 + lane];
                x &= ~no_numbers(x);
              }
              __syncwarp();
            }
          }
        }
        auto product = [&](int d, uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3) {
#pragma unroll
          for (int n = 0; n < NT; ++n) {
            mma16816<kBf16>(o[d][n], a0, a1, a2, a3, p0[n], p1[n]);
            if constexpr (kBf16) mma16816<true>(o[d][n], a0, a1, a2, a3, r0[n], r1[n]);
          }
        };
        if constexpr (C::kEight) {
#pragma unroll
          for (int c = 0; c < C::kVPieces; ++c) {
            uint32_t x[4][4];   // [key][word]
#pragma unroll
            for (int r = 0; r < 4; ++r) {
              const int j = 2 * t + (r & 1) + 8 * (r >> 1);
              if constexpr (C::kVBytes == 16) {
                const uint4 y = *reinterpret_cast<const uint4*>(vt + v_unit<C::kRowBytes, true>(j, 8 * c + g));
                x[r][0] = y.x, x[r][1] = y.y, x[r][2] = y.z, x[r][3] = y.w;
              } else {
                const uint2 y = *reinterpret_cast<const uint2*>(vt + v_unit<C::kRowBytes, true>(j, g >> 1) + (g & 1) * 8);
                x[r][0] = y.x, x[r][1] = y.y;
              }
            }
#pragma unroll
            for (int w = 0; w < C::kVBytes / 4; ++w) {
              // codes of keys (2t, 2t+1) and (2t+8, 2t+9) side by side, for dimensions 0, 1 and 2, 3 of the word
              uint32_t f[4][2];
#pragma unroll
              for (int r = 0; r < 2; ++r) {
                widen4<FMT>(__byte_perm(x[2 * r][w], x[2 * r + 1][w], 0x5140), f[0][r], f[1][r]);
                widen4<FMT>(__byte_perm(x[2 * r][w], x[2 * r + 1][w], 0x7362), f[2][r], f[3][r]);
              }
              const int d = c * (C::kVBytes / 2) + 2 * w;
              product(d, f[0][0], f[1][0], f[0][1], f[1][1]);
              product(d + 1, f[2][0], f[3][0], f[2][1], f[3][1]);
            }
          }
        } else {
          // tiles of a fragment: dims 0-7 and 8-15 of keys 0-7, then of keys 8-15
          const uint32_t v_addr = shared_addr(vt);
          const int j = (lane & 7) + ((lane & 16) >> 1), half = (lane >> 3) & 1;
#pragma unroll
          for (int d = 0; d < C::kMTiles; ++d) {
            uint32_t a0, a1, a2, a3;
            load_transposed(v_addr + v_unit<C::kRowBytes, false>(j, 2 * d + half), a0, a1, a2, a3);
            product(d, a0, a1, a2, a3);
          }
        }
      }
      __syncwarp();   // page_ids and the ring slot are free again
      slot = slot + 1 == C::kStages ? 0 : slot + 1;
      key += C::kUnit;
    }
    fresh = false;

    // an output that is not finite: a value of V may have reached rows that do not see it, or met a weight's term that is 0,
    // or the weights, which may exceed 1, brought a sum to the end of fp32's range (or its join would). This warp's part of the
    // triple is done again, values that are not finite apart and the weights at most 1 (once: the values may be seen)
    {
      bool odd = false;
#pragma unroll
      for (int n = 0; n < NT; ++n) {
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          // (8-bit: codes below 2^9 times weights below 2^15, of 2^30 keys at most, over the factor)
          bool some = C::kEight && inv[n][e & 1] < 0x1p54f / kFar;
          if constexpr (FMT != LACACHE_KV_INT8) {
#pragma unroll
            for (int d = 0; d < C::kMTiles; ++d) some |= !(fabsf(o[d][n][e]) <= kFar);
          }
          odd |= some && n * 8 + 2 * t + (e & 1) < live_rows;
        }
      }
      if (!careful && __any_sync(0xffffffffu, odd)) {
        careful = fresh = true;
        continue;
      }
      careful = false;
    }

    const int of_seq = first_of<FORM>(seq, sp), of_triple = triple, of_units = sp.units, of_base = seq_base;
    const int of_rows = rows_of<FORM>(a, sp), of_tiles = tiles_of<FORM>(a, sp);
    left -= units;
    if (first_unit + units == of_units) left -= kTripleCost;
    first_unit = 0;
    if (left > 0) {
      if (++triple == triples_of(sp)) {
        triple = 0;
        seq_base += (sp.units + kTripleCost) * triples_of(sp);
        seq = seq + 1 < seqs ? seq + 1 : seq;
        sp = span(seq);
      }
      if constexpr (kQEarly) load_q_early(seq, triple);
    }

    // ---- join the warps, scaled to the common maximum, a quarter of the dimensions at a time ----
#pragma unroll
    for (int n = 0; n < NT; ++n) {
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        float sum = l[n][h];
        sum += __shfl_xor_sync(0xffffffffu, sum, 4);
        sum += __shfl_xor_sync(0xffffffffu, sum, 8);
        sum += __shfl_xor_sync(0xffffffffu, sum, 16);
        if (g == 0) {
          stat_m[warp][n * 8 + 2 * t + h] = m[n][h];
          stat_l[warp][n * 8 + 2 * t + h] = sum;
        }
      }
    }
    __syncthreads();
    if constexpr (!kQEarly) {
      if (left > 0) load_q_early(seq, triple);
    }
    const bool whole = units == of_units;
    int c_first = block, c_last = block;   // the blocks that share the triple
    if (!whole) {
      const int begin = of_base + of_triple * (of_units + kTripleCost) + kTripleCost;
      c_first = block_of(begin);
      c_last = block_of(begin + of_units - 1);
      if (threadIdx.x == 0) {
        int* p = pending[block == c_first];
        p[0] = of_seq, p[1] = of_triple, p[2] = c_first, p[3] = c_last;
        if (FORM == kCommon) p[4] = of_rows, p[5] = of_tiles;
      }
    }
    float* mine_out = a.partial + (block * 2 + (block == c_first ? 1 : 0)) * partial_floats(DP);
    if (threadIdx.x < live_rows) {
      const int r = threadIdx.x;
      const float top = fmaxf(fmaxf(stat_m[0][r], stat_m[1][r]), fmaxf(stat_m[2][r], stat_m[3][r]));
      const float base = top == -INFINITY ? 0.f : top;
      float sum = 0.f;
#pragma unroll
      for (int w = 0; w < kAttendWarps; ++w) sum += exp2_fast(stat_m[w][r] - base) * stat_l[w][r];
      if (whole) {
        int64_t at_lse;
        row_out[r] = out_at<FORM>(a, of_seq, head, row0 + r, &at_lse);
        row_inv[r] = sum == 0.f ? 0.f : 1.f / sum;
        write_lse<FORM>(a, at_lse, top, sum);
      } else {
        *reinterpret_cast<float2*>(mine_out + C::kRows * DP + r * 2) = make_float2(top, sum);
      }
    }
#pragma unroll
    for (int n = 0; n < NT; ++n) {
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        const int r = n * 8 + 2 * t + h;
        const float top = fmaxf(fmaxf(stat_m[0][r], stat_m[1][r]), fmaxf(stat_m[2][r], stat_m[3][r]));
        // (0 x NaN stays NaN: a row whose scores are NaN has no maximum but shows it)
        m[n][h] = exp2_fast(m[n][h] - (top == -INFINITY ? 0.f : top)) * (C::kEight ? __frcp_rn(inv[n][h]) : 1.f);
      }
    }
    constexpr int kPart = C::kMTiles / 4, kPartQuads = kPart * 4;   // tiles, and quads of values, a pass
#pragma unroll
    for (int c = 0; c < 4; ++c) {
      float2* mine = reinterpret_cast<float2*>(join + warp * C::kRows * C::kOStride) + g;
#pragma unroll
      for (int n = 0; n < NT; ++n) {
#pragma unroll
        for (int h = 0; h < 2; ++h) {
#pragma unroll
          for (int d = 0; d < kPart; ++d)
            mine[(n * 8 + 2 * t + h) * (C::kOStride / 2) + d * 8] =
                make_float2(o[c * kPart + d][n][h] * m[n][h], o[c * kPart + d][n][h + 2] * m[n][h]);
        }
      }
      __syncthreads();
      for (int i = threadIdx.x; i < live_rows * kPartQuads; i += kAttendThreads) {
        const int r = i / kPartQuads, q = i % kPartQuads, quad = c * kPartQuads + q;
        float4 acc = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
        for (int w = 0; w < kAttendWarps; ++w) {
          const float4 x = *reinterpret_cast<const float4*>(join + (w * C::kRows + r) * C::kOStride + q * 4);
          acc.x += x.x, acc.y += x.y, acc.z += x.z, acc.w += x.w;
        }
        if (whole) write_quad<C, FORM>(a, row_out[r], quad, acc, row_inv[r]);
        else *reinterpret_cast<float4*>(mine_out + r * DP + quad * 4) = acc;
      }
      if (c < 3) __syncthreads();
    }
  }

  // ---- the triples that this block shares (the one it begins in and the one it ends in, at most): whichever block arrives
  // last joins the blocks' sums, in their order. Only now, so that no wait for memory holds up the triples between ----
  __syncthreads();
  if (threadIdx.x < 2) {
    int* p = pending[threadIdx.x];
    bool last = false;
    if (p[2] >= 0) {
      __threadfence();   // the block's partial sums, before its arrival; the others', after the last one's
      last = atomicAdd(a.arrived + p[2], 1u) == (unsigned int)(p[3] - p[2]);
      if (last) a.arrived[p[2]] = 0u;
      __threadfence();
    }
    if (!last) p[2] = -1;
  }
  __syncthreads();
  auto part = [&](int k, int i) {   // block i's slot of shared triple k
    return a.partial + ((int64_t)(pending[k][2] + i) * 2 + (i == 0 ? 1 : 0)) * partial_floats(DP);
  };
  auto part_ml = [&](int k, int i, int r) {
    return __ldcg(reinterpret_cast<const float2*>(part(k, i) + C::kRows * DP) + r);
  };
  auto shared_rows = [&](int k) {
    if (pending[k][2] < 0) return 0;
    const int tiles = FORM == kCommon ? pending[k][5] : a.row_tiles;
    const int left_rows = (FORM == kCommon ? pending[k][4] : a.rows) - pending[k][1] % tiles * C::kRows;
    return left_rows < C::kRows ? left_rows : C::kRows;
  };
  const int rows0 = shared_rows(0), rows1 = shared_rows(1);
  __shared__ float joint_top[2 * C::kRows];
  __shared__ int64_t joint_out[2 * C::kRows];
  __shared__ float joint_inv[2 * C::kRows];
  // the rows' common maxima and sums: eight lanes a row, eight loads in flight a lane
  for (int x0 = 0; x0 < rows0 + rows1; x0 += kAttendThreads / 8) {
    const int x = x0 + (threadIdx.x >> 3), sub = threadIdx.x & 7;
    const bool live = x < rows0 + rows1;
    const int k = x < rows0 ? 0 : 1, r = k == 0 ? x : x - rows0;
    const int n_blocks = live ? pending[k][3] - pending[k][2] + 1 : 0;
    float top = -INFINITY, sum = 0.f;
    for (int c = sub; c < n_blocks; c += 64) {
      float2 y[8];
#pragma unroll
      for (int e = 0; e < 8; ++e) y[e] = c + 8 * e < n_blocks ? part_ml(k, c + 8 * e, r) : make_float2(-INFINITY, 0.f);
      float now = top;
#pragma unroll
      for (int e = 0; e < 8; ++e) now = fmaxf(now, y[e].x);
      const float base = now == -INFINITY ? 0.f : now;
      sum *= exp2_fast(top - base);
#pragma unroll
      for (int e = 0; e < 8; ++e) sum += exp2_fast(y[e].x - base) * y[e].y;
      top = now;
    }
    float all = top;
#pragma unroll
    for (int o = 4; o; o >>= 1) all = fmaxf(all, __shfl_xor_sync(0xffffffffu, all, o));
    sum *= exp2_fast(top - (all == -INFINITY ? 0.f : all));
#pragma unroll
    for (int o = 4; o; o >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, o);
    if (live && sub == 0) {
      const int tiles = FORM == kCommon ? pending[k][5] : a.row_tiles;
      const int head = pending[k][1] / tiles, row0 = (pending[k][1] - head * tiles) * C::kRows;
      int64_t at_lse;
      joint_out[x] = out_at<FORM>(a, pending[k][0], head, row0 + r, &at_lse);
      joint_top[x] = all == -INFINITY ? 0.f : all;
      joint_inv[x] = sum == 0.f ? 0.f : 1.f / sum;
      write_lse<FORM>(a, at_lse, all, sum);
    }
  }
  __syncthreads();
  // sixteen loads in flight a thread: those of four values from up to four blocks, or of one value from sixteen
  const int values = (rows0 + rows1) * kQuads;
  const int most = max(rows0 ? pending[0][3] - pending[0][2] : 0, rows1 ? pending[1][3] - pending[1][2] : 0) + 1;
  if (most <= 4) {
    for (int j0 = threadIdx.x; j0 < values; j0 += 4 * kAttendThreads) {
      float4 y[4][4];
      float w[4][4];
#pragma unroll
      for (int v = 0; v < 4; ++v) {
        const int j = j0 + v * kAttendThreads, x = j / kQuads, quad = j % kQuads;
        const int k = x < rows0 ? 0 : 1, r = k == 0 ? x : x - rows0;
        const int n_blocks = j < values ? pending[k][3] - pending[k][2] + 1 : 0;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          y[v][e] = make_float4(0.f, 0.f, 0.f, 0.f);
          w[v][e] = -INFINITY;
          if (e < n_blocks) {
            y[v][e] = __ldcg(reinterpret_cast<const float4*>(part(k, e) + r * DP + quad * 4));
            w[v][e] = part_ml(k, e, r).x;
          }
        }
      }
#pragma unroll
      for (int v = 0; v < 4; ++v) {
        const int j = j0 + v * kAttendThreads, x = j / kQuads;
        if (j < values) {
          float4 acc = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            const float f = exp2_fast(w[v][e] - joint_top[x]);
            acc.x += f * y[v][e].x, acc.y += f * y[v][e].y, acc.z += f * y[v][e].z, acc.w += f * y[v][e].w;
          }
          write_quad<C, FORM>(a, joint_out[x], j % kQuads, acc, joint_inv[x]);
        }
      }
    }
    return;
  }
  for (int j = threadIdx.x; j < values; j += kAttendThreads) {
    const int x = j / kQuads, quad = j % kQuads;
    const int k = x < rows0 ? 0 : 1, r = k == 0 ? x : x - rows0, n_blocks = pending[k][3] - pending[k][2] + 1;
    const float base = joint_top[x];
    float4 acc = make_float4(0.f, 0.f, 0.f, 0.f);
    for (int c = 0; c < n_blocks; c += 16) {
      float4 y[16];
      float f[16];
#pragma unroll
      for (int e = 0; e < 16; ++e) {
        if (c + e < n_blocks) {
          y[e] = __ldcg(reinterpret_cast<const float4*>(part(k, c + e) + r * DP + quad * 4));
          f[e] = part_ml(k, c + e, r).x;
        }
      }
#pragma unroll
      for (int e = 0; e < 16; ++e) {
        if (c + e < n_blocks) {
          const float w = exp2_fast(f[e] - base);
          acc.x += w * y[e].x, acc.y += w * y[e].y, acc.z += w * y[e].z, acc.w += w * y[e].w;
        }
      }
    }
    write_quad<C, FORM>(a, joint_out[x], quad, acc, joint_inv[x]);
  }
}

template <int FORM>
cudaError_t launch_form(void (*kernel)(AttendArgs), int blocks, int threads, int smem, const AttendArgs& a, cudaStream_t st) {
  if (FORM == kWhole) {
    kernel<<<blocks, threads, smem, st>>>(a);
    return cudaGetLastError();
  }
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3((unsigned)blocks);
  cfg.blockDim = dim3((unsigned)threads);
  cfg.dynamicSmemBytes = (size_t)smem;
  cfg.stream = st;
  cudaLaunchAttribute attr;
  attr.id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr.val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = &attr;
  cfg.numAttrs = 1;
  return cudaLaunchKernelEx(&cfg, kernel, a);
}

template <int FMT, int DP, int NT, int FORM = kWhole>
cudaError_t launch_one(AttendArgs a, int num_sms, cudaStream_t st) {
  using C = AttendConfig<FMT, DP, NT>;
  static_assert(C::kSmem <= 227 * 1024, "shared memory");

  auto* kernel = attend_kernel<FMT, DP, NT, FORM>;
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
  const int64_t units = ((int64_t)a.max_len + 15) / C::kUnit + 1 + C::kTripleCost;
  const double tiles = FORM == kCommon ? (double)a.table.seqs * a.rows / C::kRows + a.groups : (double)a.table.seqs * a.row_tiles;
  const double most = tiles * a.kv_heads * (double)units;
  if (most >= 2147483648.0) return cudaErrorNotSupported;   // units are counted in 32 bits
  a.parts = most < (double)per_sm * num_sms ? (int)most : per_sm * num_sms;
  return launch_form<FORM>(kernel, a.parts, kAttendThreads, C::kSmem, a, st);
}

template <int FMT, int FORM = kWhole>
cudaError_t launch_format(const AttendArgs& a, int num_sms, cudaStream_t st) {
  // tiles of 32 rows where takes_tc leaves so many to this kernel (of a group's common part kv_shared_tc_common.cu has them)
  constexpr bool kWide = (FMT == LACACHE_KV_E4M3 || FMT == LACACHE_KV_INT8) && FORM != kCommon;
  const int64_t rows = FORM == kCommon ? (int64_t)a.rows * a.table.seqs / a.groups : a.rows;   // (of a group, on average)
  const int dp = padded_dim(a.head_dim), nt = rows <= 8 ? 1 : rows <= 16 || dp > 64 || !kWide ? 2 : 4;
  if constexpr (kWide) {
    if (nt == 4) return launch_one<FMT, 64, 4, FORM>(a, num_sms, st);
  }
  switch (dp * 8 + nt) {
    case 64 * 8 + 1: return launch_one<FMT, 64, 1, FORM>(a, num_sms, st);
    case 64 * 8 + 2: return launch_one<FMT, 64, 2, FORM>(a, num_sms, st);
    case 128 * 8 + 1: return launch_one<FMT, 128, 1, FORM>(a, num_sms, st);
    case 128 * 8 + 2: return launch_one<FMT, 128, 2, FORM>(a, num_sms, st);
    case 256 * 8 + 1: return launch_one<FMT, 256, 1, FORM>(a, num_sms, st);
    default: return launch_one<FMT, 256, 2, FORM>(a, num_sms, st);
  }
}

}  // namespace
}  // namespace lc
