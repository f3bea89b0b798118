// Attention of a chunk of new tokens over a paged cache, on the 5th-generation tensor cores (tcgen05, accumulators in tensor memory).
//
//   S = Q K^T,   P = 2^(c S - r),   O += P V,   l += rowsum P        c = log2(e) * scale, r a reference per row
//
// Rows.  The query heads of a key/value head's group read the same keys, so the rows of a tile are (token, head of the group):
// 128 / group whole tokens to a tile of 128 rows (the MMA's M).  A tile of 128 cached positions is a step: S is 128 x 128 in fp32 in
// tensor memory, a thread owns a row of it, writes P back as bf16 over the S that it has read, and the second MMA takes P from there.
// O stays in tensor memory for the whole item.  r only moves when a row's maximum exceeds it by more than 2^8 (then O and l are
// rescaled), which after the first tiles is rare; P <= 2^8 is as exact in bf16 as P <= 1.
//
// Two slots.  A CTA keeps two of these chains (S, O, four warps each) going so that one's MMAs run while the other's exponentials do:
//   one row tile (chunks of up to 128 rows per key/value head)   the slots take alternate tiles of positions and are merged at the end
//   PAIR (more rows)                                             the slots are two row tiles, which share every tile of positions
// Either way a key or value is read from the cache once per 128 or 256 rows.
//
// Work.  An item is a (row tile or pair, key/value head) of a sequence and the tiles of positions that it sees: all up to its last
// token, or those of the window and of the first tokens.  The items' tiles lie end to end in one index space that is cut evenly over the
// grid (one CTA per SM), so ragged batches and single long sequences fill the device alike, without the host knowing a length.  Every
// warp works its CTA's range out for itself.  Where a cut goes through an item its parts are left in scratch as (O, r, l) and
// attention_combine_kernel adds them up, in a fixed order.
//
// E4M3.  The first product takes the keys' codes as they are (kind::f8f6f4) and the queries as the sum of an e4m3 and an e5m2 part: a bf16
// has eight significant bits, four in the first part and what is left in at most three of the second.  So a row that is scaled to have its
// largest value in 224 .. 448 is exact down to 2^-6, where e4m3's normal numbers end: 2^-13.8 of the largest.  Below, up to 2^-10 is left for
// three bits: off by at most 2^-14, 2^-21.8 of the largest (every bf16 number tried).  A token's key scale multiplies its column of
// scores.  The values' codes become tiles of bf16 (exactly: a code times a power of two is a bf16 number), since weights cover far more
// binades than 8 bits do.
//
// Warps: 0-3 and 4-7 softmax of the two slots (and, for E4M3, the queries' parts); one each for loading keys, values and queries by TMA into
// rings that run on across items, and one that issues the MMAs; for E4M3 four more turn the values' codes into bf16.
//
// A value meets rows that must not see it with P = 0, and 0 * NaN is NaN.  In tiles where not every row of the item sees every position, the
// values that no row sees are therefore zeroed in shared memory, and infinities and NaN in those that only some rows see are zeroed too
// and added back to the rows that do see them (add_back).
//
// Every wait is bounded: its limit counts while the products of no further tile are issued (the next items' queries, and a slot of a pair
// that has had an item without rows, wait for as long as an item takes).  One that runs out records a code in *status, after which no
// wait waits, the rows of the step become NaN, and the CTA ends as usual.  No TMA load is a multicast load.
//
// What bounds it, and measured (1.9 GHz; us a call in a CUDA graph):
//   long bf16 contexts, few rows   bytes: 64 sequences of one token, 64 heads over 8 of 128, 500 - 8000 positions (1.1 GB) 184 - 200, 5.6 - 6.1 TB/s,
//                                  for the first 50 ms; in loops of a second (1 kW, 1.6 GHz) 202 - 217
//   chunks of 2000 over 4 - 8 k    the softmax: two slots of 2200 cycles a tile, exponentials and tensor pipe at 48 % each; 976 - 1010 = 0.91 - 0.94 PFLOP/s
//   E4M3                           turning values' codes into bf16, 3400 cycles a tile: 16 sequences of nine, 2 - 16 k positions 137 - 149, 2.0 - 2.2 TB/s
//   short contexts                 latency: start and schedule 4 us, a tile 3, the end 2; 9 tokens over 300 positions 10.0
//   a context over many SMs        its parts: 16 tokens over 30000 positions 38, of which the kernel that adds up takes 9
#pragma once
#include <cuda.h>

#include "cache_kernel.cuh"
#include "fly_common.cuh"
#include "mbarrier.cuh"

namespace fly {
namespace attn {

constexpr int kTile = 128;      // positions per step
constexpr int kTileRows = 128;  // rows per slot
constexpr int kErrAttention = 5;
__device__ __forceinline__ float quiet_nan() { return __uint_as_float(0x7fc00000u); }
// A factor of scores that fp32 may have rounded to 0: positions that are not seen have scores of -inf, and 0 * -inf is NaN.  The smallest fp32 number
// in its place is off by at most 2^-149, 2^-21 on scores of up to 2^128.
__host__ __device__ __forceinline__ float positive(float x) { return x > 0.f ? x : 1.401298464324817e-45f; }

struct Params {
  cache::View c;
  cache::Rows q, out;
  float* lse;
  const int32_t* counts;
  int B, n, heads, group;  // group: query heads per key/value head
  int window, sinks;       // window 0: none
  float scale;             // log2(e) * the softmax's scale, > 0
  int tpt;                 // tokens per row tile
  int tpi;                 // tokens per item
  int rt;                  // items per sequence and key/value head
  int groups;              // B * rt
  int item_cost;           // tiles that an item counts for besides its own: what it takes a CTA to change to it
  float4* part_o;          // [grid][2][D / 4][rows of an item]
  float2* part_ml;         // [grid][2][rows of an item]: r, l
  int* desc;               // [grid][8]: how a CTA's range begins
  int* status;
};

// The rows t0 .. t1 - 1 of a sequence's chunk that make up an item, and the tiles of positions that they see: ns tiles from 0 on, then
// those from lo_tile on, `count` in all.
struct Group {
  int b, t0, t1, L;
  int lo_tile, ns, count;
  int lo_first;  // first position in the window of the first row
  int hi;        // positions from here on are not seen
  int lo_last;   // first position in the window of the last row
};

__device__ __forceinline__ Group group_at(const Params& p, int g) {
  Group r;
  r.b = p.rt == 1 ? g : g / p.rt;
  r.t0 = (g - r.b * p.rt) * p.tpi;
  r.t1 = min(cache::count_of(p.counts, r.b, p.n), r.t0 + p.tpi);
  r.L = cache::length_of(p.c, r.b);
  r.lo_tile = r.ns = r.count = r.hi = r.lo_first = r.lo_last = 0;
  if (r.t0 >= r.t1 || r.L < 0) return r;
  r.hi = min(r.L + r.t1, p.c.capacity);
  const int lo = p.window > 0 ? max(0, r.L + r.t0 + 1 - p.window) : 0;
  r.lo_first = lo;
  r.lo_last = p.window > 0 ? max(0, r.L + r.t1 - p.window) : 0;
  const int nt = (r.hi + kTile - 1) / kTile;
  r.lo_tile = lo < r.hi ? lo / kTile : nt;  // (a window behind the table's end has no tile)
  r.ns = min(min(r.lo_tile, nt), (min(p.sinks, lo) + kTile - 1) / kTile);
  r.count = r.ns + nt - r.lo_tile;
  return r;
}
__device__ __forceinline__ int tile_start(const Group& g, int x) { return (x < g.ns ? x : g.lo_tile + x - g.ns) * kTile; }
__device__ __forceinline__ bool visible(const Params& p, int row_pos, int pos) {
  return pos <= row_pos && (p.window == 0 || pos > row_pos - p.window || pos < p.sinks);
}

// ---- PTX -------------------------------------------------------------------------------------------------------------

__device__ __forceinline__ void mbar_arrive(uint32_t bar) {
  asm volatile("mbarrier.arrive.release.cta.shared::cta.b64 _, [%0];" ::"r"(bar) : "memory");
}
__device__ __forceinline__ void tma_load_4d(uint32_t dst, const CUtensorMap* map, int x, int y, int z, int w, uint32_t bar) {
  asm volatile(
      "cp.async.bulk.tensor.4d.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3, %4, %5}], [%6];" ::"r"(dst), "l"(map),
      "r"(x), "r"(y), "r"(z), "r"(w), "r"(bar)
      : "memory");
}
__device__ __forceinline__ void tma_load_5d(uint32_t dst, const CUtensorMap* map, int x, int y, int z, int w, int v, uint32_t bar) {
  asm volatile(
      "cp.async.bulk.tensor.5d.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3, %4, %5, %6}], [%7];" ::"r"(dst), "l"(map),
      "r"(x), "r"(y), "r"(z), "r"(w), "r"(v), "r"(bar)
      : "memory");
}
__device__ __forceinline__ void tc_fence_before() { asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void tc_fence_after() { asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void async_proxy_fence() { asm volatile("fence.proxy.async.shared::cta;" ::: "memory"); }
__device__ __forceinline__ bool elect_lane() {
  uint32_t one;
  asm volatile("{\n\t.reg .pred p;\n\telect.sync _|p, 0xffffffff;\n\tselp.u32 %0, 1, 0, p;\n\t}" : "=r"(one));
  return one != 0;
}
// D[tmem] (+)= A[smem] * B[smem], bf16, fp32 accumulate, M = 128.  Descriptors as (low word, high word).
__device__ __forceinline__ void mma_ss(uint32_t d, uint32_t a_lo, uint32_t a_hi, uint32_t b_lo, uint32_t b_hi, uint32_t idesc, uint32_t accumulate) {
  asm volatile(
      "{\n\t.reg .pred p;\n\t.reg .b64 da, db;\n\tsetp.ne.b32 p, %6, 0;\n\tmov.b64 da, {%1, %2};\n\tmov.b64 db, {%3, %4};\n\t"
      "tcgen05.mma.cta_group::1.kind::f16 [%0], da, db, %5, p;\n\t}" ::"r"(d), "r"(a_lo), "r"(a_hi), "r"(b_lo), "r"(b_hi), "r"(idesc), "r"(accumulate)
      : "memory");
}
// The same for 8-bit floats.
__device__ __forceinline__ void mma_ss8(uint32_t d, uint32_t a_lo, uint32_t b_lo, uint32_t hi, uint32_t idesc, uint32_t accumulate) {
  asm volatile(
      "{\n\t.reg .pred p;\n\t.reg .b64 da, db;\n\tsetp.ne.b32 p, %5, 0;\n\tmov.b64 da, {%1, %3};\n\tmov.b64 db, {%2, %3};\n\t"
      "tcgen05.mma.cta_group::1.kind::f8f6f4 [%0], da, db, %4, p;\n\t}" ::"r"(d), "r"(a_lo), "r"(b_lo), "r"(hi), "r"(idesc), "r"(accumulate)
      : "memory");
}
// The same with A in tensor memory: lane = row, a 32-bit column = two consecutive entries of K.
__device__ __forceinline__ void mma_ts(uint32_t d, uint32_t a, uint32_t b_lo, uint32_t hi, uint32_t idesc, uint32_t accumulate) {
  asm volatile(
      "{\n\t.reg .pred p;\n\t.reg .b64 db;\n\tsetp.ne.b32 p, %5, 0;\n\tmov.b64 db, {%2, %3};\n\t"
      "tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], db, %4, p;\n\t}" ::"r"(d), "r"(a), "r"(b_lo), "r"(hi), "r"(idesc), "r"(accumulate)
      : "memory");
}
// Arrives on `bar` once every MMA issued so far by this thread has completed.
__device__ __forceinline__ void mma_commit(uint32_t bar) {
  asm volatile("tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];" ::"r"(bar) : "memory");
}
#define FLY_R8(r, i) "=r"(r[i]), "=r"(r[i + 1]), "=r"(r[i + 2]), "=r"(r[i + 3]), "=r"(r[i + 4]), "=r"(r[i + 5]), "=r"(r[i + 6]), "=r"(r[i + 7])
#define FLY_W8(r, i) "+r"(r[i]), "+r"(r[i + 1]), "+r"(r[i + 2]), "+r"(r[i + 3]), "+r"(r[i + 4]), "+r"(r[i + 5]), "+r"(r[i + 6]), "+r"(r[i + 7])
#define FLY_I8(r, i) "r"(r[i]), "r"(r[i + 1]), "r"(r[i + 2]), "r"(r[i + 3]), "r"(r[i + 4]), "r"(r[i + 5]), "r"(r[i + 6]), "r"(r[i + 7])
// 32 lanes x 32 columns: thread = lane, register i = column i.  The registers are there after tmem_wait.
__device__ __forceinline__ void tmem_ask32(uint32_t a, uint32_t (&r)[32]) {
  asm volatile(
      "tcgen05.ld.sync.aligned.32x32b.x32.b32 {%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,%16,%17,%18,%19,%20,%21,%22,%23,%24,%25,"
      "%26,%27,%28,%29,%30,%31}, [%32];"
      : FLY_R8(r, 0), FLY_R8(r, 8), FLY_R8(r, 16), FLY_R8(r, 24)
      : "r"(a)
      : "memory");
}
__device__ __forceinline__ void tmem_wait(uint32_t (&r)[32]) {
  asm volatile("tcgen05.wait::ld.sync.aligned;" : FLY_W8(r, 0), FLY_W8(r, 8), FLY_W8(r, 16), FLY_W8(r, 24) : : "memory");
}
__device__ __forceinline__ void tmem_ld32(uint32_t a, uint32_t (&r)[32]) {
  tmem_ask32(a, r);
  tmem_wait(r);
}
// The same for 16 columns, and a wait for two of them.
__device__ __forceinline__ void tmem_ask16(uint32_t a, uint32_t (&r)[16]) {
  asm volatile("tcgen05.ld.sync.aligned.32x32b.x16.b32 {%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15}, [%16];"
               : FLY_R8(r, 0), FLY_R8(r, 8)
               : "r"(a)
               : "memory");
}
__device__ __forceinline__ void tmem_wait16(uint32_t (&r)[16], uint32_t (&q)[16]) {
  asm volatile("tcgen05.wait::ld.sync.aligned;" : FLY_W8(r, 0), FLY_W8(r, 8), FLY_W8(q, 0), FLY_W8(q, 8) : : "memory");
}
__device__ __forceinline__ void tmem_st32(uint32_t a, const uint32_t (&r)[32]) {
  asm volatile(
      "tcgen05.st.sync.aligned.32x32b.x32.b32 [%0], {%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,%16,%17,%18,%19,%20,%21,%22,%23,%24,%25,"
      "%26,%27,%28,%29,%30,%31,%32};" ::"r"(a), FLY_I8(r, 0), FLY_I8(r, 8), FLY_I8(r, 16), FLY_I8(r, 24)
      : "memory");
}
__device__ __forceinline__ void tmem_st8(uint32_t a, const uint32_t (&r)[8]) {
  asm volatile("tcgen05.st.sync.aligned.32x32b.x8.b32 [%0], {%1,%2,%3,%4,%5,%6,%7,%8};" ::"r"(a), FLY_I8(r, 0) : "memory");
}
#undef FLY_R8
#undef FLY_W8
#undef FLY_I8
__device__ __forceinline__ void tmem_st_wait() { asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory"); }

// Shared-memory matrix descriptors: 128-byte swizzle; the high word has how far groups of 8 rows are apart.
__device__ __forceinline__ uint32_t desc_lo(uint32_t addr, uint32_t lbo_bytes) {
  return ((addr >> 4) & 0x3fffu) | (((lbo_bytes >> 4) & 0x3fffu) << 16);
}
__host__ __device__ constexpr uint32_t desc_hi(uint32_t group_bytes) { return (group_bytes >> 4) | (1u << 14) | (2u << 29); }
// For rows of 64 bytes: 64-byte swizzle, groups of 8 rows 512 bytes apart.
__host__ __device__ constexpr uint32_t desc_hi8(int D) { return D == 128 ? desc_hi(1024) : (512u >> 4) | (1u << 14) | (4u << 29); }
// Place of 16-byte piece `piece` of row `row` in a tile of rows of D bytes.
__device__ __forceinline__ int code_at(int D, int row, int piece) {
  return D == 128 ? row * 128 + (((piece ^ row) & 7) << 4) : row * 64 + (((piece ^ (row >> 1)) & 3) << 4);
}
// fp32 accumulator, 8-bit A (e4m3, or e5m2) and B (e4m3), both K-major, M = 128.
__host__ __device__ constexpr uint32_t instr_desc8(int n, bool a_e5m2) {
  return (1u << 4) | ((a_e5m2 ? 1u : 0u) << 7) | ((uint32_t)(n >> 3) << 17) | ((uint32_t)(kTileRows >> 4) << 24);
}
// fp32 accumulator, bf16 A and B, A K-major, M = 128.
__host__ __device__ constexpr uint32_t instr_desc(int n, bool b_mn_major) {
  return (1u << 4) | (1u << 7) | (1u << 10) | ((b_mn_major ? 1u : 0u) << 16) | ((uint32_t)(n >> 3) << 17) | ((uint32_t)(kTileRows >> 4) << 24);
}

// ---- shared memory -----------------------------------------------------------------------------------------------------

template <int D, bool E4M3, bool PAIR>
struct Shape {
  // A bf16 tile of 128 rows: 64 values of eight rows are 1024 bytes, a swizzle atom.  Queries: one half (64 columns) of all rows after the other.
  // Keys and values: eight rows after the other, both halves side by side, which is what one TMA box brings.
  static constexpr int kHalves = D / 64;
  static constexpr int kHalfBytes = 128 * 128;
  static constexpr int kGroupBytes = kHalves * 1024;        // eight rows of keys or values
  static constexpr int kTileBytes = kHalves * kHalfBytes;
  static constexpr int kCodeBytes = kTile * D;              // a tile of codes
  static constexpr int kQBufs = PAIR || !E4M3 ? 2 : 1;      // bf16 queries of one row tile: two buffers, the next item's come meanwhile
  // Ring of keys (bf16, or codes), of values in bf16, and of values' codes with their scale bytes
  static constexpr int kKBytes = E4M3 ? kCodeBytes : kTileBytes;  // (the scale bytes of a stage of codes lie by the fp32 ones)
  static constexpr int kKStages = E4M3 ? (D == 128 ? (PAIR ? 3 : 4) : 8) : (D == 128 ? 3 : 6);
  static constexpr int kVStages = E4M3 ? (D == 128 ? 2 : 4) : (D == 128 ? 2 : 6);
  static constexpr int kRawBytes = kCodeBytes + kTile;
  static constexpr int kRawStages = E4M3 ? (D == 128 ? (PAIR ? 2 : 3) : 6) : 0;
  static constexpr int kScaleRing = D == 128 ? 8 : 16;      // tiles whose key scales (fp32) are kept: two more than the ring of keys, and over
  static_assert(kScaleRing >= kKStages + 2, "");
  static constexpr int kWarpK = 8, kWarpV = 9, kWarpMma = 10, kWarpQ = 11, kWarpConv = 12;
  static constexpr int kConvWarps = E4M3 ? 4 : 0, kConvThreads = kConvWarps * 32;
  static constexpr int kThreads = (kWarpConv + kConvWarps) * 32;
  static constexpr int kItemRows = PAIR ? 2 * kTileRows : kTileRows;
  static constexpr int kOffK = kQBufs * kTileBytes;         // (E4M3: both parts of a row tile's queries take what its bf16 would)
  static constexpr int kOffV = kOffK + kKStages * kKBytes;
  static constexpr int kOffRaw = kOffV + kVStages * kTileBytes;
  static constexpr int kOffScales = kOffRaw + kRawStages * kRawBytes;
  static constexpr int kOffExchange = kOffScales + (E4M3 ? kScaleRing * kTile * 4 + kKStages * kTile : 0);  // fp32, bytes by stage
  static constexpr int kOffBar = kOffExchange + 2 * kTileRows * 8;
  static constexpr int kNumBars = 3 * kKStages + 2 * kVStages + 2 * kRawStages + 4 + 6 + 2;
  static constexpr int kOffFlags = kOffBar + kNumBars * 8;
  static constexpr int kOffMisc = kOffFlags + 2 * 16 * 4;
  static constexpr int kSmem = kOffMisc + 64;
  static_assert(kSmem <= 232448, "shared memory of one CTA");
  // Place of 16-byte piece `piece` of row `row` in a tile of keys or values.
  static __device__ __forceinline__ int piece_at(int row, int piece) {
    return (row >> 3) * kGroupBytes + (piece >> 3) * 1024 + (row & 7) * 128 + (((piece ^ row) & 7) << 4);
  }
};

// The index space that is cut: every item's tiles, behind item_cost places where nothing lies.
__device__ __forceinline__ int work_of(const Params& p, const Group& g) { return g.count > 0 ? (g.count + p.item_cost) * p.c.kv_heads : 0; }
// Few short items go to a CTA each: up to so many tiles take one CTA less than adding up their parts does (9 tokens of 64 heads over 300 positions:
// 12.0 us in parts, 10.6 whole).
constexpr int kWholeItem = 4;
// What a CTA takes of it: `tiles` places from place `off` of group g on.
struct Range {
  int share, tiles, off, g, item_cost;  // item_cost < 0: whole items, a place each
  Group gr;  // of g
};
__device__ __forceinline__ Range range_of(const Params& p) {  // (the host has seen to it that all tiles together are fewer than 2^31)
  const int lane = (int)threadIdx.x & 31;
  Range r;
  Group g0 = group_at(p, min(lane, p.groups - 1));
  const int count0 = lane < p.groups ? work_of(p, g0) : 0;
  int sum = count0;
#pragma unroll 4
  for (int g = 32 + lane; g < p.groups; g += 32) sum += work_of(p, group_at(p, g));
  int x0 = count0;  // over the first 32 groups
#pragma unroll
  for (int d = 1; d < 32; d <<= 1) {
    const int y = __shfl_up_sync(0xffffffffu, x0, d);
    if (lane >= d) x0 += y;
  }
  if (p.groups > 32) {
#pragma unroll
    for (int d = 16; d > 0; d >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, d);
  } else {
    sum = __shfl_sync(0xffffffffu, x0, 31);
  }
  r.share = max(1, (int)(((uint32_t)sum + gridDim.x - 1u) / gridDim.x));
  r.item_cost = p.item_cost;
  if (p.groups <= 32 && p.groups * p.c.kv_heads <= (int)gridDim.x && __all_sync(0xffffffffu, g0.count <= kWholeItem)) {
    const unsigned some = __ballot_sync(0xffffffffu, count0 > 0);
    sum = __popc(some) * p.c.kv_heads;
    x0 = __popc(some & (0xffffffffu >> (31 - lane))) * p.c.kv_heads;
    r.share = 1;
    r.item_cost = -1;
  }
  const uint32_t begin = (uint32_t)r.share * blockIdx.x;  // (at most sum + grid)
  r.g = r.off = r.tiles = 0;
  if (begin >= (uint32_t)sum) return r;
  const int first = (int)begin;
  r.tiles = min(r.share, sum - first);
  int run = 0;
  for (int base = 0; base < p.groups; base += 32) {
    if (base > 0) g0 = group_at(p, min(base + lane, p.groups - 1));
    const int v = base == 0 ? (r.item_cost < 0 ? min(count0, p.c.kv_heads) : count0) : base + lane < p.groups ? work_of(p, g0) : 0;
    int x = x0;
    if (base > 0) {
      x = v;
#pragma unroll
      for (int d = 1; d < 32; d <<= 1) {
        const int y = __shfl_up_sync(0xffffffffu, x, d);
        if (lane >= d) x += y;
      }
    }
    const unsigned past = __ballot_sync(0xffffffffu, run + x > first);
    if (past) {  // (first < sum: some lane is past it)
      const int at = __ffs((int)past) - 1;
      r.g = base + at;
      r.off = first - run - __shfl_sync(0xffffffffu, x - v, at);
      r.gr.b = __shfl_sync(0xffffffffu, g0.b, at);
      r.gr.t0 = __shfl_sync(0xffffffffu, g0.t0, at);
      r.gr.t1 = __shfl_sync(0xffffffffu, g0.t1, at);
      r.gr.L = __shfl_sync(0xffffffffu, g0.L, at);
      r.gr.lo_tile = __shfl_sync(0xffffffffu, g0.lo_tile, at);
      r.gr.ns = __shfl_sync(0xffffffffu, g0.ns, at);
      r.gr.count = __shfl_sync(0xffffffffu, g0.count, at);
      r.gr.lo_first = __shfl_sync(0xffffffffu, g0.lo_first, at);
      r.gr.hi = __shfl_sync(0xffffffffu, g0.hi, at);
      r.gr.lo_last = __shfl_sync(0xffffffffu, g0.lo_last, at);
      return r;
    }
    run += __shfl_sync(0xffffffffu, x, 31);
  }
  r.tiles = 0;  // (lengths that change while they are read)
  return r;
}

// A role's walk over the items of its CTA's range: tiles x0 .. x1 - 1 of item (g, kvh).
struct Walk {
  const Params& p;
  int g, kvh, x0, x1, left, item_cost;
  Group gr;
  __device__ __forceinline__ Walk(const Params& pp, const Range& r) : p(pp), g(r.g), kvh(0), x0(0), x1(0), left(r.tiles), item_cost(r.item_cost) {
    if (left > 0) {
      gr = r.gr;
      const int per = item_cost < 0 ? 1 : gr.count + item_cost;
      kvh = (int)((uint32_t)r.off / (uint32_t)per);
      begin(r.off - kvh * per);
    }
  }
  // The item from place `at` on.  (Where the range ends before its first tile the next CTA begins it.)
  __device__ __forceinline__ void begin(int at) {
    if (item_cost < 0) {
      left -= 1;
      x1 = gr.count;
      return;
    }
    const int end = min(gr.count + item_cost, at + left);
    left -= end - at;
    x0 = max(0, at - item_cost);
    x1 = end - item_cost;
  }
  __device__ __forceinline__ bool have() const { return x1 > x0; }
  __device__ __forceinline__ int tiles() const { return x1 - x0; }
  __device__ __forceinline__ void next() {
    x1 = x0;
    if (left <= 0) return;
    if (++kvh == p.c.kv_heads) {
      kvh = 0;
      do {
        if (++g >= p.groups) return;  // (does not happen: the places are counted alike)
        gr = group_at(p, g);
      } while (gr.count == 0);
    }
    begin(0);
  }
};

// Whether slot s of a pair sees anything of the tile at p0.
__device__ __forceinline__ bool slot_sees(const Params& p, const Group& g, int s, int p0) {
  const int ts0 = g.t0 + s * p.tpt, ts1 = min(g.t1, ts0 + p.tpt);
  if (ts0 >= ts1 || p0 >= g.L + ts1) return false;
  return p.window == 0 || p0 + kTile - 1 > g.L + ts0 - p.window || p0 < p.sinks;
}
// The last of the tiles x0 .. x0 + m - 1 of which slot s of a pair sees anything, counted from x0; -1: none.
__device__ __forceinline__ int last_seen(const Params& p, const Group& g, int s, int x0, int m) {
  int j = g.t0 + s * p.tpt < g.t1 ? m - 1 : -1;
  while (j >= 0 && !slot_sees(p, g, s, tile_start(g, x0 + j))) --j;  // (a few tiles from the end)
  return j;
}
// 0: no row of the item sees position pos, 1: some do, 2: all.
__device__ __forceinline__ int seen_by(const Params& p, const Group& g, int pos) {
  if (pos >= g.hi) return 0;
  const bool early = pos < p.sinks || p.window == 0;
  if (!early && pos < g.lo_first) return 0;
  return pos <= g.L + g.t0 && (early || pos >= g.lo_last) ? 2 : 1;
}
// Whether a tile holds positions that nobody sees, or that some rows see.
__device__ __forceinline__ bool tile_unseen(const Params& p, const Group& g, int p0) {
  return p0 + kTile > g.hi || (p0 < g.lo_first && p0 + kTile > p.sinks);
}
__device__ __forceinline__ bool tile_partial(const Params& p, const Group& g, int p0) {
  return (p0 + kTile > g.L + g.t0 + 1 && g.hi > max(p0, g.L + g.t0 + 1)) ||
         (p0 < g.lo_last && p0 + kTile > max(p.sinks, g.lo_first) && g.lo_first < g.lo_last);
}
// The part of a tile that the second MMA has to take, relative to the tile: positions first .. last - 1, without hole0 .. hole1 - 1 (between the
// first tokens and the window) and what stands on missing pages.
struct Span {
  int first, last, hole0, hole1;
};
__device__ __forceinline__ Span tile_span(const Params& p, const Group& g, int p0) {
  Span s;
  const int lo = g.lo_first - p0, end = min(g.hi - p0, kTile), early = p.sinks - p0;
  s.first = early > 0 ? 0 : max(lo, 0);
  s.last = early > 0 && lo >= end ? min(early, end) : end;
  s.hole0 = max(early, 0);
  s.hole1 = early > 0 ? min(lo, s.last) : 0;
  return s;
}
__device__ __forceinline__ uint32_t zero_nonfinite(uint32_t w, bool& any) {  // a pair of bf16
  if ((w & 0x7f80u) == 0x7f80u) { w &= 0xffff0000u; any = true; }
  if ((w & 0x7f800000u) == 0x7f800000u) { w &= 0xffffu; any = true; }
  return w;
}

__device__ __forceinline__ uint32_t below(int n) {  // the first n of 32 bits
  return n <= 0 ? 0u : n >= 32 ? 0xffffffffu : (1u << n) - 1u;
}
// Which of the 32 positions from c0 on a row sees: below lim, and from lo on or below snk (relative to the tile), and on a page that exists.
struct RowMask {
  int lim, lo, snk;
  uint32_t bad;  // a bit per 8 positions
  __device__ __forceinline__ uint32_t bits(int c0) const {
    uint32_t v = below(lim - c0) & (~below(lo - c0) | below(snk - c0));
    if (bad != 0)
      for (int i = 0; i < 4; ++i)
        if ((bad >> (c0 / 8 + i)) & 1u) v &= ~(0xffu << (8 * i));
    return v;
  }
};
// 32 scores times their keys' scales.
__device__ __forceinline__ void scale32(uint32_t (&r)[32], const float* scales) {
#pragma unroll
  for (int c = 0; c < 32; c += 4) {
    const float4 s = *reinterpret_cast<const float4*>(scales + c);
    float x, y;
    unpack2(mul2(pack2(__uint_as_float(r[c]), __uint_as_float(r[c + 1])), pack2(s.x, s.y)), x, y);
    r[c] = __float_as_uint(x);
    r[c + 1] = __float_as_uint(y);
    unpack2(mul2(pack2(__uint_as_float(r[c + 2]), __uint_as_float(r[c + 3])), pack2(s.z, s.w)), x, y);
    r[c + 2] = __float_as_uint(x);
    r[c + 3] = __float_as_uint(y);
  }
}
__device__ __forceinline__ float max32(const uint32_t (&r)[32], float mx) {
  float m[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) m[i] = __uint_as_float(r[i]);
#pragma unroll
  for (int c = 4; c < 32; ++c) m[c & 3] = fmaxf(m[c & 3], __uint_as_float(r[c]));
  return fmaxf(fmaxf(fmaxf(m[0], m[1]), fmaxf(m[2], m[3])), mx);
}
// 32 exponentials; their bf16 go to tensor memory at `to`.
__device__ __forceinline__ void exp32(const uint32_t (&r)[32], f2 sc2, f2 nr2, f2 (&acc)[2], uint32_t to) {
#pragma unroll
  for (int h = 0; h < 32; h += 16) {
    uint32_t w[8];
#pragma unroll
    for (int c = 0; c < 16; c += 2) {
      float x, y;
      unpack2(fma2(pack2(__uint_as_float(r[h + c]), __uint_as_float(r[h + c + 1])), sc2, nr2), x, y);
      x = ex2_approx(x);
      y = ex2_approx(y);
      acc[(c >> 1) & 1] = add2(acc[(c >> 1) & 1], pack2(x, y));
      w[c / 2] = cache::pack_bf16(x, y);
    }
    tmem_st8(to + h / 2, w);
  }
}

constexpr int kOffP = 64;  // P's first column over S: its columns are taken from the last to the first

// The row's reference moves where its maximum has passed it by 8 binades: sum and O follow.
template <int D>
__device__ __forceinline__ void move_reference(uint32_t to, float top, bool first, float& ref, float& sum) {
  const bool move = top > ref + 8.0f;  // (false for a row that has seen nothing, and for NaN)
  if (!__any_sync(0xffffffffu, move)) return;
  const float alpha = move ? (ref == -INFINITY ? 0.f : ex2_approx(ref - top)) : 1.f;
  if (move) ref = top;
  sum *= alpha;
  if (first) return;
  uint32_t a[32];
#pragma unroll 1
  for (int h = 0; h < D / 32; ++h) {
    tmem_ld32(to + h * 32, a);
#pragma unroll
    for (int c = 0; c < 32; ++c) a[c] = __float_as_uint(__uint_as_float(a[c]) * alpha);
    tmem_st32(to + h * 32, a);
  }
}

// One step of a row: S in tensor memory at `ts` becomes P there, the row's reference and sum move on, and O at `to` is rescaled if it must be.
// Columns come 32 at a time, the next ones on their way while one block is worked on; the last block of the maximum is the
// first of the exponentials.
template <int D>
__device__ __forceinline__ void softmax_step(uint32_t ts, uint32_t to, float scale, bool first, float& ref, float& sum) {
  uint32_t a[32], b[32];
  tmem_ld32(ts, a);
  tmem_ask32(ts + 32, b);
  float mx = max32(a, -INFINITY);
  tmem_wait(b);
  tmem_ask32(ts + 64, a);
  mx = max32(b, mx);
  tmem_wait(a);
  tmem_ask32(ts + 96, b);
  mx = max32(a, mx);
  tmem_wait(b);
  mx = max32(b, mx);
  move_reference<D>(to, mx * scale, first, ref, sum);
  const float nr = ref == -INFINITY ? 0.f : -ref;
  const f2 sc2 = pack2(scale, scale), nr2 = pack2(nr, nr);
  f2 acc[2] = {pack2(0.f, 0.f), pack2(0.f, 0.f)};
#pragma unroll 1
  for (int h = 1; h >= 0; --h) {
    tmem_ask32(ts + h * 64, a);
    exp32(b, sc2, nr2, acc, ts + kOffP + h * 32 + 16);
    tmem_wait(a);
    if (h != 0) tmem_ask32(ts + 32, b);
    exp32(a, sc2, nr2, acc, ts + kOffP + h * 32);
    if (h != 0) tmem_wait(b);
  }
  float x, y;
  unpack2(add2(acc[0], acc[1]), x, y);
  sum += x + y;
}

// The same in short loops over blocks b0 .. b1 - 1 of 32 columns: for tiles in which some row does not see every position (scores that it does not see
// become -inf, after the keys' scales, which may be NaN there; blocks that no row sees are left out), and for all tiles of codes, where
// more warps have code of their own: what is not in a short loop is fetched anew each time, about four cycles an instruction (16
// sequences of nine over e4m3 189 -> 158 us; bf16 chunks of 2000 1003 -> 1045, so not there).
template <int D, bool E4M3>
__device__ __forceinline__ void softmax_blocks(uint32_t ts, uint32_t to, float scale, bool first, bool masked, const RowMask& mask, int b0, int b1,
                                               const float* scales, float& ref, float& sum) {
  uint32_t a[32];
  float mx = -INFINITY;
#pragma unroll 1
  for (int h = b0; h < b1; ++h) {
    tmem_ld32(ts + h * 32, a);
    if (E4M3) scale32(a, scales + h * 32);
    if (masked) {
      const uint32_t v = mask.bits(h * 32);
#pragma unroll
      for (int c = 0; c < 32; ++c) a[c] = v & (1u << c) ? a[c] : 0xff800000u;
    }
    if (masked || E4M3) tmem_st32(ts + h * 32, a);
    mx = max32(a, mx);
  }
  if (masked || E4M3) tmem_st_wait();
  move_reference<D>(to, mx * scale, first, ref, sum);
  const float nr = ref == -INFINITY ? 0.f : -ref;
  const f2 sc2 = pack2(scale, scale), nr2 = pack2(nr, nr);
  f2 acc[2] = {pack2(0.f, 0.f), pack2(0.f, 0.f)};
#pragma unroll 1
  for (int h = b1 - 1; h >= b0; --h) {
    tmem_ld32(ts + h * 32, a);
    exp32(a, sc2, nr2, acc, ts + kOffP + h * 16);
  }
  float x, y;
  unpack2(add2(acc[0], acc[1]), x, y);
  sum += x + y;
}

// Adds back to a row what zero_nonfinite took out of the values that it sees at positions from .. to - 1; columns col0 .. col0 + 15 of row_pos are in o.
// (Only those of the tiles that O was formed from: elsewhere the row's reference may be -inf, and where an item's parts meet
// its O would count 2^-inf times infinity, which is NaN.)
template <bool E4M3>
__device__ __noinline__ void add_back(const Params& p, int b, int kvh, int row_pos, int lo_first, int lo_last, int upper, int hi, int from, int to, int col0, float* o) {
  auto visit = [&](int first, int last) {
    for (int pos = max(first, from); pos < min(last, to); ++pos) {
      if (!visible(p, row_pos, pos)) continue;
      const int page = cache::page_of(p.c, b, pos);
      if (page < 0) continue;
      const int slot = pos & ((1 << p.c.page_shift) - 1);
      const int64_t at = cache::row_at(p.c, page, slot, kvh) + col0;
      const float scale = E4M3 ? cache::scale_value(p.c.v_scales[cache::scale_at(p.c, page, slot, kvh)]) : 1.f;
      for (int c = 0; c < 16; c += 2) {
        float x, y;
        if (E4M3) {
          cache::unpack_e4m3(*reinterpret_cast<const uint16_t*>(p.c.v_pages + at + c), x, y);
          const uint32_t w = cache::pack_bf16(x * scale, y * scale);
          x = cache::bf16_lo(w);
          y = cache::bf16_hi(w);
        } else {
          const uint32_t w = *reinterpret_cast<const uint32_t*>(p.c.v_pages + 2 * (at + c));
          x = cache::bf16_lo(w);
          y = cache::bf16_hi(w);
        }
        if (!(fabsf(x) < INFINITY)) o[c] += x;
        if (!(fabsf(y) < INFINITY)) o[c + 1] += y;
      }
    }
  };
  visit(lo_first, min(lo_last, upper));  // positions that only earlier rows see
  visit(upper, hi);                      // ... and that only later ones do
}

// A row's result where a wait has run out.
__device__ __noinline__ void nan_row(const Params& p, int b, int t, int head, int D) {
  uint4* o = reinterpret_cast<uint4*>(p.out.data + 2 * ((int64_t)b * p.out.batch_stride + (int64_t)t * p.out.token_stride + (int64_t)head * p.out.head_stride));
  for (int i = 0; i < D / 8; ++i) o[i] = make_uint4(0x7fc07fc0u, 0x7fc07fc0u, 0x7fc07fc0u, 0x7fc07fc0u);
  if (p.lse) p.lse[((int64_t)b * p.n + t) * p.heads + head] = quiet_nan();
}

// Where a part of an item lies in scratch, in units of four columns of a row: neighbouring rows side by side, so that a warp's stores and
// loads are whole lines (a row after the other they took 4 - 9 thousand cycles of an item's end).
template <int D, int ROWS>
__device__ __forceinline__ int64_t part_at(int cta, bool from_start, int col4, int row) {
  return (((int64_t)cta * 2 + (from_start ? 1 : 0)) * (D / 4) + col4) * ROWS + row;
}

template <int D, bool E4M3, bool PAIR>
__global__ void __launch_bounds__(Shape<D, E4M3, PAIR>::kThreads, 1)
attention_kernel(const __grid_constant__ CUtensorMap map_q, const __grid_constant__ CUtensorMap map_k, const __grid_constant__ CUtensorMap map_v,
                 const __grid_constant__ Params p) {
  using S = Shape<D, E4M3, PAIR>;
  extern __shared__ __align__(1024) uint8_t smem[];
  const uint32_t base = smem_u32(smem);
  const uint32_t bar0 = base + S::kOffBar;
  auto k_full = [&](uint32_t s) { return bar0 + 8u * s; };                 // a stage's tile is there
  auto k_empty = [&](uint32_t s) { return bar0 + 8u * (S::kKStages + s); };  // ... has been read by its MMAs
  auto v_full = [&](uint32_t s) { return bar0 + 8u * (2 * S::kKStages + s); };
  auto v_empty = [&](uint32_t s) { return bar0 + 8u * (2 * S::kKStages + S::kVStages + s); };
  auto raw_full = [&](uint32_t s) { return bar0 + 8u * (2 * S::kKStages + 2 * S::kVStages + s); };
  auto raw_empty = [&](uint32_t s) { return bar0 + 8u * (2 * S::kKStages + 2 * S::kVStages + S::kRawStages + s); };
  constexpr uint32_t kB = 2 * S::kKStages + 2 * S::kVStages + 2 * S::kRawStages, kRaw = E4M3 ? S::kRawStages : 1;
  auto k_ready = [&](uint32_t s) { return E4M3 ? bar0 + 8u * (kB + 10 + s) : k_full(s); };  // ... and for E4M3 its keys' scales are in fp32
  const uint32_t drained = bar0 + 8u * (S::kNumBars - 1);                  // no MMA is in flight
  const uint32_t met = bar0 + 8u * (S::kNumBars - 2);                      // all warps of the two slots of one row tile are there
  auto q_full = [&](int s) { return bar0 + 8u * (kB + s); };
  auto q_empty = [&](int s) { return bar0 + 8u * (kB + 2 + s); };
  auto s_full = [&](int s) { return bar0 + 8u * (kB + 4 + s); };          // S of a slot's step is complete (and every MMA before it)
  auto p_ready = [&](int s) { return bar0 + 8u * (kB + 6 + s); };         // its P is there, O rescaled, the values' tile cleaned
  auto o_full = [&](int s) { return bar0 + 8u * (kB + 8 + s); };          // the slot's O of an item is complete
  volatile uint32_t* misc = reinterpret_cast<volatile uint32_t*>(smem + S::kOffMisc);  // [0] tensor memory, [1] a role gave up, [2] tiles whose products are issued, [8..15] items with values to add back
  volatile uint32_t* tile_bad = reinterpret_cast<volatile uint32_t*>(smem + S::kOffFlags);  // of tile number t: entry t % 16, for the conversion 16 + t % 16
  float* key_scales = reinterpret_cast<float*>(smem + S::kOffScales);  // of tile number t: entry t % kScaleRing
  uint8_t* key_bytes = smem + S::kOffScales + S::kScaleRing * kTile * 4;
  float2* exchange = reinterpret_cast<float2*>(smem + S::kOffExchange);

  const int tid = (int)threadIdx.x, lane = tid & 31, warp = __shfl_sync(0xffffffffu, tid >> 5, 0);
  if (tid == 0) {
    asm volatile("prefetch.tensormap [%0];" ::"l"(&map_q) : "memory");
    asm volatile("prefetch.tensormap [%0];" ::"l"(&map_k) : "memory");
    asm volatile("prefetch.tensormap [%0];" ::"l"(&map_v) : "memory");
    for (int s = 0; s < S::kKStages; ++s) {
      mbar_init(k_full(s), E4M3 ? 33 : 1);
      mbar_init(k_empty(s), 1);
      if (E4M3) mbar_init(k_ready(s), 1);
    }
    for (int s = 0; s < S::kVStages; ++s) { mbar_init(v_full(s), E4M3 ? S::kConvWarps : 1); mbar_init(v_empty(s), 1); }
    for (int s = 0; s < S::kRawStages; ++s) { mbar_init(raw_full(s), 33); mbar_init(raw_empty(s), S::kConvWarps); }
    for (int s = 0; s < 2; ++s) {
      mbar_init(q_full(s), E4M3 ? (PAIR ? kTileRows : 2 * kTileRows) : 1);
      mbar_init(q_empty(s), 1);
      mbar_init(s_full(s), 1);
      mbar_init(p_ready(s), kTileRows / 32);
      mbar_init(o_full(s), 1);
    }
    mbar_init(drained, 1);
    mbar_init(met, 2 * kTileRows / 32);
    misc[1] = misc[2] = 0;
    for (int i = 8; i < 16; ++i) misc[i] = 0;
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  }
  if (warp == 0) {  // all of tensor memory: shared memory already keeps it to one CTA per SM
    asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], 512;" ::"r"(base + S::kOffMisc) : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
  }
  if (!E4M3) {
    // Rows of a tile that no box brings: products with zeros take less power, and loops of 64 sequences of one token run into the limit (1 kW: 215 - 230 us,
    // with zeros 202 - 214; the first 50 ms 186, 184).  (E4M3: the softmax warps write zeros themselves.)
    const int rows = p.tpt * p.group;
    for (int i = tid; i < (kTileRows - rows) * 8; i += S::kThreads)
#pragma unroll
      for (int h = 0; h < S::kQBufs * S::kHalves; ++h) *reinterpret_cast<uint4*>(smem + h * S::kHalfBytes + rows * 128 + i * 16) = make_uint4(0u, 0u, 0u, 0u);
    async_proxy_fence();
  }
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem = misc[0];
  // The lengths and a sequence's row of the block table are asked for in L2: a prefetch reads nothing for the program, so the kernel before may still
  // be writing them.  (Which sequences a CTA will get is not known yet; as if all were as long.)
  if (warp == S::kWarpV) {
    const int b = (int)((int64_t)blockIdx.x * p.B / gridDim.x);
    if (lane * 32 < p.B) asm volatile("prefetch.global.L2 [%0];" ::"l"(p.c.lengths + lane * 32));
    if (p.counts && lane * 32 < p.B) asm volatile("prefetch.global.L2 [%0];" ::"l"(p.counts + lane * 32));
    if (((int64_t)lane * 32 << p.c.page_shift) < p.c.capacity) asm volatile("prefetch.global.L2 [%0];" ::"l"(p.c.table + b * p.c.table_stride + lane * 32));
  }
  asm volatile("griddepcontrol.wait;" ::: "memory");  // everything below reads or writes what the kernels before may be working on
  asm volatile("griddepcontrol.launch_dependents;");

  // A wait has run out, or had in a step before and nobody has looked: no wait waits any more, nothing is issued, and nothing that others
  // write is read: all that is left to do is NaN for the rows.  (One lane looks: a warp's lanes decide alike.)
  const bool pending = __shfl_sync(0xffffffffu, lane == 0 ? *reinterpret_cast<volatile int*>(p.status) : 0, 0) != 0;
  bool failed = pending;
  auto wait_warp = [&](uint32_t bar, uint32_t parity) {  // the same decision in the whole warp
    if (!failed && !__all_sync(0xffffffffu, mbar_wait_suspended(bar, parity, p.status, kErrAttention, &misc[2]))) failed = true;
  };
  const Range range = range_of(p);
  Walk walk(p, range);
  uint32_t tile_no = 0;  // tiles before this item: tile j of the item is in stage (tile_no + j) % stages of each ring

  if (warp >= 8 && warp < S::kWarpConv) {
  if (warp == S::kWarpK || warp == S::kWarpV) {
    // ---------------- keys, or values: a lane per box ----------------
    const bool values = warp == S::kWarpV;
    const int page_size = 1 << p.c.page_shift;
    // E4M3: a box is a page's part of the tile.  bf16: a box is eight rows with all their columns.
    const int rows = E4M3 ? min(page_size, kTile) : 8;
    const uint32_t box_bytes = (uint32_t)rows * D * (E4M3 ? 1 : 2);
    const int of = E4M3 ? lane * rows >> 3 : lane;  // the group of eight whose page this lane's box is on
    for (; walk.have(); walk.next()) {
      const Group& g = walk.gr;
      const int m = walk.tiles();
      // The pages of several tiles come in one load, a lane each, and those of the next tiles are asked for when these begin to be used.
      const int per_tile = max(0, 7 - p.c.page_shift), tiles_at_once = 32 >> per_tile;  // log2 of the pages of a tile
      auto ask = [&](int j) {
        const int tile = j + (lane >> per_tile), pos = tile < m ? tile_start(g, walk.x0 + tile) + ((lane & ((1 << per_tile) - 1)) << p.c.page_shift) : g.hi;
        return pos < g.hi ? p.c.table[(int64_t)g.b * p.c.table_stride + (pos >> p.c.page_shift)] : -1;
      };
      int pages = ask(0), pages_ahead = -1;
      for (int j = 0; j < m; ++j) {
        const int in = j & (tiles_at_once - 1);
        if (in == 0) {
          if (j > 0) pages = pages_ahead;
          pages_ahead = ask(j + tiles_at_once);
        }
        const int p0 = tile_start(g, walk.x0 + j), pos = p0 + 8 * lane;
        int page = __shfl_sync(0xffffffffu, pages, (in << per_tile) + ((lane & 15) * 8 >> min(7, p.c.page_shift)));  // of eight positions
        const bool need = lane < 16 && pos < g.hi;
        // What stands on a page that does not exist is not seen.  (Read behind the barrier of the keys, or of the values' codes.)
        const unsigned bad = __ballot_sync(0xffffffffu, need && (page < 0 || page >= p.c.num_pages));
        if (!need || ((bad >> lane) & 1u)) page = -1;
        const uint32_t no = tile_no + (uint32_t)j;
        uint32_t there, dst, bytes;
        if (!values) {
          const uint32_t st = no % S::kKStages;
          wait_warp(k_empty(st), ((no / S::kKStages) & 1) ^ 1);
          there = k_full(st);
          dst = base + S::kOffK + st * S::kKBytes;
          bytes = smem_u32(key_bytes) + st * kTile;
          if (lane == 0) tile_bad[no & 15] = bad;
        } else if (E4M3) {
          const uint32_t st = no % kRaw;
          wait_warp(raw_empty(st), ((no / kRaw) & 1) ^ 1);
          there = raw_full(st);
          dst = base + S::kOffRaw + st * S::kRawBytes;
          bytes = dst + S::kCodeBytes;
          if (lane == 0) tile_bad[16 + (no & 15)] = bad;
        } else {
          const uint32_t st = no % S::kVStages;
          wait_warp(v_empty(st), ((no / S::kVStages) & 1) ^ 1);
          there = v_full(st);
          dst = base + S::kOffV + st * S::kTileBytes;
          bytes = 0;
        }
        if (failed) break;
        const int pg = E4M3 ? __shfl_sync(0xffffffffu, page, of & 15) : page, at = p0 + 8 * of;
        const bool mine = of < 16 && pg >= 0 && (E4M3 || at + 8 > g.lo_first || at < p.sinks);
        const unsigned have = __ballot_sync(0xffffffffu, mine);
        if (lane == 0) mbar_expect_tx(there, (uint32_t)__popc(have) * box_bytes);
        __syncwarp();
        const int slot = at & (page_size - 1);
        const CUtensorMap* map = values ? &map_v : &map_k;
        if (E4M3) {
          if (page >= 0)  // eight scales a lane, in the same phase of the barrier
            asm volatile("cp.async.ca.shared.global [%0], [%1], 8;" ::"r"(bytes + lane * 8),
                         "l"((values ? p.c.v_scales : p.c.k_scales) + cache::scale_at(p.c, page, pos & (page_size - 1), walk.kvh))
                         : "memory");
          asm volatile("cp.async.mbarrier.arrive.noinc.shared::cta.b64 [%0];" ::"r"(there) : "memory");
          if (mine) tma_load_4d(dst + lane * rows * D, map, 0, slot, walk.kvh, pg, there);
        } else if (mine) {
          tma_load_5d(dst + lane * S::kGroupBytes, map, 0, slot, 0, walk.kvh, pg, there);
        }
        __syncwarp();
      }
      if (failed) break;
      tile_no += m;
    }
    // The last tiles have arrived before this warp lets the CTA end, whether or not somebody has taken them.
    const uint32_t stages = !values ? S::kKStages : E4M3 ? kRaw : S::kVStages;
    for (uint32_t no = tile_no > stages ? tile_no - stages : 0u; no < tile_no; ++no) {
      const uint32_t st = no % stages;
      wait_warp(!values ? k_full(st) : E4M3 ? raw_full(st) : v_full(st), (no / stages) & 1);
    }
  } else if (warp == S::kWarpQ) {
    // ---------------- queries: (heads of the group, tokens) boxes; tokens behind the chunk's end come as zeros ----------------
    // E4M3: the softmax warps take the queries apart themselves, and this one turns the keys' scale bytes into fp32, four a lane.
    uint32_t item = 0;
    for (; walk.have(); walk.next(), ++item) {
      if (E4M3) {
        const int m = walk.tiles();
        for (int j = 0; j < m; ++j) {
          const uint32_t no = tile_no + (uint32_t)j, st = no % S::kKStages;
          wait_warp(k_full(st), (no / S::kKStages) & 1);
          if (failed) break;
          const uint32_t b = *reinterpret_cast<const uint32_t*>(key_bytes + st * kTile + 4 * lane);
          *reinterpret_cast<float4*>(key_scales + (no % S::kScaleRing) * kTile + 4 * lane) =
              make_float4(cache::scale_value(b & 255u), cache::scale_value((b >> 8) & 255u), cache::scale_value((b >> 16) & 255u), cache::scale_value(b >> 24));
          __syncwarp();
          if (lane == 0) mbar_arrive(k_ready(st));
          __syncwarp();
        }
        tile_no += m;
      }
      for (int s = 0; s < (E4M3 ? 0 : PAIR ? 2 : 1); ++s) {
        const int buf = PAIR ? s : (int)(item % S::kQBufs);
        wait_warp(q_empty(buf), ((PAIR ? item : item / S::kQBufs) & 1) ^ 1);
        if (!failed && elect_lane()) {
          mbar_expect_tx(q_full(buf), (uint32_t)(p.tpt * p.group * D * 2));
          for (int h = 0; h < S::kHalves; ++h)
            tma_load_4d(base + buf * S::kTileBytes + h * S::kHalfBytes, &map_q, h * 64, walk.kvh * p.group, walk.gr.t0 + s * p.tpt, walk.gr.b, q_full(buf));
        }
        __syncwarp();
      }
    }
    for (int s = 0; s < (E4M3 ? 0 : 2); ++s) {  // (as above: the last use of each buffer)
      const uint32_t uses = PAIR ? item : (item + 1u - (uint32_t)s) / 2u;
      if (uses > 0) wait_warp(q_full(s), (uses - 1u) & 1);
    }
    // ... and the rows of sequences that hold no position at all
    for (int64_t g = blockIdx.x + (int64_t)gridDim.x * lane; g < p.groups; g += (int64_t)gridDim.x * 32) {
      const Group gr = group_at(p, (int)g);
      if (gr.count > 0) continue;
      for (int t = gr.t0; t < gr.t1; ++t)
        for (int h = 0; h < p.heads; ++h) {
          uint4* o = reinterpret_cast<uint4*>(p.out.data + 2 * ((int64_t)gr.b * p.out.batch_stride + (int64_t)t * p.out.token_stride + (int64_t)h * p.out.head_stride));
          for (int i = 0; i < D / 8; ++i) o[i] = make_uint4(0u, 0u, 0u, 0u);
          if (p.lse) p.lse[((int64_t)gr.b * p.n + t) * p.heads + h] = -INFINITY;
        }
    }
  } else if (warp == S::kWarpMma) {
    // ---------------- MMA issue ----------------
    if (lane == 0) {  // how this CTA's range begins, for the kernel that adds up
      int4* d = reinterpret_cast<int4*>(p.desc) + 2 * blockIdx.x;
      const bool any = walk.have();
      d[0] = make_int4(any ? walk.x0 : 0, any ? walk.gr.count : 0, range.share, any ? walk.kvh : 0);
      d[1] = any ? make_int4(walk.gr.b, walk.gr.t0, walk.gr.t1, 0) : make_int4(0, 0, 0, 0);
    }
    __syncwarp();
    const bool lead = elect_lane();
    constexpr uint32_t kIdescS = instr_desc(kTile, false), kIdescO = instr_desc(D, true);
    uint32_t item = 0, use0 = 0, use1 = 0;   // steps of each slot so far
    uint32_t queries0 = 0, queries1 = 0;     // items of which a slot of a pair has had its queries
    bool issued = false;
    for (; walk.have(); walk.next(), ++item) {
      const Group& g = walk.gr;
      const int m = walk.tiles();
      auto sees = [&](int s, int j) { return !PAIR || slot_sees(p, g, s, tile_start(g, walk.x0 + j)); };
      auto issue_s = [&](int s, int j) {  // S of slot s = Q x keys of tile j
        const uint32_t st = (tile_no + (uint32_t)j) % S::kKStages;
        const int buf = PAIR ? s : (int)(item % S::kQBufs);
        issued |= !failed;
        if (!failed && lead) {
          const uint32_t a = desc_lo(base + buf * S::kTileBytes, 16), b = desc_lo(base + S::kOffK + st * S::kKBytes, 16);
          if (E4M3) {
#pragma unroll
            for (int k = 0; k < D / 32; ++k) mma_ss8(tmem + s * kTile, a + k * 2, b + k * 2, desc_hi8(D), instr_desc8(kTile, false), k != 0);
#pragma unroll
            for (int k = 0; k < D / 32; ++k) mma_ss8(tmem + s * kTile, a + (S::kCodeBytes >> 4) + k * 2, b + k * 2, desc_hi8(D), instr_desc8(kTile, true), 1);
          } else {
#pragma unroll
            for (int k = 0; k < D / 16; ++k)
              mma_ss(tmem + s * kTile, a + ((uint32_t)((k / 4) * S::kHalfBytes + (k % 4) * 32) >> 4), desc_hi(1024),
                     b + ((uint32_t)((k / 4) * 1024 + (k % 4) * 32) >> 4), desc_hi(S::kGroupBytes), kIdescS, k != 0);
          }
          mma_commit(s_full(s));
        }
        __syncwarp();
      };
      auto issue_o = [&](int s, int j, bool accumulate) {  // O of slot s += P x values of tile j, 16 positions at a time
        uint32_t& use = s ? use1 : use0;
        wait_warp(p_ready(s), use & 1);
        ++use;
        const uint32_t st = (tile_no + (uint32_t)j) % S::kVStages;
        tc_fence_after();
        if (!failed && lead) {
          const uint32_t b = desc_lo(base + S::kOffV + st * S::kTileBytes, 1024);
          const uint32_t to = tmem + 2 * kTile + s * 128, from = tmem + s * kTile + kOffP;
          const Span span = tile_span(p, g, tile_start(g, walk.x0 + j));
          if (span.first == 0 && span.last == kTile) {
#pragma unroll
            for (int k = 0; k < kTile / 16; ++k)
              mma_ts(to, from + k * 8, b + ((uint32_t)(k * 2 * S::kGroupBytes) >> 4), desc_hi(S::kGroupBytes), kIdescO, accumulate || k != 0);
          } else {
            const int k0 = span.first / 16;
#pragma unroll 1
            for (int k = k0; k * 16 < span.last; ++k)
              mma_ts(to, from + k * 8, b + ((uint32_t)(k * 2 * S::kGroupBytes) >> 4), desc_hi(S::kGroupBytes), kIdescO, accumulate || k != k0);
          }
        }
        __syncwarp();
      };
      auto wait_k = [&](int j) {
        const uint32_t no = tile_no + (uint32_t)j;
        wait_warp(k_ready(no % S::kKStages), (no / S::kKStages) & 1);
      };
      auto wait_v = [&](int j) {
        const uint32_t no = tile_no + (uint32_t)j;
        wait_warp(v_full(no % S::kVStages), (no / S::kVStages) & 1);
      };
      auto commit = [&](uint32_t bar) {
        if (!failed && lead) mma_commit(bar);
        __syncwarp();
      };
      auto release_k = [&](int j) { commit(k_empty((tile_no + (uint32_t)j) % S::kKStages)); };
      auto release_v = [&](int j) {
        if (lane == 0) misc[2] = tile_no + (uint32_t)j + 1u;  // (what keeps other warps' waits from running out)
        commit(v_empty((tile_no + (uint32_t)j) % S::kVStages));
      };
      if (PAIR) {
        int last[2];
        for (int s = 0; s < 2; ++s) {
          last[s] = last_seen(p, g, s, walk.x0, m);
          if (E4M3 && last[s] < 0) continue;  // (then its warps bring no queries)
          wait_warp(q_full(s), (s ? queries1 : queries0) & 1);
          ++(s ? queries1 : queries0);
        }
        bool begun[2] = {false, false};
        wait_k(0);
        for (int s = 0; s < 2; ++s)
          if (sees(s, 0)) issue_s(s, 0);
        release_k(0);
        for (int j = 0; j < m; ++j) {
          wait_v(j);
          for (int s = 0; s < 2; ++s) {
            if (sees(s, j)) {
              issue_o(s, j, begun[s]);
              begun[s] = true;
              if (j == last[s]) commit(o_full(s));
            }
            if (j + 1 < m) {
              if (s == 0) wait_k(j + 1);
              if (sees(s, j + 1)) issue_s(s, j + 1);
            }
          }
          release_v(j);
          if (j + 1 < m) release_k(j + 1);
        }
        if (!E4M3) {
          commit(q_empty(0));
          commit(q_empty(1));
        }
      } else {
        const int buf = (int)(item % S::kQBufs);
        wait_warp(q_full(buf), (item / S::kQBufs) & 1);
        auto scores = [&](int j) {
          wait_k(j);
          issue_s(j & 1, j);
          release_k(j);
          if (!E4M3 && j == m - 1) commit(q_empty(buf));
        };
        scores(0);
        if (m > 1) scores(1);
        for (int j = 0; j < m; ++j) {
          wait_v(j);
          issue_o(j & 1, j, j >= 2);
          release_v(j);
          if (j + 2 >= m) commit(o_full(j & 1));
          if (j + 2 < m) scores(j + 2);
        }
      }
      tile_no += m;
    }
    if (issued) {  // what has been issued ends before shared and tensor memory are given back, whatever the other warps have waited for
      if (lead) mma_commit(drained);
      __syncwarp();
      if (failed) mbar_wait_quiet(drained, 0, 2000000ull);
      else wait_warp(drained, 0);
    }
    __syncwarp();
  }
  } else if (E4M3 && warp >= S::kWarpConv) {
    // ---------------- codes to tiles of bf16, 16 at a time ----------------
    // Eight neighbouring threads take four chunks of two rows, whose places in the swizzled tile share no bank.  From one of its chunks to the
    // next a thread goes on by whole groups of eight rows: its place in a row and in the swizzle stays.
    constexpr int kPer = D / 64, kConv = E4M3 ? S::kConvThreads : 128, kEach = kTile * D / 16 / kConv, kRowStep = kConv / 8 / kPer * 2;
    const int ct = tid - S::kWarpConv * 32;
    const int row0 = (ct >> 3) / kPer * 2 + ((ct >> 2) & 1), chunk = (ct >> 3) % kPer * 4 + (ct & 3);
    const int from0 = row0 * D + chunk * 16, to0 = S::piece_at(row0, chunk * 2), to1 = S::piece_at(row0, chunk * 2 + 1);
    constexpr int kToStep = kRowStep / 8 * S::kGroupBytes;
    uint32_t item = 0;
    for (; walk.have(); walk.next(), ++item) {
      const Group& g = walk.gr;
      const int m = walk.tiles();
      for (int j = 0; j < m; ++j) {
        const uint32_t no = tile_no + (uint32_t)j, rs = no % kRaw, st = no % S::kVStages;
        wait_warp(raw_full(rs), (no / kRaw) & 1);
        wait_warp(v_empty(st), ((no / S::kVStages) & 1) ^ 1);
        if (failed) break;
        const uint8_t* raw = smem + S::kOffRaw + rs * S::kRawBytes;
        uint8_t* dst = smem + S::kOffV + st * S::kTileBytes;
        const int p0 = tile_start(g, walk.x0 + j);
        const uint32_t bad = tile_bad[16 + (no & 15)];
        const bool edge = bad != 0 || tile_unseen(p, g, p0) || tile_partial(p, g, p0);
        bool any = false;
#pragma unroll 1
        for (int i0 = 0; i0 < kEach; i0 += 4) {
          uint4 codes[4];
          int scale[4];
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            codes[i] = *reinterpret_cast<const uint4*>(raw + from0 + (i0 + i) * kRowStep * D);
            scale[i] = raw[S::kCodeBytes + row0 + (i0 + i) * kRowStep];
          }
          uint32_t w[4][8];
          if (!cache::plain_e4m3<4>(codes, scale)) {
#pragma unroll
            for (int i = 0; i < 4; ++i) cache::any16_e4m3(codes[i], scale[i], w[i]);
          } else {
#pragma unroll
            for (int i = 0; i < 4; ++i) cache::plain16_e4m3(codes[i], scale[i], w[i]);
          }
          if (edge) {
#pragma unroll
            for (int i = 0; i < 4; ++i) {
              const int row = row0 + (i0 + i) * kRowStep, seen = (bad >> (row >> 3)) & 1u ? 0 : seen_by(p, g, p0 + row);
#pragma unroll
              for (int k = 0; k < 8; ++k) w[i][k] = seen == 0 ? 0u : seen == 1 ? zero_nonfinite(w[i][k], any) : w[i][k];
            }
          }
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            *reinterpret_cast<uint4*>(dst + to0 + (i0 + i) * kToStep) = make_uint4(w[i][0], w[i][1], w[i][2], w[i][3]);
            *reinterpret_cast<uint4*>(dst + to1 + (i0 + i) * kToStep) = make_uint4(w[i][4], w[i][5], w[i][6], w[i][7]);
          }
        }
        if (any) misc[8 + (item & 7)] = item + 1;
        async_proxy_fence();
        __syncwarp();
        if (lane == 0) {
          mbar_arrive(v_full(st));
          mbar_arrive(raw_empty(rs));
        }
        __syncwarp();
      }
      if (failed) break;
      tile_no += m;
    }
  } else {
    // ---------------- softmax of a slot, a thread per row ----------------
    const int slot = warp >> 2, row = tid & 127, quarter = warp & 3;
    const uint32_t lanes = (uint32_t)(quarter * 32) << 16;
    const uint32_t ts = tmem + lanes + slot * kTile, to = tmem + lanes + 2 * kTile + slot * 128;
    const int row_token = row / p.group, row_head = row - row_token * p.group;
    uint32_t use = 0, items_done = 0, item = 0, meetings = 0;
    // (A barrier with a bounded wait, not bar.sync: should lengths change during the step, the warps may not agree on how many items there are.
    // A warp that has given up does not arrive, so that the others do not go on without it.)
    auto meet = [&]() {
      __syncwarp();
      if (!failed && lane == 0) mbar_arrive(met);
      wait_warp(met, meetings++ & 1);
    };
    for (; walk.have(); walk.next(), ++item) {
      const Group& g = walk.gr;
      const int m = walk.tiles();
      const int ts0 = g.t0 + (PAIR ? slot * p.tpt : 0), ts1 = min(g.t1, ts0 + p.tpt);  // the slot's tokens
      const int t = ts0 + row_token, row_pos = g.L + t;
      const bool live = row_token < p.tpt && t < ts1;
      const bool warp_live = __any_sync(0xffffffffu, live);
      const int first_hi = min(g.L + ts0 + 1, g.hi), last_lo = p.window > 0 ? g.L + ts1 - p.window : 0;
      float ref = -INFINITY, sum = 0.f, scale = p.scale;
      bool begun = false;
      if (E4M3 && (!PAIR || last_seen(p, g, slot, walk.x0, m) >= 0)) {
        // The row's queries in two parts (of one row tile: both slots take half of the columns).  Every MMA that read the item before's is done: its O was
        // waited for.  A slot that sees nothing brings none: it waits for nothing either, and would run on past the phase that the MMAs wait for.
        constexpr int kPieces = PAIR ? D / 8 : D / 16;  // of eight values
        const int piece0 = PAIR ? 0 : slot * kPieces;
        const bool there = !failed && row_token < p.tpt && t < p.n;
        const uint4* from = reinterpret_cast<const uint4*>(p.q.data + 2 * ((int64_t)g.b * p.q.batch_stride + (int64_t)t * p.q.token_stride +
                                                                           (int64_t)(walk.kvh * p.group + row_head) * p.q.head_stride)) + piece0;
        uint32_t m2 = 0u;
        if (there) {
          if (walk.kvh + 1 < p.c.kv_heads && p.q.head_stride > 0)  // the next item's, in all likelihood
            asm volatile("prefetch.global.L2 [%0];" ::"l"(from + (int64_t)p.group * p.q.head_stride / 8));
#pragma unroll 4
          for (int i = 0; i < kPieces; ++i) {
            const uint4 v = from[i];
            m2 = __vmaxu2(m2, __vmaxu2(cache::amax2(v.x, v.y), cache::amax2(v.z, v.w)));
          }
        }
        uint32_t amax = max(m2 & 0xffffu, m2 >> 16);
        if (!PAIR) {
          exchange[slot * kTileRows + row].x = __uint_as_float(amax);
          meet();
          amax = max(amax, __float_as_uint(exchange[(slot ^ 1) * kTileRows + row].x));
        }
        const int s = cache::scale_of(amax);
        if (s == cache::kScaleNan) scale = quiet_nan();  // (so the row is)
        else scale = positive(scale * cache::scale_value(s));
        const float inv = s == cache::kScaleNan ? 0.f : __uint_as_float((uint32_t)(254 - s) << 23);
        uint8_t* hi = smem + (PAIR ? slot * S::kTileBytes : 0);
#pragma unroll 1
        for (int i = 0; i < kPieces; i += 2) {  // 16 values: 16 bytes of each part
          uint32_t w[8] = {0u, 0u, 0u, 0u, 0u, 0u, 0u, 0u};
          if (there && s != cache::kScaleNan) {
            const uint4 u = from[i], v = from[i + 1];
            const uint32_t x[8] = {u.x, u.y, u.z, u.w, v.x, v.y, v.z, v.w};
#pragma unroll
            for (int c = 0; c < 8; c += 2) cache::split_e4m3_e5m2(x[c], x[c + 1], inv, w[c / 2], w[4 + c / 2]);
          }
          if (failed) continue;
          const int at = code_at(D, row, (piece0 + i) / 2);
          *reinterpret_cast<uint4*>(hi + at) = make_uint4(w[0], w[1], w[2], w[3]);
          *reinterpret_cast<uint4*>(hi + S::kCodeBytes + at) = make_uint4(w[4], w[5], w[6], w[7]);
        }
        async_proxy_fence();
        if (!failed) mbar_arrive(q_full(PAIR ? slot : 0));
        if (!PAIR) meet();  // (the exchange is used again at the item's end)
      }
      for (int j = PAIR ? 0 : slot; j < m; j += PAIR ? 1 : 2) {
        const int p0 = tile_start(g, walk.x0 + j);
        if (PAIR && !slot_sees(p, g, slot, p0)) continue;
        wait_warp(s_full(slot), use & 1);
        if (failed) break;
        ++use;
        const uint32_t bad = tile_bad[(tile_no + (uint32_t)j) & 15];
        if (warp_live) {
          tc_fence_after();
          const bool masked = p0 + kTile > first_hi || (p0 < last_lo && p0 + kTile > p.sinks) || bad != 0;
          if (masked || E4M3) {
            RowMask mask;
            mask.bad = bad;
            mask.lim = min(row_pos + 1, g.hi) - p0;
            mask.lo = p.window > 0 ? row_pos + 1 - p.window - p0 : 0;
            mask.snk = p.sinks - p0;
            const Span span = tile_span(p, g, p0);
            softmax_blocks<D, E4M3>(ts, to, scale, !begun, masked, mask, span.first / 32, (span.last + 31) / 32, key_scales + ((tile_no + (uint32_t)j) % S::kScaleRing) * kTile, ref,
                                    sum);
          } else {
            softmax_step<D>(ts, to, scale, !begun, ref, sum);
          }
          tmem_st_wait();
          tc_fence_before();
        }
        if (!E4M3 && (bad != 0 || tile_unseen(p, g, p0) || tile_partial(p, g, p0)) && (!PAIR || slot == 0 || !slot_sees(p, g, 0, p0))) {
          // The values' tile before its MMAs (those of both slots come after this slot's p_ready), 16 bytes at a time: only what the MMAs take.
          const uint32_t no = tile_no + (uint32_t)j, st = no % S::kVStages;
          wait_warp(v_full(st), (no / S::kVStages) & 1);
          if (failed) break;
          uint8_t* tile = smem + S::kOffV + st * S::kTileBytes;
          const Span span = tile_span(p, g, p0);
          bool any = false;
          auto clean = [&](int from, int to_row, bool zero) {  // rows from .. to_row - 1
#pragma unroll 1
            for (int u = row; u < (to_row - from) * (D / 8); u += kTileRows) {
              uint4* at = reinterpret_cast<uint4*>(tile + S::piece_at(from + u / (D / 8), u % (D / 8)));
              uint4 v = zero ? make_uint4(0u, 0u, 0u, 0u) : *at;
              bool here = zero;
              if (!zero) {
                v.x = zero_nonfinite(v.x, here);
                v.y = zero_nonfinite(v.y, here);
                v.z = zero_nonfinite(v.z, here);
                v.w = zero_nonfinite(v.w, here);
                any |= here;
              }
              if (here) *at = v;
            }
          };
          const int upper = g.L + g.t0 + 1 - p0, window0 = max(max(g.lo_first, p.sinks) - p0, 0), window1 = min(g.lo_last - p0, min(upper, span.last));
#pragma unroll 1
          for (int i = 0; i < 5; ++i)  // nobody sees them | later rows only, earlier rows only
            clean(i == 0 ? span.first & ~15 : i == 1 ? span.last : i == 2 ? span.hole0 : i == 3 ? max(upper, 0) : window0,
                  i == 0 ? span.first : i == 1 ? (span.last + 15) & ~15 : i == 2 ? span.hole1 : i == 3 ? span.last : window1, i < 3);
          if (bad != 0)
            for (int r = 0; r < kTile; r += 8)
              if ((bad >> (r >> 3)) & 1u) clean(r, r + 8, true);
          if (any) misc[8 + (item & 7)] = item + 1;
          async_proxy_fence();
          __syncwarp();
        }
        begun = true;
        __syncwarp();
        if (lane == 0) mbar_arrive(p_ready(slot));
      }
      // ---- the item's end ----
      if (begun) {
        wait_warp(o_full(slot), items_done & 1);
        ++items_done;
        tc_fence_after();
      }
      const bool from_start = walk.x0 == 0, whole = from_start && walk.x1 == g.count;
      float w0 = 1.f, w1 = 0.f, r = ref, l = sum;
      bool use0 = PAIR ? begun : true, use1 = false;  // whether there is an O of each slot
      if (!PAIR) {
        exchange[slot * kTileRows + row] = make_float2(ref, failed ? quiet_nan() : sum);  // (the other slot's columns are NaN too)
        meet();  // both slots' O are complete as well
        const float2 a = exchange[row], b = exchange[kTileRows + row];
        use1 = m > 1;
        r = fmaxf(a.x, use1 ? b.x : -INFINITY);
        const float rr = r == -INFINITY ? 0.f : r;
        w0 = ex2_approx(a.x - rr);
        w1 = use1 ? ex2_approx(b.x - rr) : 0.f;
        l = a.y * w0 + (use1 ? b.y * w1 : 0.f);
        tc_fence_after();
      }
      const bool poison = misc[8 + (item & 7)] == item + 1;  // (read when both slots are done where they share the item)
      // The positions of these tiles from the window on (what only some rows see is never among the first tokens' tiles).
      const int back0 = (g.lo_tile + max(walk.x0 - g.ns, 0)) * kTile, back1 = (g.lo_tile + walk.x1 - g.ns) * kTile;
      const int head = walk.kvh * p.group + row_head;
      if (failed) {
        if (live) {
          if (whole) nan_row(p, g.b, t, head, D);
          else p.part_ml[((int64_t)blockIdx.x * 2 + (from_start ? 1 : 0)) * S::kItemRows + (PAIR ? slot * kTileRows : 0) + row] = make_float2(0.f, quiet_nan());
        }
      } else if (warp_live) {
        const float inv = whole ? (l == 0.f ? 0.f : 1.f / l) : 1.f;
        uint8_t* out = p.out.data + 2 * ((int64_t)g.b * p.out.batch_stride + (int64_t)t * p.out.token_stride + (int64_t)head * p.out.head_stride);
        const int part_row = (PAIR ? slot * kTileRows : 0) + row;
        const int h0 = PAIR ? 0 : slot * (D / 32), h1 = PAIR ? D / 16 : h0 + D / 32;  // the slots of one row tile share its columns
#pragma unroll 1
        for (int h = h0; h < h1; ++h) {
          uint32_t x[16], y[16];
          float o[16];
          if (use0) tmem_ask16(tmem + lanes + 2 * kTile + (PAIR ? slot * 128 : 0) + h * 16, x);
          if (use1) tmem_ask16(tmem + lanes + 2 * kTile + 128 + h * 16, y);
          tmem_wait16(x, y);
#pragma unroll
          for (int c = 0; c < 16; ++c) o[c] = (use0 ? __uint_as_float(x[c]) * w0 : 0.f) + (use1 ? __uint_as_float(y[c]) * w1 : 0.f);
          if (poison && live) {
            float z[16];
#pragma unroll
            for (int c = 0; c < 16; ++c) z[c] = o[c];
            add_back<E4M3>(p, g.b, walk.kvh, row_pos, g.lo_first, g.lo_last, min(g.L + g.t0 + 1, g.hi), g.hi, back0, back1, h * 16, z);
#pragma unroll
            for (int c = 0; c < 16; ++c) o[c] = z[c];
          }
#pragma unroll
          for (int c = 0; c < 16; ++c) o[c] *= inv;
          if (live) {
            if (whole) {
#pragma unroll
              for (int c = 0; c < 16; c += 8)
                *reinterpret_cast<uint4*>(out + 2 * (h * 16 + c)) = make_uint4(cache::pack_bf16(o[c], o[c + 1]), cache::pack_bf16(o[c + 2], o[c + 3]),
                                                                               cache::pack_bf16(o[c + 4], o[c + 5]), cache::pack_bf16(o[c + 6], o[c + 7]));
            } else {
#pragma unroll
              for (int c = 0; c < 16; c += 4)
                p.part_o[part_at<D, S::kItemRows>(blockIdx.x, from_start, h * 4 + c / 4, part_row)] = make_float4(o[c], o[c + 1], o[c + 2], o[c + 3]);
            }
          }
          __syncwarp();
        }
        if (live && (PAIR || slot == 0)) {
          if (!whole)
            p.part_ml[((int64_t)blockIdx.x * 2 + (from_start ? 1 : 0)) * S::kItemRows + part_row] = make_float2(r, l * inv);
          else if (p.lse)
            p.lse[((int64_t)g.b * p.n + t) * p.heads + head] = l == 0.f ? -INFINITY : kLn2 * (r + log2f(l));
        }
        tc_fence_before();
      }
      if (!PAIR) meet();  // neither slot's O is overwritten before both have read it
      tile_no += m;
    }
  }

  if (failed && !pending) misc[1] = 1;
  tc_fence_before();
  __syncthreads();
  if (misc[1] != 0) {  // stragglers among the loads
    const unsigned long long t0 = global_ns();
    while (global_ns() - t0 < 2000000ull) {}
    __syncthreads();
  }
  if (warp == 0) {
    tc_fence_after();
    asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, 512;" ::"r"(tmem) : "memory");
  }
}

// Exercises the bounded wait without any fault: one thread waits on a barrier that nothing completes.
__global__ void attention_selftest_kernel(int* status, unsigned long long limit_ns) {
  __shared__ __align__(8) unsigned long long bar;
  const uint32_t b = smem_u32(&bar);
  mbar_init(b, 1);
  asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  mbar_wait(b, 0, status, kErrAttention, limit_ns);
}

// Adds up the parts of the items that were cut: those that CTA c went on with and CTA c - 1 began.
//   r = max r_i,  l = sum 2^(r_i - r) l_i,  out = sum 2^(r_i - r) O_i / l
// Every block first lists them, so that there is no block without work but for the last ones (a block for every CTA that might have cut one took
// 5 us where none had).  Then a thread takes four columns of a row, neighbouring threads neighbouring rows.
constexpr int kCombineThreads = 256;
template <int D, int ROWS>
__global__ void __launch_bounds__(kCombineThreads) attention_combine_kernel(const __grid_constant__ Params p, int ctas) {
  asm volatile("griddepcontrol.wait;" ::: "memory");
  asm volatile("griddepcontrol.launch_dependents;");
  __shared__ int4 list[kCombineThreads][2];
  __shared__ int in_warp[kCombineThreads / 32];
  const int lane = (int)threadIdx.x & 31, warp = (int)threadIdx.x >> 5;
  const int4* desc = reinterpret_cast<const int4*>(p.desc);
  for (int c0 = 1; c0 < ctas; c0 += kCombineThreads) {  // (once, unless there are more SMs than threads)
    const int mine = c0 + (int)threadIdx.x;
    const int4 d = mine < ctas ? desc[2 * mine] : make_int4(0, 0, 0, 0);
    int4 d1 = mine < ctas ? desc[2 * mine + 1] : make_int4(0, 0, 0, 0);
    d1.w = mine;
    const bool is = d.x > 0 && d.x <= d.z;
    const unsigned others = __ballot_sync(0xffffffffu, is);
    if (lane == 0) in_warp[warp] = __popc(others);
    __syncthreads();
    int cut = 0, before = __popc(others & ((1u << lane) - 1u));
    for (int w = 0; w < kCombineThreads / 32; ++w) {
      if (w < warp) before += in_warp[w];
      cut += in_warp[w];
    }
    if (is) {  // (in the same order in every block)
      list[before][0] = d;
      list[before][1] = d1;
    }
    __syncthreads();
    const int rows = ROWS > kTileRows ? ROWS : p.tpt * p.group, per_item = rows * (D / 4);
    for (int64_t u = (int64_t)blockIdx.x * kCombineThreads + threadIdx.x; u < (int64_t)cut * per_item; u += (int64_t)gridDim.x * kCombineThreads) {
      const int k = (int)(u / per_item), in = (int)(u - (int64_t)k * per_item), col4 = in / rows, row = in - col4 * rows;
      const int4 a = list[k][0], e = list[k][1];
      const int c = e.w, x0 = a.x, count = a.y, share = a.z, kvh = a.w, b = e.x, t0 = e.y, t1 = e.z;
      const int parts = min(1 + (count - x0 + share - 1) / share, ctas - c + 1);  // (the bound: whatever lengths do meanwhile)
      const int slot = row / kTileRows, in_slot = row - slot * kTileRows, token = in_slot / p.group;
      const int t = t0 + slot * p.tpt + token;
      if (token >= p.tpt || t >= t1) continue;
      float r = -INFINITY, l = 0.f, o[4] = {0.f, 0.f, 0.f, 0.f};
      constexpr int kAtOnce = 8;
      for (int i0 = 0; i0 < parts; i0 += kAtOnce) {
        float2 ml[kAtOnce];
        float4 x[kAtOnce];
#pragma unroll
        for (int k2 = 0; k2 < kAtOnce; ++k2) {
          const int i = min(i0 + k2, parts - 1);
          ml[k2] = p.part_ml[((int64_t)(c - 1 + i) * 2 + (i == 0 ? 1 : 0)) * ROWS + row];
          x[k2] = p.part_o[part_at<D, ROWS>(c - 1 + i, i == 0, col4, row)];
        }
        float top = r;
#pragma unroll
        for (int k2 = 0; k2 < kAtOnce; ++k2) top = fmaxf(top, ml[k2].x);
        const float rr = top == -INFINITY ? 0.f : top, w0 = ex2_approx(r - rr);
        r = top;
        l *= w0;
#pragma unroll
        for (int v = 0; v < 4; ++v) o[v] *= w0;
#pragma unroll
        for (int k2 = 0; k2 < kAtOnce; ++k2) {
          if (i0 + k2 >= parts) break;
          const float w = ex2_approx(ml[k2].x - rr);
          l = fmaf(ml[k2].y, w, l);
          o[0] = fmaf(x[k2].x, w, o[0]);
          o[1] = fmaf(x[k2].y, w, o[1]);
          o[2] = fmaf(x[k2].z, w, o[2]);
          o[3] = fmaf(x[k2].w, w, o[3]);
        }
      }
      const float inv = l == 0.f ? 0.f : 1.f / l;
      const int head = kvh * p.group + in_slot - token * p.group;
      uint8_t* out = p.out.data + 2 * ((int64_t)b * p.out.batch_stride + (int64_t)t * p.out.token_stride + (int64_t)head * p.out.head_stride + col4 * 4);
      *reinterpret_cast<uint2*>(out) = make_uint2(cache::pack_bf16(o[0] * inv, o[1] * inv), cache::pack_bf16(o[2] * inv, o[3] * inv));
      if (p.lse && col4 == 0) p.lse[((int64_t)b * p.n + t) * p.heads + head] = l == 0.f ? -INFINITY : kLn2 * (r + log2f(l));
    }
    __syncthreads();
  }
}

}  // namespace attn
}  // namespace fly
