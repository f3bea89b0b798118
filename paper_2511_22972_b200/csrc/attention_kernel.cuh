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
// grid (one CTA per SM), so ragged batches and single long sequences fill the device alike, without the host knowing a length.  Where a
// cut goes through an item its parts are left in scratch as (O, r, l) and attention_combine_kernel adds them up, in a fixed order.
//
// Pages arrive by TMA, one box per page and 64 values, in a ring of stages that runs on across items.  Warps: 0-3 and 4-7 softmax of the
// two slots, 8 loads, 9 MMA issue; with E4M3 pages the boxes land in a ring of their own and warps 10.. turn them into bf16 tiles
// (exactly: a code times a power of two is a bf16 number).
//
// A value meets rows that must not see it with P = 0, and 0 * NaN is NaN.  In the tiles where some row is masked, values that no row of
// the item sees are therefore zeroed in shared memory, and infinities and NaN of those that only some rows see are zeroed and added back
// to the rows that do see them (add_back).
//
// Every wait is bounded: one that runs out records a code in *status, after which no wait waits, the rows of the step become NaN, and the
// CTA ends as usual.  No TMA load is a multicast load.
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

struct Params {
  cache::View c;
  cache::Rows out;
  float* lse;
  const int32_t* counts;
  int B, n, heads, group;  // group: query heads per key/value head
  int window, sinks;       // window 0: none
  float scale;             // log2(e) * the softmax's scale
  int tpt;                 // tokens per row tile
  int tpi;                 // tokens per item
  int rt;                  // items per sequence and key/value head
  int groups;              // B * rt
  int min_share;           // a CTA that gets work gets at least so many tiles
  int max_pages;
  float* part_o;           // [grid][2][rows of an item][D]
  float2* part_ml;         // [grid][2][rows of an item]: r, l
  int* desc;               // [grid][8]: how a CTA's range begins
  int* status;
};

// The rows t0 .. t1 - 1 of a sequence's chunk that make up an item, and the tiles of positions that they see: ns tiles from 0 on, then
// those from lo_tile on, `count` in all.
struct Group {
  int b, t0, t1, L;
  int lo_tile, ns, count;
  int hi;        // positions from here on are not seen
  int lo_last;   // first position in the window of the last row
};

__device__ __forceinline__ Group group_at(const Params& p, int g) {
  Group r;
  r.b = g / p.rt;
  r.t0 = (g - r.b * p.rt) * p.tpi;
  r.t1 = min(cache::count_of(p.counts, r.b, p.n), r.t0 + p.tpi);
  r.L = cache::length_of(p.c, r.b);
  r.lo_tile = r.ns = r.count = r.hi = r.lo_last = 0;
  if (r.t0 >= r.t1 || r.L < 0) return r;
  r.hi = min(r.L + r.t1, p.c.capacity);
  const int lo = p.window > 0 ? max(0, r.L + r.t0 + 1 - p.window) : 0;
  r.lo_last = p.window > 0 ? max(0, r.L + r.t1 - p.window) : 0;
  const int nt = (r.hi + kTile - 1) / kTile;
  r.lo_tile = lo / kTile;
  r.ns = min(min(r.lo_tile, nt), (min(p.sinks, lo) + kTile - 1) / kTile);
  r.count = r.ns + max(0, nt - r.lo_tile);
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
__device__ __forceinline__ void tc_fence_before() { asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void tc_fence_after() { asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void async_proxy_fence() { asm volatile("fence.proxy.async.shared::cta;" ::: "memory"); }
__device__ __forceinline__ bool elect_lane() {
  uint32_t one;
  asm volatile("{\n\t.reg .pred p;\n\telect.sync _|p, 0xffffffff;\n\tselp.u32 %0, 1, 0, p;\n\t}" : "=r"(one));
  return one != 0;
}
// D[tmem] (+)= A[smem] * B[smem], bf16, fp32 accumulate, M = 128.  Descriptors as (low word, high word).
__device__ __forceinline__ void mma_ss(uint32_t d, uint32_t a_lo, uint32_t b_lo, uint32_t hi, uint32_t idesc, uint32_t accumulate) {
  asm volatile(
      "{\n\t.reg .pred p;\n\t.reg .b64 da, db;\n\tsetp.ne.b32 p, %5, 0;\n\tmov.b64 da, {%1, %3};\n\tmov.b64 db, {%2, %3};\n\t"
      "tcgen05.mma.cta_group::1.kind::f16 [%0], da, db, %4, p;\n\t}" ::"r"(d), "r"(a_lo), "r"(b_lo), "r"(hi), "r"(idesc), "r"(accumulate)
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
#define FLY_I8(r, i) "r"(r[i]), "r"(r[i + 1]), "r"(r[i + 2]), "r"(r[i + 3]), "r"(r[i + 4]), "r"(r[i + 5]), "r"(r[i + 6]), "r"(r[i + 7])
// 32 lanes x 32 columns: thread = lane, register i = column i.  The registers are there when this returns.
__device__ __forceinline__ void tmem_ld32(uint32_t a, uint32_t (&r)[32]) {
  asm volatile(
      "tcgen05.ld.sync.aligned.32x32b.x32.b32 {%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,%16,%17,%18,%19,%20,%21,%22,%23,%24,%25,"
      "%26,%27,%28,%29,%30,%31}, [%32];\n\ttcgen05.wait::ld.sync.aligned;"
      : FLY_R8(r, 0), FLY_R8(r, 8), FLY_R8(r, 16), FLY_R8(r, 24)
      : "r"(a)
      : "memory");
}
__device__ __forceinline__ void tmem_st32(uint32_t a, const uint32_t (&r)[32]) {
  asm volatile(
      "tcgen05.st.sync.aligned.32x32b.x32.b32 [%0], {%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,%16,%17,%18,%19,%20,%21,%22,%23,%24,%25,"
      "%26,%27,%28,%29,%30,%31,%32};" ::"r"(a), FLY_I8(r, 0), FLY_I8(r, 8), FLY_I8(r, 16), FLY_I8(r, 24)
      : "memory");
}
__device__ __forceinline__ void tmem_st16(uint32_t a, const uint32_t (&r)[16]) {
  asm volatile("tcgen05.st.sync.aligned.32x32b.x16.b32 [%0], {%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,%16};" ::"r"(a), FLY_I8(r, 0),
               FLY_I8(r, 8)
               : "memory");
}
#undef FLY_R8
#undef FLY_I8
__device__ __forceinline__ void tmem_st_wait() { asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory"); }

// Shared-memory matrix descriptors: 128-byte swizzle, groups of 8 rows 1024 bytes apart.
__device__ __forceinline__ uint32_t desc_lo(uint32_t addr, uint32_t lbo_bytes) {
  return ((addr >> 4) & 0x3fffu) | (((lbo_bytes >> 4) & 0x3fffu) << 16);
}
constexpr uint32_t kDescHi = (1024u >> 4) | (1u << 14) | (2u << 29);
// fp32 accumulator, bf16 A and B, A K-major, M = 128.
__host__ __device__ constexpr uint32_t instr_desc(int n, bool b_mn_major) {
  return (1u << 4) | (1u << 7) | (1u << 10) | ((b_mn_major ? 1u : 0u) << 16) | ((uint32_t)(n >> 3) << 17) | ((uint32_t)(kTileRows >> 4) << 24);
}

// ---- shared memory -----------------------------------------------------------------------------------------------------

template <int D, bool E4M3, bool PAIR>
struct Shape {
  static constexpr int kHalves = D / 64;                    // of a row: 128 bytes each, a swizzle atom's width
  static constexpr int kHalfBytes = 128 * 128;              // 128 rows
  static constexpr int kTileBytes = kHalves * kHalfBytes;   // a tile of queries, keys or values in bf16
  static constexpr int kQBufs = PAIR || !E4M3 ? 2 : 1;      // (one row tile in two buffers: the next item's is loaded meanwhile)
  static constexpr int kRawTile = kTile * D;                // a tile of codes
  static constexpr int kRawBytes = kRawTile + kTile;        // ... and its scales
  static constexpr int kStages = E4M3 ? (D == 128 ? (PAIR ? 3 : 4) : 6) : (D == 128 ? 5 : 12);
  static constexpr int kRawStages = E4M3 ? (D == 128 ? 4 : 10) : 0;
  static constexpr int kOffRing = kQBufs * kTileBytes;
  static constexpr int kOffRaw = kOffRing + kStages * kTileBytes;
  static constexpr int kOffExchange = kOffRaw + kRawStages * kRawBytes;
  static constexpr int kOffBar = kOffExchange + 2 * kTileRows * 8;
  static constexpr int kNumBars = 2 * kStages + 2 * kRawStages + 4 + 6;
  static constexpr int kOffFlags = kOffBar + kNumBars * 8;
  static constexpr int kOffMisc = kOffFlags + 16 * 4;
  static constexpr int kSmem = kOffMisc + 64;
  static_assert(kSmem <= 232448, "shared memory of one CTA");
  static constexpr int kConvWarps = E4M3 ? 6 : 0;
  static constexpr int kThreads = (10 + kConvWarps) * 32;
  static constexpr int kItemRows = PAIR ? 2 * kTileRows : kTileRows;
};

constexpr int kWarpLoad = 8, kWarpMma = 9, kWarpConv = 10;

// A role's walk over the items of its CTA's range.
struct Walk {
  const Params& p;
  int g, kvh, x0, x1;
  int64_t left;
  Group gr;
  __device__ Walk(const Params& pp, int g0, int64_t off, int64_t tiles) : p(pp), g(g0), kvh(0), x0(0), x1(0), left(tiles) {
    if (left > 0) {
      gr = group_at(p, g);
      kvh = (int)(off / gr.count);
      x0 = (int)(off - (int64_t)kvh * gr.count);
      x1 = (int)min((int64_t)gr.count, x0 + left);
    }
  }
  __device__ bool have() const { return left > 0; }
  __device__ void next() {
    left -= x1 - x0;
    if (left <= 0) return;
    x0 = 0;
    if (++kvh == p.c.kv_heads) {
      kvh = 0;
      do gr = group_at(p, ++g);
      while (gr.count == 0);
    }
    x1 = (int)min((int64_t)gr.count, left);
  }
};

// Whether slot s of a pair sees anything of the tile at p0.
__device__ __forceinline__ bool slot_sees(const Params& p, const Group& g, int s, int p0) {
  const int ts0 = g.t0 + s * p.tpt, ts1 = min(g.t1, ts0 + p.tpt);
  if (ts0 >= ts1 || p0 >= g.L + ts1) return false;
  return p.window == 0 || p0 + kTile - 1 > g.L + ts0 - p.window || p0 < p.sinks;
}
// Places in the ring of an item's tiles: keys run ahead of values by as much as the MMAs do.
template <bool PAIR>
__device__ __forceinline__ int ring_k(int j) {
  return PAIR ? 2 * j : j == 0 ? 0 : 2 * j - 1;
}
template <bool PAIR>
__device__ __forceinline__ int ring_v(int j, int m) {
  return PAIR ? 2 * j + 1 : j == m - 1 ? 2 * m - 1 : 2 * j + 2;
}
// Whether a tile holds values that not every row of the item sees.
__device__ __forceinline__ bool edge_tile(const Params& p, const Group& g, int p0, uint32_t bad) {
  return p0 + kTile > min(g.L + g.t0 + 1, g.hi) || (p0 < g.lo_last && p0 + kTile > p.sinks) || bad != 0;
}
// ... of one position: 0 no row sees it, 1 some rows do, 2 all.
__device__ __forceinline__ int seen_by(const Params& p, const Group& g, int pos) {
  if (pos >= g.hi) return 0;
  const bool early = pos < p.sinks || p.window == 0;
  if (!early && pos <= g.L + g.t0 - p.window) return 0;
  return pos <= g.L + g.t0 && (early || pos >= g.lo_last) ? 2 : 1;
}
__device__ __forceinline__ uint32_t zero_nonfinite(uint32_t w, bool& any) {  // a pair of bf16
  if ((w & 0x7f80u) == 0x7f80u) { w &= 0xffff0000u; any = true; }
  if ((w & 0x7f800000u) == 0x7f800000u) { w &= 0xffffu; any = true; }
  return w;
}

// Visibility of a tile's positions to one row, relative to the tile: below lim, and from lo on or below snk, and on a page that exists.
struct RowMask {
  int lim, lo, snk;
  uint32_t bad;  // a bit per 8 positions
  __device__ __forceinline__ bool hides(int c) const { return c >= lim || (c < lo && c >= snk) || ((bad >> (c >> 3)) & 1u); }
};

// One step of a row: S in tensor memory at `ts` becomes P there, the row's reference and sum move on, and O at `to` is rescaled if it must be.
template <int D, bool MASK>
__device__ __forceinline__ void softmax_step(uint32_t ts, uint32_t to, float scale, bool first, const RowMask& mask, float& ref, float& sum) {
  float mx = -INFINITY;
  uint32_t r[32];
#pragma unroll
  for (int h = 0; h < 4; ++h) {
    tmem_ld32(ts + h * 32, r);
#pragma unroll
    for (int c = 0; c < 32; ++c) {
      if (MASK && mask.hides(h * 32 + c)) r[c] = 0xff800000u;
      mx = fmaxf(mx, __uint_as_float(r[c]));
    }
  }
  const float top = mx * scale;
  const bool move = top > ref + 8.0f;  // (false for a row that has seen nothing, and for NaN)
  if (__any_sync(0xffffffffu, move)) {
    const float alpha = move ? (ref == -INFINITY ? 0.f : ex2_approx(ref - top)) : 1.f;
    if (move) ref = top;
    sum *= alpha;
    if (!first) {
#pragma unroll
      for (int h = 0; h < D / 32; ++h) {
        tmem_ld32(to + h * 32, r);
#pragma unroll
        for (int c = 0; c < 32; ++c) r[c] = __float_as_uint(__uint_as_float(r[c]) * alpha);
        tmem_st32(to + h * 32, r);
      }
    }
  }
  const float nr = ref == -INFINITY ? 0.f : -ref;
  const f2 sc2 = pack2(scale, scale), nr2 = pack2(nr, nr);
  f2 acc = pack2(0.f, 0.f);
#pragma unroll
  for (int h = 0; h < 4; ++h) {
    tmem_ld32(ts + h * 32, r);
    uint32_t w[16];
#pragma unroll
    for (int c = 0; c < 32; c += 2) {
      float a = __uint_as_float(r[c]), b = __uint_as_float(r[c + 1]);
      if (MASK) {
        if (mask.hides(h * 32 + c)) a = -INFINITY;
        if (mask.hides(h * 32 + c + 1)) b = -INFINITY;
      }
      float x, y;
      unpack2(fma2(pack2(a, b), sc2, nr2), x, y);
      x = ex2_approx(x);
      y = ex2_approx(y);
      acc = add2(acc, pack2(x, y));
      w[c / 2] = cache::pack_bf16(x, y);
    }
    tmem_st16(ts + h * 16, w);  // over columns of S that have been read
  }
  float a, b;
  unpack2(acc, a, b);
  sum += a + b;
}

// Adds back to a row what zero_nonfinite took out of the values that it sees; columns col0 .. col0 + 31 of row_pos are in o.
template <bool E4M3>
__device__ __noinline__ void add_back(const Params& p, const Group& g, int kvh, int row_pos, int col0, float* o) {
  auto visit = [&](int from, int to) {
    for (int pos = from; pos < to; ++pos) {
      if (!visible(p, row_pos, pos)) continue;
      const int page = cache::page_of(p.c, g.b, pos);
      if (page < 0) continue;
      const int slot = pos & ((1 << p.c.page_shift) - 1);
      const int64_t at = cache::row_at(p.c, page, slot, kvh) + col0;
      const float scale = E4M3 ? cache::scale_value(p.c.v_scales[cache::scale_at(p.c, page, slot, kvh)]) : 1.f;
      for (int c = 0; c < 32; c += 2) {
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
  const int upper = min(g.L + g.t0 + 1, g.hi);                                // positions that only later rows see
  if (p.window > 0) visit(max(0, g.L + g.t0 + 1 - p.window), min(g.lo_last, upper));  // ... and that only earlier ones do
  visit(upper, g.hi);
}

template <int D, bool E4M3, bool PAIR>
__global__ void __launch_bounds__(Shape<D, E4M3, PAIR>::kThreads, 1)
attention_kernel(const __grid_constant__ CUtensorMap map_q, const __grid_constant__ CUtensorMap map_k, const __grid_constant__ CUtensorMap map_v,
                 const Params p) {
  using S = Shape<D, E4M3, PAIR>;
  extern __shared__ __align__(1024) uint8_t smem[];
  const uint32_t base = smem_u32(smem);
  const uint32_t bar0 = base + S::kOffBar;
  auto full = [&](int s) { return bar0 + 8u * s; };                       // a stage's tile is there, in bf16
  auto empty = [&](int s) { return bar0 + 8u * (S::kStages + s); };       // ... has been read by its MMAs
  auto raw_full = [&](int s) { return bar0 + 8u * (2 * S::kStages + s); };
  auto raw_empty = [&](int s) { return bar0 + 8u * (2 * S::kStages + S::kRawStages + s); };
  constexpr int kB = 2 * S::kStages + 2 * S::kRawStages;
  auto q_full = [&](int s) { return bar0 + 8u * (kB + s); };
  auto q_empty = [&](int s) { return bar0 + 8u * (kB + 2 + s); };
  auto s_full = [&](int s) { return bar0 + 8u * (kB + 4 + s); };          // S of a slot's step is complete (and every MMA before it)
  auto p_ready = [&](int s) { return bar0 + 8u * (kB + 6 + s); };         // its P is there, O rescaled, the values' tile cleaned
  auto o_full = [&](int s) { return bar0 + 8u * (kB + 8 + s); };          // the slot's O of an item is complete
  volatile uint32_t* misc = reinterpret_cast<volatile uint32_t*>(smem + S::kOffMisc);  // [0] tensor memory, [1] a role gave up, [2] an earlier step did, [4], [6..7] the range's begin, [8..15] items with values to add back
  volatile uint32_t* tile_bad = reinterpret_cast<volatile uint32_t*>(smem + S::kOffFlags);  // of tile number t: entry t % 16
  float2* exchange = reinterpret_cast<float2*>(smem + S::kOffExchange);

  const int tid = (int)threadIdx.x, lane = tid & 31, warp = __shfl_sync(0xffffffffu, tid >> 5, 0);
  if (tid == 0) {
    asm volatile("prefetch.tensormap [%0];" ::"l"(&map_q) : "memory");
    asm volatile("prefetch.tensormap [%0];" ::"l"(&map_k) : "memory");
    asm volatile("prefetch.tensormap [%0];" ::"l"(&map_v) : "memory");
    for (int s = 0; s < S::kStages; ++s) { mbar_init(full(s), E4M3 ? S::kConvWarps * 32 : 1); mbar_init(empty(s), 1); }
    for (int s = 0; s < S::kRawStages; ++s) { mbar_init(raw_full(s), 33); mbar_init(raw_empty(s), S::kConvWarps * 32); }
    for (int s = 0; s < 2; ++s) {
      mbar_init(q_full(s), 1);
      mbar_init(q_empty(s), 1);
      mbar_init(s_full(s), 1);
      mbar_init(p_ready(s), kTileRows);
      mbar_init(o_full(s), 1);
    }
    misc[1] = 0;
    for (int i = 8; i < 16; ++i) misc[i] = 0;
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  }
  if (warp == 0) {  // all of tensor memory: shared memory already keeps it to one CTA per SM
    asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], 512;" ::"r"(base + S::kOffMisc) : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
  }
  asm volatile("griddepcontrol.wait;" ::: "memory");  // everything below reads or writes what the kernels before may be working on
  asm volatile("griddepcontrol.launch_dependents;");

  // ---- this CTA's range of tiles: every thread counts a group's, a scan over the block adds them up ----
  int64_t* scan = reinterpret_cast<int64_t*>(smem + S::kOffExchange);  // [warps] sums, [32] base
  constexpr int kWarps = S::kThreads / 32;
  auto block_scan = [&](int64_t v, int64_t& before) {  // -> the block's sum; before: of the threads below
    int64_t x = v;
#pragma unroll
    for (int d = 1; d < 32; d <<= 1) {
      const int64_t y = __shfl_up_sync(0xffffffffu, x, d);
      if (lane >= d) x += y;
    }
    __syncthreads();
    if (lane == 31) scan[warp] = x;
    __syncthreads();
    int64_t sum = 0, mine = 0;
    for (int w = 0; w < kWarps; ++w) {
      const int64_t t = scan[w];
      if (w < warp) mine += t;
      sum += t;
    }
    before = mine + x - v;
    return sum;
  };
  if (tid == 0) misc[2] = *reinterpret_cast<volatile uint32_t*>(p.status);  // (one thread: the warps' decisions have to be alike)
  int64_t total = 0;
  for (int g0 = 0; g0 < p.groups; g0 += S::kThreads) {
    const int g = g0 + tid;
    Group gr;
    gr.count = 0;
    if (g < p.groups) {
      gr = group_at(p, g);
      if (gr.count == 0 && gr.t0 < gr.t1 && (unsigned)g % gridDim.x == blockIdx.x) {  // rows of a sequence that has no positions
        for (int t = gr.t0; t < gr.t1; ++t)
          for (int h = 0; h < p.heads; ++h) {
            uint4* o = reinterpret_cast<uint4*>(p.out.data + 2 * ((int64_t)gr.b * p.out.batch_stride + (int64_t)t * p.out.token_stride + (int64_t)h * p.out.head_stride));
            for (int i = 0; i < D / 8; ++i) o[i] = make_uint4(0u, 0u, 0u, 0u);
            if (p.lse) p.lse[((int64_t)gr.b * p.n + t) * p.heads + h] = -INFINITY;
          }
      }
    }
    int64_t before;
    total += block_scan((int64_t)gr.count * p.c.kv_heads, before);
  }
  int64_t share = (total + gridDim.x - 1) / gridDim.x;
  if (share < p.min_share) share = p.min_share;
  const int64_t first = share * blockIdx.x, tiles = first < total ? min(share, total - first) : 0;
  if (tiles > 0) {
    int64_t run = 0;
    for (int g0 = 0; g0 < p.groups; g0 += S::kThreads) {
      const int g = g0 + tid;
      const int64_t v = g < p.groups ? (int64_t)group_at(p, g).count * p.c.kv_heads : 0;
      int64_t before;
      const int64_t sum = block_scan(v, before);
      before += run;
      if (first >= before && first < before + v) {
        misc[4] = (uint32_t)g;
        *reinterpret_cast<volatile int64_t*>(smem + S::kOffMisc + 24) = first - before;
      }
      run += sum;
      if (run > first) break;  // (the same for all)
    }
  }
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem = misc[0];
  const int g_first = (int)misc[4];
  const int64_t off_first = *reinterpret_cast<volatile int64_t*>(smem + S::kOffMisc + 24);
  Walk walk(p, g_first, off_first, tiles);
  if (tid == 0) {
    int* d = p.desc + 8 * blockIdx.x;
    if (tiles > 0) {
      d[0] = walk.g;
      d[2] = walk.kvh;
      d[3] = walk.x0;
      d[4] = walk.gr.count;
    } else {
      d[3] = 0;
    }
    d[5] = (int)min(share, (int64_t)0x7fffffff);
  }

  // A wait has run out, or had in a step before and nobody has looked: no wait waits any more, and nothing is issued.
  bool failed = misc[2] != 0;
  auto wait = [&](uint32_t bar, uint32_t parity) {
    if (!failed && !mbar_wait(bar, parity, p.status, kErrAttention)) failed = true;
    __syncwarp();
  };
  auto wait_warp = [&](uint32_t bar, uint32_t parity) {  // the same decision in the whole warp
    if (!failed && !__all_sync(0xffffffffu, mbar_wait(bar, parity, p.status, kErrAttention))) failed = true;
  };
  uint32_t ring = 0;  // tiles of keys and values that went through the ring before this item
  uint32_t tile_no = 0;  // tiles of positions before this item

  if (warp == kWarpLoad) {
    // ---------------- loads ----------------
    const int page_size = 1 << p.c.page_shift, rows = min(page_size, kTile), parts = kTile / rows;
    const uint32_t box_bytes = (uint32_t)rows * D * (E4M3 ? 1 : 2);
    const uint32_t q_bytes = (uint32_t)(p.tpt * p.group * D * 2);
    uint32_t item = 0;
    for (; walk.have(); walk.next(), ++item) {
      const Group g = walk.gr;
      const int m = walk.x1 - walk.x0;
      // the item's queries
      const int bufs = PAIR ? 2 : 1;
      for (int s = 0; s < bufs; ++s) {
        const int buf = PAIR ? s : (int)(item % S::kQBufs);
        const uint32_t use = PAIR ? item : item / S::kQBufs;
        wait_warp(q_empty(buf), (use & 1) ^ 1);
        if (!failed && elect_lane()) {
          mbar_expect_tx(q_full(buf), q_bytes);
          for (int h = 0; h < S::kHalves; ++h)
            tma_load_4d(base + buf * S::kTileBytes + h * S::kHalfBytes, &map_q, h * 64, walk.kvh * p.group, g.t0 + s * p.tpt, g.b, q_full(buf));
        }
        __syncwarp();
      }
      // its tiles of positions; a lane per page of a tile
      auto page_for = [&](int j) {
        const int pos = tile_start(g, walk.x0 + j) + lane * rows;
        return lane < parts && pos < g.hi ? cache::page_of(p.c, g.b, pos) : -2;
      };
      auto load = [&](int place, bool values, int j, int page) {
        const uint32_t idx = ring + (uint32_t)place;
        const int p0 = tile_start(g, walk.x0 + j), slot = p0 & (page_size - 1) & ~(rows - 1);
        const unsigned have = __ballot_sync(0xffffffffu, page >= 0);
        if (E4M3) {
          const int st = (int)(idx % (uint32_t)max(1, S::kRawStages));
          wait_warp(raw_empty(st), ((idx / (uint32_t)max(1, S::kRawStages)) & 1) ^ 1);
          if (failed) return;
          const uint32_t dst = base + S::kOffRaw + st * S::kRawBytes;
          if (lane == 0) mbar_expect_tx(raw_full(st), (uint32_t)__popc(have) * box_bytes);
          __syncwarp();
          if (page >= 0) tma_load_4d(dst + lane * rows * D, values ? &map_v : &map_k, 0, slot, walk.kvh, page, raw_full(st));
          // eight scales a lane, in the same phase of the barrier
          const int at = (lane & 15) * 8, src_page = __shfl_sync(0xffffffffu, page, at / rows);
          if (lane < 16 && src_page >= 0) {
            const uint8_t* s = (values ? p.c.v_scales : p.c.k_scales) + cache::scale_at(p.c, src_page, slot + at % rows, walk.kvh);
            asm volatile("cp.async.ca.shared.global [%0], [%1], 8;" ::"r"(dst + S::kRawTile + at), "l"(s) : "memory");
          }
          asm volatile("cp.async.mbarrier.arrive.noinc.shared::cta.b64 [%0];" ::"r"(raw_full(st)) : "memory");
        } else {
          const int st = (int)(idx % S::kStages);
          wait_warp(empty(st), ((idx / S::kStages) & 1) ^ 1);
          if (failed) return;
          if (lane == 0) mbar_expect_tx(full(st), (uint32_t)__popc(have) * box_bytes);
          __syncwarp();
          if (page >= 0)
            for (int h = 0; h < S::kHalves; ++h)
              tma_load_4d(base + S::kOffRing + st * S::kTileBytes + h * S::kHalfBytes + lane * rows * 128, values ? &map_v : &map_k, h * 64, slot,
                          walk.kvh, page, full(st));
        }
      };
      int page = page_for(0), page_v = page;
      for (int j = 0; j <= m; ++j) {  // K(0) [V(0)] K(1) V(0 or 1) ...
        int ahead = -2;
        if (j < m) {
          if (j + 1 < m) ahead = page_for(j + 1);
          uint32_t bad = page == -1 ? ((1u << (rows / 8)) - 1u) << (lane * rows / 8) : 0u;
          bad = __reduce_or_sync(0xffffffffu, bad);
          if (lane == 0) tile_bad[(tile_no + (uint32_t)j) & 15] = bad;
          __syncwarp();
          load(ring_k<PAIR>(j), false, j, page);
        }
        if (PAIR ? j < m : j > 0) {
          const int jv = PAIR ? j : j - 1;
          load(ring_v<PAIR>(jv, m), true, jv, PAIR ? page : page_v);
        }
        page_v = page;
        page = ahead;
      }
      ring += 2u * m;
      tile_no += m;
    }
  } else if (warp == kWarpMma) {
    // ---------------- MMA issue ----------------
    const bool lead = elect_lane();
    constexpr uint32_t kIdescS = instr_desc(kTile, false), kIdescO = instr_desc(D, true);
    uint32_t item = 0, use0 = 0, use1 = 0;  // steps of each slot so far
    for (; walk.have(); walk.next(), ++item) {
      const Group g = walk.gr;
      const int m = walk.x1 - walk.x0;
      auto sees = [&](int s, int j) { return !PAIR || slot_sees(p, g, s, tile_start(g, walk.x0 + j)); };
      auto issue_s = [&](int s, int j) {  // S of slot s = Q x keys of tile j
        const uint32_t st = (ring + (uint32_t)ring_k<PAIR>(j)) % S::kStages;
        const int buf = PAIR ? s : (int)(item % S::kQBufs);
        if (!failed && lead) {
          const uint32_t a = desc_lo(base + buf * S::kTileBytes, 16), b = desc_lo(base + S::kOffRing + st * S::kTileBytes, 16);
#pragma unroll
          for (int k = 0; k < D / 16; ++k) {
            const uint32_t o = (uint32_t)((k / 4) * S::kHalfBytes + (k % 4) * 32) >> 4;
            mma_ss(tmem + s * kTile, a + o, b + o, kDescHi, kIdescS, k != 0);
          }
          mma_commit(s_full(s));
        }
        __syncwarp();
      };
      auto issue_o = [&](int s, int j, bool accumulate) {  // O of slot s += P x values of tile j
        uint32_t& use = s ? use1 : use0;
        wait_warp(p_ready(s), use & 1);
        ++use;
        const uint32_t st = (ring + (uint32_t)ring_v<PAIR>(j, m)) % S::kStages;
        tc_fence_after();
        if (!failed && lead) {
          const uint32_t b = desc_lo(base + S::kOffRing + st * S::kTileBytes, S::kHalfBytes);
#pragma unroll
          for (int k = 0; k < kTile / 16; ++k)
            mma_ts(tmem + 2 * kTile + s * 128, tmem + s * kTile + k * 8, b + ((k * 16 * 128) >> 4), kDescHi, kIdescO, accumulate || k != 0);
        }
        __syncwarp();
      };
      auto wait_tile = [&](int place) {
        const uint32_t idx = ring + (uint32_t)place;
        wait_warp(full((int)(idx % S::kStages)), (idx / S::kStages) & 1);
        tc_fence_after();
      };
      auto commit = [&](uint32_t bar) {
        if (!failed && lead) mma_commit(bar);
        __syncwarp();
      };
      auto release = [&](int place) { commit(empty((int)((ring + (uint32_t)place) % S::kStages))); };
      if (PAIR) {
        wait_warp(q_full(0), item & 1);
        wait_warp(q_full(1), item & 1);
        int last[2] = {-1, -1};
        for (int s = 0; s < 2; ++s)  // (a few tiles from the end, unless the slot has no token)
          if (g.t0 + s * p.tpt < g.t1)
            for (last[s] = m - 1; last[s] >= 0 && !sees(s, last[s]); --last[s]) {}
        bool begun[2] = {false, false};
        wait_tile(ring_k<PAIR>(0));
        for (int s = 0; s < 2; ++s)
          if (sees(s, 0)) issue_s(s, 0);
        release(ring_k<PAIR>(0));
        for (int j = 0; j < m; ++j) {
          wait_tile(ring_v<PAIR>(j, m));
          for (int s = 0; s < 2; ++s) {
            if (sees(s, j)) {
              issue_o(s, j, begun[s]);
              begun[s] = true;
              if (j == last[s]) commit(o_full(s));
            }
            if (j + 1 < m) {
              if (s == 0) wait_tile(ring_k<PAIR>(j + 1));
              if (sees(s, j + 1)) issue_s(s, j + 1);
            }
          }
          release(ring_v<PAIR>(j, m));
          if (j + 1 < m) release(ring_k<PAIR>(j + 1));
        }
        commit(q_empty(0));
        commit(q_empty(1));
      } else {
        const int buf = (int)(item % S::kQBufs);
        wait_warp(q_full(buf), (item / S::kQBufs) & 1);
        auto scores = [&](int j) {
          wait_tile(ring_k<PAIR>(j));
          issue_s(j & 1, j);
          release(ring_k<PAIR>(j));
          if (j == m - 1) commit(q_empty(buf));
        };
        scores(0);
        if (m > 1) scores(1);
        for (int j = 0; j < m; ++j) {
          wait_tile(ring_v<PAIR>(j, m));
          issue_o(j & 1, j, j >= 2);
          release(ring_v<PAIR>(j, m));
          if (j + 2 >= m) commit(o_full(j & 1));
          if (j + 2 < m) scores(j + 2);
        }
      }
      ring += 2u * m;
    }
    if (failed && lead) {  // what has been issued ends before shared and tensor memory are given back
      mma_commit(q_full(0));
      const unsigned long long t0 = global_ns();
      while (global_ns() - t0 < 2000000ull) {}
    }
    __syncwarp();
  } else if (E4M3 && warp >= kWarpConv) {
    // ---------------- codes to bf16 tiles ----------------
    const int ct = tid - kWarpConv * 32;
    uint32_t item = 0;
    for (; walk.have(); walk.next(), ++item) {
      const Group g = walk.gr;
      const int m = walk.x1 - walk.x0;
      auto convert = [&](int place, bool values, int j) {
        const uint32_t idx = ring + (uint32_t)place;
        const int rs = (int)(idx % (uint32_t)max(1, S::kRawStages)), st = (int)(idx % S::kStages);
        wait(raw_full(rs), (idx / (uint32_t)max(1, S::kRawStages)) & 1);
        wait(empty(st), ((idx / S::kStages) & 1) ^ 1);
        const uint8_t* raw = smem + S::kOffRaw + rs * S::kRawBytes;
        uint8_t* dst = smem + S::kOffRing + st * S::kTileBytes;
        const int p0 = tile_start(g, walk.x0 + j);
        const uint32_t bad = tile_bad[(tile_no + (uint32_t)j) & 15];
        const bool edge = values && edge_tile(p, g, p0, bad);
        bool any = false;
        // 16 codes at a time; eight neighbouring threads take four chunks of two rows, whose places in the swizzled tile share no bank
        constexpr int kChunks = kTile * D / 16, kPer = D / 16;
#pragma unroll 2
        for (int u = ct; u < kChunks; u += S::kConvWarps * 32) {
          const int quad = u & 3, odd = (u >> 2) & 1, rest = u >> 3;         // rest: (row pair, half)
          const int half = rest % (kPer / 4), row = (rest / (kPer / 4)) * 2 + odd, chunk = half * 4 + quad;
          const uint4 codes = *reinterpret_cast<const uint4*>(raw + row * D + chunk * 16);
          const float scale = cache::scale_value(raw[S::kRawTile + row]);
          uint2 a = cache::values_e4m3(codes.x, scale), b = cache::values_e4m3(codes.y, scale), c = cache::values_e4m3(codes.z, scale),
                d = cache::values_e4m3(codes.w, scale);
          if (edge) {
            const int seen = (bad >> (row >> 3)) & 1u ? 0 : seen_by(p, g, p0 + row);
            uint32_t w[8] = {a.x, a.y, b.x, b.y, c.x, c.y, d.x, d.y};
#pragma unroll
            for (int i = 0; i < 8; ++i) w[i] = seen == 0 ? 0u : seen == 1 ? zero_nonfinite(w[i], any) : w[i];
            a = make_uint2(w[0], w[1]); b = make_uint2(w[2], w[3]); c = make_uint2(w[4], w[5]); d = make_uint2(w[6], w[7]);
          }
          uint8_t* line = dst + half * S::kHalfBytes + row * 128;
          const int at = quad * 2;
          *reinterpret_cast<uint4*>(line + ((at ^ (row & 7)) << 4)) = make_uint4(a.x, a.y, b.x, b.y);
          *reinterpret_cast<uint4*>(line + (((at + 1) ^ (row & 7)) << 4)) = make_uint4(c.x, c.y, d.x, d.y);
        }
        if (any) misc[8 + (item & 7)] = item + 1;
        async_proxy_fence();
        mbar_arrive(full(st));
        mbar_arrive(raw_empty(rs));
      };
      for (int j = 0; j <= m; ++j) {
        if (j < m) convert(ring_k<PAIR>(j), false, j);
        if (PAIR ? j < m : j > 0) convert(ring_v<PAIR>(PAIR ? j : j - 1, m), true, PAIR ? j : j - 1);
      }
      ring += 2u * m;
      tile_no += m;
    }
  } else {
    // ---------------- softmax of a slot, a thread per row ----------------
    const int slot = warp >> 2, row = tid & 127, quarter = warp & 3;
    const uint32_t lanes = (uint32_t)(quarter * 32) << 16;
    const uint32_t ts = tmem + lanes + slot * kTile, to = tmem + lanes + 2 * kTile + slot * 128;
    const int row_token = row / p.group, row_head = row - row_token * p.group;
    uint32_t use = 0, items_done = 0, item = 0;
    for (; walk.have(); walk.next(), ++item) {
      const Group g = walk.gr;
      const int m = walk.x1 - walk.x0;
      const int ts0 = g.t0 + (PAIR ? slot * p.tpt : 0), ts1 = min(g.t1, ts0 + p.tpt);  // the slot's tokens
      const int t = ts0 + row_token, row_pos = g.L + t;
      const bool live = row_token < p.tpt && t < ts1;
      const bool warp_live = __any_sync(0xffffffffu, live);
      float ref = -INFINITY, sum = 0.f;
      bool begun = false;
      for (int j = PAIR ? 0 : slot; j < m; j += PAIR ? 1 : 2) {
        const int p0 = tile_start(g, walk.x0 + j);
        if (PAIR && !slot_sees(p, g, slot, p0)) continue;
        wait(s_full(slot), use & 1);
        ++use;
        const uint32_t bad = tile_bad[(tile_no + (uint32_t)j) & 15];
        if (!E4M3 && edge_tile(p, g, p0, bad) && (!PAIR || slot == 0 || !slot_sees(p, g, 0, p0))) {
          // a thread per position: the values' tile before its MMAs (those of both slots come after this slot's p_ready)
          const uint32_t idx = ring + (uint32_t)ring_v<PAIR>(j, m);
          const int st = (int)(idx % S::kStages);
          wait(full(st), (idx / S::kStages) & 1);
          const int seen = (bad >> (row >> 3)) & 1u ? 0 : seen_by(p, g, p0 + row);
          if (seen < 2) {
            bool any = false;
            for (int i = 0; i < S::kHalves * 8; ++i) {
              uint4* at = reinterpret_cast<uint4*>(smem + S::kOffRing + st * S::kTileBytes + (i >> 3) * S::kHalfBytes + row * 128 + (((i + row) & 7) << 4));
              uint4 v = make_uint4(0u, 0u, 0u, 0u);
              if (seen == 1) {
                v = *at;
                v.x = zero_nonfinite(v.x, any);
                v.y = zero_nonfinite(v.y, any);
                v.z = zero_nonfinite(v.z, any);
                v.w = zero_nonfinite(v.w, any);
              }
              *at = v;
            }
            if (any) misc[8 + (item & 7)] = item + 1;
            async_proxy_fence();
          }
          __syncwarp();
        }
        if (warp_live) {
          tc_fence_after();
          const int first_hi = min(g.L + ts0 + 1, g.hi), last_lo = p.window > 0 ? g.L + ts1 - p.window : 0;
          RowMask mask;
          mask.lim = min(row_pos + 1, g.hi) - p0;
          mask.lo = p.window > 0 ? row_pos + 1 - p.window - p0 : 0;
          mask.snk = p.sinks - p0;
          mask.bad = bad;
          if (p0 + kTile > first_hi || (p0 < last_lo && p0 + kTile > p.sinks) || bad != 0)
            softmax_step<D, true>(ts, to, p.scale, !begun, mask, ref, sum);
          else
            softmax_step<D, false>(ts, to, p.scale, !begun, mask, ref, sum);
          tmem_st_wait();
          tc_fence_before();
        }
        begun = true;
        mbar_arrive(p_ready(slot));
      }
      // ---- the item's end ----
      if (begun) {
        wait(o_full(slot), items_done & 1);
        ++items_done;
        tc_fence_after();
      }
      const bool from_start = walk.x0 == 0, whole = from_start && walk.x1 == g.count;
      float w0 = 1.f, w1 = 0.f, r = ref, l = sum;
      bool use0 = PAIR ? begun : true, use1 = false;
      if (!PAIR) {
        exchange[slot * kTileRows + row] = make_float2(ref, sum);
        asm volatile("bar.sync 1, 256;" ::: "memory");  // both slots' O are complete as well
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
      if (warp_live) {
        const float inv = failed ? __uint_as_float(0x7fc00000u) : whole ? (l == 0.f ? 0.f : 1.f / l) : 1.f;
        const int head = walk.kvh * p.group + row_head;
        uint8_t* out = p.out.data + 2 * ((int64_t)g.b * p.out.batch_stride + (int64_t)t * p.out.token_stride + (int64_t)head * p.out.head_stride);
        const int64_t part = ((int64_t)blockIdx.x * 2 + (from_start ? 1 : 0)) * S::kItemRows + (PAIR ? slot * kTileRows : 0) + row;
        const int h0 = PAIR ? 0 : slot * (D / 64), h1 = PAIR ? D / 32 : h0 + D / 64;  // the slots of one row tile share its columns
        for (int h = h0; h < h1; ++h) {
          uint32_t x[32];
          float o[32];
          if (use0) {
            tmem_ld32(tmem + lanes + 2 * kTile + (PAIR ? slot * 128 : 0) + h * 32, x);
#pragma unroll
            for (int c = 0; c < 32; ++c) o[c] = __uint_as_float(x[c]) * w0;
          } else {
#pragma unroll
            for (int c = 0; c < 32; ++c) o[c] = 0.f;
          }
          if (use1) {
            tmem_ld32(tmem + lanes + 2 * kTile + 128 + h * 32, x);
#pragma unroll
            for (int c = 0; c < 32; ++c) o[c] = fmaf(__uint_as_float(x[c]), w1, o[c]);
          }
          if (poison && live) {
            float y[32];
            for (int c = 0; c < 32; ++c) y[c] = o[c];
            add_back<E4M3>(p, g, walk.kvh, row_pos, h * 32, y);
            for (int c = 0; c < 32; ++c) o[c] = y[c];
          }
          if (live) {
            if (whole) {
#pragma unroll
              for (int c = 0; c < 32; c += 8)
                *reinterpret_cast<uint4*>(out + 2 * (h * 32 + c)) =
                    make_uint4(cache::pack_bf16(o[c] * inv, o[c + 1] * inv), cache::pack_bf16(o[c + 2] * inv, o[c + 3] * inv),
                               cache::pack_bf16(o[c + 4] * inv, o[c + 5] * inv), cache::pack_bf16(o[c + 6] * inv, o[c + 7] * inv));
            } else {
              float4* dst = reinterpret_cast<float4*>(p.part_o + part * D + h * 32);
#pragma unroll
              for (int c = 0; c < 32; c += 4) dst[c / 4] = make_float4(o[c] * inv, o[c + 1] * inv, o[c + 2] * inv, o[c + 3] * inv);
            }
          }
          __syncwarp();
        }
        if (live && (PAIR || slot == 0)) {
          if (!whole)
            p.part_ml[part] = make_float2(r, l * inv);
          else if (p.lse)
            p.lse[((int64_t)g.b * p.n + t) * p.heads + head] = failed ? inv : l == 0.f ? -INFINITY : kLn2 * (r + log2f(l));
        }
        tc_fence_before();
      }
      if (!PAIR) asm volatile("bar.sync 1, 256;" ::: "memory");  // neither slot's O is overwritten before both have read it
      ring += 2u * m;
      tile_no += m;
    }
  }

  if (failed) misc[1] = 1;
  tc_fence_before();
  __syncthreads();
  if (misc[1] != 0) {  // stragglers among the TMA loads
    const unsigned long long t0 = global_ns();
    while (global_ns() - t0 < 2000000ull) {}
  }
  __syncthreads();
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

// Adds up the parts of the items that were cut: block c takes the item that CTA c of the main kernel went on with, if CTA c - 1 began it.
//   r = max r_i,  l = sum 2^(r_i - r) l_i,  out = sum 2^(r_i - r) O_i / l
constexpr int kCombineThreads = 256;
template <int D>
__global__ void __launch_bounds__(kCombineThreads) attention_combine_kernel(const Params p, int item_rows) {
  asm volatile("griddepcontrol.wait;" ::: "memory");
  asm volatile("griddepcontrol.launch_dependents;");
  constexpr int kVals = D / 32;
  const int c = (int)blockIdx.x + 1;
  const int* d = p.desc + 8 * c;
  const int x0 = d[3], share = d[5];
  if (x0 <= 0 || x0 > share) return;
  const Group g = group_at(p, d[0]);
  const int kvh = d[2], count = d[4], parts = 1 + (count - x0 + share - 1) / share;
  const int lane = (int)threadIdx.x & 31;
  for (int row = (int)blockIdx.y * (kCombineThreads / 32) + ((int)threadIdx.x >> 5); row < item_rows; row += (int)gridDim.y * (kCombineThreads / 32)) {
    const int slot = row / kTileRows, in_slot = row - slot * kTileRows, token = in_slot / p.group;
    const int t = g.t0 + slot * p.tpt + token;
    if (token >= p.tpt || t >= g.t1) continue;
    auto part_at = [&](int i) { return ((int64_t)(c - 1 + i) * 2 + (i == 0 ? 1 : 0)) * item_rows + row; };
    float r = -INFINITY;
    for (int i = lane; i < parts; i += 32) r = fmaxf(r, p.part_ml[part_at(i)].x);
#pragma unroll
    for (int s = 16; s > 0; s >>= 1) r = fmaxf(r, __shfl_xor_sync(0xffffffffu, r, s));
    const float rr = r == -INFINITY ? 0.f : r;
    float l = 0.f, o[kVals];
#pragma unroll
    for (int v = 0; v < kVals; ++v) o[v] = 0.f;
    for (int i = 0; i < parts; ++i) {
      const int64_t at = part_at(i);
      const float2 ml = p.part_ml[at];
      const float w = ex2_approx(ml.x - rr);
      l = fmaf(ml.y, w, l);
      const float* src = p.part_o + at * D + lane * kVals;
      if (kVals == 4) {
        const float4 x = *reinterpret_cast<const float4*>(src);
        o[0] = fmaf(x.x, w, o[0]);
        o[1] = fmaf(x.y, w, o[1]);
        o[kVals - 2] = fmaf(x.z, w, o[kVals - 2]);
        o[kVals - 1] = fmaf(x.w, w, o[kVals - 1]);
      } else {
        const float2 x = *reinterpret_cast<const float2*>(src);
        o[0] = fmaf(x.x, w, o[0]);
        o[1] = fmaf(x.y, w, o[1]);
      }
    }
    const float inv = l == 0.f ? 0.f : 1.f / l;
    const int head = kvh * p.group + in_slot - token * p.group;
    uint8_t* out = p.out.data + 2 * ((int64_t)g.b * p.out.batch_stride + (int64_t)t * p.out.token_stride + (int64_t)head * p.out.head_stride + lane * kVals);
#pragma unroll
    for (int v = 0; v < kVals; v += 2) *reinterpret_cast<uint32_t*>(out + 2 * v) = cache::pack_bf16(o[v] * inv, o[v + 1] * inv);
    if (p.lse && lane == 0) p.lse[((int64_t)g.b * p.n + t) * p.heads + head] = l == 0.f ? -INFINITY : kLn2 * (r + log2f(l));
  }
}

}  // namespace attn
}  // namespace fly
