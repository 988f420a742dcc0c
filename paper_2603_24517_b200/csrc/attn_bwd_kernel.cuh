// Attention backward for sm_100a.  With S = scale Q K^T, P = exp(S - LSE) (0 where masked) and
// delta_i = sum_d dO_id O_id - dLSE_i, the gradients are
//
//     dV = P^T dO,   dP = dO V^T,   dS = P o (dP - delta),   dQ = scale dS K,   dK = scale dS^T Q.
//
// P is recomputed from Q, K and LSE tile by tile.  Two kinds of CTAs in one launch, so that every sum
// has one owner and a fixed order (no atomics, the same bits on every run):
//
//   key CTAs    one 128-key tile of one KV head: K and V stay in shared memory, the query tiles (Q, dO) of
//               every query head that shares the KV head stream past, dK and dV accumulate in tensor memory
//               (products per tile pair: K Q^T, V dO^T, P^T dO, dS^T Q);
//   query CTAs  one 128-row query tile of one head: Q and dO stay, the K / V tiles stream past, dQ accumulates
//               in tensor memory (products per tile pair: Q K^T, dO V^T, dS K).
//
// That is seven products where five would do if dQ were added up across CTAs, but those additions would
// either come in any order or wait for one another.  Each CTA (576 threads, one per SM):
//
//   warps 0-15  softmax: lane quarter w % 4 of the tile, 32 of its 128 columns (w / 4); a thread per row and quarter
//   warp  16    MMA issue (tcgen05.mma by an elected lane)
//   warps 17-18 loaders (TMA), one for each of the two streams: a ring of three 32 KB tiles for the one whose tiles
//               are read by the first and the last product of a pair (Q or K), of two for the other (dO or V)
//
// Transposed tiles in key CTAs (rows are keys) let P^T and dS^T go back to tensor memory as the left
// operand of the second products, so nothing is transposed through shared memory.
#pragma once

#include "attn_fwd_kernel.cuh"

namespace attn {
namespace bwd {

constexpr int kParts = 4;                 // softmax threads per row
constexpr int kCols = kTile / kParts;     // columns of a tile each of them handles
constexpr int kSoftmaxWarps = 4 * kParts;
constexpr int kBwdThreads = (kSoftmaxWarps + 3) * 32;
constexpr int kRingA = 3, kRingB = 2;     // slots of the two streams: Q and dO, or K and V
constexpr int kRingSlots = kRingA + kRingB;
constexpr int kStatStages = 2;
constexpr int kStatBytes = kTile * 4;  // one fp32 value per query row of a tile

constexpr int kSmemFixed = 0;  // two resident tiles
constexpr int kSmemRing = 2 * kTileBytes;
constexpr int kSmemStat = kSmemRing + kRingSlots * kTileBytes;  // [kStatStages][2][128]: -LSE log2(e), -delta
constexpr int kSmemBwdBars = kSmemStat + kStatStages * 2 * kStatBytes;
constexpr int kBwdBars = 1 + 2 * kRingSlots + 2 * kStatStages + 2 + 1 + 1 + 2 + 4 + 1 + 2;
constexpr int kSmemBwdMisc = kSmemBwdBars + kBwdBars * 8;  // tensor memory base, abort flag
constexpr int kSmemBwdBytes = kSmemBwdMisc + 8;
static_assert(kSmemBwdBytes <= 232448, "shared memory budget of one CTA");

struct BwdParams {
  int B, Hq, Hkv, Sq, Sk;
  int group;              // Hq / Hkv
  int causal;
  int off;                // Sk - Sq: key j is visible to row i iff j <= i + off
  int n_qt, n_kt;         // 128-row query tiles, 128-key tiles
  int n_key_items;        // CTAs [0, n_key_items) are key CTAs, the rest query CTAs
  float scale, scale_log2;
  const float* neg_lse2;  // [B * Hq][n_qt * 128], -LSE * log2(e); -inf in rows that see no key or do not exist
  const float* neg_delta; // same layout, -delta, 0 in those rows
  int* status;
};

// codes of expired waits: role << 8 | barrier (roles continue the forward kernels' numbering)
enum : int {
  kRoleBwdLoad = 10 << 8, kRoleBwdMma = 11 << 8, kRoleBwdSoftmax = 12 << 8,
  kBarFixed = 1, kBarRingFull = 2, kBarRingEmpty = 3, kBarStat = 4, kBarStatEmpty = 5, kBarS = 6, kBarDp = 7,
  kBarDpRead = 8, kBarP = 9, kBarDs = 10, kBarAcc = 11, kBarStage = 12
};

struct BwdBarriers {
  uint64_t* fixed_full;  // loader (TMA) -> MMA
  uint64_t* a_full;      // [kRingA]  loader (TMA) -> MMA
  uint64_t* a_empty;     // [kRingA]  MMA commit -> loader
  uint64_t* b_full;      // [kRingB]
  uint64_t* b_empty;     // [kRingB]
  uint64_t* stat_full;   // [kStatStages]  loader (bulk copy) -> softmax (key CTAs)
  uint64_t* stat_empty;  // [kStatStages]  softmax (all warps) -> loader
  uint64_t* s_full;      // [2]  MMA commit -> softmax (key CTAs use the first)
  uint64_t* dp_full;     // MMA commit -> softmax
  uint64_t* dp_read;     // softmax (all warps) -> MMA: dP is in registers (query CTAs)
  uint64_t* p_full;      // [2]  softmax warps of a half tile: its 64 columns of P are in tensor memory (key CTAs)
  uint64_t* ds_full;     // [4]  the same for dS; query CTAs alternate two pairs, one for each score buffer
  uint64_t* acc_full;    // MMA commit: the accumulators are final
  uint64_t* stage_full;  // [2]  softmax warps of a half tile: its staging area is written
};

// Untiled copy of `bytes` (a multiple of 16) from global to shared memory, counted on `bar`.
__device__ __forceinline__ void bulk_load(void* smem_dst, const void* src, uint32_t bytes, uint64_t* bar) {
  asm volatile("cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];" ::"r"(
                   smem_u32(smem_dst)),
               "l"(reinterpret_cast<uint64_t>(src)), "r"(bytes), "r"(smem_u32(bar))
               : "memory");
}

// A CTA's item: which tile it owns and which tiles stream past it.
struct BwdItem {
  int b, h;     // batch entry; KV head (key CTA) or query head (query CTA)
  int row0;     // first key / query row of the owned tile
  int first;    // first streamed tile of a head
  int per_head; // streamed tiles per head
  int n;        // streamed tiles in all (0: a query tile whose rows see no key)
};

// Launch order: tile-major over (batch, head) with the longest items first under the causal mask.
__host__ __device__ __forceinline__ BwdItem key_item(const BwdParams& p, int w) {
  BwdItem it;
  const int heads = p.B * p.Hkv;
  int kt, bh;
  if (p.causal) {  // early keys are seen by the most queries
    kt = w / heads;
    bh = w - kt * heads;
  } else {
    bh = w / p.n_kt;
    kt = w - bh * p.n_kt;
  }
  it.b = bh / p.Hkv;
  it.h = bh - it.b * p.Hkv;
  it.row0 = kt * kTile;
  const int first_row = p.causal && it.row0 > p.off ? it.row0 - p.off : 0;  // < Sq: the last row sees every key
  it.first = first_row / kTile;
  it.per_head = p.n_qt - it.first;
  it.n = it.per_head * p.group;
  return it;
}
__host__ __device__ __forceinline__ BwdItem query_item(const BwdParams& p, int w) {
  BwdItem it;
  const int heads = p.B * p.Hq;
  int qt, bh;
  if (p.causal) {  // late rows see the most keys
    qt = w / heads;
    bh = w - qt * heads;
    qt = p.n_qt - 1 - qt;
  } else {
    bh = w / p.n_qt;
    qt = w - bh * p.n_qt;
  }
  it.b = bh / p.Hq;
  it.h = bh - it.b * p.Hq;
  it.row0 = qt * kTile;
  it.first = 0;
  it.per_head = p.n_kt;
  if (p.causal) {
    const int row_end = it.row0 + kTile < p.Sq ? it.row0 + kTile : p.Sq;
    const int last_key = row_end - 1 + p.off;
    const int need = last_key < 0 ? 0 : last_key / kTile + 1;
    if (need < it.per_head) it.per_head = need;
  }
  it.n = it.per_head;
  return it;
}

// D[128 x 128] (+)= A[tmem] B for 64 of the 128 contraction rows.  A (BF16) was written over fp32 columns, by each
// softmax thread over the first half of its own kCols; B is MN-major (16 contraction rows are 2048 bytes).
__device__ __forceinline__ void issue_ts_half(bool leader, uint32_t tmem_d, uint32_t tmem_a, uint64_t b_desc, int half,
                                              bool accumulate) {
  if (leader) {
#pragma unroll
    for (int kk = 0; kk < 4; ++kk) {
      const int k16 = half * 4 + kk;           // 16 contraction rows: 8 columns of A
      const int part = k16 * 16 / kCols;
      mma_ts(tmem_d, tmem_a + part * kCols + (k16 * 8 - part * (kCols / 2)), desc_advance(b_desc, k16 * 2048), kIdescPV,
             (accumulate || kk > 0) ? 1u : 0u);
    }
  }
}

// Tensor memory columns.  Key CTAs: S (then P over it), dP (then dS over it), dV, dK.  Query CTAs: two score buffers
// (dS over the scores it comes from), dP, dQ.
constexpr uint32_t kTmS = 0, kTmDp = kTile, kTmDv = 2 * kTile, kTmDk = 3 * kTile;
constexpr uint32_t kTmQryS = 0, kTmQryDp = 2 * kTile, kTmDq = 3 * kTile;  // score buffer j % 2 at kTmQryS + (j % 2) * kTile

__device__ __forceinline__ void load_tile(uint8_t* dst, const CUtensorMap* tm, uint64_t* bar, int head, int row, int b) {
  tma_load_4d(dst, tm, bar, 0, head, row, b);
  tma_load_4d(dst + kHalfBytes, tm, bar, 64, head, row, b);
}

// Stream A (kA: Q in key CTAs, K in query CTAs) and the resident tiles, or stream B (dO, V).  Key CTAs' stream A also
// brings the row statistics of its tiles.
template <bool kKeys, bool kA>
__device__ __forceinline__ void bwd_loader(const BwdParams& p, const BwdItem& it, const BwdBarriers& bars, uint8_t* smem,
                                           WaitCtx ctx, const CUtensorMap* tm_fixed, const CUtensorMap* tm_stream) {
  constexpr int kSlots = kA ? kRingA : kRingB;
  uint64_t* full = kA ? bars.a_full : bars.b_full;
  uint64_t* empty = kA ? bars.a_empty : bars.b_empty;
  uint8_t* ring = smem + kSmemRing + (kA ? 0 : kRingA * kTileBytes);
  // each loader brings one resident tile: K or Q with stream A, V or dO with stream B
  mbar_arrive_expect_tx(bars.fixed_full, kTileBytes);
  load_tile(smem + kSmemFixed + (kA ? 0 : kTileBytes), tm_fixed, bars.fixed_full, it.h, it.row0, it.b);
  int head = kKeys ? it.h * p.group : it.h / p.group;
  int tile = it.first;
  for (int i = 0; i < it.n; ++i) {
    const int slot = i % kSlots;
    if (!mbar_wait(&empty[slot], ((i / kSlots) & 1) ^ 1, ctx, kRoleBwdLoad | kBarRingEmpty)) return;
    mbar_arrive_expect_tx(&full[slot], kTileBytes);
    load_tile(ring + slot * kTileBytes, tm_stream, &full[slot], head, tile * kTile, it.b);
    if (kKeys && kA) {
      const int st = i & 1;
      float* dst = reinterpret_cast<float*>(smem + kSmemStat) + st * 2 * kTile;
      const size_t at = (static_cast<size_t>(it.b) * p.Hq + head) * p.n_qt * kTile + static_cast<size_t>(tile) * kTile;
      if (!mbar_wait(&bars.stat_empty[st], ((i >> 1) & 1) ^ 1, ctx, kRoleBwdLoad | kBarStatEmpty)) return;
      mbar_arrive_expect_tx(&bars.stat_full[st], 2 * kStatBytes);
      bulk_load(dst, p.neg_lse2 + at, kStatBytes, &bars.stat_full[st]);
      bulk_load(dst + kTile, p.neg_delta + at, kStatBytes, &bars.stat_full[st]);
    }
    if (++tile == it.first + it.per_head) {
      tile = it.first;
      ++head;
    }
  }
}

// Shared-memory address of tile i of a stream, and the wait for it.
__device__ __forceinline__ uint32_t a_tile(uint32_t base, int i) { return base + kSmemRing + (i % kRingA) * kTileBytes; }
__device__ __forceinline__ uint32_t b_tile(uint32_t base, int i) {
  return base + kSmemRing + (kRingA + i % kRingB) * kTileBytes;
}
__device__ __forceinline__ bool wait_a(const BwdBarriers& bars, int i, WaitCtx ctx) {
  return mbar_wait_warp(&bars.a_full[i % kRingA], (i / kRingA) & 1, ctx, kRoleBwdMma | kBarRingFull);
}
__device__ __forceinline__ bool wait_b(const BwdBarriers& bars, int i, WaitCtx ctx) {
  return mbar_wait_warp(&bars.b_full[i % kRingB], (i / kRingB) & 1, ctx, kRoleBwdMma | kBarRingFull);
}

// Tensor pipe order in a key CTA, per query tile i:  P(i)^T dO(i) | K Q(i+1)^T | dS(i)^T Q(i) | V dO(i+1)^T.
// P(i+1) is exponentiated beside the last two, dS(i+1) is formed beside the next two.  P aliases the
// scores it comes from and dS the dP it comes from: a later product into the same columns is issued behind the one
// that reads them, on a pipe that executes in order.
__device__ __forceinline__ void key_mma(const BwdItem& it, const BwdBarriers& bars, uint8_t* smem, WaitCtx ctx,
                                        uint32_t tmem) {
  const bool leader = elect_one();
  const uint32_t base = smem_u32(smem);
  const uint64_t k_desc = kmajor_desc(base + kSmemFixed), v_desc = kmajor_desc(base + kSmemFixed + kTileBytes);
  if (!mbar_wait_warp(bars.fixed_full, 0, ctx, kRoleBwdMma | kBarFixed)) return;
  if (!wait_a(bars, 0, ctx)) return;
  tc_fence_after_sync();
  issue_qk(leader, tmem + kTmS, k_desc, kmajor_desc(a_tile(base, 0)));
  if (leader) mma_commit(bars.s_full);
  if (!wait_b(bars, 0, ctx)) return;
  tc_fence_after_sync();
  issue_qk(leader, tmem + kTmDp, v_desc, kmajor_desc(b_tile(base, 0)));
  if (leader) mma_commit(bars.dp_full);
  for (int i = 0; i < it.n; ++i) {
    const bool next = i + 1 < it.n;
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      if (!mbar_wait_warp(&bars.p_full[h], i & 1, ctx, kRoleBwdMma | kBarP)) return;
      tc_fence_after_sync();
      issue_ts_half(leader, tmem + kTmDv, tmem + kTmS, vtile_desc(b_tile(base, i)), h, i > 0 || h > 0);
    }
    if (leader) mma_commit(&bars.b_empty[i % kRingB]);
    if (next) {
      if (!wait_a(bars, i + 1, ctx)) return;
      tc_fence_after_sync();
      issue_qk(leader, tmem + kTmS, k_desc, kmajor_desc(a_tile(base, i + 1)));
      if (leader) mma_commit(bars.s_full);
    }
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      if (!mbar_wait_warp(&bars.ds_full[h], i & 1, ctx, kRoleBwdMma | kBarDs)) return;
      tc_fence_after_sync();
      issue_ts_half(leader, tmem + kTmDk, tmem + kTmDp, vtile_desc(a_tile(base, i)), h, i > 0 || h > 0);
    }
    if (leader) mma_commit(&bars.a_empty[i % kRingA]);
    if (next) {
      if (!wait_b(bars, i + 1, ctx)) return;
      tc_fence_after_sync();
      issue_qk(leader, tmem + kTmDp, v_desc, kmajor_desc(b_tile(base, i + 1)));
      if (leader) mma_commit(bars.dp_full);
    }
  }
  if (leader) mma_commit(bars.acc_full);
}

// Tensor pipe order in a query CTA, per key tile j:  Q K(j+1)^T | dO V(j+1)^T | dS(j) K(j).  The scores of tile j + 1 are
// computed while tile j's are exponentiated (two score buffers; dS(j) goes over the scores of tile j, and S(j+2)
// into the same columns is issued behind dS(j) K(j)); dP has one buffer, free as soon as it is in registers.
__device__ __forceinline__ void query_mma(const BwdItem& it, const BwdBarriers& bars, uint8_t* smem, WaitCtx ctx,
                                          uint32_t tmem) {
  const bool leader = elect_one();
  const uint32_t base = smem_u32(smem);
  const uint64_t q_desc = kmajor_desc(base + kSmemFixed), do_desc = kmajor_desc(base + kSmemFixed + kTileBytes);
  if (!mbar_wait_warp(bars.fixed_full, 0, ctx, kRoleBwdMma | kBarFixed)) return;
  for (int j = -1; j < it.n; ++j) {
    const int n = j + 1;
    if (n < it.n) {  // scores and dP of the next tile
      if (!wait_a(bars, n, ctx)) return;
      tc_fence_after_sync();
      issue_qk(leader, tmem + kTmQryS + (n & 1) * kTile, q_desc, kmajor_desc(a_tile(base, n)));
      if (leader) mma_commit(&bars.s_full[n & 1]);
      if (!wait_b(bars, n, ctx)) return;
      if (j >= 0 && !mbar_wait_warp(bars.dp_read, j & 1, ctx, kRoleBwdMma | kBarDpRead)) return;
      tc_fence_after_sync();
      issue_qk(leader, tmem + kTmQryDp, do_desc, kmajor_desc(b_tile(base, n)));
      if (leader) {
        mma_commit(bars.dp_full);
        mma_commit(&bars.b_empty[n % kRingB]);
      }
    }
    if (j >= 0) {
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        if (!mbar_wait_warp(&bars.ds_full[(j & 1) * 2 + h], (j >> 1) & 1, ctx, kRoleBwdMma | kBarDs)) return;
        tc_fence_after_sync();
        issue_ts_half(leader, tmem + kTmDq, tmem + kTmQryS + (j & 1) * kTile, vtile_desc(a_tile(base, j)), h, j > 0 || h > 0);
      }
      if (leader) mma_commit(&bars.a_empty[j % kRingA]);
    }
  }
  if (leader) mma_commit(bars.acc_full);
}

// 32 fp32 columns of one row -> BF16 chunks of a 128-byte-swizzled [128][64] half tile; `chunk0` is the
// first 16-byte chunk (0 or 4) in the half tile's row.
__device__ __forceinline__ void stage_row32(uint8_t* half_tile, int row, int chunk0, const uint32_t* o, float factor) {
#pragma unroll
  for (int ch = 0; ch < 4; ++ch) {
    uint4 val;
    val.x = pack_bf16x2(__uint_as_float(o[ch * 8 + 0]) * factor, __uint_as_float(o[ch * 8 + 1]) * factor);
    val.y = pack_bf16x2(__uint_as_float(o[ch * 8 + 2]) * factor, __uint_as_float(o[ch * 8 + 3]) * factor);
    val.z = pack_bf16x2(__uint_as_float(o[ch * 8 + 4]) * factor, __uint_as_float(o[ch * 8 + 5]) * factor);
    val.w = pack_bf16x2(__uint_as_float(o[ch * 8 + 6]) * factor, __uint_as_float(o[ch * 8 + 7]) * factor);
    *reinterpret_cast<uint4*>(half_tile + row * 128 + (((chunk0 + ch) ^ (row & 7)) << 4)) = val;
  }
}

// Both softmax roles: P = exp2(S * scale log2(e) - LSE log2(e)) on pairs of columns; of every eight pairs
// kBwdPolyPairs take the polynomial on the FMA pipe, the others the special-function unit.
#ifndef ATTN_BWD_POLY_PAIRS
#define ATTN_BWD_POLY_PAIRS 2
#endif
constexpr int kBwdPolyPairs = ATTN_BWD_POLY_PAIRS;
#define ATTN_F(r, i) __uint_as_float((r)[(i)])

// exp2 of kCols score columns in place, given per pair of columns the pair of -LSE log2(e).  Columns outside
// [seen_from, seen_to) become 0 where `masked`.
template <typename NegLse>
__device__ __forceinline__ void exp_row(uint32_t* x, float2 c2, NegLse neg_lse, bool masked, int seen_from, int seen_to) {
#pragma unroll
  for (int pr = 0; pr < kCols / 2; ++pr) {
    const int e = pr * 2;
    const float2 y = fma2(make_float2(ATTN_F(x, e), ATTN_F(x, e + 1)), c2, neg_lse(e));
    const float2 w = (pr & 7) < kBwdPolyPairs ? exp2_poly2(y) : make_float2(ex2_approx(y.x), ex2_approx(y.y));
    x[e] = __float_as_uint(w.x);
    x[e + 1] = __float_as_uint(w.y);
  }
  if (masked) {
#pragma unroll
    for (int e = 0; e < kCols; ++e) {
      if (e < seen_from || e >= seen_to) x[e] = 0u;
    }
  }
}

// One softmax thread: row `row` of the tile, columns [part * kCols, (part + 1) * kCols).
__device__ __forceinline__ void key_softmax(const BwdParams& p, const BwdItem& it, const BwdBarriers& bars, uint8_t* smem,
                                            WaitCtx ctx, uint32_t tmem, int part, int row, int lane,
                                            const CUtensorMap* tm_dk, const CUtensorMap* tm_dv) {
  const int half = part / (kParts / 2);
  const uint32_t lane_sel = static_cast<uint32_t>(row & ~31) << 16;
  const uint32_t t_s = tmem + lane_sel + kTmS + part * kCols, t_dp = tmem + lane_sel + kTmDp + part * kCols;
  const float2 c2 = make_float2(p.scale_log2, p.scale_log2);
  int tile = it.first;
  for (int i = 0; i < it.n; ++i) {
    const float* nl = reinterpret_cast<const float*>(smem + kSmemStat) + (i & 1) * 2 * kTile + part * kCols;
    const float* neg_delta = nl + kTile;
    bool ok = mbar_wait(&bars.stat_full[i & 1], (i >> 1) & 1, ctx, kRoleBwdSoftmax | kBarStat) &&
              mbar_wait(bars.s_full, i & 1, ctx, kRoleBwdSoftmax | kBarS);
    if (!__all_sync(0xffffffffu, ok)) return;
    tc_fence_after_sync();
    uint32_t x[kCols], pk[kCols / 2];
    tmem_ld_x32(t_s, x);
    tmem_wait_ld();
    // the key is visible to the queries of columns `seen_from` on
    const int seen_from = it.row0 + row - p.off - tile * kTile - part * kCols;
    const bool masked = p.causal && it.row0 + kTile - 1 > tile * kTile + p.off;  // CTA-uniform
    exp_row(x, c2, [&](int e) { return *reinterpret_cast<const float2*>(nl + e); }, masked, seen_from, kCols);
#pragma unroll
    for (int e = 0; e < kCols / 2; ++e) pk[e] = pack_bf16x2(ATTN_F(x, 2 * e), ATTN_F(x, 2 * e + 1));
    tmem_st_x16(t_s, pk);
    tmem_wait_st();
    tc_fence_before_sync();
    __syncwarp();
    if (lane == 0) mbar_arrive(&bars.p_full[half]);
    ok = mbar_wait(bars.dp_full, i & 1, ctx, kRoleBwdSoftmax | kBarDp);
    if (!__all_sync(0xffffffffu, ok)) return;
    tc_fence_after_sync();
    uint32_t d[kCols];
    tmem_ld_x32(t_dp, d);
    tmem_wait_ld();
#pragma unroll
    for (int e = 0; e < kCols; e += 2) {
      const float2 t = add2(make_float2(ATTN_F(d, e), ATTN_F(d, e + 1)), *reinterpret_cast<const float2*>(neg_delta + e));
      const float2 w = mul2(make_float2(ATTN_F(x, e), ATTN_F(x, e + 1)), t);
      pk[e / 2] = pack_bf16x2(w.x, w.y);
    }
    tmem_st_x16(t_dp, pk);  // over this thread's own columns, which are in registers
    tmem_wait_st();
    tc_fence_before_sync();
    __syncwarp();
    if (lane == 0) {
      mbar_arrive(&bars.ds_full[half]);
      mbar_arrive(&bars.stat_empty[i & 1]);
    }
    if (++tile == it.first + it.per_head) tile = it.first;
  }
  // Epilogue: half 0 stores dV (through V's tile in shared memory), half 1 dK (through K's); no product reads them now.
  bool ok = mbar_wait(bars.acc_full, 0, ctx, kRoleBwdSoftmax | kBarAcc);
  if (!__all_sync(0xffffffffu, ok)) return;
  tc_fence_after_sync();
  uint8_t* stage = smem + kSmemFixed + (half == 0 ? kTileBytes : 0);
  const int col0 = (part % (kParts / 2)) * 2 * kCols;  // this thread's 2 kCols columns of its accumulator
  const uint32_t t_acc = tmem + lane_sel + (half == 0 ? kTmDv : kTmDk) + col0;
  const float factor = half == 0 ? 1.f : p.scale;
#pragma unroll
  for (int cc = 0; cc < 2 * kCols / 32; ++cc) {
    uint32_t o[32];
    tmem_ld_x32(t_acc + cc * 32, o);
    tmem_wait_ld();
    const int c = col0 + cc * 32;
    stage_row32(stage + (c >> 6) * kHalfBytes, row, (c & 63) / 8, o, factor);
  }
  fence_proxy_async_smem();
  __syncwarp();
  if (lane == 0) mbar_arrive(&bars.stage_full[half]);
  if (row == 0 && part % (kParts / 2) == 0 && mbar_wait(&bars.stage_full[half], 0, ctx, kRoleBwdSoftmax | kBarStage)) {
    const CUtensorMap* tm = half == 0 ? tm_dv : tm_dk;
    tma_store_4d(tm, stage, 0, it.h, it.row0, it.b);
    tma_store_4d(tm, stage + kHalfBytes, 64, it.h, it.row0, it.b);
    tma_store_commit();
    tma_store_wait_all0();
  }
}

__device__ __forceinline__ void query_softmax(const BwdParams& p, const BwdItem& it, const BwdBarriers& bars, uint8_t* smem,
                                              WaitCtx ctx, uint32_t tmem, int part, int row, int lane,
                                              const CUtensorMap* tm_dq) {
  const int half = part / (kParts / 2);
  const uint32_t lane_sel = static_cast<uint32_t>(row & ~31) << 16;
  const uint32_t t_dp = tmem + lane_sel + kTmQryDp + part * kCols;
  const float2 c2 = make_float2(p.scale_log2, p.scale_log2);
  const size_t at = (static_cast<size_t>(it.b) * p.Hq + it.h) * p.n_qt * kTile + it.row0 + row;
  const float nl = __ldg(p.neg_lse2 + at), ndl = __ldg(p.neg_delta + at);
  const float2 nl2 = make_float2(nl, nl), ndl2 = make_float2(ndl, ndl);
  const int row_limit = p.causal ? min(p.Sk, it.row0 + row + p.off + 1) : p.Sk;   // keys this row may see
  const int tile_clear = p.causal ? min(p.Sk, it.row0 + p.off + 1) : p.Sk;        // keys every row of the tile sees
  for (int j = 0; j < it.n; ++j) {
    bool ok = mbar_wait(&bars.s_full[j & 1], (j >> 1) & 1, ctx, kRoleBwdSoftmax | kBarS);
    if (!__all_sync(0xffffffffu, ok)) return;
    tc_fence_after_sync();
    const uint32_t t_s = tmem + lane_sel + kTmQryS + (j & 1) * kTile + part * kCols;
    uint32_t x[kCols];
    tmem_ld_x32(t_s, x);
    tmem_wait_ld();
    // keys beyond Sk are masked too: their scores are 0, and exp2(nl) may be infinite
    const bool masked = (j + 1) * kTile > tile_clear;  // CTA-uniform
    exp_row(x, c2, [&](int) { return nl2; }, masked, 0, row_limit - j * kTile - part * kCols);
    ok = mbar_wait(bars.dp_full, j & 1, ctx, kRoleBwdSoftmax | kBarDp);
    if (!__all_sync(0xffffffffu, ok)) return;
    tc_fence_after_sync();
    uint32_t d[kCols], pk[kCols / 2];
    tmem_ld_x32(t_dp, d);
    tmem_wait_ld();
    tc_fence_before_sync();
    __syncwarp();
    if (lane == 0) mbar_arrive(bars.dp_read);
#pragma unroll
    for (int e = 0; e < kCols; e += 2) {
      const float2 t = add2(make_float2(ATTN_F(d, e), ATTN_F(d, e + 1)), ndl2);
      const float2 w = mul2(make_float2(ATTN_F(x, e), ATTN_F(x, e + 1)), t);
      pk[e / 2] = pack_bf16x2(w.x, w.y);
    }
    tmem_st_x16(t_s, pk);  // over this thread's own scores, read above
    tmem_wait_st();
    tc_fence_before_sync();
    __syncwarp();
    if (lane == 0) mbar_arrive(&bars.ds_full[(j & 1) * 2 + half]);
  }
  // Epilogue: each thread stores kCols columns of dQ through Q's tile, each half tile by itself.
  bool ok = mbar_wait(bars.acc_full, 0, ctx, kRoleBwdSoftmax | kBarAcc);
  if (!__all_sync(0xffffffffu, ok)) return;
  tc_fence_after_sync();
  uint8_t* stage = smem + kSmemFixed + half * kHalfBytes;
  uint32_t o[kCols];
  if (it.n > 0) {
    tmem_ld_x32(tmem + lane_sel + kTmDq + part * kCols, o);
    tmem_wait_ld();
  } else {  // no row of the tile sees a key: dQ is 0, and tensor memory holds nothing of ours
#pragma unroll
    for (int e = 0; e < kCols; ++e) o[e] = 0u;
  }
  stage_row32(stage, row, (part % (kParts / 2)) * kCols / 8, o, p.scale);
  fence_proxy_async_smem();
  __syncwarp();
  if (lane == 0) mbar_arrive(&bars.stage_full[half]);
  if (row == 0 && part % (kParts / 2) == 0 && mbar_wait(&bars.stage_full[half], 0, ctx, kRoleBwdSoftmax | kBarStage)) {
    tma_store_4d(tm_dq, stage, half * 64, it.h, it.row0, it.b);
    tma_store_commit();
    tma_store_wait_all0();
  }
}

__global__ void __launch_bounds__(kBwdThreads, 1)
attn_bwd_kernel(const __grid_constant__ CUtensorMap tm_q, const __grid_constant__ CUtensorMap tm_k,
                const __grid_constant__ CUtensorMap tm_v, const __grid_constant__ CUtensorMap tm_do,
                const __grid_constant__ CUtensorMap tm_dq, const __grid_constant__ CUtensorMap tm_dk,
                const __grid_constant__ CUtensorMap tm_dv, const BwdParams p) {
  extern __shared__ __align__(1024) uint8_t smem[];
  uint64_t* bar = reinterpret_cast<uint64_t*>(smem + kSmemBwdBars);
  BwdBarriers bars;
  bars.fixed_full = bar;
  bars.a_full = bars.fixed_full + 1;
  bars.a_empty = bars.a_full + kRingA;
  bars.b_full = bars.a_empty + kRingA;
  bars.b_empty = bars.b_full + kRingB;
  bars.stat_full = bars.b_empty + kRingB;
  bars.stat_empty = bars.stat_full + kStatStages;
  bars.s_full = bars.stat_empty + kStatStages;
  bars.dp_full = bars.s_full + 2;
  bars.dp_read = bars.dp_full + 1;
  bars.p_full = bars.dp_read + 1;
  bars.ds_full = bars.p_full + 2;
  bars.acc_full = bars.ds_full + 4;
  bars.stage_full = bars.acc_full + 1;
  uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(smem + kSmemBwdMisc);
  volatile int* abort_flag = reinterpret_cast<volatile int*>(smem + kSmemBwdMisc + 4);
  const WaitCtx ctx{abort_flag, p.status, kWaitLimitNs};
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  if ((smem_u32(smem) & 1023u) != 0) {  // the swizzled tiles need a 1024-byte aligned base
    if (tid == 0 && atomicCAS(p.status, 0, kBadSmemAlign) == 0) p.status[1] = static_cast<int>(blockIdx.x);
    return;
  }
  if (tid == 0) {
    mbar_init(bars.fixed_full, 2);
    for (int i = 0; i < kRingA; ++i) {
      mbar_init(&bars.a_full[i], 1);
      mbar_init(&bars.a_empty[i], 1);
    }
    for (int i = 0; i < kRingB; ++i) {
      mbar_init(&bars.b_full[i], 1);
      mbar_init(&bars.b_empty[i], 1);
    }
    mbar_init(bars.dp_full, 1);
    mbar_init(bars.dp_read, kSoftmaxWarps);
    mbar_init(bars.acc_full, 1);
    for (int i = 0; i < 2; ++i) {
      mbar_init(&bars.stat_full[i], 1);
      mbar_init(&bars.stat_empty[i], kSoftmaxWarps);
      mbar_init(&bars.s_full[i], 1);
      mbar_init(&bars.p_full[i], kSoftmaxWarps / 2);
      mbar_init(&bars.ds_full[i], kSoftmaxWarps / 2);
      mbar_init(&bars.ds_full[2 + i], kSoftmaxWarps / 2);
      mbar_init(&bars.stage_full[i], kSoftmaxWarps / 2);
    }
    *abort_flag = 0;
    fence_mbar_init();
  }
  if (warp == kSoftmaxWarps) {
    tmem_alloc(tmem_slot, 512);
    tmem_relinquish();
  }
  tc_fence_before_sync();
  __syncthreads();
  tc_fence_after_sync();
  const uint32_t tmem = *tmem_slot;
  const bool keys = static_cast<int>(blockIdx.x) < p.n_key_items;  // CTA-uniform
  const BwdItem it = keys ? key_item(p, blockIdx.x) : query_item(p, static_cast<int>(blockIdx.x) - p.n_key_items);

  if (warp < kSoftmaxWarps) {
    if (keys) {
      key_softmax(p, it, bars, smem, ctx, tmem, warp >> 2, tid & 127, lane, &tm_dk, &tm_dv);
    } else {
      query_softmax(p, it, bars, smem, ctx, tmem, warp >> 2, tid & 127, lane, &tm_dq);
    }
  } else if (warp == kSoftmaxWarps) {
    if (keys) {
      key_mma(it, bars, smem, ctx, tmem);
    } else {
      query_mma(it, bars, smem, ctx, tmem);
    }
  } else if (lane == 0) {
    const bool stream_a = warp == kSoftmaxWarps + 1;
    if (keys && stream_a) {
      bwd_loader<true, true>(p, it, bars, smem, ctx, &tm_k, &tm_q);
    } else if (keys) {
      bwd_loader<true, false>(p, it, bars, smem, ctx, &tm_v, &tm_do);
    } else if (stream_a) {
      bwd_loader<false, true>(p, it, bars, smem, ctx, &tm_q, &tm_k);
    } else {
      bwd_loader<false, false>(p, it, bars, smem, ctx, &tm_do, &tm_v);
    }
    if (*abort_flag) {  // let loads in flight land before the CTA's shared memory is released
      const uint64_t t0 = global_timer_ns();
      while (global_timer_ns() - t0 < 1000000ull) {
      }
    }
  }
  tc_fence_before_sync();
  __syncthreads();
  if (warp == kSoftmaxWarps) {
    tc_fence_after_sync();
    tmem_dealloc(tmem, 512);
  }
}

// Row statistics of the backward pass: -LSE log2(e) and -delta = dLSE - sum_d dO O, one half warp per
// (batch, row, head), rows padded to whole tiles.  HBM-bound: 512 bytes read per row.
constexpr int kPrepThreads = 256;
struct RowStrides {
  long long b, s, h;  // elements
};

__device__ __forceinline__ float dot2_bf16(uint32_t a, uint32_t b, float acc) {
  acc = fmaf(__uint_as_float(a << 16), __uint_as_float(b << 16), acc);
  return fmaf(__uint_as_float(a & 0xffff0000u), __uint_as_float(b & 0xffff0000u), acc);
}

__global__ void __launch_bounds__(kPrepThreads)
attn_bwd_prep_kernel(const uint16_t* __restrict__ o, const uint16_t* __restrict__ dout, RowStrides so, RowStrides sdo,
                     const float* __restrict__ lse, const float* __restrict__ dlse, float* __restrict__ neg_lse2,
                     float* __restrict__ neg_delta, int Hq, int Sq, int padded, long long n_rows) {
  const int sub = threadIdx.x & 15;
  const long long step = static_cast<long long>(gridDim.x) * (kPrepThreads / 16);
  for (long long r = static_cast<long long>(blockIdx.x) * (kPrepThreads / 16) + (threadIdx.x >> 4); r < n_rows; r += step) {
    const int h = static_cast<int>(r % Hq);
    const long long t = r / Hq;
    const int s = static_cast<int>(t % padded);
    const long long b = t / padded;
    float acc = 0.f, l = -INFINITY, dl = 0.f;
    if (s < Sq) {
      const uint4 x = __ldg(reinterpret_cast<const uint4*>(o + b * so.b + s * so.s + h * so.h) + sub);
      const uint4 y = __ldg(reinterpret_cast<const uint4*>(dout + b * sdo.b + s * sdo.s + h * sdo.h) + sub);
      const long long at = (b * Hq + h) * Sq + s;
      l = __ldg(lse + at);
      if (dlse != nullptr) dl = __ldg(dlse + at);
      acc = dot2_bf16(x.x, y.x, dot2_bf16(x.y, y.y, dot2_bf16(x.z, y.z, dot2_bf16(x.w, y.w, 0.f))));
    }
#pragma unroll
    for (int m = 8; m > 0; m >>= 1) acc += __shfl_xor_sync(0xffffffffu, acc, m);
    if (sub == 0) {
      const long long at = (b * Hq + h) * padded + s;
      const bool none = l == -INFINITY;  // the row sees no key, or does not exist: P = exp2(-inf) = 0
      neg_lse2[at] = none ? -INFINITY : -l * 1.4426950408889634f;
      neg_delta[at] = none ? 0.f : dl - acc;
    }
  }
}

#undef ATTN_F

}  // namespace bwd
}  // namespace attn
