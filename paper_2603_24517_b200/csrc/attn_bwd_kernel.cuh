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
// either come in any order or wait for one another.  Each CTA (320 threads, one per SM):
//
//   warps 0-7   softmax: lane quarter w % 4 of the tile (one thread per row), column half w / 4
//   warp  8     MMA issue (tcgen05.mma by an elected lane)
//   warp  9     loader (TMA; a ring of five 32 KB tiles beside the two resident ones)
//
// Transposed tiles in key CTAs (rows are keys) let P^T and dS^T go back to tensor memory as the left
// operand of the second products, so nothing is transposed through shared memory.
#pragma once

#include "attn_fwd_kernel.cuh"

namespace attn {
namespace bwd {

constexpr int kBwdThreads = 320;
constexpr int kRingSlots = 5;
constexpr int kStatStages = 2;
constexpr int kStatBytes = kTile * 4;  // one fp32 value per query row of a tile

constexpr int kSmemFixed = 0;  // two resident tiles
constexpr int kSmemRing = 2 * kTileBytes;
constexpr int kSmemStat = kSmemRing + kRingSlots * kTileBytes;  // [kStatStages][2][128]: -LSE log2(e), delta
constexpr int kSmemBwdBars = kSmemStat + kStatStages * 2 * kStatBytes;
constexpr int kBwdBars = 1 + 2 * kRingSlots + kStatStages + 1 + 1 + 2 + 2 + 4 + 1 + 2;
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
  const float* delta;     // same layout, 0 in those rows
  int* status;
};

// codes of expired waits: role << 8 | barrier (roles continue the forward kernels' numbering)
enum : int {
  kRoleBwdLoad = 10 << 8, kRoleBwdMma = 11 << 8, kRoleBwdSoftmax = 12 << 8,
  kBarFixed = 1, kBarRingFull = 2, kBarRingEmpty = 3, kBarStat = 4, kBarS = 5, kBarDp = 6, kBarSRead = 7, kBarP = 8,
  kBarDs = 9, kBarAcc = 10, kBarStage = 11
};

struct BwdBarriers {
  uint64_t* fixed_full;  // loader (TMA) -> MMA
  uint64_t* ring_full;   // [kRingSlots]  loader (TMA) -> MMA
  uint64_t* ring_empty;  // [kRingSlots]  MMA commit -> loader
  uint64_t* stat_full;   // [kStatStages]  loader (bulk copy) -> softmax (key CTAs)
  uint64_t* s_full;      // MMA commit -> softmax
  uint64_t* s_read;      // softmax (8 warps) -> MMA: scores are in registers (query CTAs)
  uint64_t* dp_full;     // [2]  MMA commit -> softmax
  uint64_t* p_full;      // [2]  softmax half (4 warps): its 64 columns of P are in tensor memory (key CTAs)
  uint64_t* ds_full;     // [4]  the same for dS; query CTAs, whose softmax can be a tile ahead, alternate two pairs
  uint64_t* acc_full;    // MMA commit: the accumulators are final
  uint64_t* stage_full;  // [2]  softmax half (4 warps): its staging tile is written
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

// D[128 x 128] (+)= A[tmem] B for 64 of the 128 contraction rows.  A (BF16) of half h lies in the first 32
// columns of that half's 64 fp32 columns; B is MN-major (16 contraction rows are 2048 bytes).
__device__ __forceinline__ void issue_ts_half(bool leader, uint32_t tmem_d, uint32_t tmem_a, uint64_t b_desc, int half,
                                              bool accumulate) {
  if (leader) {
#pragma unroll
    for (int kk = 0; kk < 4; ++kk) {
      mma_ts(tmem_d, tmem_a + half * 64 + kk * 8, desc_advance(b_desc, (half * 4 + kk) * 2048), kIdescPV,
             (accumulate || kk > 0) ? 1u : 0u);
    }
  }
}

constexpr uint32_t kTmS = 0, kTmDp = kTile;                          // both kinds
constexpr uint32_t kTmDv = 2 * kTile, kTmDk = 3 * kTile;             // key CTAs
constexpr uint32_t kTmDp1 = 2 * kTile, kTmDq = 3 * kTile;            // query CTAs (dP has two buffers)

__device__ __forceinline__ void load_tile(uint8_t* dst, const CUtensorMap* tm, uint64_t* bar, int head, int row, int b) {
  tma_load_4d(dst, tm, bar, 0, head, row, b);
  tma_load_4d(dst + kHalfBytes, tm, bar, 64, head, row, b);
}

// Ring order: key CTAs Q(0), dO(0), Q(1), dO(1), ...; query CTAs K(0), V(0), K(1), V(1), ...
template <bool kKeys>
__device__ __forceinline__ void bwd_loader(const BwdParams& p, const BwdItem& it, const BwdBarriers& bars, uint8_t* smem,
                                           WaitCtx ctx, const CUtensorMap* tm_q, const CUtensorMap* tm_k,
                                           const CUtensorMap* tm_v, const CUtensorMap* tm_do) {
  mbar_arrive_expect_tx(bars.fixed_full, 2 * kTileBytes);
  load_tile(smem + kSmemFixed, kKeys ? tm_k : tm_q, bars.fixed_full, it.h, it.row0, it.b);
  load_tile(smem + kSmemFixed + kTileBytes, kKeys ? tm_v : tm_do, bars.fixed_full, it.h, it.row0, it.b);
  int head = kKeys ? it.h * p.group : it.h / p.group;
  int tile = it.first;
  uint32_t cnt = 0;
  for (int i = 0; i < it.n; ++i) {
#pragma unroll
    for (int x = 0; x < 2; ++x) {
      const uint32_t slot = cnt % kRingSlots, par = (cnt / kRingSlots) & 1;
      if (!mbar_wait(&bars.ring_empty[slot], par ^ 1, ctx, kRoleBwdLoad | kBarRingEmpty)) return;
      mbar_arrive_expect_tx(&bars.ring_full[slot], kTileBytes);
      const CUtensorMap* tm = kKeys ? (x == 0 ? tm_q : tm_do) : (x == 0 ? tm_k : tm_v);
      load_tile(smem + kSmemRing + slot * kTileBytes, tm, &bars.ring_full[slot], head, tile * kTile, it.b);
      ++cnt;
    }
    if (kKeys) {
      // dO(i) took ring position 2 i + 1, i.e. the slot of position 2 i - 4 = Q(i - 2), so the wait above has
      // seen dS(i - 2)^T Q(i - 2) complete: its softmax warps have read stage i % 2 for the last time
      const int st = i & 1;
      float* dst = reinterpret_cast<float*>(smem + kSmemStat) + st * 2 * kTile;
      const size_t at = (static_cast<size_t>(it.b) * p.Hq + head) * p.n_qt * kTile + static_cast<size_t>(tile) * kTile;
      mbar_arrive_expect_tx(&bars.stat_full[st], 2 * kStatBytes);
      bulk_load(dst, p.neg_lse2 + at, kStatBytes, &bars.stat_full[st]);
      bulk_load(dst + kTile, p.delta + at, kStatBytes, &bars.stat_full[st]);
    }
    if (++tile == it.first + it.per_head) {
      tile = it.first;
      ++head;
    }
  }
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
  const uint32_t ring = base + kSmemRing;
  if (!mbar_wait_warp(bars.fixed_full, 0, ctx, kRoleBwdMma | kBarFixed)) return;
  uint32_t cnt = 0;  // ring position of Q(i)
  if (!mbar_wait_warp(&bars.ring_full[0], 0, ctx, kRoleBwdMma | kBarRingFull)) return;
  tc_fence_after_sync();
  issue_qk(leader, tmem + kTmS, k_desc, kmajor_desc(ring));
  if (leader) mma_commit(bars.s_full);
  if (!mbar_wait_warp(&bars.ring_full[1], 0, ctx, kRoleBwdMma | kBarRingFull)) return;
  tc_fence_after_sync();
  issue_qk(leader, tmem + kTmDp, v_desc, kmajor_desc(ring + kTileBytes));
  if (leader) mma_commit(&bars.dp_full[0]);
  for (int i = 0; i < it.n; ++i, cnt += 2) {
    const uint32_t q_slot = cnt % kRingSlots, do_slot = (cnt + 1) % kRingSlots;
    const bool next = i + 1 < it.n;
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      if (!mbar_wait_warp(&bars.p_full[h], i & 1, ctx, kRoleBwdMma | kBarP)) return;
      tc_fence_after_sync();
      issue_ts_half(leader, tmem + kTmDv, tmem + kTmS, vtile_desc(ring + do_slot * kTileBytes), h, i > 0 || h > 0);
    }
    if (leader) mma_commit(&bars.ring_empty[do_slot]);
    if (next) {
      const uint32_t slot = (cnt + 2) % kRingSlots, par = ((cnt + 2) / kRingSlots) & 1;
      if (!mbar_wait_warp(&bars.ring_full[slot], par, ctx, kRoleBwdMma | kBarRingFull)) return;
      tc_fence_after_sync();
      issue_qk(leader, tmem + kTmS, k_desc, kmajor_desc(ring + slot * kTileBytes));
      if (leader) mma_commit(bars.s_full);
    }
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      if (!mbar_wait_warp(&bars.ds_full[h], i & 1, ctx, kRoleBwdMma | kBarDs)) return;
      tc_fence_after_sync();
      issue_ts_half(leader, tmem + kTmDk, tmem + kTmDp, vtile_desc(ring + q_slot * kTileBytes), h, i > 0 || h > 0);
    }
    if (leader) mma_commit(&bars.ring_empty[q_slot]);
    if (next) {
      const uint32_t slot = (cnt + 3) % kRingSlots, par = ((cnt + 3) / kRingSlots) & 1;
      if (!mbar_wait_warp(&bars.ring_full[slot], par, ctx, kRoleBwdMma | kBarRingFull)) return;
      tc_fence_after_sync();
      issue_qk(leader, tmem + kTmDp, v_desc, kmajor_desc(ring + slot * kTileBytes));
      if (leader) mma_commit(&bars.dp_full[0]);
    }
  }
  if (leader) mma_commit(bars.acc_full);
}

// Tensor pipe order in a query CTA, per key tile j:  Q K(j+1)^T | dO V(j+1)^T | dS(j) K(j).  The scores are
// copied to registers before the next ones are issued (s_read); dP and the dS written over it alternate
// between two buffers.
__device__ __forceinline__ void query_mma(const BwdItem& it, const BwdBarriers& bars, uint8_t* smem, WaitCtx ctx,
                                          uint32_t tmem) {
  const bool leader = elect_one();
  const uint32_t base = smem_u32(smem);
  const uint64_t q_desc = kmajor_desc(base + kSmemFixed), do_desc = kmajor_desc(base + kSmemFixed + kTileBytes);
  const uint32_t ring = base + kSmemRing;
  if (!mbar_wait_warp(bars.fixed_full, 0, ctx, kRoleBwdMma | kBarFixed)) return;
  for (int j = 0; j <= it.n; ++j) {
    if (j < it.n) {  // scores and dP of tile j
      const uint32_t k_pos = 2 * j, v_pos = 2 * j + 1;
      if (!mbar_wait_warp(&bars.ring_full[k_pos % kRingSlots], (k_pos / kRingSlots) & 1, ctx,
                          kRoleBwdMma | kBarRingFull))
        return;
      if (j > 0 && !mbar_wait_warp(bars.s_read, (j - 1) & 1, ctx, kRoleBwdMma | kBarSRead)) return;
      tc_fence_after_sync();
      issue_qk(leader, tmem + kTmS, q_desc, kmajor_desc(ring + (k_pos % kRingSlots) * kTileBytes));
      if (leader) mma_commit(bars.s_full);
      if (!mbar_wait_warp(&bars.ring_full[v_pos % kRingSlots], (v_pos / kRingSlots) & 1, ctx,
                          kRoleBwdMma | kBarRingFull))
        return;
      tc_fence_after_sync();
      issue_qk(leader, tmem + ((j & 1) ? kTmDp1 : kTmDp), do_desc, kmajor_desc(ring + (v_pos % kRingSlots) * kTileBytes));
      if (leader) {
        mma_commit(&bars.dp_full[j & 1]);
        mma_commit(&bars.ring_empty[v_pos % kRingSlots]);
      }
    }
    if (j > 0) {  // dQ += dS(j - 1) K(j - 1)
      const int i = j - 1;
      const uint32_t k_slot = (2 * i) % kRingSlots;
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        if (!mbar_wait_warp(&bars.ds_full[(i & 1) * 2 + h], (i >> 1) & 1, ctx, kRoleBwdMma | kBarDs)) return;
        tc_fence_after_sync();
        issue_ts_half(leader, tmem + kTmDq, tmem + ((i & 1) ? kTmDp1 : kTmDp), vtile_desc(ring + k_slot * kTileBytes), h,
                      i > 0 || h > 0);
      }
      if (leader) mma_commit(&bars.ring_empty[k_slot]);
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
// kExp2PolyPairs take the polynomial, as in the forward kernel.
#define ATTN_F(r, i) __uint_as_float((r)[(i)])

// One thread: row `row` of the tile, 64 columns of half `half`.
__device__ __forceinline__ void key_softmax(const BwdParams& p, const BwdItem& it, const BwdBarriers& bars, uint8_t* smem,
                                            WaitCtx ctx, uint32_t tmem, int half, int row, int lane,
                                            const CUtensorMap* tm_dk, const CUtensorMap* tm_dv) {
  const uint32_t lane_sel = static_cast<uint32_t>(row & ~31) << 16;
  const uint32_t t_s = tmem + lane_sel + kTmS + half * 64, t_dp = tmem + lane_sel + kTmDp + half * 64;
  const float2 c2 = make_float2(p.scale_log2, p.scale_log2);
  int tile = it.first;
  for (int i = 0; i < it.n; ++i) {
    const float* nl = reinterpret_cast<const float*>(smem + kSmemStat) + (i & 1) * 2 * kTile + half * 64;
    const float* delta = nl + kTile;
    bool ok = mbar_wait(&bars.stat_full[i & 1], (i >> 1) & 1, ctx, kRoleBwdSoftmax | kBarStat) &&
              mbar_wait(bars.s_full, i & 1, ctx, kRoleBwdSoftmax | kBarS);
    if (!__all_sync(0xffffffffu, ok)) return;
    tc_fence_after_sync();
    uint32_t x[64];
    tmem_ld_x32(t_s, x);
    tmem_ld_x32(t_s + 32, x + 32);
    tmem_wait_ld();
    // columns of this half from `hidden` on see the key; the others do not
    const int q0 = tile * kTile + half * 64;
    const int hidden = p.causal ? it.row0 + row - p.off - q0 : 0;
    const bool masked = p.causal && it.row0 + kTile - 1 > tile * kTile + p.off;  // CTA-uniform
#pragma unroll
    for (int cc = 0; cc < 2; ++cc) {
      uint32_t pk[16];
#pragma unroll
      for (int pr = 0; pr < 16; ++pr) {
        const int e = cc * 32 + pr * 2;
        const float2 n2 = *reinterpret_cast<const float2*>(nl + e);
        const float2 y = fma2(make_float2(ATTN_F(x, e), ATTN_F(x, e + 1)), c2, n2);
        float2 w = (pr & 7) < kExp2PolyPairs ? exp2_poly2(y) : make_float2(ex2_approx(y.x), ex2_approx(y.y));
        if (masked) {
          if (e < hidden) w.x = 0.f;
          if (e + 1 < hidden) w.y = 0.f;
        }
        x[e] = __float_as_uint(w.x);
        x[e + 1] = __float_as_uint(w.y);
        pk[pr] = pack_bf16x2(w.x, w.y);
      }
      tmem_st_x16(t_s + cc * 16, pk);
    }
    tmem_wait_st();
    tc_fence_before_sync();
    __syncwarp();
    if (lane == 0) mbar_arrive(&bars.p_full[half]);
    ok = mbar_wait(&bars.dp_full[0], i & 1, ctx, kRoleBwdSoftmax | kBarDp);
    if (!__all_sync(0xffffffffu, ok)) return;
    tc_fence_after_sync();
    uint32_t pk[32];
#pragma unroll
    for (int cc = 0; cc < 2; ++cc) {
      uint32_t d[32];
      tmem_ld_x32(t_dp + cc * 32, d);
      tmem_wait_ld();
#pragma unroll
      for (int pr = 0; pr < 16; ++pr) {
        const int e = cc * 32 + pr * 2;
        const float2 dl = *reinterpret_cast<const float2*>(delta + e);
        const float2 t = add2(make_float2(ATTN_F(d, pr * 2), ATTN_F(d, pr * 2 + 1)), make_float2(-dl.x, -dl.y));
        const float2 w = mul2(make_float2(ATTN_F(x, e), ATTN_F(x, e + 1)), t);
        pk[cc * 16 + pr] = pack_bf16x2(w.x, w.y);
      }
    }
    // dS overwrites the first 32 of this half's own 64 columns, all of which are in registers by now
    tmem_st_x32(t_dp, pk);
    tmem_wait_st();
    tc_fence_before_sync();
    __syncwarp();
    if (lane == 0) mbar_arrive(&bars.ds_full[half]);
    if (++tile == it.first + it.per_head) tile = it.first;
  }
  // Epilogue: half 0 stores dV (through V's tile in shared memory), half 1 dK (through K's); no product reads them now.
  bool ok = mbar_wait(bars.acc_full, 0, ctx, kRoleBwdSoftmax | kBarAcc);
  if (!__all_sync(0xffffffffu, ok)) return;
  tc_fence_after_sync();
  uint8_t* stage = smem + kSmemFixed + (half == 0 ? kTileBytes : 0);
  const uint32_t t_acc = tmem + lane_sel + (half == 0 ? kTmDv : kTmDk);
  const float factor = half == 0 ? 1.f : p.scale;
#pragma unroll
  for (int cc = 0; cc < 4; ++cc) {
    uint32_t o[32];
    tmem_ld_x32(t_acc + cc * 32, o);
    tmem_wait_ld();
    stage_row32(stage + (cc >> 1) * kHalfBytes, row, (cc & 1) * 4, o, factor);
  }
  fence_proxy_async_smem();
  __syncwarp();
  if (lane == 0) mbar_arrive(&bars.stage_full[half]);
  if (row == 0 && mbar_wait(&bars.stage_full[half], 0, ctx, kRoleBwdSoftmax | kBarStage)) {
    const CUtensorMap* tm = half == 0 ? tm_dv : tm_dk;
    tma_store_4d(tm, stage, 0, it.h, it.row0, it.b);
    tma_store_4d(tm, stage + kHalfBytes, 64, it.h, it.row0, it.b);
    tma_store_commit();
    tma_store_wait_all0();
  }
}

__device__ __forceinline__ void query_softmax(const BwdParams& p, const BwdItem& it, const BwdBarriers& bars, uint8_t* smem,
                                              WaitCtx ctx, uint32_t tmem, int half, int row, int lane,
                                              const CUtensorMap* tm_dq) {
  const uint32_t lane_sel = static_cast<uint32_t>(row & ~31) << 16;
  const uint32_t t_s = tmem + lane_sel + kTmS + half * 64;
  const float2 c2 = make_float2(p.scale_log2, p.scale_log2);
  const size_t at = (static_cast<size_t>(it.b) * p.Hq + it.h) * p.n_qt * kTile + it.row0 + row;
  const float nl = __ldg(p.neg_lse2 + at), dl = -__ldg(p.delta + at);
  const float2 nl2 = make_float2(nl, nl), dl2 = make_float2(dl, dl);
  const int row_limit = p.causal ? min(p.Sk, it.row0 + row + p.off + 1) : p.Sk;   // keys this row may see
  const int tile_clear = p.causal ? min(p.Sk, it.row0 + p.off + 1) : p.Sk;        // keys every row of the tile sees
  for (int j = 0; j < it.n; ++j) {
    bool ok = mbar_wait(bars.s_full, j & 1, ctx, kRoleBwdSoftmax | kBarS);
    if (!__all_sync(0xffffffffu, ok)) return;
    tc_fence_after_sync();
    uint32_t x[64];
    tmem_ld_x32(t_s, x);
    tmem_ld_x32(t_s + 32, x + 32);
    tmem_wait_ld();
    tc_fence_before_sync();
    __syncwarp();
    if (lane == 0) mbar_arrive(bars.s_read);
    const int visible = row_limit - j * kTile - half * 64;  // columns of this half the row sees
    const bool masked = (j + 1) * kTile > tile_clear;       // CTA-uniform
#pragma unroll
    for (int pr = 0; pr < 32; ++pr) {
      const int e = pr * 2;
      const float2 y = fma2(make_float2(ATTN_F(x, e), ATTN_F(x, e + 1)), c2, nl2);
      float2 w = (pr & 7) < kExp2PolyPairs ? exp2_poly2(y) : make_float2(ex2_approx(y.x), ex2_approx(y.y));
      if (masked) {  // also keys beyond Sk, whose scores are 0 and whose exp2(nl) may be infinite
        if (e >= visible) w.x = 0.f;
        if (e + 1 >= visible) w.y = 0.f;
      }
      x[e] = __float_as_uint(w.x);
      x[e + 1] = __float_as_uint(w.y);
    }
    ok = mbar_wait(&bars.dp_full[j & 1], (j >> 1) & 1, ctx, kRoleBwdSoftmax | kBarDp);
    if (!__all_sync(0xffffffffu, ok)) return;
    tc_fence_after_sync();
    const uint32_t t_dp = tmem + lane_sel + ((j & 1) ? kTmDp1 : kTmDp) + half * 64;
    uint32_t pk[32];
#pragma unroll
    for (int cc = 0; cc < 2; ++cc) {
      uint32_t d[32];
      tmem_ld_x32(t_dp + cc * 32, d);
      tmem_wait_ld();
#pragma unroll
      for (int pr = 0; pr < 16; ++pr) {
        const int e = cc * 32 + pr * 2;
        const float2 t = add2(make_float2(ATTN_F(d, pr * 2), ATTN_F(d, pr * 2 + 1)), dl2);
        const float2 w = mul2(make_float2(ATTN_F(x, e), ATTN_F(x, e + 1)), t);
        pk[cc * 16 + pr] = pack_bf16x2(w.x, w.y);
      }
    }
    tmem_st_x32(t_dp, pk);
    tmem_wait_st();
    tc_fence_before_sync();
    __syncwarp();
    if (lane == 0) mbar_arrive(&bars.ds_full[(j & 1) * 2 + half]);
  }
  // Epilogue: each half stores its 64 columns of dQ through its half of Q's tile.
  bool ok = mbar_wait(bars.acc_full, 0, ctx, kRoleBwdSoftmax | kBarAcc);
  if (!__all_sync(0xffffffffu, ok)) return;
  tc_fence_after_sync();
  uint8_t* stage = smem + kSmemFixed + half * kHalfBytes;
#pragma unroll
  for (int cc = 0; cc < 2; ++cc) {
    uint32_t o[32];
    if (it.n > 0) {
      tmem_ld_x32(tmem + lane_sel + kTmDq + half * 64 + cc * 32, o);
      tmem_wait_ld();
    } else {  // no row of the tile sees a key: dQ is 0, and tensor memory holds nothing of ours
#pragma unroll
      for (int e = 0; e < 32; ++e) o[e] = 0u;
    }
    stage_row32(stage, row, cc * 4, o, p.scale);
  }
  fence_proxy_async_smem();
  __syncwarp();
  if (lane == 0) mbar_arrive(&bars.stage_full[half]);
  if (row == 0 && mbar_wait(&bars.stage_full[half], 0, ctx, kRoleBwdSoftmax | kBarStage)) {
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
  bars.ring_full = bars.fixed_full + 1;
  bars.ring_empty = bars.ring_full + kRingSlots;
  bars.stat_full = bars.ring_empty + kRingSlots;
  bars.s_full = bars.stat_full + kStatStages;
  bars.s_read = bars.s_full + 1;
  bars.dp_full = bars.s_read + 1;
  bars.p_full = bars.dp_full + 2;
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
    mbar_init(bars.fixed_full, 1);
    for (int i = 0; i < kRingSlots; ++i) {
      mbar_init(&bars.ring_full[i], 1);
      mbar_init(&bars.ring_empty[i], 1);
    }
    mbar_init(bars.s_full, 1);
    mbar_init(bars.s_read, 8);
    mbar_init(bars.acc_full, 1);
    for (int i = 0; i < 2; ++i) {
      mbar_init(&bars.stat_full[i], 1);
      mbar_init(&bars.dp_full[i], 1);
      mbar_init(&bars.p_full[i], 4);
      mbar_init(&bars.ds_full[i], 4);
      mbar_init(&bars.ds_full[2 + i], 4);
      mbar_init(&bars.stage_full[i], 4);
    }
    *abort_flag = 0;
    fence_mbar_init();
  }
  if (warp == 8) {
    tmem_alloc(tmem_slot, 512);
    tmem_relinquish();
  }
  tc_fence_before_sync();
  __syncthreads();
  tc_fence_after_sync();
  const uint32_t tmem = *tmem_slot;
  const bool keys = static_cast<int>(blockIdx.x) < p.n_key_items;  // CTA-uniform
  const BwdItem it = keys ? key_item(p, blockIdx.x) : query_item(p, static_cast<int>(blockIdx.x) - p.n_key_items);

  if (warp < 8) {
    if (keys) {
      key_softmax(p, it, bars, smem, ctx, tmem, warp >> 2, tid & 127, lane, &tm_dk, &tm_dv);
    } else {
      query_softmax(p, it, bars, smem, ctx, tmem, warp >> 2, tid & 127, lane, &tm_dq);
    }
  } else if (warp == 8) {
    if (keys) {
      key_mma(it, bars, smem, ctx, tmem);
    } else {
      query_mma(it, bars, smem, ctx, tmem);
    }
  } else if (lane == 0) {
    if (keys) {
      bwd_loader<true>(p, it, bars, smem, ctx, &tm_q, &tm_k, &tm_v, &tm_do);
    } else {
      bwd_loader<false>(p, it, bars, smem, ctx, &tm_q, &tm_k, &tm_v, &tm_do);
    }
    if (*abort_flag) {  // let loads in flight land before the CTA's shared memory is released
      const uint64_t t0 = global_timer_ns();
      while (global_timer_ns() - t0 < 1000000ull) {
      }
    }
  }
  tc_fence_before_sync();
  __syncthreads();
  if (warp == 8) {
    tc_fence_after_sync();
    tmem_dealloc(tmem, 512);
  }
}

// Row statistics of the backward pass: -LSE log2(e) and delta = sum_d dO O - dLSE, one half warp per
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
                     float* __restrict__ delta, int Hq, int Sq, int padded, long long n_rows) {
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
      delta[at] = none ? 0.f : acc - dl;
    }
  }
}

#undef ATTN_F

}  // namespace bwd
}  // namespace attn
