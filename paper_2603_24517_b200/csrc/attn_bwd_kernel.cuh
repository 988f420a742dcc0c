// Attention backward for sm_100a.  With S = scale Q K^T, P = exp(S - LSE) (0 where masked) and
// delta_i = sum_d dO_id O_id - dLSE_i, the gradients are
//
//     dV = P^T dO,   dP = dO V^T,   dS = P o (dP - delta),   dQ = scale dS K,   dK = scale dS^T Q.
//
// P is recomputed from Q, K and LSE tile by tile.  Two kinds of work items in one launch, so that every sum
// has one owner and a fixed order (no atomics, the same bits on every run):
//
//   key items    one 128-key tile of one KV head: K and V stay in shared memory, the query tiles (Q, dO) of
//                every query head that shares the KV head stream past, dK and dV accumulate in tensor memory
//                (products per tile pair: K Q^T, V dO^T, P^T dO, dS^T Q);
//   query items  one 128-row query tile of one head: Q and dO stay, the K / V tiles stream past, dQ accumulates
//                in tensor memory (products per tile pair: Q K^T, dO V^T, dS K).
//
// That is seven products where five would do if dQ were added up across key tiles, but those additions would
// either come in any order or wait for one another.  A long item of a problem with few tiles can be split along its
// stream; its parts leave fp32 partial sums that attn_bwd_join_kernel adds up in order.
//
// One CTA per SM (640 threads) works through items: the grid has a CTA per item, and a running CTA takes over CTAs
// that have not started yet (clusterlaunchcontrol), so the hardware's own queue balances the work and nothing is
// left in memory between launches.  Roles:
//
//   warps 0-15  softmax: lane quarter w % 4 of the tile, 16 columns of each half of it (part w / 4); four threads a row.
//               All warps do their share of the first half, hand it over, and do the second while the product that
//               reads the first already runs.  Also the accumulators' way out (tensor memory -> BF16 -> shared memory)
//   warps 16-17 MMA issue (tcgen05.mma by an elected lane).  Barrier polls and commits take a warp longer than the few
//               instructions that the tensor pipe queues behind an issuer last, so one warp alone leaves the pipe
//               idle; two warps feed it by turns.  Products that must keep an order share a warp:
//               16: scores and the products that read P (key items) or dS (query items); 17: dP, and dK
//   warp  18    loader (TMA).  Stream A (Q or K), whose tiles are read by the first and the last product of a pair, has
//               a ring of three 32 KB tiles, stream B (dO or V) one of two; it also fetches the next item
//   warp  19    TMA stores of the results
//
// The results are staged in ring slots, which the loader sets aside at the end of an item, so the next
// item's tiles are already on their way while the results leave.
//
// Transposed tiles in key items (rows are keys) let P^T and dS^T go back to tensor memory as the left
// operand of the second products, so nothing is transposed through shared memory.
//
// Precision: every sum is fp32; P and dS are rounded to BF16 as operands, which adds to a result about as much as its own
// rounding does: 0.0024 of it, where that one alone is 0.0017.  In sums of few terms the rounding of one weight shows in
// full (up to 0.0037); for such problems (kFine) P and dS are handed over as the sum of two BF16 numbers, with a second
// product each, and 0.0017 is left.
#pragma once

#include "attn_fwd_kernel.cuh"

namespace attn {
namespace bwd {

constexpr int kParts = 4;                 // softmax threads per row
constexpr int kCols = kTile / kParts / 2; // columns of each half tile that each of them handles
constexpr int kSoftmaxWarps = 4 * kParts;
constexpr int kBwdThreads = (kSoftmaxWarps + 4) * 32;
// Registers a thread after the re-split (setmaxnreg): the block is launched with 96 each.
constexpr int kRegsSoftmax = 104, kRegsOther = 56;
static_assert(kSoftmaxWarps * kRegsSoftmax + 4 * kRegsOther <= kBwdThreads / 32 * 96, "register split");
constexpr int kRingA = 3, kRingB = 2;     // slots of the two streams: Q and dO, or K and V
constexpr int kRingSlots = kRingA + kRingB;
constexpr int kStatStages = 2;
constexpr int kStatBytes = kTile * 4;  // one fp32 value per query row of a tile

constexpr int kSmemFixed = 0;  // two resident tiles
constexpr int kSmemRing = 2 * kTileBytes;
constexpr int kSmemStat = kSmemRing + kRingSlots * kTileBytes;  // [kStatStages][2][128]: -LSE log2(e), -delta
constexpr int kSmemBwdBars = kSmemStat + kStatStages * 2 * kStatBytes;
constexpr int kBwdBars = 4 + 2 * kRingSlots + 2 * kStatStages + 2 + 1 + 1 + 2 + 4 + 2 + 1 + 2 + 4 + 2;
constexpr int kItemInts = 12;
constexpr int kSmemBwdClc = (kSmemBwdBars + kBwdBars * 8 + 15) / 16 * 16;  // [2] 16-byte answers of the launch queue
constexpr int kSmemBwdItems = kSmemBwdClc + 32;                            // [2][kItemInts] mailbox of work items
constexpr int kSmemBwdMisc = kSmemBwdItems + 2 * kItemInts * 4;            // tensor memory base, abort flag
constexpr int kSmemBwdBytes = kSmemBwdMisc + 8;
static_assert(kSmemBwdBytes <= 232448, "shared memory budget of one CTA");

// Packed query tiles (short query sequences of GQA groups): a tile's 128 rows hold 128 >> pack_log2 query rows of all
// 1 << pack_log2 heads of a group, row r being query row r >> pack_log2 of head r % group.  To everything but the masks
// and the addresses of query tiles that is a problem with Hq = Hkv and Sq << pack_log2 rows; Hq, group, Sq and
// n_qt below describe it as such.
struct BwdParams {
  int B, Hq, Hkv, Sq, Sk;
  int group;              // Hq / Hkv
  int pack_log2;
  int causal;
  int off;                // keys minus query rows: key j is visible to query row i (a tile's row >> pack_log2) iff j <= i + off
  int n_qt, n_kt;         // 128-row query tiles, 128-key tiles
  int key_splits, qry_splits;  // parts of a key / query item's stream
  int n_items;            // B * Hkv * (n_kt * key_splits + group * n_qt * qry_splits)
  int run, run_extra;     // launch order, see decode_item
  int queries_first;      // in a run: 1: query items before key items
  float scale, scale_log2;
  const float* neg_lse2;  // [B * Hq][n_qt * 128], -LSE * log2(e); -inf in rows that see no key or do not exist
  const float* neg_delta; // same layout, -delta, 0 in those rows
  float *dq_part, *dk_part, *dv_part;  // fp32 partial sums of split items, [split][head of the batch][padded rows][128]
  int* status;
};

// codes of expired waits: role << 8 | barrier (roles continue the forward kernels' numbering)
enum : int {
  kRoleBwdLoad = 10 << 8, kRoleBwdMma = 11 << 8, kRoleBwdSoftmax = 12 << 8, kRoleBwdStore = 13 << 8, kRoleBwdMma2 = 14 << 8,
  kBarFixed = 1, kBarRingFull = 2, kBarRingEmpty = 3, kBarStat = 4, kBarStatEmpty = 5, kBarS = 6, kBarDp = 7,
  kBarDpRead = 8, kBarP = 9, kBarDs = 10, kBarAcc = 11, kBarAccEmpty = 12, kBarStageFree = 13, kBarStage = 14, kBarItem = 15,
  kBarItemEmpty = 16, kBarClc = 17, kBarFixedEmpty = 18
};

struct BwdBarriers {
  uint64_t* fixed_full;  // [2]  loader (TMA) -> MMA: K or Q, V or dO
  uint64_t* fixed_empty; // [2]  MMA commit after an item's last use -> loader
  uint64_t* a_full;      // [kRingA]  loader (TMA) -> MMA
  uint64_t* a_empty;     // [kRingA]  two MMA commits, one for each product that reads the tile -> loader
  uint64_t* b_full;      // [kRingB]
  uint64_t* b_empty;     // [kRingB]
  uint64_t* stat_full;   // [kStatStages]  loader (bulk copy) -> softmax (key items)
  uint64_t* stat_empty;  // [kStatStages]  softmax (all warps) -> loader
  uint64_t* s_full;      // [2]  MMA commit -> softmax (key items use the first)
  uint64_t* dp_full;     // MMA commit -> softmax
  uint64_t* dp_read;     // softmax (all warps) -> MMA: dP is in registers (query items)
  uint64_t* p_full;      // [2]  softmax (all warps): a half tile's columns of P are in tensor memory (key items)
  uint64_t* ds_full;     // [4]  the same for dS; query items alternate two pairs, one for each score buffer
  uint64_t* acc_full;    // commits of both MMA warps: the accumulators are final
  uint64_t* acc_empty;   // softmax (all warps) -> MMA: they are in registers
  uint64_t* stage_free;  // store warp -> softmax: it has come to this item (keeps them from running further ahead)
  uint64_t* stage_full;  // [2]  softmax warps of a half tile -> store warp
  uint64_t* item_full;   // [2]  loader -> everybody else: the next item is in the mailbox
  uint64_t* item_empty;  // [2]
  uint64_t* clc_full;    // [2]  the launch queue's answer has arrived
};

// Untiled copy of `bytes` (a multiple of 16) from global to shared memory, counted on `bar`.
__device__ __forceinline__ void bulk_load(void* smem_dst, const void* src, uint32_t bytes, uint64_t* bar) {
  asm volatile("cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];" ::"r"(
                   smem_u32(smem_dst)),
               "l"(reinterpret_cast<uint64_t>(src)), "r"(bytes), "r"(smem_u32(bar))
               : "memory");
}

// The launch queue: asks for a CTA that has not started yet (16-byte answer, counted on `bar`), and reads the answer:
// the index of the CTA taken over, or -1 if none is left.
__device__ __forceinline__ void clc_request(void* answer, uint64_t* bar) {
  asm volatile("clusterlaunchcontrol.try_cancel.async.shared::cta.mbarrier::complete_tx::bytes.b128 [%0], [%1];" ::"r"(
                   smem_u32(answer)),
               "r"(smem_u32(bar))
               : "memory");
}
__device__ __forceinline__ int clc_answer(const void* answer) {
  uint32_t got, x;
  asm volatile(
      "{\n\t"
      ".reg .pred p;\n\t"
      ".reg .b128 r;\n\t"
      "ld.shared.b128 r, [%2];\n\t"
      "mov.u32 %1, 0;\n\t"
      "clusterlaunchcontrol.query_cancel.is_canceled.pred.b128 p, r;\n\t"
      "selp.u32 %0, 1, 0, p;\n\t"
      "@p clusterlaunchcontrol.query_cancel.get_first_ctaid::x.b32.b128 %1, r;\n\t"
      "}\n"
      : "=&r"(got), "=&r"(x)  // no output may share the address's register
      : "r"(smem_u32(answer))
      : "memory");
  return got != 0 ? static_cast<int>(x) : -1;
}

// A work item: the tile it owns and the tiles that stream past it.  Streamed tile t (t0 <= t < t0 + n) is tile
// first + t % per_head of the t / per_head-th head of the group (key items), or tile t (query items).
struct BwdItem {
  int keys;         // 1: key item, 0: query item
  int b, h;         // batch entry; KV head (key item) or query head (query item)
  int row0;         // first key / query row of the owned tile
  int first, per_head;
  int t0, n;        // n = 0: nothing streams past, the result is 0
  int split;        // which part of the stream this is, of key_splits / qry_splits
};

// Launch order.  A unit is a (batch, KV head) with its query heads: n_kt key tiles and group * n_qt query tiles, each
// in its number of parts.  Units are taken in runs of `run` (the first `run_extra` runs) or run - 1 units whose
// tensors together fit L2; in a run come first all items of the kind with the longer streams, then all of the other.  Under the causal mask each kind
// goes rank by rank over the run's units, longest ranks (early keys, late rows) first, so that a run ends on
// short items.  Without it items are alike and go unit by unit: neighbours then read the same stream at about the same
// time, which the L2 answers with fewer requests (8 heads of 16384: 3 % over a mixed order).
__host__ __device__ __forceinline__ BwdItem decode_item(const BwdParams& p, int w) {
  const int unit_keys = p.n_kt * p.key_splits;
  const int per_unit = unit_keys + p.group * p.n_qt * p.qry_splits;
  const int big = p.run * per_unit;
  int first, g, rem;
  if (w < p.run_extra * big) {
    first = w / big;
    rem = w - first * big;
    first *= p.run;
    g = p.run;
  } else {
    const int small = big - per_unit;
    const int n = (w - p.run_extra * big) / small;
    rem = (w - p.run_extra * big) - n * small;
    first = p.run_extra * p.run + n * (p.run - 1);
    g = p.run - 1;
  }
  BwdItem it;
  const int run_keys = g * unit_keys, run_queries = g * (per_unit - unit_keys);
  it.keys = (p.queries_first ? rem >= run_queries : rem < run_keys) ? 1 : 0;
  if (p.queries_first && it.keys) rem -= run_queries;
  if (!p.queries_first && !it.keys) rem -= run_keys;
  int splits;
  if (it.keys) {
    splits = p.key_splits;
    const int u = p.causal ? rem % g : rem / unit_keys;
    const int rank = p.causal ? rem / g : rem - u * unit_keys, unit = first + u;
    const int kt = rank / splits;
    it.split = rank - kt * splits;
    it.b = unit / p.Hkv;
    it.h = unit - it.b * p.Hkv;
    it.row0 = kt * kTile;
    const int first_row = p.causal && it.row0 > p.off ? (it.row0 - p.off) << p.pack_log2 : 0;  // < Sq: the last row sees all
    it.first = first_row / kTile;
    it.per_head = p.n_qt - it.first;
    it.n = it.per_head * p.group;
  } else {
    splits = p.qry_splits;
    const int wide = g * p.group, per_head = p.n_qt * splits;
    const int x = p.causal ? rem % wide : rem / per_head;  // which head of the run
    const int rank = p.causal ? rem / wide : rem - x * per_head;
    const int unit = first + x / p.group;
    const int qt = rank / splits;
    it.split = rank - qt * splits;
    it.b = unit / p.Hkv;
    it.h = (unit - it.b * p.Hkv) * p.group + x % p.group;
    it.row0 = (p.causal ? p.n_qt - 1 - qt : qt) * kTile;
    it.first = 0;
    it.per_head = p.n_kt;
    if (p.causal) {
      const int row_end = it.row0 + kTile < p.Sq ? it.row0 + kTile : p.Sq;
      const int last_key = ((row_end - 1) >> p.pack_log2) + p.off;
      const int need = last_key < 0 ? 0 : last_key / kTile + 1;
      if (need < it.per_head) it.per_head = need;
    }
    it.n = it.per_head;
  }
  it.t0 = 0;
  if (splits > 1) {  // equal parts of this item's own stream
    const long long n = it.n;
    it.t0 = static_cast<int>(n * it.split / splits);
    it.n = static_cast<int>(n * (it.split + 1) / splits) - it.t0;
  }
  return it;
}
// Whether the item's result goes out as BF16 through a staging slot (else as an fp32 partial sum).
__device__ __forceinline__ bool staged(const BwdParams& p, const BwdItem& it) {
  return (it.keys ? p.key_splits : p.qry_splits) == 1;
}

__device__ __forceinline__ void put_item(volatile int* slot, const BwdItem& it) {
  slot[1] = it.keys; slot[2] = it.b; slot[3] = it.h; slot[4] = it.row0; slot[5] = it.first; slot[6] = it.per_head;
  slot[7] = it.t0; slot[8] = it.n; slot[9] = it.split;
}

// Item number k of this CTA for a consuming warp: false when there are no more, or after an expired wait.  One
// arrival per warp hands the mailbox slot back.
__device__ __forceinline__ bool next_item(const BwdBarriers& bars, const volatile int* box, int k, WaitCtx ctx, int role,
                                          bool whole_warp, bool arrives, BwdItem& it) {
  bool ok = mbar_wait(&bars.item_full[k & 1], (k >> 1) & 1, ctx, role | kBarItem);
  if (whole_warp) ok = __all_sync(0xffffffffu, ok);
  if (!ok) return false;
  const int* slot = const_cast<const int*>(box) + (k & 1) * kItemInts;
  const int valid = slot[0];
  it.keys = slot[1]; it.b = slot[2]; it.h = slot[3]; it.row0 = slot[4]; it.first = slot[5]; it.per_head = slot[6];
  it.t0 = slot[7]; it.n = slot[8]; it.split = slot[9];
  if (whole_warp) __syncwarp();
  if (arrives) mbar_arrive(&bars.item_empty[k & 1]);
  return valid != 0;
}
constexpr int kItemConsumers = kSoftmaxWarps + 3;  // softmax warps, MMA warps, store warp

// D[128 x 128] (+)= A[tmem] B for one half (64) of the contraction rows.  A (BF16) was written over fp32 columns, by each
// softmax thread over the first half of its own 16 (kFine: and what that rounding left over the second half); B is
// MN-major (16 contraction rows are 2048 bytes).
template <bool kFine>
__device__ __forceinline__ void issue_ts_half(bool leader, uint32_t tmem_d, uint32_t tmem_a, uint64_t b_desc, int half,
                                              bool accumulate) {
  if (leader) {
#pragma unroll
    for (int kk = 0; kk < 4; ++kk) {
      mma_ts(tmem_d, tmem_a + half * 64 + kk * kCols, desc_advance(b_desc, (half * 4 + kk) * 2048), kIdescPV,
             (accumulate || kk > 0) ? 1u : 0u);
      if (kFine) {
        mma_ts(tmem_d, tmem_a + half * 64 + kk * kCols + kCols / 2, desc_advance(b_desc, (half * 4 + kk) * 2048), kIdescPV, 1u);
      }
    }
  }
}

// Tensor memory columns.  Key items: S (then P over it), dP (then dS over it), dV, dK.  Query items: two score buffers
// (dS over the scores it comes from), dP, dQ.
constexpr uint32_t kTmS = 0, kTmDp = kTile, kTmDv = 2 * kTile, kTmDk = 3 * kTile;
constexpr uint32_t kTmQryS = 0, kTmQryDp = 2 * kTile, kTmDq = 3 * kTile;  // score buffer j % 2 at kTmQryS + (j % 2) * kTile

__device__ __forceinline__ void load_tile(uint8_t* dst, const CUtensorMap* tm, uint64_t* bar, int head, int row, int b) {
  tma_load_4d(dst, tm, bar, 0, head, row, b);
  tma_load_4d(dst + kHalfBytes, tm, bar, 64, head, row, b);
}

// A position in a ring of N slots: the slot and the parity of its current phase.
template <int N>
struct RingPos {
  uint32_t slot = 0, par = 0;
  __device__ __forceinline__ void next() {
    if (++slot == N) {
      slot = 0;
      par ^= 1u;
    }
  }
  __device__ __forceinline__ void skip(uint32_t n) {
    const uint32_t c = (par * N + slot + n) % (2 * N);
    par = c >= N ? 1u : 0u;
    slot = c - par * N;
  }
};
typedef RingPos<kRingA> RingPosA;
typedef RingPos<kRingB> RingPosB;

// The loader's counts: ring positions, resident tiles, statistics tiles so far.
struct LoaderState {
  RingPosA a;
  RingPosB b;
  uint32_t fixed = 0, stats = 0;
};

// One item's tiles: the resident ones, then the streams, pair by pair; key items' stream A also brings the row
// statistics of its tiles.  False after an expired wait.
__device__ __forceinline__ bool load_item(const BwdParams& p, const BwdItem& it, const BwdBarriers& bars, uint8_t* smem,
                                          WaitCtx ctx, const CUtensorMap* fixed_a, const CUtensorMap* fixed_b,
                                          const CUtensorMap* stream_a, const CUtensorMap* stream_b, LoaderState& ls,
                                          void* clc_buf, uint64_t* clc_bar) {
  uint8_t* ring_a = smem + kSmemRing;
  uint8_t* ring_b = ring_a + kRingA * kTileBytes;
  // query tiles are addressed by the first of their heads and their first query row
  const int fixed_pack = it.keys ? 0 : p.pack_log2, stream_pack = it.keys ? p.pack_log2 : 0;
  const int head0 = it.keys ? it.h * p.group : it.h / p.group;
  int head = head0 + it.t0 / (it.per_head > 0 ? it.per_head : 1);
  int tile = it.first + it.t0 - (head - head0) * it.per_head;
  for (int i = 0; i < it.n; ++i) {
#pragma unroll
    for (int x = 0; x < 2; ++x) {
      if (i == 0) {  // the resident tile of the product that comes first
        if (!mbar_wait(&bars.fixed_empty[x], (ls.fixed & 1) ^ 1, ctx, kRoleBwdLoad | kBarFixedEmpty)) return false;
        mbar_arrive_expect_tx(&bars.fixed_full[x], kTileBytes);
        load_tile(smem + kSmemFixed + x * kTileBytes, x == 0 ? fixed_a : fixed_b, &bars.fixed_full[x], it.h << fixed_pack,
                  it.row0 >> fixed_pack, it.b);
      }
      if (x == 0) {
        if (!mbar_wait(&bars.a_empty[ls.a.slot], ls.a.par ^ 1, ctx, kRoleBwdLoad | kBarRingEmpty)) return false;
        mbar_arrive_expect_tx(&bars.a_full[ls.a.slot], kTileBytes);
        load_tile(ring_a + ls.a.slot * kTileBytes, stream_a, &bars.a_full[ls.a.slot], head << stream_pack,
                  (tile * kTile) >> stream_pack, it.b);
        ls.a.next();
      } else {
        if (!mbar_wait(&bars.b_empty[ls.b.slot], ls.b.par ^ 1, ctx, kRoleBwdLoad | kBarRingEmpty)) return false;
        mbar_arrive_expect_tx(&bars.b_full[ls.b.slot], kTileBytes);
        load_tile(ring_b + ls.b.slot * kTileBytes, stream_b, &bars.b_full[ls.b.slot], head << stream_pack,
                  (tile * kTile) >> stream_pack, it.b);
        ls.b.next();
      }
    }
    if (it.keys) {
      const uint32_t st = ls.stats & 1;
      float* dst = reinterpret_cast<float*>(smem + kSmemStat) + st * 2 * kTile;
      const size_t at = (static_cast<size_t>(it.b) * p.Hq + head) * p.n_qt * kTile + static_cast<size_t>(tile) * kTile;
      if (!mbar_wait(&bars.stat_empty[st], ((ls.stats >> 1) & 1) ^ 1, ctx, kRoleBwdLoad | kBarStatEmpty)) return false;
      mbar_arrive_expect_tx(&bars.stat_full[st], 2 * kStatBytes);
      bulk_load(dst, p.neg_lse2 + at, kStatBytes, &bars.stat_full[st]);
      bulk_load(dst + kTile, p.neg_delta + at, kStatBytes, &bars.stat_full[st]);
      ++ls.stats;
    }
    if (++tile == it.first + it.per_head) {
      tile = it.first;
      ++head;
    }
  }
  if (it.n > 0) ++ls.fixed;
  // Ask for the next item only now that this one's last tiles are on their way (two tile pairs or so are still to be
  // computed, longer than the answer takes): a CTA that reserved it earlier would keep others from it.
  fence_proxy_async_smem();  // the answer this one overwrites was read through the generic proxy
  mbar_arrive_expect_tx(clc_bar, 16);
  clc_request(clc_buf, clc_bar);
  return true;
}
// The slots for the item's results.
__device__ __forceinline__ bool load_stage_slots(const BwdParams& p, const BwdItem& it, const BwdBarriers& bars, WaitCtx ctx,
                                                 LoaderState& ls) {
  if (staged(p, it)) {
    // The slots behind the last tiles take the results: the `full` barriers of these positions tell the softmax warps.
    if (!mbar_wait(&bars.a_empty[ls.a.slot], ls.a.par ^ 1, ctx, kRoleBwdLoad | kBarRingEmpty)) return false;
    mbar_arrive(&bars.a_full[ls.a.slot]);
    ls.a.next();
    if (it.keys) {
      if (!mbar_wait(&bars.b_empty[ls.b.slot], ls.b.par ^ 1, ctx, kRoleBwdLoad | kBarRingEmpty)) return false;
      mbar_arrive(&bars.b_full[ls.b.slot]);
      ls.b.next();
    }
  }
  return true;
}

__device__ __forceinline__ void role_loader(const BwdParams& p, const BwdBarriers& bars, uint8_t* smem, volatile int* box,
                                            WaitCtx ctx, const CUtensorMap* tm_q, const CUtensorMap* tm_k,
                                            const CUtensorMap* tm_v, const CUtensorMap* tm_do) {
  LoaderState ls;
  BwdItem it = decode_item(p, static_cast<int>(blockIdx.x));
  put_item(box, it);
  box[0] = 1;
  mbar_arrive(&bars.item_full[0]);
  for (int k = 0;; ++k) {
    uint8_t* answer = smem + kSmemBwdClc + (k & 1) * 16;
    uint64_t* clc_bar = &bars.clc_full[k & 1];
    const bool ok = it.keys ? load_item(p, it, bars, smem, ctx, tm_k, tm_v, tm_q, tm_do, ls, answer, clc_bar)
                            : load_item(p, it, bars, smem, ctx, tm_q, tm_do, tm_k, tm_v, ls, answer, clc_bar);
    if (!ok || !mbar_wait(clc_bar, (k >> 1) & 1, ctx, kRoleBwdLoad | kBarClc)) return;
    const int w = clc_answer(answer);
    // the divisions of the next item's index, before the wait for slots that this item's last products hold
    const BwdItem coming = decode_item(p, w >= 0 ? w : 0);
    if (!load_stage_slots(p, it, bars, ctx, ls)) return;
    const int n = k + 1;
    if (!mbar_wait(&bars.item_empty[n & 1], ((n >> 1) & 1) ^ 1, ctx, kRoleBwdLoad | kBarItemEmpty)) return;
    volatile int* slot = box + (n & 1) * kItemInts;
    it = coming;
    if (w >= 0) put_item(slot, it);
    slot[0] = w >= 0 ? 1 : 0;
    mbar_arrive(&bars.item_full[n & 1]);
    if (w < 0) return;
  }
}

// For a wait that lasts as long as an item of `n` tile pairs: each of them (1.5 us or so) adds to the limit.
__device__ __forceinline__ WaitCtx whole_item(WaitCtx ctx, int n) {
  return WaitCtx{ctx.abort_flag, ctx.status, ctx.limit_ns + static_cast<uint64_t>(n) * 20000};
}

// TMA stores of the staged results; hands the slots back to the loader once they have been read.
__device__ __forceinline__ void role_store(const BwdParams& p, const BwdBarriers& bars, uint8_t* smem,
                                           const volatile int* box, WaitCtx ctx, const CUtensorMap* tm_dq,
                                           const CUtensorMap* tm_dk, const CUtensorMap* tm_dv) {
  uint32_t pos_a = 0, pos_b = 0, stores = 0;
  BwdItem it;
  int unstaged = 0;  // tile pairs of the item before, if this warp does nothing for it and waits until its tiles are loaded
  for (int k = 0; next_item(bars, box, k, whole_item(ctx, unstaged), kRoleBwdStore, false, true, it); ++k) {
    pos_a += it.n;
    pos_b += it.n;
    unstaged = staged(p, it) ? 0 : it.n;
    if (!staged(p, it)) continue;
    uint8_t* slot_a = smem + kSmemRing + (pos_a % kRingA) * kTileBytes;
    uint8_t* slot_b = smem + kSmemRing + (kRingA + pos_b % kRingB) * kTileBytes;
    mbar_arrive(bars.stage_free);
#pragma unroll
    for (int half = 0; half < 2; ++half) {
      if (!mbar_wait(&bars.stage_full[half], stores & 1, whole_item(ctx, it.n), kRoleBwdStore | kBarStage)) return;
      if (it.keys) {  // half 0: dV in stream B's slot, half 1: dK in stream A's
        const CUtensorMap* tm = half == 0 ? tm_dv : tm_dk;
        uint8_t* src = half == 0 ? slot_b : slot_a;
        tma_store_4d(tm, src, 0, it.h, it.row0, it.b);
        tma_store_4d(tm, src + kHalfBytes, 64, it.h, it.row0, it.b);
      } else {
        tma_store_4d(tm_dq, slot_a + half * kHalfBytes, half * 64, it.h << p.pack_log2, it.row0 >> p.pack_log2, it.b);
      }
      tma_store_commit();
    }
    ++stores;
    tma_store_wait_read0();
    // in the place of the two products that read a tile
    mbar_arrive(&bars.a_empty[pos_a % kRingA]);
    mbar_arrive(&bars.a_empty[pos_a % kRingA]);
    ++pos_a;
    if (it.keys) {
      mbar_arrive(&bars.b_empty[pos_b % kRingB]);
      mbar_arrive(&bars.b_empty[pos_b % kRingB]);
      ++pos_b;
    }
  }
}

// Shared-memory address of the tile at a ring position, and the wait for it.
__device__ __forceinline__ uint32_t tile_at(uint32_t base, const RingPosA& r) { return base + kSmemRing + r.slot * kTileBytes; }
__device__ __forceinline__ uint32_t tile_at(uint32_t base, const RingPosB& r) {
  return base + kSmemRing + (kRingA + r.slot) * kTileBytes;
}
__device__ __forceinline__ bool wait_tile(const BwdBarriers& bars, const RingPosA& r, WaitCtx ctx, int role) {
  return mbar_wait_warp(&bars.a_full[r.slot], r.par, ctx, role | kBarRingFull);
}
__device__ __forceinline__ bool wait_tile(const BwdBarriers& bars, const RingPosB& r, WaitCtx ctx, int role) {
  return mbar_wait_warp(&bars.b_full[r.slot], r.par, ctx, role | kBarRingFull);
}

// Phases of the barriers that count tile pairs across items; every role that waits for them keeps its own copy.
struct Phases {
  uint32_t s = 0;    // bit x: uses of score buffer x so far (s_full[x], ds_full[2 x], ds_full[2 x + 1])
  uint32_t dp = 0;   // tile pairs so far (dp_full)
  uint32_t key = 0;  // tile pairs of key items (p_full, stat_full, stat_empty)
  uint32_t qry = 0;  // tile pairs of query items (dp_read)
};

// What both MMA warps know of the item they work on.
struct MmaItem {
  uint32_t base, tmem;
  RingPosA a;                    // ring positions: of its first tiles, and behind its last ones afterwards
  RingPosB b;
  uint32_t fixed;                // resident tiles before it
  uint32_t k;                    // its number
  bool leader;
  bool after_other;              // the item before was of the other kind
};

// Key item, first MMA warp:  S(0) | P(i)^T dO(i), S(i+1) | ...    (S = K Q^T)
// Key item, second MMA warp: dP(0) | dS(i)^T Q(i), dP(i+1) | ...  (dP = V dO^T)
// P(i+1) is exponentiated beside the second warp's products, dS(i+1) is formed beside the first warp's.  P aliases the
// scores it comes from and dS the dP it comes from: a later product into the same columns is issued behind the one
// that reads them by the same warp, and the pipe executes in order.  Waits that are over early (the tiles) come while
// there is nothing to issue.  Across items the same order holds between items of one kind; products into columns that
// the item before used otherwise, and into its accumulators, wait until its results have left tensor memory
// (acc_empty).
template <bool kFine>
__device__ __forceinline__ bool key_mma_1(const BwdItem& it, MmaItem& m, const BwdBarriers& bars, WaitCtx ctx, Phases& ph) {
  constexpr int kRole = kRoleBwdMma;
  const uint64_t k_desc = kmajor_desc(m.base + kSmemFixed);
  if (!mbar_wait_warp(&bars.fixed_full[0], m.fixed & 1, ctx, kRole | kBarFixed) || !wait_tile(bars, m.a, ctx, kRole)) return false;
  tc_fence_after_sync();
  issue_qk(m.leader, m.tmem + kTmS, k_desc, kmajor_desc(tile_at(m.base, m.a)));
  if (m.leader) {
    mma_commit(&bars.s_full[0]);
    mma_commit(&bars.a_empty[m.a.slot]);
    if (it.n == 1) mma_commit(&bars.fixed_empty[0]);  // that was the last use of K
  }
  m.a.next();
  if (!mbar_wait_warp(bars.acc_empty, (m.k & 1) ^ 1, ctx, kRole | kBarAccEmpty)) return false;
  for (int i = 0; i < it.n; ++i) {
    const bool next = i + 1 < it.n;
    if (!wait_tile(bars, m.b, ctx, kRole)) return false;             // dO(i)
    if (next && !wait_tile(bars, m.a, ctx, kRole)) return false;     // Q(i + 1)
    const uint64_t do_desc = vtile_desc(tile_at(m.base, m.b));
    const uint64_t q_desc = kmajor_desc(tile_at(m.base, m.a));
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      if (!mbar_wait_warp(&bars.p_full[h], ph.key & 1, ctx, kRole | kBarP)) return false;
      tc_fence_after_sync();
      issue_ts_half<kFine>(m.leader, m.tmem + kTmDv, m.tmem + kTmS, do_desc, h, i > 0 || h > 0);
    }
    if (next) {
      issue_qk(m.leader, m.tmem + kTmS, k_desc, q_desc);
      if (m.leader) {
        mma_commit(&bars.s_full[0]);
        mma_commit(&bars.a_empty[m.a.slot]);
        if (i + 2 == it.n) mma_commit(&bars.fixed_empty[0]);
      }
      m.a.next();
    }
    if (m.leader) mma_commit(&bars.b_empty[m.b.slot]);
    m.b.next();
    ++ph.key;
  }
  ph.s ^= it.n & 1;  // the other warp waits for dS
  return true;
}
template <bool kFine>
__device__ __forceinline__ bool key_mma_2(const BwdItem& it, MmaItem& m, const BwdBarriers& bars, WaitCtx ctx, Phases& ph) {
  constexpr int kRole = kRoleBwdMma2;
  const uint64_t v_desc = kmajor_desc(m.base + kSmemFixed + kTileBytes);
  // dP's columns were a score buffer of a query item, which the first MMA warp's products read
  if (m.after_other && !mbar_wait_warp(bars.acc_empty, (m.k & 1) ^ 1, ctx, kRole | kBarAccEmpty)) return false;
  if (!mbar_wait_warp(&bars.fixed_full[1], m.fixed & 1, ctx, kRole | kBarFixed) || !wait_tile(bars, m.b, ctx, kRole)) return false;
  tc_fence_after_sync();
  issue_qk(m.leader, m.tmem + kTmDp, v_desc, kmajor_desc(tile_at(m.base, m.b)));
  if (m.leader) {
    mma_commit(bars.dp_full);
    mma_commit(&bars.b_empty[m.b.slot]);
    if (it.n == 1) mma_commit(&bars.fixed_empty[1]);  // that was the last use of V
  }
  m.b.next();
  if (!m.after_other && !mbar_wait_warp(bars.acc_empty, (m.k & 1) ^ 1, ctx, kRole | kBarAccEmpty)) return false;
  for (int i = 0; i < it.n; ++i) {
    const bool next = i + 1 < it.n;
    if (next && !wait_tile(bars, m.b, ctx, kRole)) return false;     // dO(i + 1)
    const uint64_t q_desc = vtile_desc(tile_at(m.base, m.a));        // Q(i): dS(i) comes from its scores
    const uint64_t do_desc = kmajor_desc(tile_at(m.base, m.b));
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      if (!mbar_wait_warp(&bars.ds_full[h], ph.s & 1, ctx, kRole | kBarDs)) return false;
      tc_fence_after_sync();
      issue_ts_half<kFine>(m.leader, m.tmem + kTmDk, m.tmem + kTmDp, q_desc, h, i > 0 || h > 0);
    }
    if (next) {
      issue_qk(m.leader, m.tmem + kTmDp, v_desc, do_desc);
      if (m.leader) {
        mma_commit(bars.dp_full);
        mma_commit(&bars.b_empty[m.b.slot]);
        if (i + 2 == it.n) mma_commit(&bars.fixed_empty[1]);
      }
      m.b.next();
    }
    if (m.leader) mma_commit(&bars.a_empty[m.a.slot]);
    m.a.next();
    ph.s ^= 1u;
  }
  return true;
}

// Query item, first MMA warp:  S(0), S(1) | dS(j) K(j), S(j+2) | ...  (S = Q K^T).  The scores of tile j + 1 are computed
// while tile j's are exponentiated: two score buffers, dS(j) goes over the scores of tile j, and S(j+2) into the same
// columns is issued behind dS(j) K(j).
// Second MMA warp: dP(j) = dO V(j)^T into one buffer, free as soon as the softmax warps have it in registers.
template <bool kFine>
__device__ __forceinline__ bool query_mma_1(const BwdItem& it, MmaItem& m, const BwdBarriers& bars, WaitCtx ctx, Phases& ph) {
  constexpr int kRole = kRoleBwdMma;
  const uint64_t q_desc = kmajor_desc(m.base + kSmemFixed);
  RingPosA done = m.a;  // position of K(j); m.a: of K(j + 2)
  if (!mbar_wait_warp(&bars.fixed_full[0], m.fixed & 1, ctx, kRole | kBarFixed)) return false;
  for (int j = -2; j < it.n; ++j) {
    const int n = j + 2;
    const uint32_t scores = m.tmem + kTmQryS + (n & 1) * kTile;  // buffer of tiles j and j + 2
    // buffer 1 was a key item's dP, which the second MMA warp's products read
    if (j == -1 && m.after_other && !mbar_wait_warp(bars.acc_empty, (m.k & 1) ^ 1, ctx, kRole | kBarAccEmpty)) return false;
    if (j >= 0) {  // dQ += dS(j) K(j)
      if (j == 0 && !m.after_other && !mbar_wait_warp(bars.acc_empty, (m.k & 1) ^ 1, ctx, kRole | kBarAccEmpty)) return false;
      const int x = j & 1;
      const uint64_t kv_desc = vtile_desc(tile_at(m.base, done));
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        if (!mbar_wait_warp(&bars.ds_full[2 * x + h], (ph.s >> x) & 1, ctx, kRole | kBarDs)) return false;
        tc_fence_after_sync();
        issue_ts_half<kFine>(m.leader, m.tmem + kTmDq, scores, kv_desc, h, j > 0 || h > 0);
      }
      if (m.leader) mma_commit(&bars.a_empty[done.slot]);
      done.next();
      ph.s ^= 1u << x;
    }
    if (n < it.n) {
      if (!wait_tile(bars, m.a, ctx, kRole)) return false;
      tc_fence_after_sync();
      issue_qk(m.leader, scores, q_desc, kmajor_desc(tile_at(m.base, m.a)));
      if (m.leader) {
        mma_commit(&bars.s_full[n & 1]);
        mma_commit(&bars.a_empty[m.a.slot]);
        if (n + 1 == it.n) mma_commit(&bars.fixed_empty[0]);
      }
      m.a.next();
    }
  }
  m.b.skip(it.n);
  return true;
}
__device__ __forceinline__ bool query_mma_2(const BwdItem& it, MmaItem& m, const BwdBarriers& bars, WaitCtx ctx, Phases& ph) {
  constexpr int kRole = kRoleBwdMma2;
  const uint64_t do_desc = kmajor_desc(m.base + kSmemFixed + kTileBytes);
  if (!mbar_wait_warp(&bars.fixed_full[1], m.fixed & 1, ctx, kRole | kBarFixed) ||
      !mbar_wait_warp(bars.acc_empty, (m.k & 1) ^ 1, ctx, kRole | kBarAccEmpty))
    return false;
  for (int j = 0; j < it.n; ++j) {
    if (!wait_tile(bars, m.b, ctx, kRole)) return false;
    if (j > 0) {  // dP(j - 1) has been read
      if (!mbar_wait_warp(bars.dp_read, ph.qry & 1, ctx, kRole | kBarDpRead)) return false;
      ++ph.qry;
    }
    tc_fence_after_sync();
    issue_qk(m.leader, m.tmem + kTmQryDp, do_desc, kmajor_desc(tile_at(m.base, m.b)));
    if (m.leader) {
      mma_commit(bars.dp_full);
      mma_commit(&bars.b_empty[m.b.slot]);
      mma_commit(&bars.b_empty[m.b.slot]);  // the tile's only reader stands for two
      if (j + 1 == it.n) mma_commit(&bars.fixed_empty[1]);
    }
    m.b.next();
  }
  ++ph.qry;  // the last tile's phase: over by the time that the next item gets past acc_empty
  ph.s ^= (((it.n + 1) >> 1) & 1) | (((it.n >> 1) & 1) << 1);  // the other warp waits for dS
  m.a.skip(it.n);
  return true;
}

template <bool kFirst, bool kFine>
__device__ __forceinline__ void role_mma(const BwdParams& p, const BwdBarriers& bars, uint8_t* smem, const volatile int* box,
                                         WaitCtx ctx, uint32_t tmem, int lane) {
  constexpr int kRole = kFirst ? kRoleBwdMma : kRoleBwdMma2;
  MmaItem m;
  m.base = smem_u32(smem);
  m.tmem = tmem;
  m.fixed = 0;
  m.leader = elect_one();
  Phases ph;
  BwdItem it;
  int kind_before = -1;
  for (int k = 0; next_item(bars, box, k, ctx, kRole, true, lane == 0, it); ++k) {
    m.k = k;
    m.after_other = k > 0 && it.keys != kind_before;
    if (it.n > 0) {
      bool ok;
      if (kFirst) {
        ok = it.keys ? key_mma_1<kFine>(it, m, bars, ctx, ph) : query_mma_1<kFine>(it, m, bars, ctx, ph);
      } else {
        ok = it.keys ? key_mma_2<kFine>(it, m, bars, ctx, ph) : query_mma_2(it, m, bars, ctx, ph);
      }
      if (!ok) return;
      ++m.fixed;
      kind_before = it.keys;
    } else if (!mbar_wait_warp(bars.acc_empty, (k & 1) ^ 1, ctx, kRole | kBarAccEmpty)) {
      return;
    }
    if (m.leader) mma_commit(bars.acc_full);
    if (staged(p, it)) {
      m.a.next();
      if (it.keys) m.b.next();
    }
  }
}

// 32 fp32 columns of one row, times `factor`, as BF16 words.
__device__ __forceinline__ void pack_row32(const uint32_t* o, float factor, uint32_t* pk) {
#pragma unroll
  for (int e = 0; e < 16; ++e) pk[e] = pack_bf16x2(__uint_as_float(o[2 * e]) * factor, __uint_as_float(o[2 * e + 1]) * factor);
}
// Four 16-byte chunks of a row of a 128-byte-swizzled [128][64] half tile; `chunk0` is the first (0 or 4).
__device__ __forceinline__ void stage_row32(uint8_t* half_tile, int row, int chunk0, const uint32_t* pk) {
#pragma unroll
  for (int ch = 0; ch < 4; ++ch) {
    *reinterpret_cast<uint4*>(half_tile + row * 128 + (((chunk0 + ch) ^ (row & 7)) << 4)) =
        make_uint4(pk[ch * 4], pk[ch * 4 + 1], pk[ch * 4 + 2], pk[ch * 4 + 3]);
  }
}
// The same columns as an fp32 partial sum of a split item.
__device__ __forceinline__ void store_part32(float* dst, const uint32_t* o, float factor) {
#pragma unroll
  for (int e = 0; e < 32; e += 4) {
    *reinterpret_cast<float4*>(dst + e) = make_float4(__uint_as_float(o[e]) * factor, __uint_as_float(o[e + 1]) * factor,
                                                      __uint_as_float(o[e + 2]) * factor, __uint_as_float(o[e + 3]) * factor);
  }
}

// Both softmax roles: P = exp2(S * scale log2(e) - LSE log2(e)) on pairs of columns; of every eight pairs
// kPolyPairs take the polynomial on the FMA pipe, the others the special-function unit.  Key items have the tensor pipe
// waiting for P, so the two units share the work; query items have the next scores ready and want the fewest
// instructions (8 heads of 16384, warm GPU, key / query pairs of eight: 0 / 0 3060 us, 1 / 1 2990, 2 / 1 2950, 4 / 1 2980,
// 2 / 2 2960).
constexpr int kKeyPolyPairs = 2, kQryPolyPairs = 1;
#define ATTN_F(r, i) __uint_as_float((r)[(i)])

// exp2 of kCols score columns in place, given per pair of columns the pair of -LSE log2(e).  Columns outside
// [seen_from, seen_to) become 0 where `masked`.
template <int kPolyPairs, typename NegLse>
__device__ __forceinline__ void exp_row(uint32_t* x, float2 c2, NegLse neg_lse, bool masked, int seen_from, int seen_to) {
#pragma unroll
  for (int pr = 0; pr < kCols / 2; ++pr) {
    const int e = pr * 2;
    const float2 y = fma2(make_float2(ATTN_F(x, e), ATTN_F(x, e + 1)), c2, neg_lse(e));
    const float2 w = (pr & 7) < kPolyPairs ? exp2_poly2(y) : make_float2(ex2_approx(y.x), ex2_approx(y.y));
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

// A thread's kCols columns of an operand as BF16 words; kFine: and then what their rounding left.
template <bool kFine>
struct Operand {
  uint32_t word[kFine ? kCols : kCols / 2];
  __device__ __forceinline__ void put(int e, float a, float b) {  // columns e, e + 1
    const uint32_t w = pack_bf16x2(a, b);
    word[e / 2] = w;
    if constexpr (kFine) word[(kCols + e) / 2] = pack_bf16x2(a - __uint_as_float(w << 16), b - __uint_as_float(w & 0xffff0000u));
  }
};

// dS = P o (dP - delta) of kCols columns, given per pair of columns the pair of -delta.
template <bool kFine, typename NegDelta>
__device__ __forceinline__ void ds_row(const uint32_t* x, const uint32_t* d, NegDelta neg_delta, Operand<kFine>& out) {
#pragma unroll
  for (int e = 0; e < kCols; e += 2) {
    const float2 t = add2(make_float2(ATTN_F(d, e), ATTN_F(d, e + 1)), neg_delta(e));
    const float2 w = mul2(make_float2(ATTN_F(x, e), ATTN_F(x, e + 1)), t);
    out.put(e, w.x, w.y);
  }
}
// A finished operand into tensor memory, and the word to the MMA warp that waits for it.
template <bool kFine>
__device__ __forceinline__ void hand_over(uint32_t taddr, const Operand<kFine>& op, uint64_t* bar, int lane) {
  if constexpr (kFine) {
    tmem_st_x16(taddr, op.word);
  } else {
    tmem_st_x8(taddr, op.word);
  }
  tmem_wait_st();
  tc_fence_before_sync();
  __syncwarp();
  if (lane == 0) mbar_arrive(bar);
}

// kCols row statistics, 16 bytes at a time (every thread of a warp reads the same ones).
__device__ __forceinline__ void load_stats(const float* src, float2* f) {
#pragma unroll
  for (int i = 0; i < kCols / 4; ++i) {
    const float4 v = *reinterpret_cast<const float4*>(src + 4 * i);
    f[2 * i] = make_float2(v.x, v.y);
    f[2 * i + 1] = make_float2(v.z, v.w);
  }
}

// One softmax thread of a key item: row `row` of the tile (a key), columns part * kCols + [0, kCols) of each half.
template <bool kFine>
__device__ __forceinline__ bool key_softmax(const BwdParams& p, const BwdItem& it, const BwdBarriers& bars,
                                            const uint8_t* smem, WaitCtx ctx, uint32_t tmem_row, int part, int row, int lane,
                                            Phases& ph) {
  const uint32_t t_s = tmem_row + kTmS + part * kCols, t_dp = tmem_row + kTmDp + part * kCols;
  const float2 c2 = make_float2(p.scale_log2, p.scale_log2);
  int tile = it.first + it.t0 % it.per_head;
  for (int i = 0; i < it.n; ++i) {
    const uint32_t st = ph.key & 1;
    const float* nl = reinterpret_cast<const float*>(smem + kSmemStat) + st * 2 * kTile + part * kCols;
    const float* neg_delta = nl + kTile;
    bool ok = mbar_wait(&bars.stat_full[st], (ph.key >> 1) & 1, ctx, kRoleBwdSoftmax | kBarStat) &&
              mbar_wait(&bars.s_full[0], ph.s & 1, ctx, kRoleBwdSoftmax | kBarS);
    if (!__all_sync(0xffffffffu, ok)) return false;
    tc_fence_after_sync();
    uint32_t x[2][kCols], d[2][kCols];
    Operand<kFine> op;
    tmem_ld_x16(t_s, x[0]);
    tmem_ld_x16(t_s + 64, x[1]);
    tmem_wait_ld();
    // the key is visible to the queries of columns `seen_from` on
    const int seen_from = (max(0, it.row0 + row - p.off) << p.pack_log2) - tile * kTile - part * kCols;
    const bool masked = p.causal && it.row0 + kTile - 1 > ((tile * kTile) >> p.pack_log2) + p.off;  // the same for the whole CTA
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      float2 st2[kCols / 2];
      load_stats(nl + h * 64, st2);
      exp_row<kKeyPolyPairs>(x[h], c2, [&](int e) { return st2[e / 2]; }, masked, seen_from - h * 64, kCols);
#pragma unroll
      for (int e = 0; e < kCols; e += 2) op.put(e, ATTN_F(x[h], e), ATTN_F(x[h], e + 1));
      hand_over<kFine>(t_s + h * 64, op, &bars.p_full[h], lane);
    }
    ok = mbar_wait(bars.dp_full, ph.dp & 1, ctx, kRoleBwdSoftmax | kBarDp);
    if (!__all_sync(0xffffffffu, ok)) return false;
    tc_fence_after_sync();
    tmem_ld_x16(t_dp, d[0]);
    tmem_ld_x16(t_dp + 64, d[1]);
    tmem_wait_ld();
#pragma unroll
    for (int h = 0; h < 2; ++h) {  // over this thread's own columns, which are in registers
      float2 st2[kCols / 2];
      load_stats(neg_delta + h * 64, st2);
      ds_row<kFine>(x[h], d[h], [&](int e) { return st2[e / 2]; }, op);
      hand_over<kFine>(t_dp + h * 64, op, &bars.ds_full[h], lane);
    }
    if (lane == 0) mbar_arrive(&bars.stat_empty[st]);
    ph.s ^= 1u;
    ++ph.dp;
    ++ph.key;
    if (++tile == it.first + it.per_head) tile = it.first;
  }
  return true;
}

// The same for a query item: row `row` is a query, the columns are keys.
template <bool kFine>
__device__ __forceinline__ bool query_softmax(const BwdParams& p, const BwdItem& it, const BwdBarriers& bars, WaitCtx ctx,
                                              uint32_t tmem_row, int part, int row, int lane, Phases& ph) {
  const uint32_t t_dp = tmem_row + kTmQryDp + part * kCols;
  const float2 c2 = make_float2(p.scale_log2, p.scale_log2);
  const size_t at = (static_cast<size_t>(it.b) * p.Hq + it.h) * p.n_qt * kTile + it.row0 + row;
  const float nl = __ldg(p.neg_lse2 + at), ndl = __ldg(p.neg_delta + at);
  const float2 nl2 = make_float2(nl, nl), ndl2 = make_float2(ndl, ndl);
  const int row_limit = p.causal ? min(p.Sk, ((it.row0 + row) >> p.pack_log2) + p.off + 1) : p.Sk;  // keys this row may see
  const int tile_clear = p.causal ? min(p.Sk, (it.row0 >> p.pack_log2) + p.off + 1) : p.Sk;          // keys every row of the tile sees
  for (int j = 0; j < it.n; ++j) {
    const int x_buf = j & 1;
    bool ok = mbar_wait(&bars.s_full[x_buf], (ph.s >> x_buf) & 1, ctx, kRoleBwdSoftmax | kBarS);
    if (!__all_sync(0xffffffffu, ok)) return false;
    tc_fence_after_sync();
    const uint32_t t_s = tmem_row + kTmQryS + x_buf * kTile + part * kCols;
    uint32_t x[2][kCols], d[2][kCols];
    Operand<kFine> op;
    tmem_ld_x16(t_s, x[0]);
    tmem_ld_x16(t_s + 64, x[1]);
    tmem_wait_ld();
    // keys beyond Sk are masked too: their scores are 0, and exp2(nl) may be infinite
    const bool masked = (it.t0 + j + 1) * kTile > tile_clear;  // the same for the whole CTA
    const int seen_to = row_limit - (it.t0 + j) * kTile - part * kCols;
#pragma unroll
    for (int h = 0; h < 2; ++h)
      exp_row<kQryPolyPairs>(x[h], c2, [&](int) { return nl2; }, masked, 0, seen_to - h * 64);
    ok = mbar_wait(bars.dp_full, ph.dp & 1, ctx, kRoleBwdSoftmax | kBarDp);
    if (!__all_sync(0xffffffffu, ok)) return false;
    tc_fence_after_sync();
    tmem_ld_x16(t_dp, d[0]);
    tmem_ld_x16(t_dp + 64, d[1]);
    tmem_wait_ld();
    tc_fence_before_sync();
    __syncwarp();
    if (lane == 0) mbar_arrive(bars.dp_read);
#pragma unroll
    for (int h = 0; h < 2; ++h) {  // over this thread's own scores, read above
      ds_row<kFine>(x[h], d[h], [&](int) { return ndl2; }, op);
      hand_over<kFine>(t_s + h * 64, op, &bars.ds_full[2 * x_buf + h], lane);
    }
    ph.s ^= 1u << x_buf;
    ++ph.dp;
  }
  return true;
}

// The results' way out.  Key items: half 0 takes dV, half 1 dK, 64 columns a thread; query items: 32 columns of dQ.
// pos_a, pos_b: ring positions of the slots set aside; `stored`: items that were staged so far.
__device__ __forceinline__ bool write_results(const BwdParams& p, const BwdItem& it, const BwdBarriers& bars, uint8_t* smem,
                                              WaitCtx ctx, uint32_t tmem_row, int part, int row, int lane, int item,
                                              uint32_t pos_a, uint32_t pos_b, uint32_t stored) {
  const int half = part / (kParts / 2);
  const int n32 = it.keys ? 2 : 1;  // 32-column pieces of this thread
  const int col0 = it.keys ? (part % (kParts / 2)) * 64 : part * 32;
  const uint32_t t_acc = tmem_row + (it.keys ? (half == 0 ? kTmDv : kTmDk) : kTmDq) + col0;
  const float factor = it.keys && half == 0 ? 1.f : p.scale;
  bool ok = mbar_wait(bars.acc_full, item & 1, ctx, kRoleBwdSoftmax | kBarAcc);
  if (!__all_sync(0xffffffffu, ok)) return false;
  tc_fence_after_sync();
  const bool out_bf16 = staged(p, it);
  float* part_dst = nullptr;
  if (!out_bf16) {
    const int heads = it.keys ? p.Hkv : p.Hq, rows = (it.keys ? p.n_kt : p.n_qt) * kTile;
    float* buf = it.keys ? (half == 0 ? p.dv_part : p.dk_part) : p.dq_part;
    part_dst = buf + (((static_cast<size_t>(it.split) * p.B + it.b) * heads + it.h) * rows + it.row0 + row) * kHeadDim + col0;
  }
  uint32_t pk[32];
#pragma unroll
  for (int cc = 0; cc < 2; ++cc) {
    if (cc < n32) {
      uint32_t o[32];
      if (it.n > 0) {
        tmem_ld_x32(t_acc + cc * 32, o);
        tmem_wait_ld();
      } else {  // nothing streamed past: the result is 0, and tensor memory holds nothing of this item
#pragma unroll
        for (int e = 0; e < 32; ++e) o[e] = 0u;
      }
      if (out_bf16) {
        pack_row32(o, factor, pk + cc * 16);
      } else {
        store_part32(part_dst + cc * 32, o, factor);
      }
    }
  }
  tc_fence_before_sync();
  __syncwarp();
  if (lane == 0) mbar_arrive(bars.acc_empty);
  if (!out_bf16) return true;
  ok = mbar_wait(bars.stage_free, stored & 1, ctx, kRoleBwdSoftmax | kBarStageFree) &&
       mbar_wait(&bars.a_full[pos_a % kRingA], (pos_a / kRingA) & 1, ctx, kRoleBwdSoftmax | kBarRingFull) &&
       (!it.keys || mbar_wait(&bars.b_full[pos_b % kRingB], (pos_b / kRingB) & 1, ctx, kRoleBwdSoftmax | kBarRingFull));
  if (!__all_sync(0xffffffffu, ok)) return false;
  uint8_t* slot_a = smem + kSmemRing + (pos_a % kRingA) * kTileBytes;
  uint8_t* slot_b = smem + kSmemRing + (kRingA + pos_b % kRingB) * kTileBytes;
  uint8_t* stage = (it.keys && half == 0 ? slot_b : slot_a) + (col0 >> 6) * kHalfBytes;
#pragma unroll
  for (int cc = 0; cc < 2; ++cc) {
    if (cc < n32) stage_row32(stage, row, ((col0 & 63) + cc * 32) / 8, pk + cc * 16);
  }
  fence_proxy_async_smem();
  __syncwarp();
  if (lane == 0) mbar_arrive(&bars.stage_full[half]);
  return true;
}

template <bool kFine>
__device__ __forceinline__ void role_softmax(const BwdParams& p, const BwdBarriers& bars, uint8_t* smem, const volatile int* box,
                                             WaitCtx ctx, uint32_t tmem, int part, int row, int lane) {
  const uint32_t tmem_row = tmem + (static_cast<uint32_t>(row & ~31) << 16);
  uint32_t pos_a = 0, pos_b = 0, stored = 0;
  Phases ph;
  BwdItem it;
  for (int k = 0; next_item(bars, box, k, ctx, kRoleBwdSoftmax, true, lane == 0, it); ++k) {
    bool ok = true;
    if (it.n > 0) {
      ok = it.keys ? key_softmax<kFine>(p, it, bars, smem, ctx, tmem_row, part, row, lane, ph)
                   : query_softmax<kFine>(p, it, bars, ctx, tmem_row, part, row, lane, ph);
    }
    pos_a += it.n;
    pos_b += it.n;
    if (!ok || !write_results(p, it, bars, smem, ctx, tmem_row, part, row, lane, k, pos_a, pos_b, stored)) return;
    if (staged(p, it)) {
      ++pos_a;
      ++stored;
      if (it.keys) ++pos_b;
    }
  }
}

template <bool kFine>
__global__ void __launch_bounds__(kBwdThreads, 1)
attn_bwd_kernel(const __grid_constant__ CUtensorMap tm_q, const __grid_constant__ CUtensorMap tm_k,
                const __grid_constant__ CUtensorMap tm_v, const __grid_constant__ CUtensorMap tm_do,
                const __grid_constant__ CUtensorMap tm_dq, const __grid_constant__ CUtensorMap tm_dk,
                const __grid_constant__ CUtensorMap tm_dv, const BwdParams p) {
  extern __shared__ __align__(1024) uint8_t smem[];
  uint64_t* bar = reinterpret_cast<uint64_t*>(smem + kSmemBwdBars);
  BwdBarriers bars;
  bars.fixed_full = bar;
  bars.fixed_empty = bars.fixed_full + 2;
  bars.a_full = bars.fixed_empty + 2;
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
  bars.acc_empty = bars.acc_full + 1;
  bars.stage_free = bars.acc_empty + 1;
  bars.stage_full = bars.stage_free + 1;
  bars.item_full = bars.stage_full + 2;
  bars.item_empty = bars.item_full + 2;
  bars.clc_full = bars.item_empty + 2;
  volatile int* box = reinterpret_cast<volatile int*>(smem + kSmemBwdItems);
  uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(smem + kSmemBwdMisc);
  volatile int* abort_flag = reinterpret_cast<volatile int*>(smem + kSmemBwdMisc + 4);
  const WaitCtx ctx{abort_flag, p.status, kWaitLimitNs};
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  if ((smem_u32(smem) & 1023u) != 0) {  // the swizzled tiles need a 1024-byte aligned base
    if (tid == 0 && atomicCAS(p.status, 0, kBadSmemAlign) == 0) p.status[1] = static_cast<int>(blockIdx.x);
    return;
  }
  if (tid == 0) {
    for (int i = 0; i < kRingA; ++i) {
      mbar_init(&bars.a_full[i], 1);
      mbar_init(&bars.a_empty[i], 2);
    }
    for (int i = 0; i < kRingB; ++i) {
      mbar_init(&bars.b_full[i], 1);
      mbar_init(&bars.b_empty[i], 2);
    }
    mbar_init(bars.dp_full, 1);
    mbar_init(bars.dp_read, kSoftmaxWarps);
    mbar_init(bars.stage_free, 1);
    mbar_init(bars.acc_full, 2);
    mbar_init(bars.acc_empty, kSoftmaxWarps);
    for (int i = 0; i < 2; ++i) {
      mbar_init(&bars.fixed_full[i], 1);
      mbar_init(&bars.fixed_empty[i], 1);
      mbar_init(&bars.stat_full[i], 1);
      mbar_init(&bars.stat_empty[i], kSoftmaxWarps);
      mbar_init(&bars.s_full[i], 1);
      mbar_init(&bars.p_full[i], kSoftmaxWarps);
      mbar_init(&bars.ds_full[i], kSoftmaxWarps);
      mbar_init(&bars.ds_full[2 + i], kSoftmaxWarps);
      mbar_init(&bars.stage_full[i], kSoftmaxWarps / 2);
      mbar_init(&bars.item_full[i], 1);
      mbar_init(&bars.item_empty[i], kItemConsumers);
      mbar_init(&bars.clc_full[i], 1);
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

  if (warp < kSoftmaxWarps) {
    reg_alloc<kRegsSoftmax>();
    role_softmax<kFine>(p, bars, smem, box, ctx, tmem, warp >> 2, tid & 127, lane);
  } else {
    reg_dealloc<kRegsOther>();
    if (warp == kSoftmaxWarps) {
      role_mma<true, kFine>(p, bars, smem, box, ctx, tmem, lane);
    } else if (warp == kSoftmaxWarps + 1) {
      role_mma<false, kFine>(p, bars, smem, box, ctx, tmem, lane);
    } else if (lane != 0) {
      // the loader and the store warp are one thread each
    } else if (warp == kSoftmaxWarps + 2) {
      role_loader(p, bars, smem, box, ctx, &tm_q, &tm_k, &tm_v, &tm_do);
    } else {
      role_store(p, bars, smem, box, ctx, &tm_dq, &tm_dk, &tm_dv);
    }
    if (lane == 0 && *abort_flag) {  // let copies in flight land before the CTA's shared memory is released
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

// Row statistics of the backward pass: -LSE log2(e) and -delta = dLSE - sum_d dO O, rows padded to whole tiles.
// HBM-bound: 512 bytes read per row.  A block takes 256 rows, heads fastest as they lie in memory, half a warp a row
// with four rows in flight; the sums pass through shared memory so that they are written along the sequence.
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
                     float* __restrict__ neg_delta, int Hq, int Sq, int padded, int pack_log2, int heads_log2, int n_blocks) {
  __shared__ float sums[kPrepThreads];  // [sequence][head]
  const int sub = threadIdx.x & 15;
  const int heads = 1 << heads_log2, rows = kPrepThreads >> heads_log2;  // heads and sequence positions of a block
  const int h_blocks = (Hq + heads - 1) >> heads_log2, s_blocks = (padded + rows - 1) / rows;
  for (int blk = blockIdx.x; blk < n_blocks; blk += gridDim.x) {
    const int hb = blk % h_blocks, t = blk / h_blocks;
    const int sb = t % s_blocks;
    const long long b = t / s_blocks;
    const uint16_t* ob = o + b * so.b;
    const uint16_t* db = dout + b * sdo.b;
#pragma unroll
    for (int i = 0; i < 16; i += 4) {
      uint4 x[4], y[4];
#pragma unroll
      for (int u = 0; u < 4; ++u) {
        const int r = (i + u) * 16 + (threadIdx.x >> 4);
        const int h = (hb << heads_log2) + (r & (heads - 1)), s = sb * rows + (r >> heads_log2);
        x[u] = y[u] = make_uint4(0u, 0u, 0u, 0u);
        if (h < Hq && s < Sq) {
          x[u] = __ldg(reinterpret_cast<const uint4*>(ob + s * so.s + h * so.h) + sub);
          y[u] = __ldg(reinterpret_cast<const uint4*>(db + s * sdo.s + h * sdo.h) + sub);
        }
      }
#pragma unroll
      for (int u = 0; u < 4; ++u) {
        float acc = dot2_bf16(x[u].x, y[u].x, dot2_bf16(x[u].y, y[u].y, dot2_bf16(x[u].z, y[u].z, dot2_bf16(x[u].w, y[u].w, 0.f))));
#pragma unroll
        for (int m = 8; m > 0; m >>= 1) acc += __shfl_xor_sync(0xffffffffu, acc, m);
        if (sub == 0) sums[(i + u) * 16 + (threadIdx.x >> 4)] = acc;
      }
    }
    __syncthreads();
    // `padded`: positions of a head, to whole tiles
    const int h = (hb << heads_log2) + threadIdx.x / rows, s = sb * rows + threadIdx.x % rows;
    if (h < Hq && s < padded) {
      float l = -INFINITY, dl = 0.f;
      if (s < Sq) {
        const long long at = (b * Hq + h) * Sq + s;
        l = __ldg(lse + at);
        if (dlse != nullptr) dl = __ldg(dlse + at);
      }
      // [B][Hq][padded], or packed [B][Hkv][padded][group]
      const long long at = ((((b * Hq + h) >> pack_log2) * padded + s) << pack_log2) + (h & ((1 << pack_log2) - 1));
      // The row sees no key, or does not exist.  Its P is not always an exact 0 (the polynomial stops at 2^-126): rows that
      // see no key vanish by the mask, rows that do not exist by their dO, which TMA fills with zeros, and delta 0.
      const bool none = l == -INFINITY;
      neg_lse2[at] = none ? -INFINITY : -l * 1.4426950408889634f;
      neg_delta[at] = none ? 0.f : dl - sums[(threadIdx.x % rows) * heads + threadIdx.x / rows];
    }
    __syncthreads();
  }
}

// Adds up the fp32 partial sums of split items in order and rounds once: one warp a row of 128, rows in the
// order of the output [B][S][H]; blockIdx.y picks the output.  HBM-bound, and small: only problems with few tiles are
// split.
constexpr int kJoinThreads = 256;
struct JoinOut {
  const float* part;  // [splits][B][H][padded][128]
  uint16_t* out;
  RowStrides strides;
  int splits, H, S, padded, pack_log2;
  long long n_rows, part_stride;
};
struct JoinParams {
  JoinOut o[3];
};
__global__ void __launch_bounds__(kJoinThreads) attn_bwd_join_kernel(const __grid_constant__ JoinParams p) {
  const JoinOut& j = p.o[blockIdx.y];
  const int lane = threadIdx.x & 31;
  const long long step = static_cast<long long>(gridDim.x) * (kJoinThreads / 32);
  for (long long r = static_cast<long long>(blockIdx.x) * (kJoinThreads / 32) + (threadIdx.x >> 5); r < j.n_rows; r += step) {
    const int h = static_cast<int>(r % j.H);
    const long long t = r / j.H;
    const long long s = t % j.S, b = t / j.S;
    const float* src = j.part + ((b * j.H + h) * j.padded + s) * kHeadDim + lane * 4;
    float4 v = make_float4(0.f, 0.f, 0.f, 0.f);
    for (int i = 0; i < j.splits; ++i) {
      const float4 x = __ldg(reinterpret_cast<const float4*>(src + i * j.part_stride));
      v.x += x.x; v.y += x.y; v.z += x.z; v.w += x.w;
    }
    const long long head = (static_cast<long long>(h) << j.pack_log2) + (s & ((1 << j.pack_log2) - 1));
    *reinterpret_cast<uint2*>(j.out + b * j.strides.b + (s >> j.pack_log2) * j.strides.s + head * j.strides.h + lane * 4) =
        make_uint2(pack_bf16x2(v.x, v.y), pack_bf16x2(v.z, v.w));
  }
}

}  // namespace bwd
}  // namespace attn
