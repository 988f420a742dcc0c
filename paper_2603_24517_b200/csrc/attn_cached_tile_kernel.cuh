// Attention of new tokens over a paged 8-bit cache, for many query rows a key head (prompts, chunks): tensor cores.
//
// The scheme of the forward kernel: a CTA holds two 128-row query tiles ("stages") against one stream of 128-key tiles, S and
// O in tensor memory, one softmax thread a row.  A query tile's rows are (token, head of the group), heads fastest, so a key
// head is read once for its group.  What differs:
//
//   warps 0-7    softmax; each thread also brings its row of Q into shared memory, as f16 scaled by a power of two of the row
//   warp  12     tcgen05.mma, f16 operands
//   warp  13     fetch: walks the CTA's piece of the work and publishes its items; page numbers and scales two and one steps
//                ahead; codes by TMA, a page a copy (any page size and strides), into 32 KB of staging
//   warps 8-11,  converters: codes exactly to f16 in the swizzled ring of K / V tiles, zeros behind the last token; 8-11 also
//         14-15  write O / l -> BF16 -> memory, or an fp32 part where the tile's keys are spread over CTAs
//
// Scales: 16 keys lie in one page, 32 or 64 where pages have as many slots (GRAN, "a granule").  K's scale multiplies the row's
// factor granule by granule, V's enters the exponent as its log2 and is taken out of the row sum again granule by granule, so both
// products run on bare codes.
//
// Work: the line of (sequence, key head, tile pair, 128 keys) steps cut into equal pieces, as in the decoding kernel.  A tile whose
// rows fit one stage takes its keys on both stages in turn and joins the two results.
//
// Bound by the chain softmax -> P V -> Q K^T of the forward kernel, which the converters beside it and the five roles'
// instruction fetches lengthen: 8192 rows on 32768 keys (32 / 8 heads, E4M3) 3.20 ms, 1200 TFLOP/s, replayed on a GPU with
// nothing else to do (INT8 3.39), where the forward kernel takes 2.92 on BF16 keys laid out one after another; 3.63 ms, 1060
// TFLOP/s, in calls one behind the other at the power limit.  Without the conversion (a timing copy) 6 % less.  A step of a tile
// pair takes 2.1 us, of one stage's rows 1.9 us.  The softmax warps spill 128 to 152 bytes a thread (a row's 128 scores fill the
// 128 registers the kernel compiles for).  Code that runs once an item is kept in short loops: straight-line code that is not in
// the instruction cache takes about 20 clocks an instruction here (an item's switch 14000 clocks, in loops 7000).
#pragma once

#include "attn_cached_kernel.cuh"

namespace attn {
namespace kv {

constexpr int kTileRows = 256;  // rows of a work item: two stages
constexpr int kConvWarps = 6;
constexpr int kItemReaders = 1 + 8 + kConvWarps;  // warps that read an item: MMA, softmax, converters (four of them write results)
// registers of a thread after the split of the CTA's 64K: 8 softmax, 8 other warps
constexpr int kTRegsSoftmax = 192, kTRegsOther = 64;
static_assert(8 * kTRegsSoftmax + 8 * kTRegsOther <= 2048, "register split");

constexpr int kTSmemQ = 0;
constexpr int kTSmemKv = 2 * kTileBytes;
constexpr int kTSmemRaw = kTSmemKv + kKvSlots * kTileBytes;      // codes of one K and one V tile
constexpr int kTSmemStats = kTSmemRaw + 2 * kTile * kKvDim;      // float [2 stages][2][128]
constexpr int kMetaSteps = 4;
constexpr int kMetaFloats = 27;
constexpr int kItemSlots = 5;      // the fetching warp looks two steps (items) ahead of the codes it requests, results follow one behind
constexpr int kItemInts = 11;
constexpr int kTSmemMeta = kTSmemStats + 2 * 2 * kTile * 4;
constexpr int kTSmemItems = kTSmemMeta + kMetaSteps * kMetaFloats * 4;
constexpr int kTSmemBars = (kTSmemItems + kItemSlots * kItemInts * 4 + 7) / 8 * 8;
constexpr int kTNumBars = 2 + 4 + 2 * kKvSlots + 2 * 7 + kMetaSteps + 2 * kItemSlots;
constexpr int kTSmemMisc = kTSmemBars + kTNumBars * 8;
constexpr int kTSmemBytes = kTSmemMisc + 8;
static_assert(kTSmemBytes <= 232448, "shared memory budget of one CTA");
static_assert(kTSmemBars % 8 == 0 && kTSmemMeta % 16 == 0 && kTSmemStats % 16 == 0 && kTSmemMisc % 8 == 0, "alignment");
static_assert(kHeadDim == kKvDim && kTile == kStepKeys, "one head dimension, one tile");

// What the converters tell the softmax warps about a step.
enum : int { kMetaK = 0, kMetaV = 8, kMetaInv = 16, kMetaFloor = 24, kMetaBad = 25, kMetaValid = 26 };

struct TileBarriers {
  uint64_t* q_full;    // [2] softmax (4 warps): the stage's Q is in shared memory -> MMA
  uint64_t* raw_full;  // [2] TMA: the codes of the keys, of the values -> converters
  uint64_t* raw_empty; // [2] converters (kConvWarps warps) -> fetching warp
  uint64_t* kv_full;   // [kKvSlots] converters (kConvWarps warps) -> MMA
  uint64_t* kv_empty;  // [kKvSlots] MMA commit -> converters
  uint64_t* s_full;    // [2] MMA commit -> softmax
  uint64_t* p_half;    // [2] softmax (4 warps): the first 64 keys of P -> MMA
  uint64_t* p_full;    // [2] softmax (4 warps) -> MMA
  uint64_t* o_full;    // [2] MMA commit (last P V) -> epilogue
  uint64_t* o_empty;   // [2] epilogue (4 warps) -> MMA
  uint64_t* l_full;    // [2] softmax (128 threads) -> epilogue
  uint64_t* l_empty;   // [2] epilogue (128 threads) -> softmax
  uint64_t* meta_full; // [kMetaSteps] fetching warp -> softmax; converters read the entry too, behind raw_full
  uint64_t* item_full;  // [kItemSlots] fetching warp -> MMA, softmax, converters
  uint64_t* item_empty; // [kItemSlots] those kItemReaders warps -> fetching warp
};
enum : int { kRoleConvert = 6 << 8, kBarMeta = 20 };

constexpr uint32_t make_idesc_f16(uint32_t b_mn_major) {  // as make_idesc_bf16, both operand formats 0
  return (1u << 4) | (b_mn_major << 16) | ((kTile >> 3) << 17) | ((kTile >> 4) << 24);
}
constexpr uint32_t kIdescQKf16 = make_idesc_f16(0);
constexpr uint32_t kIdescPVf16 = make_idesc_f16(1);

// One tile pair, or the CTA's piece of it, as the fetching warp publishes it: the roles keep no place on the line of work
// themselves (the softmax warps have no registers for it).
struct Item {
  int n;            // steps; 0: no more items
  int t_first;      // the first of them
  bool two;         // the second stage has rows of its own
  bool split;       // it has not: the stages take the steps in turn, and their parts are joined at the end
  bool whole;       // all of the tile's steps
  int b, h, tile;
  SeqWork s;
  int last;         // the last CTA with a part of the tile
};
__device__ __forceinline__ void publish_item(int* box, const CachedParams& p, const Line& line, const Cursor<kTileRows>& c, long long at) {
  const int n = static_cast<int>(min(static_cast<long long>(c.steps - c.t), line.end - at));
  const bool two = c.tile * kTileRows + kTile < c.s.n * p.group;
  box[0] = n;
  box[1] = c.t;
  box[2] = (two ? 1 : 0) | (c.t == 0 && n == c.steps ? 2 : 0) | (!two && n > 1 ? 4 : 0);
  box[3] = c.b;
  box[4] = c.h;
  box[5] = c.tile;
  box[6] = c.s.row0;
  box[7] = c.s.n;
  box[8] = c.s.len;
  box[9] = c.s.keys;
  box[10] = static_cast<int>(line.owner(at - c.t + c.steps - 1));
}
__device__ __forceinline__ const int* item_box(const uint8_t* smem, uint32_t k) {
  return reinterpret_cast<const int*>(smem + kTSmemItems) + (k % kItemSlots) * kItemInts;
}
// The k-th item of this CTA, once a whole warp of a consuming role has waited for it.
__device__ __forceinline__ bool wait_item(const TileBarriers& bars, uint32_t k, WaitCtx ctx, int role) {
  return mbar_wait_warp(&bars.item_full[k % kItemSlots], (k / kItemSlots) & 1, ctx, role | kBarSchedFull);
}
__device__ __forceinline__ void read_item(const uint8_t* smem, uint32_t k, Item& it) {
  const int* box = item_box(smem, k);
  it.n = box[0];
  it.t_first = box[1];
  it.two = (box[2] & 1) != 0;
  it.whole = (box[2] & 2) != 0;
  it.split = (box[2] & 4) != 0;
  it.b = box[3];
  it.h = box[4];
  it.tile = box[5];
  it.s = SeqWork{box[6], box[7], box[8], box[9]};
  it.last = box[10];
}
__device__ __forceinline__ void drop_item(const TileBarriers& bars, uint32_t k, int lane) {
  __syncwarp();
  if (lane == 0) mbar_arrive(&bars.item_empty[k % kItemSlots]);
}
__device__ __forceinline__ bool take_item(const TileBarriers& bars, const uint8_t* smem, uint32_t k, WaitCtx ctx, int role, int lane, Item& it) {
  if (!wait_item(bars, k, ctx, role)) return false;
  read_item(smem, k, it);
  drop_item(bars, k, lane);
  return true;
}

// ---- the pages' codes -------------------------------------------------------------------------------------------------
struct StepPlace {  // where a step's codes are; `page` is that of granule (lane & 7): -1 does not exist, -2 behind the last token
  int page, h, key0, keys;
  bool first;       // of its item in this CTA
};

// Looks pages up two steps ahead and their scales one, requests the codes page by page and writes what the softmax warps need.
__device__ __forceinline__ void role_fetch(const CachedParams& p, const TileBarriers& bars, uint8_t* smem, WaitCtx ctx,
                                           const Line& line, Cursor<kTileRows> ahead, int lane, const CUtensorMap* tm_k,
                                           const CUtensorMap* tm_v) {
  const CacheView& c = p.c;
  long long left = line.end - line.begin;  // steps whose pages have not been looked up yet
  bool first = true, ended = false, ok = true;
  uint32_t items = 0;
  auto publish = [&](bool some) {
    const uint32_t slot = items % kItemSlots;
    ok = ok && mbar_wait_warp(&bars.item_empty[slot], ((items / kItemSlots) & 1) ^ 1, ctx, kRoleLoad | kBarSchedEmpty);
    ++items;
    if (!ok) return;
    if (lane == 0) {
      int* box = reinterpret_cast<int*>(smem + kTSmemItems) + slot * kItemInts;
      if (some) {
        publish_item(box, p, line, ahead, line.end - left);
      } else {
        box[0] = 0;
      }
      mbar_arrive(&bars.item_full[slot]);
    }
    __syncwarp();
  };
  auto look_up = [&]() {
    StepPlace f;
    f.keys = 0;
    f.page = -2;
    f.h = f.key0 = 0;
    f.first = false;
    if (left <= 0) {
      if (!ended) publish(false);
      ended = true;
    } else {
      if (first || ahead.t == 0) publish(true);
      --left;
      f.h = ahead.h;
      f.key0 = ahead.t * kStepKeys;
      f.keys = ahead.s.keys;
      f.first = first || ahead.t == 0;
      first = false;
      const int key = f.key0 + (lane & 7) * 16;
      if (key < f.keys) f.page = page_of(c, ahead.b, key >> c.page_log2);
      if (++ahead.t >= ahead.steps && left > 0) ahead.next_tile(p);
    }
    return f;
  };
  auto scale_of = [&](const StepPlace& f) {  // lanes 0-7: K's of granule lane, 8-15: V's of granule lane - 8
    return lane < 16 && f.page >= 0 ? __ldg(c.scales[lane >> 3] + static_cast<long long>(f.page) * c.Hkv + f.h) : 0.f;
  };
  StepPlace now = look_up(), next = look_up();
  float scale_now = scale_of(now);
  float top_scale = kScaleLeast;  // log2 of the largest V scale of the item so far
  const bool asks = lane < 8 && ((lane * 16) & ((1 << c.page_log2) - 1)) == 0;  // one lane a page
  const uint32_t steps = static_cast<uint32_t>(line.end - line.begin);
  for (uint32_t i = 0; i < steps; ++i) {
    const StepPlace after = look_up();
    if (!ok) return;
    const float scale_next = scale_of(next);
    const float lv = lg2_approx(scale_now);
    float top = lane >= 8 && lane < 16 ? lv : kScaleLeast;
#pragma unroll
    for (int m = 4; m > 0; m >>= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, m));
    top = __shfl_sync(0xffffffffu, top, 8);
    top_scale = fmaxf(now.first ? kScaleLeast : top_scale, top);
    const unsigned bad = __ballot_sync(0xffffffffu, lane < 8 && now.page == -1);
    float* meta = reinterpret_cast<float*>(smem + kTSmemMeta) + (i % kMetaSteps) * kMetaFloats;
#pragma unroll 1
    for (int kv = 0; kv < 2; ++kv) {
      // the step's entry may be written once the codes of the keys of the step before have been converted: that needed the
      // slot of the keys two steps before that, so the scores of i - 3 are complete and the weights of i - 4 were taken
      if (!mbar_wait_warp(&bars.raw_empty[kv], (i & 1) ^ 1, ctx, kRoleLoad | kBarKvEmpty)) return;
      if (kv == 0) {
        if (lane < 8) {
          meta[kMetaK + lane] = scale_now;
        } else if (lane < 16) {
          const float counts = now.page >= 0 ? fmaxf(lv, top_scale - kScaleZero) : top_scale;
          meta[kMetaV + lane - 8] = counts;
          meta[kMetaInv + lane - 8] = ex2_approx(-counts);
        } else if (lane == 16) {
          meta[kMetaFloor] = top_scale - kScaleSpan;
          reinterpret_cast<int*>(meta)[kMetaBad] = bad != 0 ? (__ffs(bad) - 1) * 16 : kStepKeys;
          reinterpret_cast<int*>(meta)[kMetaValid] = now.keys - now.key0;
        }
        __syncwarp();
        if (lane == 0) mbar_arrive(&bars.meta_full[i % kMetaSteps]);
      }
      if (lane == 0) mbar_arrive_expect_tx(&bars.raw_full[kv], kTile * kKvDim);
      __syncwarp();
      if (asks)  // a page that is not there lies behind the last one: zeros
        tma_load_4d(smem + kTSmemRaw + kv * kTile * kKvDim + lane * 16 * kKvDim, kv == 0 ? tm_k : tm_v, &bars.raw_full[kv], 0, 0,
                    now.h, now.page >= 0 ? now.page : c.n_pages);
      __syncwarp();
    }
    now = next;
    next = after;
    scale_now = scale_next;
  }
}

// The codes of step i (keys, then values) to f16: converter warp cw's rows of the tiles.  A lane takes 16 codes of one of 8 rows at
// a time, odd rows the other half of the head dimension than even ones, so neither its reads nor its writes meet another
// lane's bank.
template <int TYPE>
__device__ __forceinline__ bool convert_step(const TileBarriers& bars, uint8_t* smem, WaitCtx ctx, uint32_t i, int cw, int lane) {
  const int sub = lane >> 2, ch = (lane & 3) * 2;
#pragma unroll 1
  for (int kv = 0; kv < 2; ++kv) {
    const uint32_t kv_cnt = 2 * i + kv, slot = kv_cnt % kKvSlots;
    bool ok = mbar_wait(&bars.raw_full[kv], i & 1, ctx, kRoleConvert | kBarKvFull);
    ok = ok && mbar_wait(&bars.kv_empty[slot], ((kv_cnt / kKvSlots) & 1) ^ 1, ctx, kRoleConvert | kBarKvEmpty);
    if (!__all_sync(0xffffffffu, ok)) return false;
    const int valid = reinterpret_cast<const int*>(smem + kTSmemMeta)[(i % kMetaSteps) * kMetaFloats + kMetaValid];
    const uint8_t* raw = smem + kTSmemRaw + kv * kTile * kKvDim + sub * kKvDim + (lane & 3) * 16;
    uint8_t* tile = smem + kTSmemKv + slot * kTileBytes + sub * 128;
#pragma unroll 1
    for (int rg = cw; rg < 16; rg += kConvWarps) {
#pragma unroll
      for (int k = 0; k < 2; ++k) {
        const int half = k ^ (sub & 1);
        uint4 w = *reinterpret_cast<const uint4*>(raw + rg * 8 * kKvDim + half * 64);
        if (valid < kTile && rg * 8 + sub >= valid) w = make_uint4(0, 0, 0, 0);  // behind the last token: zeros
        uint4 lo, hi;
        codes_to_f16<TYPE>(w.x, lo.x, lo.y);
        codes_to_f16<TYPE>(w.y, lo.z, lo.w);
        codes_to_f16<TYPE>(w.z, hi.x, hi.y);
        codes_to_f16<TYPE>(w.w, hi.z, hi.w);
        uint8_t* row = tile + rg * 8 * 128 + half * kHalfBytes;
        *reinterpret_cast<uint4*>(row + ((ch ^ sub) << 4)) = lo;
        *reinterpret_cast<uint4*>(row + (((ch + 1) ^ sub) << 4)) = hi;
      }
    }
    fence_proxy_async_smem();
    __syncwarp();
    if (lane == 0) {
      mbar_arrive(&bars.raw_empty[kv]);
      mbar_arrive(&bars.kv_full[slot]);
    }
  }
  return true;
}

// ---- MMA --------------------------------------------------------------------------------------------------------------
__device__ __forceinline__ void issue_qk_f16(bool leader, uint32_t tmem_s, uint64_t q_desc, uint64_t k_desc) {
  if (leader) {
#pragma unroll
    for (int kk = 0; kk < 8; ++kk) {
      const uint32_t off = (kk >> 2) * kHalfBytes + (kk & 3) * 32;
      mma_ss(tmem_s, desc_advance(q_desc, off), desc_advance(k_desc, off), kIdescQKf16, kk > 0);
    }
  }
}
__device__ __forceinline__ void issue_pv_f16(bool leader, uint32_t tmem_o, uint32_t tmem_p, uint64_t v_desc, bool accumulate,
                                             int kk_begin, int kk_end) {
  if (leader) {
#pragma unroll
    for (int kk = 0; kk < 8; ++kk) {
      if (kk >= kk_begin && kk < kk_end) {
        mma_ts(tmem_o, tmem_p + kk * 8, desc_advance(v_desc, kk * 2048), kIdescPVf16, (accumulate || kk > 0) ? 1u : 0u);
      }
    }
  }
}

__device__ __forceinline__ void role_tile_mma(const TileBarriers& bars, uint8_t* smem, WaitCtx ctx,                                              uint32_t tmem, int lane) {
  const bool leader = elect_one();
  const uint32_t base = smem_u32(smem);
  const uint64_t q_desc[2] = {kmajor_desc(base + kTSmemQ), kmajor_desc(base + kTSmemQ + kTileBytes)};
  uint32_t kv_cnt = 0;
  uint32_t q_cnt[2] = {0, 0};
  uint32_t sp_cnt[2] = {0, 0};
  for (uint32_t k = 0;; ++k) {
    Item it;
    if (!take_item(bars, smem, k, ctx, kRoleMma, lane, it) || it.n == 0) return;
    if (it.split) {
      // The first two steps' scores, then per step j: P V, and the scores of step j + 2 in the place it leaves.  The keys of step
      // j + 1 are given back only now: the entry of step j + 4 goes by them, and step j's weights have been taken now
      const uint32_t first = kv_cnt;  // tiles K(j), V(j) are first + 2 j, first + 2 j + 1
      auto tile_ready = [&](uint32_t t) { return mbar_wait_warp(&bars.kv_full[t % kKvSlots], (t / kKvSlots) & 1, ctx, kRoleMma | kBarKvFull); };
#pragma unroll 1
      for (int j = -2; j < it.n; ++j) {
        const int s = j & 1;  // selected, not indexed: the counters stay in registers
        const uint32_t q_par = (s ? q_cnt[1] : q_cnt[0]) & 1, sp_par = (s ? sp_cnt[1] : sp_cnt[0]) & 1;
        const uint32_t vt = first + 2 * j + 1, kt = first + 2 * (j + 2);
        if (j >= 0) {
          if (!tile_ready(vt)) return;
          const uint64_t v_desc = vtile_desc(base + kTSmemKv + (vt % kKvSlots) * kTileBytes);
          const uint32_t t_o = tmem + 2 * kTile + s * kTile, t_p = tmem + s * kTile;
          if (j < 2 && !mbar_wait_warp(&bars.o_empty[s], q_par ^ 1, ctx, kRoleMma | kBarOEmpty)) return;
          if (!mbar_wait_warp(&bars.p_half[s], sp_par, ctx, kRoleMma | kBarPHalf)) return;
          tc_fence_after_sync();
          issue_pv_f16(leader, t_o, t_p, v_desc, j >= 2, 0, 4);
          if (!mbar_wait_warp(&bars.p_full[s], sp_par, ctx, kRoleMma | kBarPFull)) return;
          if (s) {
            ++sp_cnt[1];
          } else {
            ++sp_cnt[0];
          }
          tc_fence_after_sync();
          issue_pv_f16(leader, t_o, t_p, v_desc, j >= 2, 4, 8);
          if (leader) {
            mma_commit(&bars.kv_empty[vt % kKvSlots]);
            if (j + 1 < it.n) mma_commit(&bars.kv_empty[(vt + 1) % kKvSlots]);
            if (j + 2 >= it.n) mma_commit(&bars.o_full[s]);
          }
        }
        if (j + 2 < it.n) {
          if (!tile_ready(kt)) return;
          if (j < 0 && !mbar_wait_warp(&bars.q_full[s], q_par, ctx, kRoleMma | kBarQFull)) return;
          tc_fence_after_sync();
          issue_qk_f16(leader, tmem + s * kTile, s ? q_desc[1] : q_desc[0], kmajor_desc(base + kTSmemKv + (kt % kKvSlots) * kTileBytes));
          if (leader) mma_commit(&bars.s_full[s]);
        }
        if (leader && j == -2) mma_commit(&bars.kv_empty[kt % kKvSlots]);
      }
      kv_cnt = first + 2 * it.n;
      ++q_cnt[0];
      ++q_cnt[1];
      continue;
    }
    {
      const uint32_t slot = kv_cnt % kKvSlots, par = (kv_cnt / kKvSlots) & 1;
      if (!mbar_wait_warp(&bars.kv_full[slot], par, ctx, kRoleMma | kBarKvFull)) return;
      const uint64_t k_desc = kmajor_desc(base + kTSmemKv + slot * kTileBytes);
#pragma unroll
      for (int s = 0; s < 2; ++s) {
        if (s == 0 || it.two) {
          if (!mbar_wait_warp(&bars.q_full[s], q_cnt[s] & 1, ctx, kRoleMma | kBarQFull)) return;
          tc_fence_after_sync();
          issue_qk_f16(leader, tmem + s * kTile, q_desc[s], k_desc);
          if (leader) mma_commit(&bars.s_full[s]);
        }
      }
      if (leader) mma_commit(&bars.kv_empty[slot]);
      ++kv_cnt;
    }
    for (int j = 0; j < it.n; ++j) {
      const uint32_t vslot = kv_cnt % kKvSlots, vpar = (kv_cnt / kKvSlots) & 1;
      ++kv_cnt;
      const bool has_next = j + 1 < it.n;
      uint32_t kslot = 0, kpar = 0;
      if (has_next) {
        kslot = kv_cnt % kKvSlots;
        kpar = (kv_cnt / kKvSlots) & 1;
        ++kv_cnt;
      }
      if (!mbar_wait_warp(&bars.kv_full[vslot], vpar, ctx, kRoleMma | kBarKvFull)) return;
      bool k_ready = false;
      const uint64_t v_desc = vtile_desc(base + kTSmemKv + vslot * kTileBytes);
      const uint64_t k_desc = kmajor_desc(base + kTSmemKv + kslot * kTileBytes);
#pragma unroll
      for (int s = 0; s < 2; ++s) {
        if (s == 0 || it.two) {
          if (j == 0) {  // the previous item's O must have left tensor memory
            if (!mbar_wait_warp(&bars.o_empty[s], (q_cnt[s] & 1) ^ 1, ctx, kRoleMma | kBarOEmpty)) return;
          }
          if (!mbar_wait_warp(&bars.p_half[s], sp_cnt[s] & 1, ctx, kRoleMma | kBarPHalf)) return;
          tc_fence_after_sync();
          issue_pv_f16(leader, tmem + 2 * kTile + s * kTile, tmem + s * kTile, v_desc, j > 0, 0, 4);
          if (!mbar_wait_warp(&bars.p_full[s], sp_cnt[s] & 1, ctx, kRoleMma | kBarPFull)) return;
          ++sp_cnt[s];
          tc_fence_after_sync();
          issue_pv_f16(leader, tmem + 2 * kTile + s * kTile, tmem + s * kTile, v_desc, j > 0, 4, 8);
          if (leader && !has_next) mma_commit(&bars.o_full[s]);
          if (leader && (s == 1 || !it.two)) mma_commit(&bars.kv_empty[vslot]);
          if (has_next) {
            if (!k_ready) {
              if (!mbar_wait_warp(&bars.kv_full[kslot], kpar, ctx, kRoleMma | kBarKvFull)) return;
              tc_fence_after_sync();
              k_ready = true;
            }
            issue_qk_f16(leader, tmem + s * kTile, q_desc[s], k_desc);
            if (leader) mma_commit(&bars.s_full[s]);
          }
        }
      }
      if (leader && has_next) mma_commit(&bars.kv_empty[kslot]);
    }
    ++q_cnt[0];
    if (it.two) ++q_cnt[1];
  }
}

__device__ __forceinline__ void cp_async16(uint32_t dst, const void* src, bool take) {
  const int bytes = take ? 16 : 0;  // 0: zeros are written, nothing is read
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst), "l"(src), "r"(bytes) : "memory");
}
__device__ __forceinline__ void cp_async_wait_all() { asm volatile("cp.async.wait_all;" ::: "memory"); }

// ---- softmax: one thread owns one row of stage `s` ------------------------------------------------------------------------
template <int GRAN>
__device__ __forceinline__ void role_tile_softmax(const CachedParams& p, const TileBarriers& bars, uint8_t* smem, WaitCtx ctx,
                                                  uint32_t tmem, int s, int row, int lane) {
  const uint32_t lane_sel = static_cast<uint32_t>(row & ~31) << 16;
  const uint32_t t_s = tmem + lane_sel + s * kTile;
  const uint32_t t_o = tmem + lane_sel + 2 * kTile + s * kTile;
  float* stats = reinterpret_cast<float*>(smem + kTSmemStats) + s * 2 * kTile;
  uint32_t s_cnt = 0, l_cnt = 0, step = 0;
  for (uint32_t k = 0;; ++k) {
    int n, key0;  // steps of the item, first key of the step
    int first, stride;  // the stage's first step, and from one of its steps to the next
    bool idle;    // none of the warp's rows is real: it only keeps the barriers going
    int limit;    // keys the row sees; rows that are not real see all
    int clear;    // keys that all rows of the stage see: steps up to there need no mask
    float factor;
    bool used;
    bool seen;    // the row sees a key here
    {
      Item it;
      if (!take_item(bars, smem, k, ctx, kRoleSoftmax, lane, it) || it.n == 0) return;
      n = it.n;
      used = s == 0 || it.two || it.split;
      first = it.split ? s : 0;
      stride = it.split ? 2 : 1;
      if (used) {
        // Q: the stage's last product that reads it has completed (its scores have been taken)
        const int r0 = it.tile * kTileRows + (it.two ? s * kTile : 0);
        const TilePlace w = tile_place(p, it.s, it.h, r0 + row);
        limit = w.real ? visible(it.s, w.token, p.causal) : it.s.keys;
        clear = visible(it.s, min(r0 / p.group, it.s.n - 1), p.causal);
        key0 = (it.t_first + first) * kStepKeys;
        seen = limit > key0;
        idle = !__any_sync(0xffffffffu, w.real);
        // This code runs once an item, so it is never in the instruction cache: short loops take a fifth of the time that the same
        // work takes unrolled.  Half a warp brings a row, 16 bytes a lane, to its place in the swizzled order; then each
        // thread reads its own row, every lane beginning at another 16 bytes, and turns it into f16 in place
        const long long at = w.real ? row_offset(p, p.sq, it.b, it.s, w) : -1;
        uint8_t* tile = smem + kTSmemQ + s * kTileBytes + (row & ~31) * 128;
        {
          const uint32_t dst = smem_u32(tile) + ((lane & 15) >> 3) * kHalfBytes;
          const uint16_t* q = p.q + (lane & 15) * 8;
#pragma unroll 2
          for (int r = lane >> 4; r < 32; r += 2) {
            const long long from = __shfl_sync(0xffffffffu, at, r);
            cp_async16(dst + r * 128 + (((lane & 7) ^ (r & 7)) << 4), q + max(from, 0ll), from >= 0);
          }
          cp_async_wait_all();
          __syncwarp();
        }
        uint8_t* mine = tile + lane * 128;
        float largest = 0.f;
#pragma unroll 2
        for (int i = 0; i < 16; ++i) {
          const uint4 x = *reinterpret_cast<const uint4*>(mine + (i >> 3) * kHalfBytes + (((i + lane) & 7) << 4));
          const uint32_t words[4] = {x.x, x.y, x.z, x.w};
#pragma unroll
          for (int m = 0; m < 4; ++m) {
            const float2 f = unpack_bf16x2(words[m]);
            largest = max3(largest, fabsf(f.x), fabsf(f.y));
          }
        }
        const float my_up = row_factor(largest);
#pragma unroll 2
        for (int i = 0; i < 16; ++i) {
          uint4* place = reinterpret_cast<uint4*>(mine + (i >> 3) * kHalfBytes + (((i + lane) & 7) << 4));
          const uint4 x = *place;
          const uint32_t words[4] = {x.x, x.y, x.z, x.w};
          uint32_t y[4];
#pragma unroll
          for (int m = 0; m < 4; ++m) {
            const float2 f = unpack_bf16x2(words[m]);
            y[m] = pack_f16x2(f.x * my_up, f.y * my_up);
          }
          *place = make_uint4(y[0], y[1], y[2], y[3]);
        }
        factor = p.scale_log2 / my_up;
        fence_proxy_async_smem();
        __syncwarp();
        if (lane == 0) mbar_arrive(&bars.q_full[s]);
      }
    }
    if (used) {
      float m_used = -INFINITY;  // reference maximum, log2 units, an integer
      float l = 0.f;
      for (int j = first; j < n; j += stride, key0 += stride * kStepKeys) {
        if (idle) {
          bool ok = mbar_wait(&bars.s_full[s], s_cnt & 1, ctx, kRoleSoftmax | kBarSFull);
          if (!__all_sync(0xffffffffu, ok)) return;
          ++s_cnt;
          if (lane == 0) {
            mbar_arrive(&bars.p_half[s]);
            mbar_arrive(&bars.p_full[s]);
          }
          continue;
        }
        const uint32_t q = (step + j) % kMetaSteps;
        bool ok = mbar_wait(&bars.meta_full[q], ((step + j) / kMetaSteps) & 1, ctx, kRoleSoftmax | kBarMeta);
        const float* meta = reinterpret_cast<const float*>(smem + kTSmemMeta) + q * kMetaFloats;
        float cg[kTile / GRAN];
#pragma unroll
        for (int g = 0; g < kTile / GRAN; ++g) cg[g] = fmaxf(meta[kMetaK + g * (GRAN / 16)] * factor, 1e-37f);  // not 0: -inf stays -inf
        ok = ok && mbar_wait(&bars.s_full[s], s_cnt & 1, ctx, kRoleSoftmax | kBarSFull);
        ok = __all_sync(0xffffffffu, ok);
        if (!ok) return;
        ++s_cnt;
        tc_fence_after_sync();
        uint32_t xr[kTile];
        tmem_ld_x32(t_s + 0, xr + 0);
        tmem_ld_x32(t_s + 32, xr + 32);
        tmem_ld_x32(t_s + 64, xr + 64);
        tmem_ld_x32(t_s + 96, xr + 96);
        tmem_wait_ld();
#define X(i) __uint_as_float(xr[(i)])
        if (key0 + kStepKeys > clear) {  // warp-uniform
          const int vis = limit - key0;
#pragma unroll
          for (int i = 0; i < kTile; ++i) {
            if (i >= vis) xr[i] = 0xff800000u;
          }
        }
        float m_blk = -INFINITY;
        const float floor = meta[kMetaFloor];
#pragma unroll
        for (int g = 0; g < kTile / GRAN; ++g) {
          float top[4];
#pragma unroll
          for (int c = 0; c < 4; ++c) {
            const int i = g * GRAN + c * (GRAN / 4);
            top[c] = max3(X(i), X(i + 1), X(i + 2));
#pragma unroll
            for (int k = 3; k + 1 < GRAN / 4; k += 2) top[c] = max3(top[c], X(i + k), X(i + k + 1));
            top[c] = fmaxf(top[c], X(i + GRAN / 4 - 1));
          }
          m_blk = fmaxf(m_blk, fmaf(fmaxf(fmaxf(top[0], top[1]), fmaxf(top[2], top[3])), cg[g], fmaxf(meta[kMetaV + g * (GRAN / 16)], floor)));
        }
        if (j == first) {
          m_used = m_blk == -INFINITY ? 0.f : ceilf(m_blk);
        } else {
          if (__any_sync(0xffffffffu, m_blk - m_used > kWeightLag)) {
            // P V of the step before has completed (S of this one was issued after it): O is quiescent
            const float m_new = fmaxf(m_used, ceilf(m_blk));
            const float f = ex2_approx(m_used - m_new);
            l *= f > 0.f ? f : 0x1p-126f;
            if (f == 0.f) l *= ex2_approx(m_used - m_new + 126.f);  // scales far apart: what is nothing beside O may be most of the row sum
            m_used = m_new;
#pragma unroll
            for (int cc = 0; cc < 8; ++cc) {
              uint32_t o[16];
              tmem_ld_x16(t_o + cc * 16, o);
              tmem_wait_ld();
#pragma unroll
              for (int i = 0; i < 16; ++i) o[i] = __float_as_uint(__uint_as_float(o[i]) * f);
              tmem_st_x16(t_o + cc * 16, o);
            }
          }
        }
        const float neg_m = kWeightShift - m_used;
        float2 sum = make_float2(0.f, 0.f), part = make_float2(0.f, 0.f);
#pragma unroll
        for (int cc = 0; cc < 4; ++cc) {
          uint32_t pk[16];
#pragma unroll
          for (int h = 0; h < 2; ++h) {  // 16 keys
            const int g = (cc * 2 + h) * 16 / GRAN;
            const float add = neg_m + meta[kMetaV + g * (GRAN / 16)];
            const float2 c2 = make_float2(cg[g], cg[g]), a2 = make_float2(add, add);
#pragma unroll
            for (int k = 0; k < 8; ++k) {
              const int i = (cc * 2 + h) * 16 + k * 2;
              const float2 x = fma2(make_float2(X(i), X(i + 1)), c2, a2);
              const float2 e = make_float2(ex2_approx(x.x), ex2_approx(x.y));
              part = add2(part, e);
              pk[h * 8 + k] = pack_f16x2(e.x, e.y);
            }
            if (((cc * 2 + h) * 16 + 16) % GRAN == 0) {
              const float inv = meta[kMetaInv + g * (GRAN / 16)];
              sum = fma2(part, make_float2(inv, inv), sum);
              part = make_float2(0.f, 0.f);
            }
          }
          tmem_st_x16(t_s + cc * 16, pk);
          if (cc == 1) {
            tmem_wait_st();
            tc_fence_before_sync();
            if (lane == 0) mbar_arrive(&bars.p_half[s]);
          }
        }
#undef X
        l += sum.x + sum.y;
        const int bad = reinterpret_cast<const int*>(meta)[kMetaBad];
        if (bad < kStepKeys && key0 + bad < limit) l = __int_as_float(0x7fffffff);
        tmem_wait_st();
        tc_fence_before_sync();
        if (lane == 0) mbar_arrive(&bars.p_full[s]);
      }
      bool ok = mbar_wait(&bars.l_empty[s], (l_cnt & 1) ^ 1, ctx, kRoleSoftmax | kBarLEmpty);
      ok = __all_sync(0xffffffffu, ok);
      if (!ok) return;
      // a row that has seen no key here has the sum 0 by definition, and no maximum
      stats[row] = seen ? l : 0.f;
      stats[kTile + row] = seen ? m_used : -INFINITY;
      mbar_arrive(&bars.l_full[s]);
      ++l_cnt;
    }
    step += n;
  }
}

// A thread writes rows of its own, so every store of a warp meets 32 lines: the fewer and wider the stores, the better.
__device__ __forceinline__ void store_32_bytes(void* at, const uint32_t* v, bool aligned) {
  if (aligned) {
    asm volatile("st.global.v8.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};" ::"l"(at), ATTN_W4(v, 0), ATTN_W4(v, 4) : "memory");
  } else {
    reinterpret_cast<uint4*>(at)[0] = make_uint4(v[0], v[1], v[2], v[3]);
    reinterpret_cast<uint4*>(at)[1] = make_uint4(v[4], v[5], v[6], v[7]);
  }
}

// ---- results ----------------------------------------------------------------------------------------------------------------
__device__ __forceinline__ bool write_item(const CachedParams& p, const TileBarriers& bars, const uint8_t* smem, WaitCtx ctx, uint32_t tmem,
                                           uint32_t k, uint32_t* cnt, int row, int lane) {
  const uint32_t lane_sel = static_cast<uint32_t>(row & ~31) << 16;
  Item it;
  read_item(smem, k, it);
#pragma unroll 1
  for (int s = 0; s < 2; ++s) {
    if (s == 1 && !it.two) continue;
    float l = 0.f, m = -INFINITY, f[2] = {0.f, 0.f};  // the stage's part, or both stages' joined: O = f[0] O0 + f[1] O1
    {
      float lq[2], mq[2];
#pragma unroll
      for (int q = 0; q < 2; ++q) {
        if (q == 1 && !it.split) break;
        const float* stats = reinterpret_cast<const float*>(smem + kTSmemStats) + (s + q) * 2 * kTile;
        const bool ok = mbar_wait(&bars.l_full[s + q], cnt[s + q] & 1, ctx, kRoleEpilogue | kBarLFull);
        if (!__all_sync(0xffffffffu, ok)) return false;
        lq[q] = stats[row];
        mq[q] = stats[kTile + row];
        mbar_arrive(&bars.l_empty[s + q]);
        m = fmaxf(m, mq[q]);
      }
#pragma unroll
      for (int q = 0; q < 2; ++q) {
        if (q == 1 && !it.split) break;
        const bool ok = mbar_wait(&bars.o_full[s + q], cnt[s + q] & 1, ctx, kRoleEpilogue | kBarOFull);
        if (!__all_sync(0xffffffffu, ok)) return false;
        ++cnt[s + q];
        const float h = mq[q] == -INFINITY ? 0.f : ex2_approx(0.5f * (mq[q] - m));
        l += mq[q] == -INFINITY ? lq[q] : lq[q] * h * h;  // the sum of a row that has seen no key is 0
        f[q] = h * h;
      }
    }
    tc_fence_after_sync();
    const int r = s * kTile + row;
    const TilePlace w = tile_place(p, it.s, it.h, it.tile * kTileRows + r);
    // keys beyond the table's reach
    if (w.real && it.s.len > it.s.keys && (!p.causal || it.s.len - it.s.n + w.token >= it.s.keys)) l = __int_as_float(0x7fffffff);
    const uint32_t t_o = tmem + lane_sel + 2 * kTile + s * kTile;
    const long long slot = 2ll * blockIdx.x + (it.t_first == 0 ? 1 : 0);
    if (it.whole) {
      const float inv = l == 0.f ? 0.f : __fdividef(1.f, l);
      f[0] *= inv;
      f[1] *= inv;
    }
    uint16_t* out = p.o + row_offset(p, p.so, it.b, it.s, w);
    float* part = p.parts + (slot * kTileRows + r) * kKvDim;
#pragma unroll 2
    for (int cc = 0; cc < 8; ++cc) {
      uint32_t o[16], o1[16];
      tmem_ld_x16(t_o + cc * 16, o);
      if (it.split) tmem_ld_x16(t_o + kTile + cc * 16, o1);
      tmem_wait_ld();
#pragma unroll
      for (int i = 0; i < 16; ++i) {
        float x = __uint_as_float(o[i]) * f[0];
        if (it.split) x = fmaf(__uint_as_float(o1[i]), f[1], x);
        o[i] = __float_as_uint(x);
      }
      if (w.real && it.whole) {
        uint32_t val[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) val[i] = pack_bf16x2(__uint_as_float(o[2 * i]), __uint_as_float(o[2 * i + 1]));
        store_32_bytes(out + cc * 16, val, p.wide_o);
      } else if (w.real) {
        store_32_bytes(part + cc * 16, o, true);
        store_32_bytes(part + cc * 16 + 8, o + 8, true);
      }
      __syncwarp();
    }
    tc_fence_before_sync();
    __syncwarp();
    if (lane == 0) {
      mbar_arrive(&bars.o_empty[s]);
      if (it.split) mbar_arrive(&bars.o_empty[1]);
    }
    if (it.whole) {
      if (w.real && p.lse != nullptr)
        p.lse[lse_index(p, it.b, it.s, w)] = lse_of(m, l);
    } else {
      reinterpret_cast<float2*>(p.parts + 2ll * p.ctas * kTileRows * kKvDim)[slot * kTileRows + r] = make_float2(m, l);
      if (r == 0 && it.t_first == 0) {
        p.pieces[2 * blockIdx.x] = make_int4(it.b, it.h, it.tile, it.last);
        p.pieces[2 * blockIdx.x + 1] = make_int4(it.s.row0, it.s.n, 0, 0);
      }
    }
  }
  drop_item(bars, k, lane);
  return true;
}

// Converter warps.  Those that `write` write an item's results one step into the next one, when its last product is long done;
// the two steps of tiles that lie converted by then keep the tensor pipe busy meanwhile.
template <int TYPE>
__device__ __forceinline__ void role_convert(const CachedParams& p, const TileBarriers& bars, uint8_t* smem, WaitCtx ctx, uint32_t tmem,
                                             int cw, bool writes, int row, int lane) {
  uint32_t cnt[2] = {0, 0};
  uint32_t step = 0;
  for (uint32_t k = 0;; ++k) {
    if (!wait_item(bars, k, ctx, kRoleEpilogue)) return;
    const int n = item_box(smem, k)[0];
    if (!writes) drop_item(bars, k, lane);
    for (int j = 0; j < max(n, 1); ++j, ++step) {
      if (n > 0 && !convert_step<TYPE>(bars, smem, ctx, step, cw, lane)) return;
      if (writes && j == 0 && k > 0 && !write_item(p, bars, smem, ctx, tmem, k - 1, cnt, row, lane)) return;
    }
    if (n == 0) return;
  }
}

template <int TYPE, int GRAN>
__global__ void __launch_bounds__(kThreads, 1) attn_cached_tile_kernel(const __grid_constant__ CUtensorMap tm_k,
                                                                     const __grid_constant__ CUtensorMap tm_v, const CachedParams p) {
  extern __shared__ __align__(1024) uint8_t smem[];
  uint64_t* bar_mem = reinterpret_cast<uint64_t*>(smem + kTSmemBars);
  TileBarriers bars;
  bars.q_full = bar_mem;
  bars.raw_full = bars.q_full + 2;
  bars.raw_empty = bars.raw_full + 2;
  bars.kv_full = bars.raw_empty + 2;
  bars.kv_empty = bars.kv_full + kKvSlots;
  bars.s_full = bars.kv_empty + kKvSlots;
  bars.p_half = bars.s_full + 2;
  bars.p_full = bars.p_half + 2;
  bars.o_full = bars.p_full + 2;
  bars.o_empty = bars.o_full + 2;
  bars.l_full = bars.o_empty + 2;
  bars.l_empty = bars.l_full + 2;
  bars.meta_full = bars.l_empty + 2;
  bars.item_full = bars.meta_full + kMetaSteps;
  bars.item_empty = bars.item_full + kItemSlots;
  uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(smem + kTSmemMisc);
  volatile int* abort_flag = reinterpret_cast<volatile int*>(smem + kTSmemMisc + 4);
  const WaitCtx ctx{abort_flag, p.status, kWaitLimitNs};
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;

  if (tid == 0) p.pieces[2 * blockIdx.x] = make_int4(0, 0, 0, -1);
  if ((smem_u32(smem) & 1023u) != 0) {  // the swizzled tiles need a 1024-byte aligned base
    if (tid == 0 && atomicCAS(p.status, 0, kBadSmemAlign) == 0) p.status[1] = static_cast<int>(blockIdx.x);
    return;
  }
  if (tid == 0) {
    tma_prefetch_desc(&tm_k);
    tma_prefetch_desc(&tm_v);
  }
  Line line;
  Cursor<kTileRows> cur;
  if (!find_piece<kTileRows>(p, line, cur, reinterpret_cast<long long*>(smem))) return;
  if (tid == 0) {
    for (int i = 0; i < 2; ++i) {
      mbar_init(&bars.q_full[i], 4);
      mbar_init(&bars.raw_full[i], 1);
      mbar_init(&bars.raw_empty[i], kConvWarps);
      mbar_init(&bars.s_full[i], 1);
      mbar_init(&bars.p_half[i], 4);
      mbar_init(&bars.p_full[i], 4);
      mbar_init(&bars.o_full[i], 1);
      mbar_init(&bars.o_empty[i], 4);
      mbar_init(&bars.l_full[i], kTile);
      mbar_init(&bars.l_empty[i], kTile);
    }
    for (int i = 0; i < kKvSlots; ++i) {
      mbar_init(&bars.kv_full[i], kConvWarps);
      mbar_init(&bars.kv_empty[i], 1);
    }
    for (int i = 0; i < kMetaSteps; ++i) mbar_init(&bars.meta_full[i], 1);
    for (int i = 0; i < kItemSlots; ++i) {
      mbar_init(&bars.item_full[i], 1);
      mbar_init(&bars.item_empty[i], kItemReaders);
    }
    *abort_flag = 0;
    fence_mbar_init();
  }
  if (warp == 12) {
    tmem_alloc(tmem_slot, 512);
    tmem_relinquish();
  }
  tc_fence_before_sync();
  __syncthreads();
  tc_fence_after_sync();
  const uint32_t tmem = *tmem_slot;
  let_next_start();

  if (warp < 8) {
    reg_alloc<kTRegsSoftmax>();
    role_tile_softmax<GRAN>(p, bars, smem, ctx, tmem, warp >> 2, tid & 127, lane);
  } else {
    reg_dealloc<kTRegsOther>();
    if (warp == 12) {
      role_tile_mma(bars, smem, ctx, tmem, lane);
    } else if (warp == 13) {
      role_fetch(p, bars, smem, ctx, line, cur, lane, &tm_k, &tm_v);
      if (*abort_flag) {  // let loads in flight land before the CTA's shared memory is released
        const uint64_t t0 = global_timer_ns();
        while (global_timer_ns() - t0 < 1000000ull) {
        }
      }
    } else {
      role_convert<TYPE>(p, bars, smem, ctx, tmem, warp < 12 ? warp - 8 : warp - 10, warp < 12, tid & 127, lane);
    }
  }
  tc_fence_before_sync();
  __syncthreads();
  if (warp == 12) {
    tc_fence_after_sync();
    tmem_dealloc(tmem, 512);
  }
}

}  // namespace kv
}  // namespace attn
