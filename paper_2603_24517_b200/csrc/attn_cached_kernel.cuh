// Attention of new tokens over a paged 8-bit cache, for few query rows a key head (decoding).
//
//     s_ij = scale k_scale(page of j) q_i . c^K_j,    o_i = sum_j softmax_j(s_ij) v_scale(page of j) c^V_j
//
// Bound by HBM: 256 bytes a cached token and key head, read once for all query heads of the group.  A query tile is 8 or 16
// rows (token, head of the group), heads fastest.  All work is a line of (sequence, key head, query tile, 128 keys) steps, cut
// into equal contiguous pieces, one a CTA, whatever the lengths are; the cut is computed on the device from the lengths.  A
// CTA that holds a whole tile's keys writes its result, the others leave fp32 parts, which a second kernel joins in order.
//
// In a CTA each of 8 warps owns 16 keys of a step and works alone until its piece of a tile ends: its own ring of 4 KB stages
// filled by TMA, its own running maximum, sum and accumulator.  16 keys lie in one page, so the scales are one factor a warp
// and step.  The products are S^T = K Q^T and O^T = V^T P^T by mma.m16n8k16 (f16): the keys, then the head dimension fill the 16
// rows of the left operand, so 8 query rows leave nothing idle (with the queries on the left, 16 rows were computed for any
// group).  Codes go from shared memory to the left operand without a transpose: the inner index of a product may be in
// any order, so a lane takes 16 consecutive head dimensions of its keys (K) or of four keys (V) and the queries are loaded in the
// same order; the weights change sides by movmatrix.  Which key and which 16 dimensions a lane takes is chosen (`spread`) so that
// the reads of a 128-byte-swizzled stage meet no bank twice.
// Codes are exact in f16; queries are scaled by a power of two of their row, weights are held as 2^6 exp(s - m) with a maximum
// that may lag by a factor of 2^8 (so it is reduced over the lanes only when one of them meets a larger score), which leaves
// f16 its 11 bits of both; V's scale is part of the exponent (below).
//
// 64 sequences of up to 8192 tokens (32 / 8 heads, E4M3, 744 MB): 132 us, 5.6 TB/s, 88 % of the copy rate; INT8 codes take 10 %
// longer.  One token on 512: 10.0 us, all latency (lengths, pages, codes, merge, join).  What a lone warp of a scheduler could not
// hide bounded the first form (8 warps an SM, 217 us).  Measured slower: tiles of 16 rows at two CTAs an SM (186 us for 16
// sequences where one CTA takes 112: spills), of 32 rows (213), the merge in loops (9.9 against 9.5 us for the short one).
#pragma once

#include "attn_fwd_kernel.cuh"
#include "kv_cache_kernel.cuh"

namespace attn {
namespace kv {

constexpr int kDecWarps = 8;
constexpr int kDecThreads = kDecWarps * 32;
constexpr int kStepKeys = 128;                         // keys a CTA takes in one step: 16 a warp
constexpr int kWarpStageBytes = 2 * 16 * kKvDim;       // K then V
constexpr float kWeightShift = 6.f;   // weights are held as 2^kWeightShift exp(s - m)
constexpr float kWeightLag = 8.f;     // log2 units the reference maximum may lag

// A key's weight in the product with the values is 2^(s_j + log2 vs_j - M): s_j the score in log2 units, vs_j the V scale of its page
// and head, M a running maximum of s_j + log2 vs_j over the keys that the row sees, rounded up to an integer.  So the weights of
// what counts most in the row's result have the full f16 precision whatever the scales are, nothing overflows for values near the
// end of their range, and tokens that the row does not see have no part in it.  The row sum takes the scale out again,
// l = sum_j 2^(s_j + log2 vs_j - M) / vs_j, and O / l needs no factor.  M is an integer, so that it costs no rounding in the exponents
// and in the log-sum-exp.
// Scales of 0 need a number: with R the largest log2 vs so far (at least kScaleLeast), log2 vs counts as R - kScaleZero at least, and as R -
// kScaleSpan at least in the maximum.  A weight of such a page is then 2^(6 + 8 - 40) at most, which is 0 in f16, while its part of the row
// sum stays a normal fp32 number.
constexpr float kScaleLeast = -20.f;
constexpr float kScaleSpan = 64.f;
constexpr float kScaleZero = 104.f;
static_assert(kScaleZero - kScaleSpan - kWeightShift - kWeightLag > 25.f, "weights of scale 0 vanish in f16");
static_assert(kScaleZero - kScaleLeast < 126.f, "the inverse of the least scale is a normal number");

// Query tiles of 8 NB rows.  8 rows: two CTAs an SM, so that one's start and end run beside the other's steps; 16 rows need
// 233 registers.
template <int NB>
struct Dec {
  static constexpr int kRows = 8 * NB;
  static constexpr int kCtasPerSm = NB == 1 ? 2 : 1;
  static constexpr int kStages = NB == 1 ? 2 : 4;
  static constexpr int kRing = kDecWarps * kStages * kWarpStageBytes;
  static constexpr int kMerge = kDecWarps * kRows * kKvDim * 4;
  static constexpr int kStats = kDecWarps * kRows * 8;
  static constexpr int kBars = kDecWarps * kStages * 8;
  static constexpr int kSmem = kRing + kMerge + kStats + kBars + 16 + 1024;  // 1024: the ring starts at a multiple of it
};

struct CachedParams {
  CacheView c;
  const uint16_t* q;
  uint16_t* o;
  float* lse;             // [B, Hq, S], or [Hq, S] with starts; may be null
  RowStrides sq, so;
  int Hq, group, causal;
  int rows_above, rows_up_to;  // the launch is for sequences of more than / at most so many rows (tokens times heads of the group)
  float scale_log2;       // scale * log2(e)
  float* parts;           // [2 ctas][rows][kKvDim], then [2 ctas][rows][2] (reference maximum in log2 units, sum)
  int4* pieces;           // [ctas][2]: {sequence, head, tile, last CTA with a part or -1}, {first row, rows of the sequence} of the
                          // tile that the CTA began and did not end
  int ctas;
  int wide_o;             // rows of o begin at multiples of 32 bytes
  int* status;            // bounded waits that ran out, see WaitCtx
};

// One sequence of the line of work.
struct SeqWork {
  int row0, n;       // its rows
  int len;           // tokens in all, at least 0
  int keys;          // of them in the table's reach
};
__device__ __forceinline__ SeqWork seq_work(const CachedParams& p, int b) {
  const CacheView& c = p.c;
  SeqWork s;
  rows_of(c, b, s.row0, s.n);
  const int rows = s.n * p.group;
  if (rows <= p.rows_above || rows > p.rows_up_to) s.n = 0;  // another launch's
  s.len = max(__ldg(c.lens + b), 0);
  s.keys = static_cast<int>(min(static_cast<long long>(s.len), static_cast<long long>(c.max_blocks) << c.page_log2));
  return s;
}
// Keys that row token i of the sequence sees (0: none).
__device__ __forceinline__ int visible(const SeqWork& s, int i, int causal) {
  return causal ? min(s.keys, max(s.len - s.n + i + 1, 0)) : s.keys;
}
// Steps of a tile whose last row token is i: at least one, so that rows that see nothing are written too.
__device__ __forceinline__ int steps_of(const SeqWork& s, int i, int causal) {
  return max((visible(s, i, causal) + kStepKeys - 1) / kStepKeys, 1);
}

template <int ROWS>
__device__ __forceinline__ int tile_steps(const CachedParams& p, const SeqWork& s, int tile) {
  return steps_of(s, min((tile * ROWS + ROWS - 1) / p.group, s.n - 1), p.causal);
}
template <int ROWS>
__device__ __forceinline__ int tiles_of(const CachedParams& p, const SeqWork& s) {
  return (s.n * p.group + ROWS - 1) / ROWS;
}

// A place on the line of work.
template <int ROWS>
struct Cursor {
  int b, h, tile, t, steps, tiles;
  SeqWork s;
  __device__ __forceinline__ void enter_tile(const CachedParams& p) {
    steps = tile_steps<ROWS>(p, s, tile);
  }
  __device__ __forceinline__ void enter_sequence(const CachedParams& p) {
    s = seq_work(p, b);
    tiles = tiles_of<ROWS>(p, s);
  }
  __device__ __forceinline__ void next_tile(const CachedParams& p) {  // of the head, then the next head, the next sequence
    t = 0;
    if (++tile >= tiles) {
      tile = 0;
      if (++h >= p.c.Hkv) {
        h = 0;
        do {
          if (++b >= p.c.B) return;
          enter_sequence(p);
        } while (tiles == 0);
      }
    }
    enter_tile(p);
  }
};

// Steps of one head of a sequence.
template <int ROWS>
__device__ __forceinline__ long long head_steps(const CachedParams& p, const SeqWork& s) {
  const int tiles = tiles_of<ROWS>(p, s);
  if (tiles == 0) return 0;
  if (!p.causal) return static_cast<long long>(tiles) * steps_of(s, s.n - 1, 0);
  long long sum = 0;
  for (int k = 0; k < tiles; ++k) sum += tile_steps<ROWS>(p, s, k);
  return sum;
}
// The same by a whole warp (one sequence in all lanes): 8192 tokens of four heads are 128 tiles, 10 us for one lane.
template <int ROWS>
__device__ __forceinline__ long long head_steps_warp(const CachedParams& p, const SeqWork& s, int lane) {
  const int tiles = tiles_of<ROWS>(p, s);
  if (!p.causal || tiles <= 1) return head_steps<ROWS>(p, s);
  long long sum = 0;
  for (int k = lane; k < tiles; k += 32) sum += tile_steps<ROWS>(p, s, k);
#pragma unroll
  for (int m = 16; m > 0; m >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, m);
  return sum;
}
// Which tile holds step `left` of a head, and the step within it.
template <int ROWS>
__device__ __forceinline__ void find_tile(const CachedParams& p, const SeqWork& s, long long left, int lane, int& tile, int& t) {
  if (!p.causal) {  // tiles of equal length
    const int steps = steps_of(s, s.n - 1, 0);
    tile = static_cast<int>(left / steps);
    t = static_cast<int>(left - static_cast<long long>(tile) * steps);
    return;
  }
  if (ROWS <= 16) {  // decoding: a tile or two
    tile = 0;
    for (int n = tile_steps<ROWS>(p, s, 0); left >= n; n = tile_steps<ROWS>(p, s, ++tile)) left -= n;
    t = static_cast<int>(left);
    return;
  }
  const int tiles = tiles_of<ROWS>(p, s);
  for (int k0 = 0;; k0 += 32) {
    const int mine = k0 + lane < tiles ? tile_steps<ROWS>(p, s, k0 + lane) : 0;
    long long upto = mine;
#pragma unroll
    for (int m = 1; m < 32; m <<= 1) {
      const long long other = __shfl_up_sync(0xffffffffu, upto, m);
      if (lane >= m) upto += other;
    }
    const unsigned beyond = __ballot_sync(0xffffffffu, left < upto);
    if (beyond != 0 || k0 + 32 >= tiles) {
      const int src = beyond != 0 ? __ffs(beyond) - 1 : 31;
      tile = k0 + src;
      t = static_cast<int>(left - __shfl_sync(0xffffffffu, upto - mine, src));
      return;
    }
    left -= __shfl_sync(0xffffffffu, upto, 31);
  }
}

// The line of work as one CTA sees it.
struct Line {
  long long total;   // steps in all
  long long ctas;    // CTAs that have a piece
  long long begin, end;
  __device__ __forceinline__ long long owner(long long step) const { return ((step + 1) * ctas - 1) / total; }
};

// This CTA's piece of a line of `total` steps; false: it has none.
__device__ __forceinline__ bool cut_line(const CachedParams& p, Line& line, long long total) {
  line.total = total;
  line.ctas = min(static_cast<long long>(p.ctas), total);
  if (blockIdx.x >= line.ctas) return false;
  if (total < 1 << 20) {  // at most 2^11 CTAs: 32-bit divisions
    const uint32_t t = static_cast<uint32_t>(total), c = static_cast<uint32_t>(line.ctas);
    line.begin = t * blockIdx.x / c;
    line.end = t * (blockIdx.x + 1) / c;
  } else {
    line.begin = total * blockIdx.x / line.ctas;
    line.end = total * (blockIdx.x + 1) / line.ctas;
  }
  return true;
}

// Cuts the line and finds where this CTA's piece begins.  All threads call; `scratch` holds threads / 32 + 2 long longs.  Up to 32
// sequences a warp does it by itself; beyond, a thread's sequences are neighbours, so their sums are scanned once and only the
// thread that holds the place looks closer.  False for a CTA without a piece (of all its threads).
template <int ROWS>
__device__ __forceinline__ bool find_piece(const CachedParams& p, Line& line, Cursor<ROWS>& at, long long* scratch) {
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, warps = blockDim.x >> 5;
  const bool small = p.c.B <= 32;
  const int threads = small ? 32 : static_cast<int>(blockDim.x), me = small ? lane : static_cast<int>(threadIdx.x);
  const int per = (p.c.B + threads - 1) / threads;
  const int b0 = me * per, b1 = min(b0 + per, p.c.B);
  long long mine = 0;
  if (small && ROWS > 16) {
    // lane b has sequence b; those of many tiles are counted by the whole warp, one after another
    SeqWork s;
    s.n = s.row0 = s.len = s.keys = 0;
    if (lane < p.c.B) s = seq_work(p, lane);
    const bool many = p.causal && tiles_of<ROWS>(p, s) > 8;
    if (!many) mine = head_steps<ROWS>(p, s) * p.c.Hkv;
    for (unsigned left = __ballot_sync(0xffffffffu, many); left != 0; left &= left - 1) {
      const int src = __ffs(left) - 1;
      SeqWork x;
      x.row0 = 0;
      x.n = __shfl_sync(0xffffffffu, s.n, src);
      x.len = __shfl_sync(0xffffffffu, s.len, src);
      x.keys = __shfl_sync(0xffffffffu, s.keys, src);
      const long long sum = head_steps_warp<ROWS>(p, x, lane) * p.c.Hkv;
      if (lane == src) mine = sum;
    }
  } else {
    for (int b = b0; b < b1; ++b) mine += head_steps<ROWS>(p, seq_work(p, b)) * p.c.Hkv;
  }
  long long upto = mine;
#pragma unroll
  for (int m = 1; m < 32; m <<= 1) {
    const long long other = __shfl_up_sync(0xffffffffu, upto, m);
    if (lane >= m) upto += other;
  }
  long long found_at = 0;
  if (small) {
    if (!cut_line(p, line, __shfl_sync(0xffffffffu, upto, 31))) return false;
    const unsigned here = __ballot_sync(0xffffffffu, line.begin >= upto - mine && line.begin < upto);
    at.b = __ffs(here) - 1;
    found_at = __shfl_sync(0xffffffffu, upto - mine, at.b);
  } else {
    if (lane == 31) scratch[warp] = upto;
    __syncthreads();
    long long total = 0, before = 0;
    for (int w = 0; w < warps; ++w) {
      if (w == warp) before = total;
      total += scratch[w];
    }
    if (!cut_line(p, line, total)) return false;
    long long* found = scratch + warps;  // sequence, its first step
    long long from = before + upto - mine;
    if (line.begin >= from && line.begin < from + mine) {
      for (int b = b0; b < b1; ++b) {
        const long long cost = head_steps<ROWS>(p, seq_work(p, b)) * p.c.Hkv;
        if (line.begin < from + cost) {
          found[0] = b;
          found[1] = from;
          break;
        }
        from += cost;
      }
    }
    __syncthreads();
    at.b = static_cast<int>(found[0]);
    found_at = found[1];
  }
  long long left = line.begin - found_at;
  at.enter_sequence(p);
  const long long per_head = ROWS > 16 ? head_steps_warp<ROWS>(p, at.s, lane) : head_steps<ROWS>(p, at.s);
  at.h = line.total < 1 << 20 ? static_cast<int>(static_cast<uint32_t>(left) / static_cast<uint32_t>(per_head)) : static_cast<int>(left / per_head);
  left -= at.h * per_head;
  find_tile<ROWS>(p, at.s, left, lane, at.tile, at.t);
  at.enter_tile(p);
  return true;
}
// The launch behind this one may start to take its place on the SMs; it waits for this one's results itself.
__device__ __forceinline__ void let_next_start() { asm volatile("griddepcontrol.launch_dependents;" ::: "memory"); }
__device__ __forceinline__ void wait_for_launch_before() { asm volatile("griddepcontrol.wait;" ::: "memory"); }

__device__ __forceinline__ void mma_f16(float* d, const uint32_t* a, uint32_t b0, uint32_t b1) {
  asm volatile(
      "mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
      : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
      : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}
__device__ __forceinline__ uint32_t pack_f16x2(float lo, float hi) {
  uint32_t y;
  asm("cvt.rn.f16x2.f32 %0, %1, %2;" : "=r"(y) : "f"(hi), "f"(lo));
  return y;
}
// The power of two that brings a row's largest magnitude to [2^8, 2^9): all but values 2^22 times smaller are then exact in f16.
__device__ __forceinline__ float row_factor(float largest) {
  if (!(largest > 0.f) || !(largest < 3.4e38f)) return 1.f;
  const int e = static_cast<int>(__float_as_uint(largest) >> 23) - 127;
  return __uint_as_float(static_cast<uint32_t>(min(max(8 - e, -126), 126) + 127) << 23);
}

struct TilePlace {
  int token, head;  // row's token of the sequence, query head
  bool real;
};
__device__ __forceinline__ TilePlace tile_place(const CachedParams& p, const SeqWork& s, int h, int r) {
  TilePlace w;
  w.token = r / p.group;  // rows are below 2^30
  w.head = h * p.group + (r - w.token * p.group);
  w.real = w.token < s.n;
  return w;
}
__device__ __forceinline__ long long row_offset(const CachedParams& p, const RowStrides& st, int b, const SeqWork& s, const TilePlace& w) {
  return (p.c.starts == nullptr ? b * st.b : 0ll) + (static_cast<long long>(s.row0) + w.token) * st.s + w.head * st.h;
}
__device__ __forceinline__ long long lse_index(const CachedParams& p, int b, const SeqWork& s, const TilePlace& w) {
  return p.c.starts == nullptr ? (static_cast<long long>(b) * p.Hq + w.head) * p.c.S + w.token
                               : static_cast<long long>(w.head) * p.c.S + s.row0 + w.token;
}

// x 2^d; d may lie far outside the exponents of one factor.
__device__ __forceinline__ float times_exp2(float x, float d) {
  const float h = ex2_approx(0.5f * d);
  return x * h * h;
}
// The row's log-sum-exp from its reference maximum (an integer) and its sum, 0 where it sees no key, NaN where a page was missing.  The
// sum's exponent is added as an integer, so that the logarithm is one of a number in [1, 2).  Without branches: it runs once an item, so
// its code is never in the instruction cache (0.6 us of the short single token's 10 with a branch for NaN).
__device__ __forceinline__ float lse_of(float m, float l) {
  const uint32_t bits = __float_as_uint(l);
  const float k = static_cast<float>(static_cast<int>(bits >> 23) - 127);
  const float z = (m - kWeightShift + k) + lg2_approx(__uint_as_float((bits & 0x7fffffu) | 0x3f800000u));
  return l == 0.f ? -INFINITY : fmaf(l, 0.f, z * kLn2);
}

// Transpose of an 8 x 8 matrix of 16-bit numbers that lies over the warp, two a lane.
__device__ __forceinline__ uint32_t transpose8x8(uint32_t x) {
  uint32_t y;
  asm volatile("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(y) : "r"(x));
  return y;
}
// 0..7 in an order in which neighbours 2 i, 2 i + 1 lie four apart.
__device__ __forceinline__ int spread(int g) { return (g & 1) << 2 | g >> 1; }

template <int TYPE, int NB>
__global__ void __launch_bounds__(kDecThreads, Dec<NB>::kCtasPerSm)
attn_cached_decode_kernel(const __grid_constant__ CUtensorMap tm_k, const __grid_constant__ CUtensorMap tm_v, const CachedParams p) {
  using D = Dec<NB>;
  constexpr int kRows = D::kRows;
  extern __shared__ uint8_t smem_raw[];
  uint8_t* smem = smem_raw + ((1024u - (smem_u32(smem_raw) & 1023u)) & 1023u);  // the swizzle goes by the address
  uint8_t* merge = smem + D::kRing;
  float2* row_stats = reinterpret_cast<float2*>(merge + D::kMerge);  // [warp][row]{m, l}
  uint64_t* bars = reinterpret_cast<uint64_t*>(merge + D::kMerge + D::kStats);
  volatile int* abort_flag = reinterpret_cast<volatile int*>(merge + D::kMerge + D::kStats + D::kBars);
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, g = lane >> 2, t4 = lane & 3;
  const WaitCtx ctx{abort_flag, p.status, kWaitLimitNs};

  if (threadIdx.x == 0) {
    tma_prefetch_desc(&tm_k);
    tma_prefetch_desc(&tm_v);
  }
  Line line;
  Cursor<kRows> now;
  const bool works = find_piece<kRows>(p, line, now, reinterpret_cast<long long*>(merge));
  if (threadIdx.x == 0) {
    p.pieces[2 * blockIdx.x] = make_int4(0, 0, 0, -1);
    for (int i = 0; i < kDecWarps * D::kStages; ++i) mbar_init(&bars[i], 1);
    *abort_flag = 0;
    fence_mbar_init();
  }
  __syncthreads();  // also: the scratch of find_piece is the merge buffer
  let_next_start();
  if (!works) return;

  Cursor<kRows> ahead = now;  // the step whose codes are requested next
  long long left_ahead = line.end - line.begin;
  uint8_t* ring = smem + warp * D::kStages * kWarpStageBytes;
  uint64_t* full = bars + warp * D::kStages;
  const int slot_mask = (1 << p.c.page_log2) - 1;
  // page of this warp's keys in the step `ahead` stands at: -1 does not exist, -2 no key there
  auto look_up = [&]() {
    const int key = ahead.t * kStepKeys + warp * 16;
    return left_ahead > 0 && key < ahead.s.keys ? page_of(p.c, ahead.b, key >> p.c.page_log2) : -2;
  };
  int page = look_up(), put = 0;
  float2 scales[D::kStages];  // of the requested steps, the oldest first; keys of a page that does not exist: -1
  // requests the 16 keys of that step and moves on to the next
  auto request = [&](float2& scale) {
    scale = make_float2(0.f, 0.f);
    if (page != -2) {
      if (lane == 0) {
        uint8_t* dst = ring + put * kWarpStageBytes;
        const int at = page >= 0 ? page : p.c.n_pages;  // behind the last page: zeros
        const int slot = (ahead.t * kStepKeys + warp * 16) & slot_mask;
        mbar_arrive_expect_tx(&full[put], kWarpStageBytes);
        tma_load_4d(dst, &tm_k, &full[put], 0, slot, ahead.h, at);
        tma_load_4d(dst + 16 * kKvDim, &tm_v, &full[put], 0, slot, ahead.h, at);
      }
      if (page >= 0) {
        const long long at = static_cast<long long>(page) * p.c.Hkv + ahead.h;
        scale = make_float2(__ldg(p.c.scales[0] + at), __ldg(p.c.scales[1] + at));
      } else {
        scale.x = -1.f;
      }
    }
    put = put + 1 == D::kStages ? 0 : put + 1;
    if (left_ahead > 0) {
      --left_ahead;
      if (++ahead.t >= ahead.steps && left_ahead > 0) ahead.next_tile(p);
      page = look_up();
    }
  };
#pragma unroll
  for (int i = 0; i < D::kStages; ++i) request(scales[i]);

  int get = 0;
  uint32_t phase = 0;  // a bit a stage
  long long at = line.begin;
  while (at < line.end) {
    // ---- one tile, or this CTA's piece of it ----
    const int t_first = now.t;
    const int n_steps = static_cast<int>(min(static_cast<long long>(now.steps - now.t), line.end - at));
    const long long tile_begin = at - now.t;
    const int row_first = now.tile * kRows;
    // queries (right operand): lane (g, t4) has row g; step i of the product takes d = 64 (i / 4) + 16 t4 + 4 (i % 4) + 0..3, the
    // order that a lane's codes of K have.  Scores: lane (g, t4) has rows 2 t4, 2 t4 + 1 of keys spread(g), 8 + spread(g)
    uint32_t qf[NB][8][2];
    float factor[NB][2];
    int limit[NB][2];  // keys the row sees
#pragma unroll
    for (int nb = 0; nb < NB; ++nb) {
      const TilePlace w = tile_place(p, now.s, now.h, row_first + 8 * nb + g);
      uint32_t raw[16];
#pragma unroll
      for (int i = 0; i < 16; ++i) raw[i] = 0;
      if (w.real) {
        const uint16_t* row = p.q + row_offset(p, p.sq, now.b, now.s, w) + t4 * 16;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const uint4 x = __ldg(reinterpret_cast<const uint4*>(row + (i >> 1) * 64 + (i & 1) * 8));
          raw[4 * i] = x.x;
          raw[4 * i + 1] = x.y;
          raw[4 * i + 2] = x.z;
          raw[4 * i + 3] = x.w;
        }
      }
      float largest = 0.f;
#pragma unroll
      for (int i = 0; i < 16; ++i) {
        const float2 f = unpack_bf16x2(raw[i]);
        largest = max3(largest, fabsf(f.x), fabsf(f.y));
      }
      largest = fmaxf(largest, __shfl_xor_sync(0xffffffffu, largest, 1));
      largest = fmaxf(largest, __shfl_xor_sync(0xffffffffu, largest, 2));
      const float up = row_factor(largest);
      const float down = p.scale_log2 / up;
      const int sees = w.real ? visible(now.s, w.token, p.causal) : 0;
#pragma unroll
      for (int e = 0; e < 2; ++e) {  // row 2 t4 + e is with the lanes of g = 2 t4 + e
        factor[nb][e] = __shfl_sync(0xffffffffu, down, 8 * t4 + 4 * e);
        limit[nb][e] = __shfl_sync(0xffffffffu, sees, 8 * t4 + 4 * e);
      }
#pragma unroll
      for (int i = 0; i < 16; ++i) {  // word i: d = 64 (i / 8) + 16 t4 + 2 (i % 8)
        const float2 f = unpack_bf16x2(raw[i]);
        qf[nb][i >> 1][i & 1] = pack_f16x2(f.x * up, f.y * up);
      }
    }
    // keys that all rows see: steps up to there need no mask
    const int clear = visible(now.s, min(row_first / p.group, now.s.n - 1), p.causal);
    float acc[NB][8][4];  // d = 16 spread(g) + 2 mt (values 0, 1) and + 1 (2, 3); rows 2 t4 (0, 2) and 2 t4 + 1 (1, 3)
    float m[NB][2], l[NB][2], top_scale = kScaleLeast;  // log2 of the largest V scale
#pragma unroll
    for (int nb = 0; nb < NB; ++nb) {
#pragma unroll
      for (int mt = 0; mt < 8; ++mt) acc[nb][mt][0] = acc[nb][mt][1] = acc[nb][mt][2] = acc[nb][mt][3] = 0.f;
      m[nb][0] = m[nb][1] = -INFINITY;
      l[nb][0] = l[nb][1] = 0.f;
    }

#pragma unroll 1
    for (int step = 0; step < n_steps; ++step) {
      const int key0 = (t_first + step) * kStepKeys + warp * 16;
      float k_scale = scales[0].x;
      const float v_scale = scales[0].y;
      if (key0 < now.s.keys) {  // else nothing was requested
        // a wait that runs out leaves the codes as they are: the status word says that the results are void
        mbar_wait_warp(&full[get], phase >> get & 1, ctx, kRoleLoad | kBarKvFull);
        phase ^= 1u << get;
        const uint8_t* stage = ring + get * kWarpStageBytes;
        const bool bad = k_scale < 0.f;
        if (bad) k_scale = 0.f;
        float s[NB][4];
#pragma unroll
        for (int nb = 0; nb < NB; ++nb) s[nb][0] = s[nb][1] = s[nb][2] = s[nb][3] = 0.f;
        const int kr = spread(g);
#pragma unroll
        for (int half = 0; half < 2; ++half) {
          const uint8_t* src = stage + kr * kKvDim + (((half * 4 + t4) ^ kr) << 4);
          const uint4 w0 = *reinterpret_cast<const uint4*>(src), w1 = *reinterpret_cast<const uint4*>(src + 8 * kKvDim);
          const uint32_t x0[4] = {w0.x, w0.y, w0.z, w0.w}, x1[4] = {w1.x, w1.y, w1.z, w1.w};
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            uint32_t a[4];
            codes_to_f16<TYPE>(x0[i], a[0], a[2]);
            codes_to_f16<TYPE>(x1[i], a[1], a[3]);
#pragma unroll
            for (int nb = 0; nb < NB; ++nb) mma_f16(s[nb], a, qf[nb][half * 4 + i][0], qf[nb][half * 4 + i][1]);
          }
        }
        const float lv0 = lg2_approx(v_scale);
        top_scale = fmaxf(top_scale, lv0);
        const float lv = fmaxf(lv0, top_scale - kScaleZero), extra = fmaxf(lv, top_scale - kScaleSpan) - lv;
        const float v_inverse = ex2_approx(-lv), lag = kWeightLag - extra;
        bool grow = false;
#pragma unroll
        for (int nb = 0; nb < NB; ++nb) {
#pragma unroll
          for (int e = 0; e < 2; ++e) {
            const float f = factor[nb][e] * k_scale;
            s[nb][e] = fmaf(s[nb][e], f, lv);
            s[nb][2 + e] = fmaf(s[nb][2 + e], f, lv);
            if (key0 + 16 > clear) {  // warp-uniform
              if (key0 + kr >= limit[nb][e]) s[nb][e] = -INFINITY;
              if (key0 + 8 + kr >= limit[nb][e]) s[nb][2 + e] = -INFINITY;
              if (bad && key0 < limit[nb][e]) l[nb][e] = __int_as_float(0x7fffffff);
            } else if (bad) {
              l[nb][e] = __int_as_float(0x7fffffff);
            }
            grow = grow || fmaxf(s[nb][e], s[nb][2 + e]) > m[nb][e] + lag;
          }
        }
        if (__any_sync(0xffffffffu, grow)) {
#pragma unroll
          for (int nb = 0; nb < NB; ++nb) {
            float a[2];
#pragma unroll
            for (int e = 0; e < 2; ++e) {
              float top = fmaxf(s[nb][e], s[nb][2 + e]);
#pragma unroll
              for (int x = 4; x < 32; x <<= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, x));
              const float to = fmaxf(m[nb][e], ceilf(top + extra));
              const float h = m[nb][e] == -INFINITY ? 0.f : ex2_approx(0.5f * (m[nb][e] - to));
              a[e] = h * h;
              m[nb][e] = to;
              l[nb][e] = l[nb][e] * h * h;
            }
#pragma unroll
            for (int mt = 0; mt < 8; ++mt) {
              acc[nb][mt][0] *= a[0];
              acc[nb][mt][1] *= a[1];
              acc[nb][mt][2] *= a[0];
              acc[nb][mt][3] *= a[1];
            }
          }
        }
        uint32_t pf[NB][2];
#pragma unroll
        for (int nb = 0; nb < NB; ++nb) {
          float x[4];
#pragma unroll
          for (int e = 0; e < 2; ++e) {
            const float ref = m[nb][e] == -INFINITY ? 0.f : m[nb][e] - kWeightShift;
            x[e] = ex2_approx(s[nb][e] - ref);
            x[2 + e] = ex2_approx(s[nb][2 + e] - ref);
            l[nb][e] = fmaf(x[e] + x[2 + e], v_inverse, l[nb][e]);
          }
          pf[nb][0] = transpose8x8(pack_f16x2(x[0], x[1]));
          pf[nb][1] = transpose8x8(pack_f16x2(x[2], x[3]));
        }
        // V^T: inner indices 2 t4, 2 t4 + 1 are keys t4, t4 + 4, and 8 more those + 8; a lane takes d = 16 spread(g) .. + 15 of them
        uint4 w[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const int r = t4 + 4 * i;
          w[i] = *reinterpret_cast<const uint4*>(stage + (16 + r) * kKvDim + ((kr ^ (r & 7)) << 4));
          if (key0 + 16 > now.s.keys && key0 + r >= now.s.keys) w[i] = make_uint4(0, 0, 0, 0);  // behind the last token: anything
        }
#pragma unroll
        for (int word = 0; word < 4; ++word) {
          uint32_t x[4], a[4], b[4];
#pragma unroll
          for (int i = 0; i < 4; ++i) x[i] = word == 0 ? w[i].x : word == 1 ? w[i].y : word == 2 ? w[i].z : w[i].w;
          codes_to_f16<TYPE>(__byte_perm(x[0], x[1], 0x5140), a[0], a[1]);
          codes_to_f16<TYPE>(__byte_perm(x[2], x[3], 0x5140), a[2], a[3]);
          codes_to_f16<TYPE>(__byte_perm(x[0], x[1], 0x7362), b[0], b[1]);
          codes_to_f16<TYPE>(__byte_perm(x[2], x[3], 0x7362), b[2], b[3]);
#pragma unroll
          for (int nb = 0; nb < NB; ++nb) {
            mma_f16(acc[nb][2 * word], a, pf[nb][0], pf[nb][1]);
            mma_f16(acc[nb][2 * word + 1], b, pf[nb][0], pf[nb][1]);
          }
        }
      }
      __syncwarp();
      get = get + 1 == D::kStages ? 0 : get + 1;
#pragma unroll
      for (int i = 0; i + 1 < D::kStages; ++i) scales[i] = scales[i + 1];
      request(scales[D::kStages - 1]);
    }

    // ---- the eight warps' parts of the tile ----
#pragma unroll
    for (int nb = 0; nb < NB; ++nb) {
#pragma unroll
      for (int e = 0; e < 2; ++e) {
#pragma unroll
        for (int x = 4; x < 32; x <<= 1) l[nb][e] += __shfl_xor_sync(0xffffffffu, l[nb][e], x);
        if (g == 0) row_stats[warp * kRows + 8 * nb + 2 * t4 + e] = make_float2(m[nb][e], l[nb][e]);
      }
    }
    __syncthreads();
    const int swz = t4 | (g & 1) << 2;
#pragma unroll
    for (int nb = 0; nb < NB; ++nb) {
#pragma unroll
      for (int e = 0; e < 2; ++e) {
        const int r = 8 * nb + 2 * t4 + e;
        float to = -INFINITY;
#pragma unroll
        for (int w = 0; w < kDecWarps; ++w) to = fmaxf(to, row_stats[w * kRows + r].x);
        const float a = m[nb][e] == -INFINITY ? 0.f : ex2_approx(m[nb][e] - to);
        float4* row = reinterpret_cast<float4*>(merge) + (warp * kRows + r) * (kKvDim / 4);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          row[(4 * spread(g) + i) ^ swz] = make_float4(acc[nb][2 * i][e] * a, acc[nb][2 * i][2 + e] * a, acc[nb][2 * i + 1][e] * a,
                                                       acc[nb][2 * i + 1][2 + e] * a);
        }
      }
    }
    __syncthreads();
#pragma unroll 1
    for (int nb = 0; nb < NB; ++nb) {  // a warp a row, four columns a lane
      const int r = 8 * nb + warp;
      const TilePlace w = tile_place(p, now.s, now.h, row_first + r);
      if (!w.real) break;
      // lane i has warp i % 8's maximum and sum
      const float2 mine = row_stats[(lane & 7) * kRows + r];
      float to = mine.x;
#pragma unroll
      for (int x = 1; x < kDecWarps; x <<= 1) to = fmaxf(to, __shfl_xor_sync(0xffffffffu, to, x));
      float sum = mine.x == -INFINITY ? mine.y : times_exp2(mine.y, mine.x - to);
#pragma unroll
      for (int x = 1; x < kDecWarps; x <<= 1) sum += __shfl_xor_sync(0xffffffffu, sum, x);
      float4 o = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
      for (int i = 0; i < kDecWarps; ++i) {
        const float4 x = reinterpret_cast<const float4*>(merge)[(i * kRows + r) * (kKvDim / 4) + (lane ^ ((r >> 1 & 3) | (lane >> 4) << 2))];
        o.x += x.x;
        o.y += x.y;
        o.z += x.z;
        o.w += x.w;
      }
      // a row that sees keys beyond the table's reach is NaN, as one that needs a page that does not exist
      if (now.s.len > now.s.keys && (!p.causal || now.s.len - now.s.n + w.token >= now.s.keys)) sum = __int_as_float(0x7fffffff);
      if (t_first == 0 && n_steps == now.steps) {
        const float inv = sum > 0.f ? 1.f / sum : sum == 0.f ? 0.f : sum;  // 0: a row that sees no key
        *reinterpret_cast<uint2*>(p.o + row_offset(p, p.so, now.b, now.s, w) + lane * 4) =
            make_uint2(pack_bf16x2(o.x * inv, o.y * inv), pack_bf16x2(o.z * inv, o.w * inv));
        if (lane == 0 && p.lse != nullptr)
          p.lse[lse_index(p, now.b, now.s, w)] = lse_of(to, sum);
      } else {  // slot 2 i: a tile begun by an earlier CTA; 2 i + 1: one begun here
        const long long slot = 2ll * blockIdx.x + (t_first == 0 ? 1 : 0);
        reinterpret_cast<float4*>(p.parts + (slot * kRows + r) * kKvDim)[lane] = o;
        if (lane == 0)
          reinterpret_cast<float2*>(p.parts + 2ll * p.ctas * kRows * kKvDim)[slot * kRows + r] = make_float2(to, sum);
      }
    }
    if (threadIdx.x == 0 && t_first == 0 && n_steps != now.steps) {
      p.pieces[2 * blockIdx.x] = make_int4(now.b, now.h, now.tile, static_cast<int>(line.owner(tile_begin + now.steps - 1)));
      p.pieces[2 * blockIdx.x + 1] = make_int4(now.s.row0, now.s.n, 0, 0);
    }
    __syncthreads();
    at += n_steps;
    if (at < line.end) now.next_tile(p);
  }
  if (*abort_flag && lane == 0) {  // let loads in flight land before the CTA's shared memory is released
    const uint64_t t0 = global_timer_ns();
    while (global_timer_ns() - t0 < 1000000ull) {
    }
  }
}

// Joins the parts of a tile that several CTAs worked on: sum_i 2^(m_i - m) O_i / sum_i 2^(m_i - m) l_i, parts in order.
//
// A row is 512 bytes of every part.  Where a tile has few parts a warp takes kJoinRows rows at once, so that their loads are in
// flight together; where it has many, the eight warps of a block share the parts of one row.  Block (i, y) looks at the tile that
// CTA i began and did not end; ROWS / 8 blocks a tile.  The launch starts while the kernel before it ends.
constexpr int kJoinRows = 4;
constexpr int kJoinMany = 12;

struct JoinSum {
  float m, l;
  float4 o;
};
__device__ __forceinline__ void join_part(JoinSum& j, const float2 ml, const float4 x) {
  const float to = fmaxf(j.m, ml.x);
  const float g = j.m == -INFINITY ? 0.f : ex2_approx(0.5f * (j.m - to)), h = ml.x == -INFINITY ? 0.f : ex2_approx(0.5f * (ml.x - to));
  const float a = g * g, f = h * h;
  // a part that has seen no key has the sum 0, or NaN where a page was missing
  j.l = (j.m == -INFINITY ? j.l : j.l * g * g) + (ml.x == -INFINITY ? ml.y : ml.y * h * h);
  j.m = to;
  j.o.x = j.o.x * a + x.x * f;
  j.o.y = j.o.y * a + x.y * f;
  j.o.z = j.o.z * a + x.z * f;
  j.o.w = j.o.w * a + x.w * f;
}
__device__ __forceinline__ void join_write(const CachedParams& p, const JoinSum& j, int b, const SeqWork& s, const TilePlace& w, int lane) {
  const float inv = j.l > 0.f ? 1.f / j.l : j.l == 0.f ? 0.f : j.l;
  *reinterpret_cast<uint2*>(p.o + row_offset(p, p.so, b, s, w) + lane * 4) =
      make_uint2(pack_bf16x2(j.o.x * inv, j.o.y * inv), pack_bf16x2(j.o.z * inv, j.o.w * inv));
  if (lane == 0 && p.lse != nullptr)
    p.lse[lse_index(p, b, s, w)] = lse_of(j.m, j.l);
}

template <int ROWS>
__global__ void __launch_bounds__(256) attn_cached_join_kernel(const CachedParams p) {
  __shared__ float4 sums[8][32];
  __shared__ float2 stat[8];
  wait_for_launch_before();
  const int4 piece = p.pieces[2 * blockIdx.x], rows = p.pieces[2 * blockIdx.x + 1];
  if (piece.w < 0) return;
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const int first = blockIdx.x, n = piece.w - first + 1;
  SeqWork s;
  s.row0 = rows.x;
  s.n = rows.y;
  const float2* stats = reinterpret_cast<const float2*>(p.parts + 2ll * p.ctas * ROWS * kKvDim);
  const float4* parts = reinterpret_cast<const float4*>(p.parts);
  const int tile_row = piece.z * ROWS;
  if (n <= kJoinMany) {
    for (int r0 = (blockIdx.y * 8 + warp) * kJoinRows; r0 < ROWS; r0 += static_cast<int>(gridDim.y) * 8 * kJoinRows) {
      if (!tile_place(p, s, piece.y, tile_row + r0).real) return;  // rows are in order: none behind it is
      JoinSum j[kJoinRows];
#pragma unroll
      for (int k = 0; k < kJoinRows; ++k) j[k] = JoinSum{-INFINITY, 0.f, make_float4(0.f, 0.f, 0.f, 0.f)};
#pragma unroll 2
      for (int i = 0; i < n; ++i) {
        const long long at = (2ll * (first + i) + (i == 0 ? 1 : 0)) * ROWS + r0;
        float2 ml[kJoinRows];
        float4 x[kJoinRows];
#pragma unroll
        for (int k = 0; k < kJoinRows; ++k) {
          ml[k] = stats[at + k];
          x[k] = parts[(at + k) * (kKvDim / 4) + lane];
        }
#pragma unroll
        for (int k = 0; k < kJoinRows; ++k) join_part(j[k], ml[k], x[k]);
      }
#pragma unroll
      for (int k = 0; k < kJoinRows; ++k) {
        const TilePlace w = tile_place(p, s, piece.y, tile_row + r0 + k);
        if (w.real) join_write(p, j[k], piece.x, s, w, lane);
      }
    }
    return;
  }
  for (int r = blockIdx.y; r < ROWS; r += gridDim.y) {
    const TilePlace w = tile_place(p, s, piece.y, tile_row + r);
    if (!w.real) return;
    JoinSum j{-INFINITY, 0.f, make_float4(0.f, 0.f, 0.f, 0.f)};
#pragma unroll 4
    for (int i = warp; i < n; i += 8) {
      const long long at = (2ll * (first + i) + (i == 0 ? 1 : 0)) * ROWS + r;
      join_part(j, stats[at], parts[at * (kKvDim / 4) + lane]);
    }
    __syncthreads();  // the row before has been read
    sums[warp][lane] = j.o;
    if (lane == 0) stat[warp] = make_float2(j.m, j.l);
    __syncthreads();
    if (warp != 0) continue;
#pragma unroll
    for (int i = 1; i < 8; ++i) join_part(j, stat[i], sums[i][lane]);
    join_write(p, j, piece.x, s, w, lane);
  }
}

}  // namespace kv
}  // namespace attn
