// Attention of new tokens over a paged 8-bit cache, for few query rows a key head (decoding).
//
//     s_ij = scale k_scale(page of j) q_i . c^K_j,    o_i = sum_j softmax_j(s_ij) v_scale(page of j) c^V_j
//
// Bound by HBM: 256 bytes a cached token and key head, read once for all query heads of the group.  A query tile is 16 rows
// (token, head of the group), heads fastest.  All work is a line of (sequence, key head, query tile, 128 keys) steps, cut into
// equal contiguous pieces, one a CTA, whatever the lengths are; the cut is computed on the device from the lengths.  A CTA
// that holds a whole tile's keys writes its result, the others leave fp32 parts, which a second kernel joins in order.
//
// In a CTA each of 8 warps owns 16 keys of a step and works alone until its piece of a tile ends: its own ring of four 4 KB
// stages filled by 16-byte asynchronous copies three steps ahead, its own running maximum, sum and 16 x 128 accumulator.
// 16 keys lie in one page, so the scales are one factor a warp and step.  Keys go from shared memory to the operands of
// mma.m16n8k16 (f16) without a transpose: the products' inner index may be in any order, so a lane takes 16 consecutive head
// dimensions of its key (K) or of four keys (V), and the queries are loaded in the same order.  Codes are exact in f16;
// queries are scaled by a power of two of their row, weights are held as 2^6 exp(s - m) with a maximum that may lag by a
// factor of 2^8, so f16 keeps 11 bits of both; V's scale enters as its ratio to the largest one met so far.
#pragma once

#include "attn_fwd_kernel.cuh"
#include "kv_cache_kernel.cuh"

namespace attn {
namespace kv {

constexpr int kDecWarps = 8;
constexpr int kDecThreads = kDecWarps * 32;
constexpr int kDecRows = 16;
constexpr int kDecStages = 4;
constexpr int kStepKeys = 128;                         // keys a CTA takes in one step: 16 a warp
constexpr int kWarpStageBytes = 2 * 16 * kKvDim;       // K then V
constexpr int kDecRingBytes = kDecWarps * kDecStages * kWarpStageBytes;  // 128 KB
constexpr int kDecMergeBytes = kDecWarps * kDecRows * kKvDim * 4;        // 64 KB
constexpr int kDecSmemBytes = kDecRingBytes + kDecMergeBytes + kDecWarps * kDecStages * 16 + kDecWarps * kDecRows * 8;
constexpr float kWeightShift = 6.f;   // weights are held as 2^kWeightShift exp(s - m)
constexpr float kWeightLag = 8.f;     // log2 units the reference maximum may lag

struct CachedParams {
  CacheView c;
  const uint16_t* q;
  uint16_t* o;
  float* lse;             // [B, Hq, S], or [Hq, S] with starts; may be null
  RowStrides sq, so;
  int Hq, group, causal;
  float scale_log2;       // scale * log2(e)
  float* parts;           // [2 ctas][rows][kKvDim], then [2 ctas][rows][2] (reference maximum in log2 units, sum)
  int4* pieces;           // [ctas]: {sequence, head, tile, last CTA with a part} of the tile the CTA began and did not end
  int ctas;
  int min_steps;          // a piece has at least about so many
  int* status;            // bounded waits that ran out, see WaitCtx
};

// One sequence of the line of work.
struct SeqWork {
  int row0, n;       // its rows
  int len;           // tokens in all, at least 0
  int keys;          // of them in the table's reach
};
__device__ __forceinline__ SeqWork seq_work(const CacheView& c, int b) {
  SeqWork s;
  rows_of(c, b, s.row0, s.n);
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

// A place on the line of work.
template <int ROWS>
struct Cursor {
  int b, h, tile, t, steps, tiles;
  SeqWork s;
  __device__ __forceinline__ void enter_tile(const CachedParams& p) {
    steps = steps_of(s, min((tile * ROWS + ROWS - 1) / p.group, s.n - 1), p.causal);
  }
  __device__ __forceinline__ void enter_sequence(const CachedParams& p) {
    s = seq_work(p.c, b);
    tiles = static_cast<int>((static_cast<long long>(s.n) * p.group + ROWS - 1) / ROWS);
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
  const long long rows = static_cast<long long>(s.n) * p.group;
  const int tiles = static_cast<int>((rows + ROWS - 1) / ROWS);
  if (tiles == 0) return 0;
  if (!p.causal) return static_cast<long long>(tiles) * steps_of(s, s.n - 1, 0);
  long long sum = 0;
  for (int k = 0; k < tiles; ++k) sum += steps_of(s, min((k * ROWS + ROWS - 1) / p.group, s.n - 1), 1);
  return sum;
}

// The line of work as one CTA sees it.
struct Line {
  long long total;   // steps in all
  long long ctas;    // CTAs that have a piece
  long long begin, end;
  __device__ __forceinline__ long long owner(long long step) const { return ((step + 1) * ctas - 1) / total; }
};

// Cuts the line and finds where this CTA's piece begins.  All threads call; `scratch` holds 2 * (threads / 32) + 8 long longs.
template <int ROWS>
__device__ __forceinline__ bool find_piece(const CachedParams& p, Line& line, Cursor<ROWS>& at, long long* scratch) {
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, warps = blockDim.x >> 5;
  long long mine = 0;
  for (int b = threadIdx.x; b < p.c.B; b += blockDim.x) mine += head_steps<ROWS>(p, seq_work(p.c, b)) * p.c.Hkv;
#pragma unroll
  for (int m = 16; m > 0; m >>= 1) mine += __shfl_xor_sync(0xffffffffu, mine, m);
  if (lane == 0) scratch[warp] = mine;
  __syncthreads();
  long long total = 0;
  for (int w = 0; w < warps; ++w) total += scratch[w];
  line.total = total;
  line.ctas = min(static_cast<long long>(p.ctas), (total + p.min_steps - 1) / p.min_steps);
  if (blockIdx.x >= line.ctas) return false;
  line.begin = total * blockIdx.x / line.ctas;
  line.end = total * (blockIdx.x + 1) / line.ctas;
  // the sequence that holds step line.begin: a scan over the sequences, a block of them at a time
  long long* found = scratch + warps;  // sequence, its first step
  long long before = 0;
  for (int b0 = 0; b0 < p.c.B; b0 += blockDim.x) {
    __syncthreads();
    const int b = b0 + threadIdx.x;
    const long long cost = b < p.c.B ? head_steps<ROWS>(p, seq_work(p.c, b)) * p.c.Hkv : 0;
    long long upto = cost;
#pragma unroll
    for (int m = 1; m < 32; m <<= 1) {
      const long long other = __shfl_up_sync(0xffffffffu, upto, m);
      if (lane >= m) upto += other;
    }
    if (lane == 31) scratch[warp] = upto;
    __syncthreads();
    long long base = before, block = 0;
    for (int w = 0; w < warps; ++w) {
      if (w < warp) base += scratch[w];
      block += scratch[w];
    }
    const long long from = base + upto - cost;
    if (cost > 0 && line.begin >= from && line.begin < from + cost) {
      found[0] = b;
      found[1] = from;
    }
    before += block;
    if (before > line.begin) break;
  }
  __syncthreads();
  at.b = static_cast<int>(found[0]);
  long long left = line.begin - found[1];
  at.enter_sequence(p);
  const long long per_head = head_steps<ROWS>(p, at.s);
  at.h = static_cast<int>(left / per_head);
  left -= at.h * per_head;
  at.tile = 0;
  at.enter_tile(p);
  if (!p.causal) {  // tiles of equal length
    at.tile = static_cast<int>(left / at.steps);
    left -= static_cast<long long>(at.tile) * at.steps;
  } else {
    while (left >= at.steps) {
      left -= at.steps;
      ++at.tile;
      at.enter_tile(p);
    }
  }
  at.t = static_cast<int>(left);
  return true;
}

__device__ __forceinline__ void cp_async16(uint32_t dst, const void* src, bool take) {
  const int bytes = take ? 16 : 0;  // 0: zeros are written, nothing is read
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst), "l"(src), "r"(bytes) : "memory");
}
__device__ __forceinline__ void cp_async4(uint32_t dst, const void* src, bool take) {
  const int bytes = take ? 4 : 0;
  asm volatile("cp.async.ca.shared.global [%0], [%1], 4, %2;" ::"r"(dst), "l"(src), "r"(bytes) : "memory");
}
__device__ __forceinline__ void cp_async_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int N>
__device__ __forceinline__ void cp_async_wait() {
  asm volatile("cp.async.wait_group %0;" ::"n"(N) : "memory");
}
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
__device__ __forceinline__ TilePlace tile_place(const CachedParams& p, const SeqWork& s, int h, long long r) {
  TilePlace w;
  w.token = static_cast<int>(r / p.group);
  w.head = h * p.group + static_cast<int>(r - static_cast<long long>(w.token) * p.group);
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

template <int TYPE>
__global__ void __launch_bounds__(kDecThreads, 1) attn_cached_decode_kernel(const CachedParams p) {
  extern __shared__ __align__(128) uint8_t smem[];
  uint8_t* merge = smem + kDecRingBytes;
  float2* scale_ring = reinterpret_cast<float2*>(merge + kDecMergeBytes);          // [warp][stage]{k, v}, 16 bytes apart
  float2* row_stats = reinterpret_cast<float2*>(merge + kDecMergeBytes + kDecWarps * kDecStages * 16);  // [warp][row]{m, l}
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, g = lane >> 2, t4 = lane & 3;

  Line line;
  Cursor<kDecRows> now;
  const bool works = find_piece<kDecRows>(p, line, now, reinterpret_cast<long long*>(merge));
  __syncthreads();  // the scratch is the merge buffer
  if (threadIdx.x == 0) p.pieces[blockIdx.x] = make_int4(0, 0, 0, -1);
  if (!works) return;
  Cursor<kDecRows> ahead = now;          // what is requested next
  long long left_ahead = line.end - line.begin;

  const uint32_t ring = smem_u32(smem) + warp * kDecStages * kWarpStageBytes;
  const uint32_t scales = smem_u32(scale_ring) + warp * kDecStages * 16;
  volatile int* bad_ring = reinterpret_cast<volatile int*>(scale_ring) + warp * kDecStages * 4 + 2;
  int put = 0;
  // requests 16 keys of the step `ahead` stands at and moves on
  auto request = [&]() {
    if (left_ahead > 0) {
      --left_ahead;
      const int key0 = ahead.t * kStepKeys + warp * 16;
      const bool any = key0 < ahead.s.keys;
      const int page = any ? page_of(p.c, ahead.b, key0 >> p.c.page_log2) : -1;
      const int slot0 = key0 & ((1 << p.c.page_log2) - 1);
#pragma unroll
      for (int kv = 0; kv < 2; ++kv) {
        const uint8_t* base = p.c.codes[kv] + max(page, 0) * p.c.sp[kv] + ahead.h * p.c.sh[kv] + slot0 * p.c.ss[kv];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const int r = 4 * i + (lane >> 3), u = lane & 7;
          const int swz = kv == 0 ? u ^ ((r & 1) << 2) : u ^ (r & 6);
          const bool take = page >= 0 && key0 + r < ahead.s.keys;
          cp_async16(ring + put * kWarpStageBytes + kv * 16 * kKvDim + r * kKvDim + swz * 16,
                     take ? base + r * p.c.ss[kv] + u * 16 : p.c.codes[kv], take);
        }
      }
      if (lane < 2) {
        cp_async4(scales + put * 16 + lane * 4,
                  p.c.scales[lane] + (page >= 0 ? static_cast<long long>(page) * p.c.Hkv + ahead.h : 0ll), page >= 0);
      }
      if (lane == 2) bad_ring[put * 4] = any && page < 0;
      if (++ahead.t >= ahead.steps) ahead.next_tile(p);
    }
    cp_async_commit();
    put = put + 1 == kDecStages ? 0 : put + 1;
  };
  for (int i = 0; i < kDecStages - 1; ++i) request();

  int get = 0;
  long long at = line.begin;
  while (at < line.end) {
    // ---- one tile, or this CTA's piece of it ----
    const int t_first = now.t;
    const int n_steps = static_cast<int>(min(static_cast<long long>(now.steps - now.t), line.end - at));
    const long long tile_begin = at - now.t;
    // queries, in the order that a lane's K bytes have: step i of the product takes d = 64 (i / 4) + 16 t4 + 4 (i % 4) + 0..3
    uint32_t qf[8][4];
    float factor[2];
    int limit[2];  // keys the row sees
#pragma unroll
    for (int rr = 0; rr < 2; ++rr) {
      const TilePlace w = tile_place(p, now.s, now.h, static_cast<long long>(now.tile) * kDecRows + g + 8 * rr);
      uint32_t raw[16];
#pragma unroll
      for (int i = 0; i < 16; ++i) raw[i] = 0;
      limit[rr] = 0;
      if (w.real) {
        limit[rr] = visible(now.s, w.token, p.causal);
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
        largest = fmaxf(largest, fmaxf(fabsf(f.x), fabsf(f.y)));
      }
      largest = fmaxf(largest, __shfl_xor_sync(0xffffffffu, largest, 1));
      largest = fmaxf(largest, __shfl_xor_sync(0xffffffffu, largest, 2));
      const float up = row_factor(largest);
      factor[rr] = p.scale_log2 / up;
#pragma unroll
      for (int i = 0; i < 16; ++i) {  // word i: d = 64 (i / 8) + 16 t4 + 2 (i % 8)
        const float2 f = unpack_bf16x2(raw[i]);
        qf[i >> 1][(i & 1) * 2 + rr] = pack_f16x2(f.x * up, f.y * up);
      }
    }
    float acc[16][4];
#pragma unroll
    for (int i = 0; i < 16; ++i) acc[i][0] = acc[i][1] = acc[i][2] = acc[i][3] = 0.f;
    float m[2] = {-INFINITY, -INFINITY}, l[2] = {0.f, 0.f}, vref = 0.f;

    for (int step = 0; step < n_steps; ++step) {
      request();
      cp_async_wait<kDecStages - 1>();
      __syncwarp();
      const int key0 = (t_first + step) * kStepKeys + warp * 16;
      if (key0 < now.s.keys) {
        const uint8_t* stage = smem + warp * kDecStages * kWarpStageBytes + get * kWarpStageBytes;
        const float* sc = reinterpret_cast<const float*>(scale_ring) + (warp * kDecStages + get) * 4;
        const float k_scale = sc[0], v_scale = sc[1];
        const bool bad = bad_ring[get * 4] != 0;
        float s[2][4];
#pragma unroll
        for (int j = 0; j < 2; ++j) {
          s[j][0] = s[j][1] = s[j][2] = s[j][3] = 0.f;
          const int r = 8 * j + g;
#pragma unroll
          for (int half = 0; half < 2; ++half) {
            const uint4 w = *reinterpret_cast<const uint4*>(stage + r * kKvDim + ((half * 4 + t4) ^ ((r & 1) << 2)) * 16);
            const uint32_t words[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
            for (int i = 0; i < 4; ++i) {
              uint32_t b0, b1;
              codes_to_f16<TYPE>(words[i], b0, b1);
              mma_f16(s[j], qf[half * 4 + i], b0, b1);
            }
          }
        }
        // columns 2 t4 + e of n-tile j are keys key0 + 8 j + 2 t4 + e; rows g (values 0, 1) and g + 8 (2, 3)
        float top[2];
#pragma unroll
        for (int rr = 0; rr < 2; ++rr) {
          const float f = factor[rr] * k_scale;
#pragma unroll
          for (int j = 0; j < 2; ++j) {
#pragma unroll
            for (int e = 0; e < 2; ++e) {
              const float x = s[j][2 * rr + e] * f;
              s[j][2 * rr + e] = key0 + 8 * j + 2 * t4 + e < limit[rr] ? x : -INFINITY;
            }
          }
          top[rr] = fmaxf(fmaxf(s[0][2 * rr], s[0][2 * rr + 1]), fmaxf(s[1][2 * rr], s[1][2 * rr + 1]));
          top[rr] = fmaxf(top[rr], __shfl_xor_sync(0xffffffffu, top[rr], 1));
          top[rr] = fmaxf(top[rr], __shfl_xor_sync(0xffffffffu, top[rr], 2));
        }
        if (__any_sync(0xffffffffu, top[0] > m[0] + kWeightLag || top[1] > m[1] + kWeightLag)) {
          float a[2];
#pragma unroll
          for (int rr = 0; rr < 2; ++rr) {
            const float to = fmaxf(m[rr], top[rr]);
            a[rr] = m[rr] == -INFINITY ? 0.f : ex2_approx(m[rr] - to);
            m[rr] = to;
            l[rr] *= a[rr];
          }
#pragma unroll
          for (int i = 0; i < 16; ++i) {
            acc[i][0] *= a[0];
            acc[i][1] *= a[0];
            acc[i][2] *= a[1];
            acc[i][3] *= a[1];
          }
        }
        if (v_scale > vref) {
          const float a = __fdividef(vref, v_scale);
          vref = v_scale;
#pragma unroll
          for (int i = 0; i < 16; ++i) {
#pragma unroll
            for (int e = 0; e < 4; ++e) acc[i][e] *= a;
          }
        }
        const float ratio = vref > 0.f ? __fdividef(v_scale, vref) : 0.f;
        uint32_t pf[4];
#pragma unroll
        for (int rr = 0; rr < 2; ++rr) {
          const float ref = m[rr] == -INFINITY ? 0.f : m[rr] - kWeightShift;
#pragma unroll
          for (int j = 0; j < 2; ++j) {
            const float x = ex2_approx(s[j][2 * rr] - ref), y = ex2_approx(s[j][2 * rr + 1] - ref);
            l[rr] += x + y;
            pf[2 * j + rr] = pack_f16x2(x * ratio, y * ratio);
          }
          if (bad && key0 < limit[rr]) l[rr] = __int_as_float(0x7fffffff);
        }
        // V: lane (g, t4) takes d = 16 g .. 16 g + 15 of keys 2 t4, 2 t4 + 1, 2 t4 + 8, 2 t4 + 9; n-tile i is d = 16 g + i
        const uint8_t* v = stage + 16 * kKvDim;
        uint4 w[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const int r = 2 * t4 + (i & 1) + 8 * (i >> 1);
          w[i] = *reinterpret_cast<const uint4*>(v + r * kKvDim + (g ^ (r & 6)) * 16);
        }
#pragma unroll
        for (int word = 0; word < 4; ++word) {
          uint32_t x[4], b0[4], b1[4];
#pragma unroll
          for (int i = 0; i < 4; ++i) x[i] = word == 0 ? w[i].x : word == 1 ? w[i].y : word == 2 ? w[i].z : w[i].w;
          codes_to_f16<TYPE>(__byte_perm(x[0], x[1], 0x5140), b0[0], b0[1]);
          codes_to_f16<TYPE>(__byte_perm(x[0], x[1], 0x7362), b0[2], b0[3]);
          codes_to_f16<TYPE>(__byte_perm(x[2], x[3], 0x5140), b1[0], b1[1]);
          codes_to_f16<TYPE>(__byte_perm(x[2], x[3], 0x7362), b1[2], b1[3]);
#pragma unroll
          for (int i = 0; i < 4; ++i) mma_f16(acc[word * 4 + i], pf, b0[i], b1[i]);
        }
      }
      __syncwarp();
      get = get + 1 == kDecStages ? 0 : get + 1;
    }

    // ---- the eight warps' parts of the tile ----
#pragma unroll
    for (int rr = 0; rr < 2; ++rr) {
      l[rr] += __shfl_xor_sync(0xffffffffu, l[rr], 1);
      l[rr] += __shfl_xor_sync(0xffffffffu, l[rr], 2);
      if (t4 == 0) row_stats[warp * kDecRows + g + 8 * rr] = make_float2(m[rr], l[rr]);
    }
    __syncthreads();
    float a[2];
#pragma unroll
    for (int rr = 0; rr < 2; ++rr) {
      float to = -INFINITY;
#pragma unroll
      for (int w = 0; w < kDecWarps; ++w) to = fmaxf(to, row_stats[w * kDecRows + g + 8 * rr].x);
      a[rr] = m[rr] == -INFINITY ? 0.f : ex2_approx(m[rr] - to) * vref;
    }
#pragma unroll
    for (int rr = 0; rr < 2; ++rr) {
      const int r = g + 8 * rr;
      float4* row = reinterpret_cast<float4*>(merge) + (warp * kDecRows + r) * (kKvDim / 4);
      const int swz = t4 | (r & 1) << 2;
#pragma unroll
      for (int e = 0; e < 2; ++e) {  // column 2 t4 + e of n-tile i is d = 16 (2 t4 + e) + i
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          row[(8 * t4 + 4 * e + i) ^ swz] = make_float4(acc[4 * i][2 * rr + e] * a[rr], acc[4 * i + 1][2 * rr + e] * a[rr],
                                                        acc[4 * i + 2][2 * rr + e] * a[rr], acc[4 * i + 3][2 * rr + e] * a[rr]);
        }
      }
    }
    __syncthreads();
    {
      const int r = threadIdx.x >> 4, c8 = threadIdx.x & 15;  // row, eight columns
      float to = -INFINITY;
#pragma unroll
      for (int w = 0; w < kDecWarps; ++w) to = fmaxf(to, row_stats[w * kDecRows + r].x);
      float sum = 0.f;
      float o[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int w = 0; w < kDecWarps; ++w) {
        const float2 ml = row_stats[w * kDecRows + r];
        sum += ml.x == -INFINITY ? ml.y : ml.y * ex2_approx(ml.x - to);
        const float4* row = reinterpret_cast<const float4*>(merge) + (w * kDecRows + r) * (kKvDim / 4);
#pragma unroll
        for (int i = 0; i < 2; ++i) {
          const int u = 2 * c8 + i;
          const float4 x = row[u ^ (u >> 3 | (r & 1) << 2)];
          o[4 * i] += x.x;
          o[4 * i + 1] += x.y;
          o[4 * i + 2] += x.z;
          o[4 * i + 3] += x.w;
        }
      }
      const TilePlace w = tile_place(p, now.s, now.h, static_cast<long long>(now.tile) * kDecRows + r);
      // a row that sees keys beyond the table's reach is NaN, as one that needs a page that does not exist
      if (w.real && now.s.len > now.s.keys && (!p.causal || now.s.len - now.s.n + w.token >= now.s.keys)) sum = __int_as_float(0x7fffffff);
      if (t_first == 0 && n_steps == now.steps) {
        if (w.real) {
          const float inv = sum > 0.f ? 1.f / sum : sum == 0.f ? 0.f : sum;  // 0: a row that sees no key
          uint4 x;
          x.x = pack_bf16x2(o[0] * inv, o[1] * inv);
          x.y = pack_bf16x2(o[2] * inv, o[3] * inv);
          x.z = pack_bf16x2(o[4] * inv, o[5] * inv);
          x.w = pack_bf16x2(o[6] * inv, o[7] * inv);
          *reinterpret_cast<uint4*>(p.o + row_offset(p, p.so, now.b, now.s, w) + c8 * 8) = x;
          if (c8 == 0 && p.lse != nullptr) {
            p.lse[lse_index(p, now.b, now.s, w)] = sum == 0.f ? -INFINITY : (to - kWeightShift + log2f(sum)) * kLn2;
          }
        }
      } else {  // slot 2 i: a tile begun by an earlier CTA; 2 i + 1: one begun here
        const long long slot = 2ll * blockIdx.x + (t_first == 0 ? 1 : 0);
        float4* part = reinterpret_cast<float4*>(p.parts + (slot * kDecRows + r) * kKvDim) + 2 * c8;
        part[0] = make_float4(o[0], o[1], o[2], o[3]);
        part[1] = make_float4(o[4], o[5], o[6], o[7]);
        if (c8 == 0) {
          reinterpret_cast<float2*>(p.parts + 2ll * p.ctas * kDecRows * kKvDim)[slot * kDecRows + r] = make_float2(to, sum);
        }
        if (threadIdx.x == 0 && t_first == 0) {
          p.pieces[blockIdx.x] = make_int4(now.b, now.h, now.tile, static_cast<int>(line.owner(tile_begin + now.steps - 1)));
        }
      }
    }
    __syncthreads();
    at += n_steps;
    if (at < line.end) now.next_tile(p);
  }
  cp_async_wait<0>();
}

// Joins the parts of a tile that several CTAs worked on: sum_i 2^(m_i - m) O_i / sum_i 2^(m_i - m) l_i, parts in order.
// Grid: (ctas, ROWS / 8); a block joins 8 rows of the tile that CTA blockIdx.x began and did not end, a warp a row.  Where a tile
// is spread over many CTAs the block takes the rows one after another and its warps share the parts.
constexpr int kJoinRows = 8;
constexpr int kJoinMany = 12;

struct JoinRow {
  float top, sum;
};
// The joint maximum and sum of a row, in every lane: the lanes' terms and then the lanes in a fixed order.
template <class Slot>
__device__ __forceinline__ JoinRow join_stats(const float2* stats, const Slot& slot, int n, int lane) {
  JoinRow j{-INFINITY, 0.f};
  for (int i = lane; i < n; i += 32) j.top = fmaxf(j.top, stats[slot(i)].x);
#pragma unroll
  for (int k = 16; k > 0; k >>= 1) j.top = fmaxf(j.top, __shfl_xor_sync(0xffffffffu, j.top, k));
  for (int i = lane; i < n; i += 32) {
    const float2 ml = stats[slot(i)];
    j.sum += ml.x == -INFINITY ? ml.y : ml.y * ex2_approx(ml.x - j.top);
  }
#pragma unroll
  for (int k = 16; k > 0; k >>= 1) j.sum += __shfl_xor_sync(0xffffffffu, j.sum, k);
  return j;
}

template <int ROWS>
__global__ void __launch_bounds__(256) attn_cached_join_kernel(const CachedParams p) {
  __shared__ float4 sums[8][32];
  const int4 piece = p.pieces[blockIdx.x];
  if (piece.w < 0) return;
  const SeqWork s = seq_work(p.c, piece.x);
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const int first = blockIdx.x, n = piece.w - first + 1;
  const float2* stats = reinterpret_cast<const float2*>(p.parts + 2ll * p.ctas * ROWS * kKvDim);
  const bool many = n > kJoinMany;
  for (int k = many ? 0 : warp; k < kJoinRows; k += many ? 1 : kJoinRows) {
    const int r = blockIdx.y * kJoinRows + k;
    const TilePlace w = tile_place(p, s, piece.y, static_cast<long long>(piece.z) * ROWS + r);
    if (!w.real) break;  // rows are in order: none behind it is
    auto slot = [&](int i) { return (2ll * (first + i) + (i == 0 ? 1 : 0)) * ROWS + r; };
    const JoinRow j = join_stats(stats, slot, n, lane);
    float4 o = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll 4
    for (int i = many ? warp : 0; i < n; i += many ? 8 : 1) {
      const float m = stats[slot(i)].x;
      const float4 x = reinterpret_cast<const float4*>(p.parts + slot(i) * kKvDim)[lane];
      const float f = m == -INFINITY ? 0.f : ex2_approx(m - j.top);
      o.x += x.x * f;
      o.y += x.y * f;
      o.z += x.z * f;
      o.w += x.w * f;
    }
    if (many) {
      __syncthreads();  // the row before has been read
      sums[warp][lane] = o;
      __syncthreads();
      if (warp != 0) continue;
#pragma unroll
      for (int i = 1; i < 8; ++i) {
        const float4 x = sums[i][lane];
        o.x += x.x;
        o.y += x.y;
        o.z += x.z;
        o.w += x.w;
      }
    }
    const float inv = j.sum > 0.f ? 1.f / j.sum : j.sum == 0.f ? 0.f : j.sum;
    const uint2 y = make_uint2(pack_bf16x2(o.x * inv, o.y * inv), pack_bf16x2(o.z * inv, o.w * inv));
    *reinterpret_cast<uint2*>(p.o + row_offset(p, p.so, piece.x, s, w) + lane * 4) = y;
    if (lane == 0 && p.lse != nullptr)
      p.lse[lse_index(p, piece.x, s, w)] = j.sum == 0.f ? -INFINITY : (j.top - kWeightShift + log2f(j.sum)) * kLn2;
  }
}

}  // namespace kv
}  // namespace attn
