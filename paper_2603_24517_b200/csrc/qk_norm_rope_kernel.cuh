// Norm of every query and key head with the position rotation in the same pass, and its gradient.
//
//     n = x r w,   r = 1 / sqrt(mean(x^2) + eps),   y = Rot(pos) n          (x: one head's 128 values)
//
// Rot turns each pair (a, b) of the first `rot` values by the angle of (position, pair):
// (a c - b s, b c + a s); the other values pass.  With g = Rot^T dy:
//
//     dw = sum over rows of g x r,    dx = r (g w - x r^2 mean(g w x)).
//
// Elementwise with one 128-value reduction per row: bound by HBM (4 bytes a value forward, 6 backward) as long as the
// instructions stay few.  Half a warp owns a row, 16 bytes a lane, so a row is one 256-byte access and its sums are four
// shuffles; the partner of a value sits in the same lane (adjacent pairs) or `rot / 16` lanes away (halves), where four
// shuffles of the packed BF16 words fetch it.  A warp works on 8 rows of one token and one tensor at a time: four
// independent row loads per lane are in flight and the token's angles are read once for them; it does all its query
// units before its key units, so weights and weight sums stay in registers; the arithmetic is in packed fp32 pairs.
// Rows go through the caches as streams (evict first).  32768 tokens of 32 + 8 heads: forward 130 us, 5.2 TB/s,
// gradient 203 us, 5.0 TB/s, as replayed launches (calls on a busy GPU 136 and 215 us; a timing copy with the same accesses
// and no arithmetic 111 and 196 us, so the gradient is held by its access plan).  Measured slower: two rows a
// lane (219 us), eight (176 us), the next unit's rows fetched ahead into registers (145 and 236 us) or shared memory (175
// and 224 us: a warp's own chain of sums is what takes the time, and both cost resident warps or instructions),
// more CTAs than resident (135 us); in the forward pass, rows in pairs with shared sums (131 us).
#pragma once

#include "attn_merge_kernel.cuh"
#include "ptx.cuh"

namespace attn {
namespace rope {

constexpr int kRopeThreads = 256;
constexpr int kRopeWarps = kRopeThreads / 32;
constexpr int kRowsPerLane = 4;                   // rows a half warp holds at once
constexpr int kUnitRows = 2 * kRowsPerLane;       // rows of one token a warp works on at a time
constexpr int kRopeDim = 128;
constexpr int kDwCtas = 296;                      // CTAs of the gradient kernel, each with one partial of both dw

struct RopeStrides {
  long long b, s, h;  // elements
};

struct RopeParams {
  const uint16_t* x[2];  // queries, keys
  const uint16_t* dy[2]; // gradient kernel only
  uint16_t* out[2];      // y, or dx
  RopeStrides sx[2], sdy[2], sout[2];
  const void* w[2];      // may be null (weight 1)
  int w_bf16;
  const float* cos_tab;  // [n_positions][rot / 2]
  const float* sin_tab;
  const void* positions; // may be null: the token's index in its sequence
  int positions_64;
  long long pos_b, pos_s;  // strides of positions
  long long n_positions;
  int S, heads[2], units[2];  // units: ceil(heads / kUnitRows), per token
  int rot;
  float eps;
  uint32_t n_units[2];   // B * S * units
  float* partials;       // gradient kernel: [gridDim.x][2][128], or null
};

struct Unit {
  long long b;
  int s, h0;  // token of the sequence, first head
};
// 32-bit division: a 64-bit one costs more instructions than the arithmetic of the unit's rows.
__device__ __forceinline__ Unit unit_of(const RopeParams& p, int t, uint32_t u) {
  const uint32_t per = p.units[t];
  const uint32_t token = u / per, b = token / static_cast<uint32_t>(p.S);
  Unit r;
  r.h0 = static_cast<int>(u - token * per) * kUnitRows;
  r.b = b;
  r.s = static_cast<int>(token - b * p.S);
  return r;
}

// Eight values of a lane as four pairs.
__device__ __forceinline__ void unpack8(const uint4& v, float2* f) {
  f[0] = make_float2(bf16_lo(v.x), bf16_hi(v.x));
  f[1] = make_float2(bf16_lo(v.y), bf16_hi(v.y));
  f[2] = make_float2(bf16_lo(v.z), bf16_hi(v.z));
  f[3] = make_float2(bf16_lo(v.w), bf16_hi(v.w));
}
__device__ __forceinline__ uint4 pack8(const float2* f) {
  return make_uint4(pack_bf16x2(f[0].x, f[0].y), pack_bf16x2(f[1].x, f[1].y), pack_bf16x2(f[2].x, f[2].y),
                    pack_bf16x2(f[3].x, f[3].y));
}
__device__ __forceinline__ void load8(const float* src, float2* f) {
  const float4 a = __ldg(reinterpret_cast<const float4*>(src)), b = __ldg(reinterpret_cast<const float4*>(src) + 1);
  f[0] = make_float2(a.x, a.y);
  f[1] = make_float2(a.z, a.w);
  f[2] = make_float2(b.x, b.y);
  f[3] = make_float2(b.z, b.w);
}
// 8 weights starting at value `at` (a multiple of 8)
__device__ __forceinline__ void load_weights(const RopeParams& p, int t, int at, float2* f) {
  if (p.w[t] == nullptr) {
#pragma unroll
    for (int i = 0; i < 4; ++i) f[i] = make_float2(1.f, 1.f);
  } else if (p.w_bf16) {
    unpack8(__ldg(reinterpret_cast<const uint4*>(p.w[t]) + at / 8), f);
  } else {
    load8(static_cast<const float*>(p.w[t]) + at, f);
  }
}
__device__ __forceinline__ float sum16(float v) {  // over the half warp
#pragma unroll
  for (int m = 8; m > 0; m >>= 1) v += __shfl_xor_sync(0xffffffffu, v, m);
  return v;
}
// Four sums at once: the lanes first share out the values among themselves, so nine shuffles do what sixteen would, in a
// chain hardly longer than one sum's.
__device__ __forceinline__ void sum16x4(float* v, int lane) {
  const bool b8 = lane & 8, b4 = lane & 4;
  const float a0 = (b8 ? v[2] : v[0]) + __shfl_xor_sync(0xffffffffu, b8 ? v[0] : v[2], 8);
  const float a1 = (b8 ? v[3] : v[1]) + __shfl_xor_sync(0xffffffffu, b8 ? v[1] : v[3], 8);
  float c = (b4 ? a1 : a0) + __shfl_xor_sync(0xffffffffu, b4 ? a0 : a1, 4);
  c += __shfl_xor_sync(0xffffffffu, c, 2);
  c += __shfl_xor_sync(0xffffffffu, c, 1);
#pragma unroll
  for (int i = 0; i < 4; ++i) v[i] = __shfl_sync(0xffffffffu, c, (lane & 16) + (i >> 1) * 8 + (i & 1) * 4);
}
__device__ __forceinline__ uint4 shfl4(const uint4& v, int lane) {
  return make_uint4(__shfl_sync(0xffffffffu, v.x, lane), __shfl_sync(0xffffffffu, v.y, lane),
                    __shfl_sync(0xffffffffu, v.z, lane), __shfl_sync(0xffffffffu, v.w, lane));
}

// What a lane needs of the rotation: per value the cosine and the signed sine that goes with the pair's other value
// (-sin for the first of a pair, +sin for the second; cosine 1 and sine 0 behind the rotated values).
struct Turn {
  float2 c[4], s[4];
};
// The lane that holds the other values of this lane's pairs (its own where they are in the lane or not rotated).
template <bool kInterleaved>
__device__ __forceinline__ int partner_lane(const RopeParams& p, int lane) {
  const int sub = lane & 15, half_lanes = p.rot >> 4;  // lanes that hold the first half of the rotated values
  if (kInterleaved || sub >= 2 * half_lanes) return lane;
  return sub < half_lanes ? lane + half_lanes : lane - half_lanes;
}

// False: the position lies outside the tables; the token's rows become NaN, nothing is read out of bounds.
template <bool kInterleaved>
__device__ __forceinline__ bool load_turn(const RopeParams& p, const Unit& u, int lane, Turn* tn) {
  const int sub = lane & 15, half_lanes = p.rot >> 4;
  long long pos = u.s;
  if (p.positions != nullptr) {
    const long long at = u.b * p.pos_b + u.s * p.pos_s;
    pos = p.positions_64 ? __ldg(static_cast<const long long*>(p.positions) + at)
                         : static_cast<long long>(__ldg(static_cast<const int*>(p.positions) + at));
  }
  const bool good = pos >= 0 && pos < p.n_positions;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    tn->c[i] = make_float2(1.f, 1.f);
    tn->s[i] = make_float2(0.f, 0.f);
  }
  if (sub >= 2 * half_lanes || !good) return good;
  const long long row = pos * (p.rot >> 1);
  if (kInterleaved) {
    const float4 c = __ldg(reinterpret_cast<const float4*>(p.cos_tab + row) + sub);
    const float4 s = __ldg(reinterpret_cast<const float4*>(p.sin_tab + row) + sub);
    const float cc[4] = {c.x, c.y, c.z, c.w}, ss[4] = {s.x, s.y, s.z, s.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      tn->c[i] = make_float2(cc[i], cc[i]);
      tn->s[i] = make_float2(-ss[i], ss[i]);
    }
  } else {
    const bool first = sub < half_lanes;
    const int at = (first ? sub : sub - half_lanes) * 8;
    load8(p.cos_tab + row + at, tn->c);
    load8(p.sin_tab + row + at, tn->s);
    const float sign = first ? -1.f : 1.f;
#pragma unroll
    for (int i = 0; i < 4; ++i) tn->s[i] = mul2(tn->s[i], make_float2(sign, sign));
  }
  return good;
}

// The other value of each of the lane's pairs, as packed words.
template <bool kInterleaved>
__device__ __forceinline__ uint4 partner(const uint4& v, int lane) {
  if (kInterleaved) return make_uint4(v.x << 16 | v.x >> 16, v.y << 16 | v.y >> 16, v.z << 16 | v.z >> 16, v.w << 16 | v.w >> 16);
  return shfl4(v, lane);
}

__device__ __forceinline__ float sum_squares(const float2* f) {  // of the lane's values
  float2 a = mul2(f[0], f[0]), b = mul2(f[1], f[1]);
  a = fma2(f[2], f[2], a);
  b = fma2(f[3], f[3], b);
  a = add2(a, b);
  return a.x + a.y;
}
// 1 / sqrt(mean + eps) of a row, NaN for a token whose position lies outside the tables
__device__ __forceinline__ float inv_rms(float squares, float eps, bool good) {
  return good ? rsqrtf(fmaf(squares, 1.f / kRopeDim, eps)) : __int_as_float(0x7fffffff);
}

// The warp's units `un`, un + step, ... of tensor t.  Returns the first number beyond them, minus n_units[t]: the warps'
// numbering goes on through the other tensor's units.
template <bool kInterleaved, int t>
__device__ __forceinline__ uint32_t forward_units(const RopeParams& p, uint32_t un, uint32_t step, int lane) {
  const int sub = lane & 15, hw = lane >> 4, other = partner_lane<kInterleaved>(p, lane);
  const RopeStrides sx = p.sx[t], so = p.sout[t];
  const int heads = p.heads[t];
  float2 w[4], wp[4];
  if (un < p.n_units[t]) {
    load_weights(p, t, sub * 8, w);
    load_weights(p, t, (other & 15) * 8, wp);
    if (kInterleaved) {
#pragma unroll
      for (int i = 0; i < 4; ++i) wp[i] = make_float2(w[i].y, w[i].x);
    }
  }
  for (; un < p.n_units[t]; un += step) {
    const Unit u = unit_of(p, t, un);
    const int h0 = u.h0 + hw;
    // streaming, but coherent loads: y may be x itself (a lane's rows are read before they are written)
    const uint16_t* src = p.x[t] + u.b * sx.b + u.s * sx.s + h0 * sx.h + sub * 8;
    uint16_t* dst = p.out[t] + u.b * so.b + u.s * so.s + h0 * so.h + sub * 8;
    uint4 x[kRowsPerLane];
#pragma unroll
    for (int i = 0; i < kRowsPerLane; ++i) {
      x[i] = make_uint4(0u, 0u, 0u, 0u);
      if (h0 + 2 * i < heads) x[i] = __ldcs(reinterpret_cast<const uint4*>(src + 2 * i * sx.h));
    }
    Turn tn;
    const bool good = load_turn<kInterleaved>(p, u, lane, &tn);
#pragma unroll
    for (int i = 0; i < 4; ++i) {  // y = r (x * w c + x_partner * w_partner s)
      tn.c[i] = mul2(tn.c[i], w[i]);
      tn.s[i] = mul2(tn.s[i], wp[i]);
    }
#pragma unroll
    for (int i = 0; i < kRowsPerLane; ++i) {
      float2 f[4], g[4];
      unpack8(x[i], f);
      unpack8(partner<kInterleaved>(x[i], other), g);
      const float r = inv_rms(sum16(sum_squares(f)), p.eps, good);
      const float2 r2 = make_float2(r, r);
#pragma unroll
      for (int e = 0; e < 4; ++e) f[e] = mul2(fma2(f[e], tn.c[e], mul2(g[e], tn.s[e])), r2);
      if (h0 + 2 * i < heads) __stcs(reinterpret_cast<uint4*>(dst + 2 * i * so.h), pack8(f));
    }
  }
  return un - p.n_units[t];
}

template <bool kInterleaved>
__global__ void __launch_bounds__(kRopeThreads, 3)
qk_norm_rope_kernel(const __grid_constant__ RopeParams p) {
  const int lane = threadIdx.x & 31;
  const uint32_t step = gridDim.x * kRopeWarps;
  const uint32_t un = blockIdx.x * kRopeWarps + (threadIdx.x >> 5);
  forward_units<kInterleaved, 1>(p, forward_units<kInterleaved, 0>(p, un, step, lane), step, lane);
}

// The same for the gradient; dw: the sums of g x r over the lane's values of all its rows.
template <bool kInterleaved, int t>
__device__ __forceinline__ uint32_t backward_units(const RopeParams& p, uint32_t un, uint32_t step, int lane, float2* dw) {
  const int sub = lane & 15, hw = lane >> 4, other = partner_lane<kInterleaved>(p, lane);
  const RopeStrides sx = p.sx[t], sg = p.sdy[t], so = p.sout[t];
  const int heads = p.heads[t];
  float2 w[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) dw[i] = make_float2(0.f, 0.f);
  if (un < p.n_units[t]) load_weights(p, t, sub * 8, w);
  for (; un < p.n_units[t]; un += step) {
    const Unit u = unit_of(p, t, un);
    const int h0 = u.h0 + hw;
    const uint16_t* src = p.x[t] + u.b * sx.b + u.s * sx.s + h0 * sx.h + sub * 8;
    const uint16_t* grd = p.dy[t] + u.b * sg.b + u.s * sg.s + h0 * sg.h + sub * 8;
    uint16_t* dst = p.out[t] + u.b * so.b + u.s * so.s + h0 * so.h + sub * 8;
    uint4 x[kRowsPerLane], y[kRowsPerLane];
#pragma unroll
    for (int i = 0; i < kRowsPerLane; ++i) {
      x[i] = y[i] = make_uint4(0u, 0u, 0u, 0u);
      if (h0 + 2 * i < heads) {
        x[i] = __ldcs(reinterpret_cast<const uint4*>(src + 2 * i * sx.h));
        y[i] = __ldcs(reinterpret_cast<const uint4*>(grd + 2 * i * sg.h));
      }
    }
    Turn tn;
    const bool good = load_turn<kInterleaved>(p, u, lane, &tn);
#pragma unroll
    for (int i = 0; i < 4; ++i) tn.s[i] = mul2(tn.s[i], make_float2(-1.f, -1.f));  // the transposed rotation
#pragma unroll
    for (int i = 0; i < kRowsPerLane; i += 2) {  // two rows at a time
      float2 g[2][4];
      float sums[4];  // squares, and g w x, of both rows
#pragma unroll
      for (int v = 0; v < 2; ++v) {
        float2 f[4], q[4];
        unpack8(x[i + v], f);
        unpack8(y[i + v], g[v]);
        unpack8(partner<kInterleaved>(y[i + v], other), q);
        float2 gx = make_float2(0.f, 0.f);
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          g[v][e] = fma2(g[v][e], tn.c[e], mul2(q[e], tn.s[e]));
          gx = fma2(mul2(g[v][e], w[e]), f[e], gx);
        }
        sums[v] = sum_squares(f);
        sums[2 + v] = gx.x + gx.y;
      }
      sum16x4(sums, lane);
#pragma unroll
      for (int v = 0; v < 2; ++v) {  // rows beyond the last head hold zeros and add nothing to dw
        float2 f[4];
        unpack8(x[i + v], f);
        const float r = inv_rms(sums[v], p.eps, good), k = -sums[2 + v] * (1.f / kRopeDim) * r * r;
        const float2 r2 = make_float2(r, r), k2 = make_float2(k, k);
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          dw[e] = fma2(g[v][e], mul2(f[e], r2), dw[e]);
          f[e] = mul2(fma2(f[e], k2, mul2(g[v][e], w[e])), r2);
        }
        if (h0 + 2 * (i + v) < heads) __stcs(reinterpret_cast<uint4*>(dst + 2 * (i + v) * so.h), pack8(f));
      }
    }
  }
  return un - p.n_units[t];
}

// dx, and per CTA the sums of g x r over its rows, added up in a fixed order.
template <bool kInterleaved>
__global__ void __launch_bounds__(kRopeThreads, 2)
qk_norm_rope_bwd_kernel(const __grid_constant__ RopeParams p) {
  __shared__ float sums[kRopeWarps * 2][2][kRopeDim];
  const int lane = threadIdx.x & 31, sub = lane & 15, hw = lane >> 4;
  const uint32_t step = gridDim.x * kRopeWarps;
  float2 dw[2][4];
  const uint32_t un = backward_units<kInterleaved, 0>(p, blockIdx.x * kRopeWarps + (threadIdx.x >> 5), step, lane, dw[0]);
  backward_units<kInterleaved, 1>(p, un, step, lane, dw[1]);
  if (p.partials == nullptr) return;
#pragma unroll
  for (int t = 0; t < 2; ++t) {
#pragma unroll
    for (int e = 0; e < 4; ++e) *reinterpret_cast<float2*>(&sums[(threadIdx.x >> 5) * 2 + hw][t][sub * 8 + e * 2]) = dw[t][e];
  }
  __syncthreads();
  const int t = threadIdx.x >> 7, c = threadIdx.x & 127;
  float v = 0.f;
#pragma unroll
  for (int i = 0; i < kRopeWarps * 2; ++i) v += sums[i][t][c];
  p.partials[(static_cast<size_t>(blockIdx.x) * 2 + t) * kRopeDim + c] = v;
}

// dw[t][c] = sum over the n partials, 8 columns a CTA, 32 threads a column, added up in a fixed order.
__global__ void __launch_bounds__(256)
qk_norm_rope_dw_kernel(const float* __restrict__ partials, int n, float* dw_q, float* dw_k) {
  __shared__ float part[32][9];
  const int col = blockIdx.x * 8 + (threadIdx.x & 7), grp = threadIdx.x >> 3;  // col in [0, 256): both tensors
  float v = 0.f;
  for (int i = grp; i < n; i += 32) v += __ldg(partials + static_cast<size_t>(i) * 2 * kRopeDim + col);
  part[grp][threadIdx.x & 7] = v;
  __syncthreads();
  if (threadIdx.x < 8) {
    float s = 0.f;
#pragma unroll
    for (int i = 0; i < 32; ++i) s += part[i][threadIdx.x];
    const int c = blockIdx.x * 8 + threadIdx.x;
    float* out = c < kRopeDim ? dw_q : dw_k;
    if (out != nullptr) out[c & (kRopeDim - 1)] = s;
  }
}

}  // namespace rope
}  // namespace attn
