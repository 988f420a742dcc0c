// Norm of every query and key head with the position rotation in the same pass, and its gradient.
//
//     n = x r w,   r = 1 / sqrt(mean(x^2) + eps),   y = Rot(pos) n          (x: one head's 128 values)
//
// Rot turns each pair (a, b) of the first `rot` values by the angle of (position, pair):
// (a c - b s, b c + a s); the other values pass.  With g = Rot^T dy:
//
//     dw = sum over rows of g x r,    dx = r (g w - x r^2 mean(g w x)).
//
// Elementwise with one 128-value reduction per row: bound by HBM (4 bytes a value forward, 6 backward).  Half a
// warp owns a row, 16 bytes a lane, so a row is one 256-byte access and its sums are four shuffles; the partner
// of a value sits in the same lane (adjacent pairs) or `rot / 16` lanes away (halves), where four shuffles of the
// packed BF16 words fetch it.  A warp works on 8 rows of one token and one tensor at a time: four independent row
// loads per lane are in flight, and the token's angles and the weights are read once for them.
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
  int S, heads[2], units[2];  // units: ceil(heads / kUnitRows)
  int rot;
  float eps;
  int n_units;           // B * S * (units[0] + units[1])
  float* partials;       // gradient kernel: [gridDim.x][2][128], or null
};

struct Unit {
  long long b;
  int s, t, h0;  // token, tensor (0 queries, 1 keys), first head
};
// 32-bit division: a 64-bit one costs more instructions than the arithmetic of the unit's rows.
__device__ __forceinline__ Unit unit_of(const RopeParams& p, uint32_t u) {
  const uint32_t per = p.units[0] + p.units[1];
  const uint32_t token = u / per, b = token / static_cast<uint32_t>(p.S);
  const int k = static_cast<int>(u - token * per);
  Unit r;
  r.t = k >= p.units[0] ? 1 : 0;
  r.h0 = (r.t ? k - p.units[0] : k) * kUnitRows;
  r.b = b;
  r.s = static_cast<int>(token - b * p.S);
  return r;
}

__device__ __forceinline__ void unpack8(const uint4& v, float* f) {
  f[0] = bf16_lo(v.x); f[1] = bf16_hi(v.x); f[2] = bf16_lo(v.y); f[3] = bf16_hi(v.y);
  f[4] = bf16_lo(v.z); f[5] = bf16_hi(v.z); f[6] = bf16_lo(v.w); f[7] = bf16_hi(v.w);
}
__device__ __forceinline__ uint4 pack8(const float* f) {
  return make_uint4(pack_bf16x2(f[0], f[1]), pack_bf16x2(f[2], f[3]), pack_bf16x2(f[4], f[5]), pack_bf16x2(f[6], f[7]));
}
__device__ __forceinline__ void load8(const float* src, float* f) {
  const float4 a = __ldg(reinterpret_cast<const float4*>(src)), b = __ldg(reinterpret_cast<const float4*>(src) + 1);
  f[0] = a.x; f[1] = a.y; f[2] = a.z; f[3] = a.w; f[4] = b.x; f[5] = b.y; f[6] = b.z; f[7] = b.w;
}
// 8 weights starting at value `at` (a multiple of 8)
__device__ __forceinline__ void load_weights(const RopeParams& p, int t, int at, float* f) {
  if (p.w[t] == nullptr) {
#pragma unroll
    for (int i = 0; i < 8; ++i) f[i] = 1.f;
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
__device__ __forceinline__ uint4 shfl4(const uint4& v, int lane) {
  return make_uint4(__shfl_sync(0xffffffffu, v.x, lane), __shfl_sync(0xffffffffu, v.y, lane),
                    __shfl_sync(0xffffffffu, v.z, lane), __shfl_sync(0xffffffffu, v.w, lane));
}

// What a lane needs of the rotation: per value the cosine and the signed sine that goes with the pair's other value
// (-sin for the first of a pair, +sin for the second), and in the halves layout the lane of the other value.
struct Turn {
  float c[8], s[8];
  int lane;
  bool inside;  // this lane's values are rotated
};

// `good` false: the position lies outside the tables; the token's rows become NaN, nothing is read out of bounds.
template <bool kInterleaved>
__device__ __forceinline__ void load_turn(const RopeParams& p, const Unit& u, int lane, Turn* tn, bool* good) {
  const int sub = lane & 15, half_lanes = p.rot >> 4;  // lanes that hold the first half of the rotated values
  long long pos = u.s;
  if (p.positions != nullptr) {
    const long long at = u.b * p.pos_b + u.s * p.pos_s;
    pos = p.positions_64 ? __ldg(static_cast<const long long*>(p.positions) + at)
                         : static_cast<long long>(__ldg(static_cast<const int*>(p.positions) + at));
  }
  *good = pos >= 0 && pos < p.n_positions;
  tn->inside = sub < 2 * half_lanes;
  tn->lane = lane;
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    tn->c[i] = 1.f;
    tn->s[i] = 0.f;
  }
  if (!tn->inside || !*good) return;
  const long long row = pos * (p.rot >> 1);
  if (kInterleaved) {
    const float4 c = __ldg(reinterpret_cast<const float4*>(p.cos_tab + row) + sub);
    const float4 s = __ldg(reinterpret_cast<const float4*>(p.sin_tab + row) + sub);
    const float cc[4] = {c.x, c.y, c.z, c.w}, ss[4] = {s.x, s.y, s.z, s.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      tn->c[2 * i] = tn->c[2 * i + 1] = cc[i];
      tn->s[2 * i] = -ss[i];
      tn->s[2 * i + 1] = ss[i];
    }
  } else {
    const bool first = sub < half_lanes;
    const int at = (first ? sub : sub - half_lanes) * 8;
    load8(p.cos_tab + row + at, tn->c);
    load8(p.sin_tab + row + at, tn->s);
    tn->lane = first ? lane + half_lanes : lane - half_lanes;
#pragma unroll
    for (int i = 0; i < 8; ++i) tn->s[i] = first ? -tn->s[i] : tn->s[i];
  }
}

// The other value of each of the lane's pairs, as packed words.
template <bool kInterleaved>
__device__ __forceinline__ uint4 partner(const uint4& v, int lane) {
  if (kInterleaved) return make_uint4(v.x << 16 | v.x >> 16, v.y << 16 | v.y >> 16, v.z << 16 | v.z >> 16, v.w << 16 | v.w >> 16);
  return shfl4(v, lane);
}

template <bool kInterleaved>
__global__ void __launch_bounds__(kRopeThreads)
qk_norm_rope_kernel(const __grid_constant__ RopeParams p) {
  const int lane = threadIdx.x & 31, sub = lane & 15, hw = lane >> 4;
  const uint32_t step = gridDim.x * kRopeWarps;
  for (uint32_t un = blockIdx.x * kRopeWarps + (threadIdx.x >> 5); un < static_cast<uint32_t>(p.n_units); un += step) {
    const Unit u = unit_of(p, un);
    const RopeStrides sx = p.sx[u.t], so = p.sout[u.t];
    // no restrict qualifiers and no non-coherent loads: y may be x itself (a lane's rows are read before written)
    const uint16_t* src = p.x[u.t] + u.b * sx.b + u.s * sx.s;
    uint4 x[kRowsPerLane];
#pragma unroll
    for (int i = 0; i < kRowsPerLane; ++i) {
      const int h = u.h0 + 2 * i + hw;
      x[i] = make_uint4(0u, 0u, 0u, 0u);
      if (h < p.heads[u.t]) x[i] = *(reinterpret_cast<const uint4*>(src + h * sx.h) + sub);
    }
    Turn tn;
    bool good;
    load_turn<kInterleaved>(p, u, lane, &tn, &good);
    float w[8], wp[8];
    load_weights(p, u.t, sub * 8, w);
    if (kInterleaved) {
#pragma unroll
      for (int i = 0; i < 8; ++i) wp[i] = w[i ^ 1];
    } else {
      load_weights(p, u.t, (tn.lane & 15) * 8, wp);
    }
#pragma unroll
    for (int i = 0; i < 8; ++i) {  // y = r (x * w c + x_partner * w_partner s)
      w[i] *= tn.c[i];
      wp[i] *= tn.s[i];
    }
#pragma unroll
    for (int i = 0; i < kRowsPerLane; ++i) {
      const int h = u.h0 + 2 * i + hw;
      float f[8], g[8], ss = 0.f;
      unpack8(x[i], f);
      unpack8(partner<kInterleaved>(x[i], tn.lane), g);
#pragma unroll
      for (int e = 0; e < 8; ++e) ss = fmaf(f[e], f[e], ss);
      const float r = good ? rsqrtf(sum16(ss) * (1.f / kRopeDim) + p.eps) : __int_as_float(0x7fffffff);
#pragma unroll
      for (int e = 0; e < 8; ++e) f[e] = r * fmaf(f[e], w[e], tn.inside ? g[e] * wp[e] : 0.f);
      if (h < p.heads[u.t])
        *(reinterpret_cast<uint4*>(p.out[u.t] + u.b * so.b + u.s * so.s + h * so.h) + sub) = pack8(f);
    }
  }
}

// dx, and per CTA the sums of g x r over its rows, added up in a fixed order.
template <bool kInterleaved>
__global__ void __launch_bounds__(kRopeThreads)
qk_norm_rope_bwd_kernel(const __grid_constant__ RopeParams p) {
  __shared__ float sums[kRopeWarps * 2][2][kRopeDim];
  const int lane = threadIdx.x & 31, sub = lane & 15, hw = lane >> 4;
  const uint32_t step = gridDim.x * kRopeWarps;
  float dw[2][8];
#pragma unroll
  for (int i = 0; i < 8; ++i) dw[0][i] = dw[1][i] = 0.f;
  for (uint32_t un = blockIdx.x * kRopeWarps + (threadIdx.x >> 5); un < static_cast<uint32_t>(p.n_units); un += step) {
    const Unit u = unit_of(p, un);
    const RopeStrides sx = p.sx[u.t], sg = p.sdy[u.t], so = p.sout[u.t];
    const uint16_t* src = p.x[u.t] + u.b * sx.b + u.s * sx.s;
    const uint16_t* grd = p.dy[u.t] + u.b * sg.b + u.s * sg.s;
    uint4 x[kRowsPerLane], y[kRowsPerLane];
#pragma unroll
    for (int i = 0; i < kRowsPerLane; ++i) {
      const int h = u.h0 + 2 * i + hw;
      x[i] = y[i] = make_uint4(0u, 0u, 0u, 0u);
      if (h < p.heads[u.t]) {
        x[i] = *(reinterpret_cast<const uint4*>(src + h * sx.h) + sub);
        y[i] = *(reinterpret_cast<const uint4*>(grd + h * sg.h) + sub);
      }
    }
    Turn tn;
    bool good;
    load_turn<kInterleaved>(p, u, lane, &tn, &good);
    float w[8], acc[8];
    load_weights(p, u.t, sub * 8, w);
#pragma unroll
    for (int i = 0; i < 8; ++i) acc[i] = 0.f;
#pragma unroll
    for (int i = 0; i < kRowsPerLane; ++i) {
      const int h = u.h0 + 2 * i + hw;
      float f[8], g[8], q[8], ss = 0.f, gx = 0.f;
      unpack8(x[i], f);
      unpack8(y[i], g);
      unpack8(partner<kInterleaved>(y[i], tn.lane), q);
#pragma unroll
      for (int e = 0; e < 8; ++e) {  // the transposed rotation: the sines change sign
        g[e] = fmaf(g[e], tn.c[e], tn.inside ? -(q[e] * tn.s[e]) : 0.f);
        ss = fmaf(f[e], f[e], ss);
        gx = fmaf(g[e] * w[e], f[e], gx);
      }
      const float r = good ? rsqrtf(sum16(ss) * (1.f / kRopeDim) + p.eps) : __int_as_float(0x7fffffff);
      const float k = sum16(gx) * (1.f / kRopeDim) * r * r;
      const bool row = h < p.heads[u.t];
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        if (row) acc[e] = fmaf(g[e], f[e] * r, acc[e]);
        f[e] = r * fmaf(-f[e], k, g[e] * w[e]);
      }
      if (row) *(reinterpret_cast<uint4*>(p.out[u.t] + u.b * so.b + u.s * so.s + h * so.h) + sub) = pack8(f);
    }
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      dw[0][e] += u.t == 0 ? acc[e] : 0.f;
      dw[1][e] += u.t == 1 ? acc[e] : 0.f;
    }
  }
  if (p.partials == nullptr) return;
#pragma unroll
  for (int t = 0; t < 2; ++t) {
#pragma unroll
    for (int e = 0; e < 8; ++e) sums[(threadIdx.x >> 5) * 2 + hw][t][sub * 8 + e] = dw[t][e];
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
