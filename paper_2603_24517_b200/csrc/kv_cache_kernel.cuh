// A paged key/value cache in 8 bits: new tokens' keys and values quantised into their pages, and the way back.
//
// Position p of sequence b is slot p % page of page table[b][p / page].  A page and head has one scale s for its keys and one
// for its values; a code c stands for c s.  With A the largest finite magnitude among the new values of a page and head,
//
//     E4M3:  s = the smallest power of two with A <= 448 s       INT8:  s = A (1 / 127)   (0 where A = 0)
//     s <- max(s, the page's scale), if the page holds earlier tokens;  c = round(x / s), ties to even
//
// and where s grew, the codes the page already holds become round(c s_old / s).  A power of two moves E4M3 codes to a
// larger scale without a rounding error outside the smallest binades, and x / s is exact; the price is less than one bit of
// range, which a floating code does not miss.
//
// Both directions move 3 bytes a value, which bounds them (all but the append in INT8, below).  One CTA owns one page and head
// of the keys or of the values, a warp 16 slots of it, so the largest magnitude is known in the CTA, nobody else touches the
// scale, and eight 16-byte (codes: 8-byte) accesses are in flight in each lane.  Which page that is follows from the CTA's index
// alone: sequence b owns the units from starts[b] / page + 2 b on, which is at least as many as it has pages, so a warp finds b
// by a search over `starts` and no list of pages has to be made first.  32768 tokens of 8 heads: 37.8 us to append, 35.5 to read
// back, 5.3 and 5.7 TB/s, in INT8 81.0 (not profiled: the codes take a dozen instructions a value and a branch around a
// division) and 36.4; three CTAs of 256 threads' worth of registers (80, a few spills) against two without spills: 38 and 45 us.
#pragma once

#include <cuda_fp16.h>

#include "ptx.cuh"

namespace attn {
namespace kv {

constexpr int kKvDim = 128;
constexpr int kSlotsPerWarp = 16;   // slots of a page a warp works on; page sizes are 16 .. 128
constexpr int kE4m3 = 0;
constexpr int kInt8 = 1;
constexpr float kMinScale = 7.888609052210118e-31f;  // 2^-100: x / s stays in range for every BF16 x

// What the entry points know about the cache.  Everything in device memory that came from the caller (page numbers, lengths,
// starts) is checked where it is read: a wrong one loses its own sequence's results and touches nothing else.
struct CacheView {
  uint8_t* codes[2];       // keys, values
  float* scales[2];        // [n_pages][Hkv]
  long long sp[2], ss[2], sh[2];  // strides of page, slot and head in bytes
  const int* table;        // [B][max_blocks]
  long long table_stride;
  const int* lens;         // [B] tokens of each sequence, the new ones included
  const int* starts;       // [B + 1] rows of each sequence in a packed batch, or null: S rows each
  int B, S, Hkv, n_pages, page_log2, max_blocks;  // S: rows a sequence, or rows in all with `starts`
  int type;
};

// Rows of sequence b: the first one in its batch and how many.
__device__ __forceinline__ void rows_of(const CacheView& c, int b, int& row0, int& n) {
  if (c.starts == nullptr) {
    row0 = 0;
    n = c.S;
  } else {
    const int a = __ldg(c.starts + b), e = __ldg(c.starts + b + 1);
    row0 = min(max(a, 0), c.S);
    n = max(min(e, c.S) - row0, 0);
  }
}

// Page of block j of sequence b, or -1 where there is none.
__device__ __forceinline__ int page_of(const CacheView& c, int b, int j) {
  if (j < 0 || j >= c.max_blocks) return -1;
  const int page = __ldg(c.table + b * c.table_stride + j);
  return static_cast<unsigned>(page) < static_cast<unsigned>(c.n_pages) ? page : -1;
}

// Units of the page-wise kernels.
__host__ __device__ __forceinline__ long long units_per_sequence(int S, int page_log2) {
  return S <= 1 ? 1 : ((S - 2) >> page_log2) + 2;
}
__host__ __device__ __forceinline__ long long unit_count(bool packed, int B, int S, int page_log2) {
  return packed ? (S >> page_log2) + 2ll * B : B * units_per_sequence(S, page_log2);
}
__device__ __forceinline__ long long first_unit(const CacheView& c, int b) {
  return (min(max(__ldg(c.starts + b), 0), c.S) >> c.page_log2) + 2ll * b;
}

// Sequence and block (counted from the sequence's first block of this call) of a unit; every lane of a full warp calls.
__device__ __forceinline__ void unit_place(const CacheView& c, long long u, int lane, int& b, long long& j) {
  if (c.starts == nullptr) {
    const long long per = units_per_sequence(c.S, c.page_log2);
    b = static_cast<int>(u / per);
    j = u - b * per;
    return;
  }
  int lo = 0, hi = c.B;  // the answer is in [lo, hi): the last b whose first unit is not beyond u
  while (hi - lo > 1) {
    const int step = (hi - lo + 31) >> 5;
    const int probe = lo + lane * step;
    const bool reached = probe < hi && first_unit(c, probe) <= u;
    const unsigned votes = __ballot_sync(0xffffffffu, reached);  // lane 0's holds by construction for u >= 0
    const int last = votes == 0 ? 0 : 31 - __clz(votes);
    lo += last * step;
    hi = min(hi, lo + step);
  }
  b = lo;
  j = u - first_unit(c, b);
}

// ---- codes ------------------------------------------------------------------------------------------------------
__device__ __forceinline__ float2 unpack_bf16x2(uint32_t w) {
  return make_float2(__uint_as_float(w << 16), __uint_as_float(w & 0xffff0000u));
}
__device__ __forceinline__ __half2 bits_half2(uint32_t w) { return *reinterpret_cast<__half2*>(&w); }
__device__ __forceinline__ uint32_t half2_bits(__half2 h) { return *reinterpret_cast<uint32_t*>(&h); }

// Four codes of one word as four f16, exactly: lo = bytes 0, 1, hi = bytes 2, 3.
template <int TYPE>
__device__ __forceinline__ void codes_to_f16(uint32_t w, uint32_t& lo, uint32_t& hi) {
  if (TYPE == kE4m3) {
    asm("{\n\t.reg .b16 l, h;\n\tmov.b32 {l, h}, %2;\n\tcvt.rn.f16x2.e4m3x2 %0, l;\n\tcvt.rn.f16x2.e4m3x2 %1, h;\n\t}\n"
        : "=r"(lo), "=r"(hi)
        : "r"(w));
  } else {  // 0x6400 | (c + 128) is the f16 number 1024 + c + 128
    const uint32_t u = w ^ 0x80808080u;
    const __half2 bias = bits_half2(0x64806480u);
    lo = half2_bits(__hsub2(bits_half2(__byte_perm(u, 0x64646464u, 0x4140)), bias));
    hi = half2_bits(__hsub2(bits_half2(__byte_perm(u, 0x64646464u, 0x4342)), bias));
  }
}

// Scale of a page and head whose new values' largest finite magnitude is `a`.
template <int TYPE>
__device__ __forceinline__ float scale_for(float a) {
  if (!(a > 0.f)) return 0.f;
  float s;
  if (TYPE == kE4m3) {  // 448 = 1.75 * 2^8: the exponent of a, one more where its fraction is above 1.75
    const int e = static_cast<int>((__float_as_uint(a) + 0x1fffffu) >> 23) - 127 - 8;
    s = e < -100 ? kMinScale : __uint_as_float(static_cast<uint32_t>(e + 127) << 23);
  } else {
    s = __fmul_rn(a, 1.f / 127.f);  // the product defines the scale, not the quotient
  }
  return fmaxf(s, kMinScale);
}

struct Quantiser {
  float scale, inverse;  // scale 0 (nothing but zeros): codes of x itself
};
__device__ __forceinline__ Quantiser quantiser(float scale) {
  const float s = scale > 0.f ? scale : 1.f;
  return Quantiser{s, __fdiv_rn(1.f, s)};
}

// round(x / s) of four values, packed.
template <int TYPE>
__device__ __forceinline__ uint32_t encode4(const float* x, const Quantiser& q) {
  if (TYPE == kE4m3) {  // the scale is a power of two, so the product is the quotient; caches from elsewhere are only read
    uint16_t lo, hi;
    asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;" : "=h"(lo) : "f"(x[1] * q.inverse), "f"(x[0] * q.inverse));
    asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;" : "=h"(hi) : "f"(x[3] * q.inverse), "f"(x[2] * q.inverse));
    return lo | static_cast<uint32_t>(hi) << 16;
  }
  uint32_t w = 0;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    float y = x[i] * q.inverse;  // within 2^-22 of the quotient: the division decides only next to a tie
    float r = rintf(y);
    if (fabsf(fabsf(y - r) - 0.5f) < 1e-3f) r = rintf(__fdiv_rn(x[i], q.scale));
    r = fminf(fmaxf(r, -127.f), 127.f);
    const int c = x[i] == x[i] ? static_cast<int>(r) : 0;
    w |= (static_cast<uint32_t>(c) & 0xffu) << (8 * i);
  }
  return w;
}

// ---- new tokens into their pages -----------------------------------------------------------------------------------
struct RowStrides {
  long long b, s, h;  // elements
};

// Grid: (units, 2 Hkv), one CTA of page / 16 warps each.
template <int TYPE>
__global__ void __launch_bounds__(256, 3) kv_append_kernel(const CacheView c, const uint16_t* __restrict__ k_rows,
                                                        const uint16_t* __restrict__ v_rows, const RowStrides ks,
                                                        const RowStrides vs) {
  __shared__ float warp_max[8];
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  int b;
  long long j;
  unit_place(c, blockIdx.x, lane, b, j);
  int row0, n;
  rows_of(c, b, row0, n);
  if (n == 0) return;
  const int t = blockIdx.y & 1, h = blockIdx.y >> 1;
  const int begin = max(__ldg(c.lens + b), 0) - n;  // position of the sequence's first row here; negative: no place for it
  const long long block = (begin >> c.page_log2) + j;
  const long long slot0 = block << c.page_log2;     // position of the page's slot 0
  const long long first = max(slot0, static_cast<long long>(max(begin, 0)));
  const long long last = min(slot0 + (1 << c.page_log2), static_cast<long long>(begin) + n);
  if (first >= last) return;
  const int lo = static_cast<int>(first - slot0), hi = static_cast<int>(last - slot0);  // slots written: [lo, hi)

  // the rows are on their way while the page is looked up
  const RowStrides st = t ? vs : ks;
  const uint16_t* rows = (t ? v_rows : k_rows) + (c.starts == nullptr ? b * st.b : 0ll) + h * st.h +
                         (row0 + slot0 - begin) * st.s + (lane & 15) * 8;
  uint4 x[8];
  float largest = 0.f;
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const int slot = warp * kSlotsPerWarp + 2 * i + (lane >> 4);
    x[i] = make_uint4(0, 0, 0, 0);
    if (slot >= lo && slot < hi) x[i] = __ldcs(reinterpret_cast<const uint4*>(rows + slot * st.s));
  }
  const int page = page_of(c, b, static_cast<int>(min(block, 0x7fffffffll)));
  if (page < 0) return;
  uint8_t* codes = c.codes[t] + page * c.sp[t] + h * c.sh[t] + (lane & 15) * 8;
  float* scale_at = c.scales[t] + static_cast<long long>(page) * c.Hkv + h;
  const bool holds = lo > 0;
  const float before = holds ? *scale_at : 0.f;

#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const uint32_t w[4] = {x[i].x, x[i].y, x[i].z, x[i].w};
#pragma unroll
    for (int m = 0; m < 4; ++m) {
      const float2 f = unpack_bf16x2(w[m]);
      const float a = fabsf(f.x), d = fabsf(f.y);
      if (a <= 3.4e38f) largest = fmaxf(largest, a);  // infinities and NaN take no part
      if (d <= 3.4e38f) largest = fmaxf(largest, d);
    }
  }
#pragma unroll
  for (int m = 16; m > 0; m >>= 1) largest = fmaxf(largest, __shfl_xor_sync(0xffffffffu, largest, m));
  if (blockDim.x > 32) {
    if (lane == 0) warp_max[warp] = largest;
    __syncthreads();
    for (int w = 0; w < static_cast<int>(blockDim.x >> 5); ++w) largest = fmaxf(largest, warp_max[w]);
  }
  const float scale = fmaxf(scale_for<TYPE>(largest), before);
  const Quantiser q = quantiser(scale);
  if (holds && scale > before) {  // the tokens the page already holds, at the larger scale
    for (int slot = warp * 2 + (lane >> 4); slot < lo; slot += static_cast<int>(blockDim.x >> 4)) {
      uint2* at = reinterpret_cast<uint2*>(codes + slot * c.ss[t]);
      uint2 w = *at;
      uint32_t* word = reinterpret_cast<uint32_t*>(&w);
#pragma unroll
      for (int m = 0; m < 2; ++m) {
        uint32_t f16[2];
        codes_to_f16<TYPE>(word[m], f16[0], f16[1]);
        const float2 f = __half22float2(bits_half2(f16[0])), g = __half22float2(bits_half2(f16[1]));
        const float old[4] = {__fmul_rn(f.x, before), __fmul_rn(f.y, before), __fmul_rn(g.x, before), __fmul_rn(g.y, before)};
        word[m] = encode4<TYPE>(old, q);
      }
      *at = w;
    }
  }
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const int slot = warp * kSlotsPerWarp + 2 * i + (lane >> 4);
    if (slot < lo || slot >= hi) continue;
    const float2 f[4] = {unpack_bf16x2(x[i].x), unpack_bf16x2(x[i].y), unpack_bf16x2(x[i].z), unpack_bf16x2(x[i].w)};
    const float* v = reinterpret_cast<const float*>(f);
    *reinterpret_cast<uint2*>(codes + slot * c.ss[t]) = make_uint2(encode4<TYPE>(v, q), encode4<TYPE>(v + 4, q));
  }
  // every thread's read of the old scale lies before the barrier above, or in this warp
  __syncwarp();
  if (threadIdx.x == 0) *scale_at = scale;
}

// ---- the last tokens of each sequence back in BF16 -------------------------------------------------------------------
template <int TYPE>
__global__ void __launch_bounds__(256) kv_read_kernel(const CacheView c, uint16_t* __restrict__ k_rows,
                                                      uint16_t* __restrict__ v_rows, const RowStrides ks, const RowStrides vs) {
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  int b;
  long long j;
  unit_place(c, blockIdx.x, lane, b, j);
  int row0, n;
  rows_of(c, b, row0, n);
  if (n == 0) return;
  const int t = blockIdx.y & 1, h = blockIdx.y >> 1;
  const int begin = max(__ldg(c.lens + b), 0) - n;
  const long long block = (begin >> c.page_log2) + j;
  const long long slot0 = block << c.page_log2;
  const int lo = static_cast<int>(max(begin - slot0, 0ll));
  const int hi = static_cast<int>(min(1ll << c.page_log2, static_cast<long long>(begin) + n - slot0));
  if (lo >= hi) return;
  const int page = page_of(c, b, static_cast<int>(min(block, 0x7fffffffll)));
  const RowStrides st = t ? vs : ks;
  uint16_t* rows = (t ? v_rows : k_rows) + (c.starts == nullptr ? b * st.b : 0ll) + h * st.h +
                   (row0 + slot0 - begin) * st.s + (lane & 15) * 8;
  const uint8_t* codes = c.codes[t] + max(page, 0) * c.sp[t] + h * c.sh[t] + (lane & 15) * 8;
  const float scale = page < 0 ? 0.f : __ldg(c.scales[t] + static_cast<long long>(page) * c.Hkv + h);
  uint2 x[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const int slot = warp * kSlotsPerWarp + 2 * i + (lane >> 4);
    x[i] = make_uint2(0, 0);
    if (slot >= lo && slot < hi && page >= 0) x[i] = __ldg(reinterpret_cast<const uint2*>(codes + slot * c.ss[t]));
  }
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const int slot = warp * kSlotsPerWarp + 2 * i + (lane >> 4);
    if (slot < lo || slot >= hi) continue;
    uint32_t f16[4], out[4];
    codes_to_f16<TYPE>(x[i].x, f16[0], f16[1]);
    codes_to_f16<TYPE>(x[i].y, f16[2], f16[3]);
#pragma unroll
    for (int m = 0; m < 4; ++m) {
      const float2 f = __half22float2(bits_half2(f16[m]));
      out[m] = pack_bf16x2(f.x * scale, f.y * scale);
      // positions before the sequence's first token are zeros; a page that does not exist gives NaN
      if (page < 0) out[m] = block < 0 ? 0u : 0x7fff7fffu;
    }
    *reinterpret_cast<uint4*>(rows + slot * st.s) = make_uint4(out[0], out[1], out[2], out[3]);
  }
}

}  // namespace kv
}  // namespace attn
