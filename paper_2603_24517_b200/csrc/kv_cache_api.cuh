// Host side of attn_kv_append, attn_kv_read and attn_fwd_cached.  Included by attn_api.cu.
#pragma once

namespace {

using attn::kv::CachedParams;
using attn::kv::CacheView;
using attn::kv::RowStrides;

// Checks what all three share and fills the kernels' view of the cache.  `S`: rows a sequence, or rows in all with starts.
attn_status_t cache_view(const attn_kv_cache_t* c, int S, CacheView* v) {
  if (c == nullptr || c->k == nullptr || c->v == nullptr || c->k_scale == nullptr || c->v_scale == nullptr ||
      c->block_table == nullptr || c->seq_lens == nullptr)
    return ATTN_ERR_NULL;
  if (c->B <= 0 || c->Hkv <= 0 || c->D <= 0 || c->n_pages <= 0 || c->page_size <= 0 || c->max_blocks <= 0 || S <= 0)
    return ATTN_ERR_SHAPE;
  if (c->D != attn::kv::kKvDim) return ATTN_ERR_UNSUPPORTED;
  int page_log2 = 4;
  while (page_log2 < 7 && (1 << page_log2) != c->page_size) ++page_log2;
  if ((1 << page_log2) != c->page_size) return ATTN_ERR_UNSUPPORTED;
  if (c->type != ATTN_KV_E4M3 && c->type != ATTN_KV_INT8) return ATTN_ERR_UNSUPPORTED;
  // 32-bit positions and units
  if (static_cast<long long>(c->max_blocks) * c->page_size > (1ll << 30) || c->Hkv > 32767) return ATTN_ERR_UNSUPPORTED;
  if (S > (1 << 30) / (c->starts != nullptr ? 1 : c->B) || c->B > (1 << 24)) return ATTN_ERR_UNSUPPORTED;
  if (misaligned(c->k, 15) || misaligned(c->v, 15) || misaligned(c->k_scale, 3) || misaligned(c->v_scale, 3) ||
      misaligned(c->block_table, 3) || misaligned(c->seq_lens, 3) || misaligned(c->starts, 3))
    return ATTN_ERR_ALIGN;
  const long long* strides[2] = {c->k_strides, c->v_strides};
  for (int t = 0; t < 2; ++t) {
    for (int i = 0; i < 3; ++i) {
      if (strides[t][i] <= 0) return ATTN_ERR_SHAPE;
      if (strides[t][i] % 16 != 0) return ATTN_ERR_ALIGN;
      if (strides[t][i] >= (1ll << 39)) return ATTN_ERR_UNSUPPORTED;
    }
    if (strides[t][1] < attn::kv::kKvDim || strides[t][2] < attn::kv::kKvDim) return ATTN_ERR_SHAPE;
    v->sp[t] = strides[t][0];
    v->ss[t] = strides[t][1];
    v->sh[t] = strides[t][2];
  }
  if (c->table_stride < 0) return ATTN_ERR_SHAPE;
  v->codes[0] = static_cast<uint8_t*>(c->k);
  v->codes[1] = static_cast<uint8_t*>(c->v);
  v->scales[0] = c->k_scale;
  v->scales[1] = c->v_scale;
  v->table = c->block_table;
  v->table_stride = c->table_stride;
  v->lens = c->seq_lens;
  v->starts = c->starts;
  v->B = c->B;
  v->S = S;
  v->Hkv = c->Hkv;
  v->n_pages = c->n_pages;
  v->page_log2 = page_log2;
  v->max_blocks = c->max_blocks;
  v->type = c->type;
  return ATTN_OK;
}

// Strides of rows [B, S, H, D], or [S, H, D] of a packed batch (the first one is then not used).
attn_status_t row_strides(const long long* s, bool packed, int S, int H, RowStrides* out) {
  if (s == nullptr) {
    const Strides3 c = contiguous_strides(S, H);
    *out = RowStrides{c.b, c.s, c.h};
    return ATTN_OK;
  }
  const long long checked[3] = {packed ? 128 : s[0], s[1], s[2]};
  const attn_status_t st = check_strides(checked);
  if (st == ATTN_OK) *out = RowStrides{checked[0], checked[1], checked[2]};
  return st;
}

// What attn_kv_append and attn_kv_read share: arguments and the launch by pages.
struct PageLaunch {
  CacheView c;
  RowStrides ks, vs;
  dim3 grid;
  int threads;
};
attn_status_t page_launch(const attn_kv_cache_t* cache, const void* k, const void* v, int S, const long long* k_strides,
                          const long long* v_strides, PageLaunch* l) {
  if (k == nullptr || v == nullptr) return ATTN_ERR_NULL;
  attn_status_t st = cache_view(cache, S, &l->c);
  if (st != ATTN_OK) return st;
  if (misaligned(k, 15) || misaligned(v, 15)) return ATTN_ERR_ALIGN;
  st = row_strides(k_strides, cache->starts != nullptr, S, cache->Hkv, &l->ks);
  if (st == ATTN_OK) st = row_strides(v_strides, cache->starts != nullptr, S, cache->Hkv, &l->vs);
  if (st != ATTN_OK) return st;
  const long long units = attn::kv::unit_count(cache->starts != nullptr, l->c.B, S, l->c.page_log2);
  if (units > 0x7fffffffLL) return ATTN_ERR_UNSUPPORTED;
  l->grid = dim3(static_cast<unsigned>(units), 2u * l->c.Hkv);
  l->threads = (cache->page_size / attn::kv::kSlotsPerWarp) * 32;
  return ATTN_OK;
}

// The codes [n_pages, Hkv, page, D] as a 4-D tensor; a box is `rows` slots of one head.  A page number of n_pages reads zeros.
bool make_page_map(CUtensorMap* tm, const attn_kv_cache_t* c, int t, int rows, CUtensorMapSwizzle swizzle) {
  const long long* st = t == 0 ? c->k_strides : c->v_strides;
  const cuuint64_t dims[4] = {attn::kv::kKvDim, static_cast<cuuint64_t>(c->page_size), static_cast<cuuint64_t>(c->Hkv),
                              static_cast<cuuint64_t>(c->n_pages)};
  const cuuint64_t strides[3] = {static_cast<cuuint64_t>(st[1]), static_cast<cuuint64_t>(st[2]), static_cast<cuuint64_t>(st[0])};
  const cuuint32_t box[4] = {attn::kv::kKvDim, static_cast<cuuint32_t>(rows), 1, 1};
  const cuuint32_t elem_strides[4] = {1, 1, 1, 1};
  return g_encode(tm, CU_TENSOR_MAP_DATA_TYPE_UINT8, 4, t == 0 ? c->k : c->v, dims, strides, box, elem_strides,
                  CU_TENSOR_MAP_INTERLEAVE_NONE, swizzle, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
                  CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

// A part of a tile for every CTA that may end in one or begin in one.
size_t cached_parts(int ctas, int rows) { return 2ull * ctas * rows; }
size_t cached_workspace(int ctas, int rows) {
  return cached_parts(ctas, rows) * (attn::kv::kKvDim + 2) * sizeof(float) + static_cast<size_t>(ctas) * 2 * sizeof(int4) + 32;
}
constexpr int kWorkspaceSms = 160;  // SMs of a device at most
// In a packed batch with long sequences, single tokens and what else fits 8 rows go to the decoding kernel first (a step of 24
// sequences, 21 of them single tokens: 318 us all in tiles of 256 rows, 275 so; 4 us where there are none; 16 rows of two
// tokens stay, 16 sequences of 16 to 32 rows take a quarter more time apart; nor is it worth a launch where none has over 64).
// Tokens of 9 to 16 rows take tiles of 16, which read their keys once (64 sequences, groups of 16: 314 us in tiles of 8, 305 of 16; 48
// sequences, groups of 12: 652 and 637; all in tiles of 256 rows 339 and 736, but 24 sequences of 2 key heads 176 where these take 192).
// More than 16 heads a key head: a single token has too many rows itself, so nothing is split off (16 sequences, groups of 32: 60.0 us
// with the launches for nothing in front, 54.6 without).
int short_rows(int group) { return group <= 8 ? 8 : group <= 16 ? group : 0; }
int short_tile(int group) { return group <= 8 ? 8 : 16; }

// Rows of a query tile for the longest sequence's (token, head of a group) rows.  Decoding, 16 sequences of 12000 tokens, 8 key heads,
// E4M3: 8 rows 76 us in tiles of 8, 106 of 16, 168 of 256; 16 rows 131, 108 and 168; 32 rows 251, 201 and 170.
int tile_rows(int Hq, int Hkv, int max_new) {
  const long long rows = static_cast<long long>(Hq / Hkv) * max_new;
  return rows <= 8 ? 8 : rows <= 16 ? 16 : attn::kv::kTileRows;
}
int cached_ctas(int sms, int rows) { return rows == 8 ? sms * attn::kv::Dec<1>::kCtasPerSm : sms; }

// Places the parts of a launch at `at`; returns the first byte behind them.
uintptr_t place_parts(CachedParams* p, uintptr_t at, int sms, int rows) {
  at = (at + 31) & ~static_cast<uintptr_t>(31);
  p->ctas = cached_ctas(sms, rows);
  p->parts = reinterpret_cast<float*>(at);
  p->pieces = reinterpret_cast<int4*>(p->parts + cached_parts(p->ctas, rows) * (attn::kv::kKvDim + 2));
  return reinterpret_cast<uintptr_t>(p->pieces + 2 * p->ctas);
}

template <int NB>
bool prepare_decode() {
  return cudaFuncSetAttribute(attn::kv::attn_cached_decode_kernel<attn::kv::kE4m3, NB>, cudaFuncAttributeMaxDynamicSharedMemorySize,
                              attn::kv::Dec<NB>::kSmem) == cudaSuccess &&
         cudaFuncSetAttribute(attn::kv::attn_cached_decode_kernel<attn::kv::kInt8, NB>, cudaFuncAttributeMaxDynamicSharedMemorySize,
                              attn::kv::Dec<NB>::kSmem) == cudaSuccess;
}

template <int GRAN>
bool prepare_tile() {
  return cudaFuncSetAttribute(attn::kv::attn_cached_tile_kernel<attn::kv::kE4m3, GRAN>, cudaFuncAttributeMaxDynamicSharedMemorySize,
                              attn::kv::kTSmemBytes) == cudaSuccess &&
         cudaFuncSetAttribute(attn::kv::attn_cached_tile_kernel<attn::kv::kInt8, GRAN>, cudaFuncAttributeMaxDynamicSharedMemorySize,
                              attn::kv::kTSmemBytes) == cudaSuccess;
}

// Done by the first call of attn_fwd_cached on a device: the other entry points neither wait for these ten kernels (the first attn_fwd of a
// process takes 5.5 ms, with them 6.0) nor fail with them.  Calls at once may both do it.
bool prepare_cached(DeviceState* dev) {
  if (dev->cached_ready.load(std::memory_order_acquire)) return true;
  if (!prepare_decode<1>() || !prepare_decode<2>() || !prepare_tile<16>() || !prepare_tile<32>() || !prepare_tile<64>()) return false;
  dev->cached_ready.store(true, std::memory_order_release);
  return true;
}

// The join as a launch that may begin before the one in front of it has ended (it waits for that one's results on the device).
template <int ROWS>
attn_status_t launch_join(const CachedParams& p, int blocks, cudaStream_t s) {
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(p.ctas, blocks);
  cfg.blockDim = dim3(256);
  cfg.stream = s;
  cudaLaunchAttribute at;
  at.id = cudaLaunchAttributeProgrammaticStreamSerialization;
  at.val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = &at;
  cfg.numAttrs = 1;
  return cudaLaunchKernelEx(&cfg, attn::kv::attn_cached_join_kernel<ROWS>, p) == cudaSuccess ? ATTN_OK : ATTN_ERR_CUDA;
}

template <int NB>
attn_status_t launch_decode(const CachedParams& p, const CUtensorMap& tm_k, const CUtensorMap& tm_v, cudaStream_t s) {
  using D = attn::kv::Dec<NB>;
  if (p.c.type == ATTN_KV_E4M3) {
    attn::kv::attn_cached_decode_kernel<attn::kv::kE4m3, NB><<<p.ctas, attn::kv::kDecThreads, D::kSmem, s>>>(tm_k, tm_v, p);
  } else {
    attn::kv::attn_cached_decode_kernel<attn::kv::kInt8, NB><<<p.ctas, attn::kv::kDecThreads, D::kSmem, s>>>(tm_k, tm_v, p);
  }
  if (cudaGetLastError() != cudaSuccess) return ATTN_ERR_CUDA;
  return launch_join<D::kRows>(p, D::kRows, s);
}

// GRAN: keys that share their scales.  Three prompts of 700 rows on 4700 keys, pages of 32: 200 us by 16 keys, 191 by 32.
template <int GRAN>
attn_status_t launch_tile(const CachedParams& p, const CUtensorMap& tm_k, const CUtensorMap& tm_v, cudaStream_t s) {
  if (p.c.type == ATTN_KV_E4M3) {
    attn::kv::attn_cached_tile_kernel<attn::kv::kE4m3, GRAN><<<p.ctas, attn::kThreads, attn::kv::kTSmemBytes, s>>>(tm_k, tm_v, p);
  } else {
    attn::kv::attn_cached_tile_kernel<attn::kv::kInt8, GRAN><<<p.ctas, attn::kThreads, attn::kv::kTSmemBytes, s>>>(tm_k, tm_v, p);
  }
  if (cudaGetLastError() != cudaSuccess) return ATTN_ERR_CUDA;
  return launch_join<attn::kv::kTileRows>(p, attn::kv::kTileRows / (8 * attn::kv::kJoinRows), s);
}

}  // namespace

extern "C" {

attn_status_t attn_kv_append(const attn_kv_cache_t* cache, const void* k, const void* v, int S, const long long* k_strides,
                             const long long* v_strides, void* stream) {
  PageLaunch l;
  attn_status_t st = page_launch(cache, k, v, S, k_strides, v_strides, &l);
  if (st != ATTN_OK) return st;
  if (k == cache->k || k == cache->v || v == cache->k || v == cache->v || cache->k == cache->v || cache->k_scale == cache->v_scale)
    return ATTN_ERR_UNSUPPORTED;
  if (device_state(&st) == nullptr) return st;
  const uint16_t *kp = static_cast<const uint16_t*>(k), *vp = static_cast<const uint16_t*>(v);
  cudaStream_t s = static_cast<cudaStream_t>(stream);
  if (l.c.type == ATTN_KV_E4M3) {
    attn::kv::kv_append_kernel<attn::kv::kE4m3><<<l.grid, l.threads, 0, s>>>(l.c, kp, vp, l.ks, l.vs);
  } else {
    attn::kv::kv_append_kernel<attn::kv::kInt8><<<l.grid, l.threads, 0, s>>>(l.c, kp, vp, l.ks, l.vs);
  }
  return cudaGetLastError() == cudaSuccess ? ATTN_OK : ATTN_ERR_CUDA;
}

attn_status_t attn_kv_read(const attn_kv_cache_t* cache, void* k, void* v, int S, const long long* k_strides,
                           const long long* v_strides, void* stream) {
  PageLaunch l;
  attn_status_t st = page_launch(cache, k, v, S, k_strides, v_strides, &l);
  if (st != ATTN_OK) return st;
  if (k == v || k == cache->k || k == cache->v || v == cache->k || v == cache->v) return ATTN_ERR_UNSUPPORTED;
  if (device_state(&st) == nullptr) return st;
  uint16_t *kp = static_cast<uint16_t*>(k), *vp = static_cast<uint16_t*>(v);
  cudaStream_t s = static_cast<cudaStream_t>(stream);
  if (l.c.type == ATTN_KV_E4M3) {
    attn::kv::kv_read_kernel<attn::kv::kE4m3><<<l.grid, l.threads, 0, s>>>(l.c, kp, vp, l.ks, l.vs);
  } else {
    attn::kv::kv_read_kernel<attn::kv::kInt8><<<l.grid, l.threads, 0, s>>>(l.c, kp, vp, l.ks, l.vs);
  }
  return cudaGetLastError() == cudaSuccess ? ATTN_OK : ATTN_ERR_CUDA;
}

size_t attn_fwd_cached_workspace_bytes(int Hq, int Hkv, int max_new) {
  if (Hq <= 0 || Hkv <= 0 || Hq % Hkv != 0 || max_new <= 0) return 0;
  const int rows = tile_rows(Hq, Hkv, max_new);
  const size_t bytes = cached_workspace(cached_ctas(kWorkspaceSms, rows), rows);
  if (rows != attn::kv::kTileRows || short_rows(Hq / Hkv) == 0) return bytes;
  const int tile = short_tile(Hq / Hkv);
  return bytes + cached_workspace(cached_ctas(kWorkspaceSms, tile), tile);
}

attn_status_t attn_fwd_cached(const attn_kv_cache_t* cache, const void* q, void* o, float* lse, int Hq, int S, int max_new,
                              int causal, float scale, const long long* q_strides, const long long* o_strides, void* workspace,
                              size_t workspace_bytes, void* stream) {
  if (q == nullptr || o == nullptr || workspace == nullptr) return ATTN_ERR_NULL;
  CachedParams p;
  std::memset(&p, 0, sizeof(p));
  attn_status_t st = cache_view(cache, S, &p.c);
  if (st != ATTN_OK) return st;
  if (Hq <= 0 || Hq % cache->Hkv != 0 || max_new <= 0) return ATTN_ERR_SHAPE;
  if (!std::isfinite(scale) || !(scale > 0.f)) return ATTN_ERR_UNSUPPORTED;
  if (static_cast<long long>(S) * (Hq / cache->Hkv) > (1ll << 30)) return ATTN_ERR_UNSUPPORTED;
  if (misaligned(q, 15) || misaligned(o, 15) || misaligned(lse, 3) || misaligned(workspace, 15)) return ATTN_ERR_ALIGN;
  st = row_strides(q_strides, cache->starts != nullptr, S, Hq, &p.sq);
  if (st == ATTN_OK) st = row_strides(o_strides, cache->starts != nullptr, S, Hq, &p.so);
  if (st != ATTN_OK) return st;
  if (o == q || o == cache->k || o == cache->v || workspace == q || workspace == o || workspace == cache->k || workspace == cache->v)
    return ATTN_ERR_UNSUPPORTED;
  if (workspace_bytes < attn_fwd_cached_workspace_bytes(Hq, cache->Hkv, max_new)) return ATTN_ERR_TOO_LARGE;
  DeviceState* dev = device_state(&st);
  if (dev == nullptr) return st;
  if (!prepare_cached(dev)) return ATTN_ERR_CUDA;
  p.q = static_cast<const uint16_t*>(q);
  p.o = static_cast<uint16_t*>(o);
  p.lse = lse;
  p.Hq = Hq;
  p.group = Hq / cache->Hkv;
  p.causal = causal ? 1 : 0;
  p.scale_log2 = scale * 1.4426950408889634f;
  const int rows = tile_rows(Hq, cache->Hkv, max_new);
  const int sms = dev->sm_count < kWorkspaceSms ? dev->sm_count : kWorkspaceSms;
  p.status = dev->status;
  p.wide_o = !misaligned(o, 31) && p.so.b % 16 == 0 && p.so.s % 16 == 0 && p.so.h % 16 == 0;
  p.rows_above = 0;
  p.rows_up_to = 0x7fffffff;
  uintptr_t at = place_parts(&p, reinterpret_cast<uintptr_t>(workspace), sms, rows);
  cudaStream_t s = static_cast<cudaStream_t>(stream);
  CUtensorMap tm_k, tm_v;
  const bool many = rows == attn::kv::kTileRows;
  const bool split = many && cache->starts != nullptr && cache->B > 1 && p.group * static_cast<long long>(max_new) > 64 && short_rows(p.group) > 0;
  if (!many || split) {
    if (!make_page_map(&tm_k, cache, 0, 16, CU_TENSOR_MAP_SWIZZLE_128B) || !make_page_map(&tm_v, cache, 1, 16, CU_TENSOR_MAP_SWIZZLE_128B))
      return ATTN_ERR_CUDA;
    if (rows == 8) return launch_decode<1>(p, tm_k, tm_v, s);
    if (rows == 16) return launch_decode<2>(p, tm_k, tm_v, s);
    CachedParams few = p;
    const int tile = short_tile(p.group);
    place_parts(&few, at, sms, tile);
    few.rows_up_to = p.rows_above = short_rows(p.group);
    st = tile == 8 ? launch_decode<1>(few, tm_k, tm_v, s) : launch_decode<2>(few, tm_k, tm_v, s);
    if (st != ATTN_OK) return st;
  }
  if (!make_page_map(&tm_k, cache, 0, cache->page_size, CU_TENSOR_MAP_SWIZZLE_NONE) ||
      !make_page_map(&tm_v, cache, 1, cache->page_size, CU_TENSOR_MAP_SWIZZLE_NONE))
    return ATTN_ERR_CUDA;
  if (cache->page_size == 16) return launch_tile<16>(p, tm_k, tm_v, s);
  if (cache->page_size == 32) return launch_tile<32>(p, tm_k, tm_v, s);
  return launch_tile<64>(p, tm_k, tm_v, s);
}

}  // extern "C"
