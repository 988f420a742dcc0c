// Host side of the backward entry points: argument checks, plan, TMA descriptors, launches.
// Included by attn_api.cu (uses its device state and descriptor helpers).
#pragma once

namespace {

using attn::bwd::BwdParams;

// Bytes of one row-statistics array: fp32 [B * Hq][ceil(Sq / 128) * 128].
size_t bwd_stat_bytes(int B, int Hq, int Sq) {
  const size_t padded = (static_cast<size_t>(Sq) + attn::kTile - 1) / attn::kTile * attn::kTile;
  return static_cast<size_t>(B) * Hq * padded * sizeof(float);
}

constexpr int kPlanSms = 148;  // the plan, and with it the workspace, does not depend on the device
constexpr int kMaxParts = 32;

// Bytes of the partial sums of `splits` parts: fp32 [splits][B][H][tiles * 128][128]; none without a split.
size_t bwd_part_bytes(int splits, int B, int H, int tiles) {
  return splits > 1 ? static_cast<size_t>(splits) * B * H * tiles * attn::kTile * attn::kHeadDim * sizeof(float) : 0;
}

// Problem geometry and launch order (no device access).  False if the launch grid cannot hold the items.
bool fill_bwd_plan(BwdParams* p, int B, int Hq, int Hkv, int Sq, int Sk, int causal) {
  std::memset(p, 0, sizeof(*p));
  p->B = B; p->Hq = Hq; p->Hkv = Hkv; p->Sq = Sq; p->Sk = Sk;
  p->group = Hq / Hkv;
  p->causal = causal ? 1 : 0;
  p->off = Sk - Sq;
  p->n_qt = (Sq + attn::kTile - 1) / attn::kTile;
  p->n_kt = (Sk + attn::kTile - 1) / attn::kTile;
  // Parts of an item's stream.  An item's cost is counted in products (a key tile pair has four, a query tile pair three);
  // where the longest item exceeds a quarter of what an SM has to do on average, it is cut, so that no SM works on
  // alone at the end, but not below 24 products: a part costs its partial sums and a third launch adds them up.
  // (One head, 64 rows on 9000 keys, and the like; 512 rows on 65536 keys, 16 heads: 1.50 -> SPLIT_E.)
  const long long units = static_cast<long long>(B) * Hkv;
  const long long key_tiles = units * p->n_kt, qry_tiles = units * p->group * p->n_qt;
  const long long key_cost = 4LL * p->group * p->n_qt, qry_cost = 3LL * p->n_kt;  // of the longest items
  const double total = (static_cast<double>(key_tiles) * key_cost + static_cast<double>(qry_tiles) * qry_cost) *
                       (causal && Sk >= Sq ? 1.0 - 0.5 * Sq / Sk : causal ? 0.5 * Sk / Sq : 1.0);
  const double part = std::fmax(total / kPlanSms / 4, 24.0);
  auto parts = [part](long long cost) {
    const double n = std::ceil(static_cast<double>(cost) / part);
    return n < 1 ? 1 : n > kMaxParts ? kMaxParts : static_cast<int>(n);
  };
  p->key_splits = parts(key_cost);
  p->qry_splits = parts(qry_cost);
  const long long items = key_tiles * p->key_splits + qry_tiles * p->qry_splits;
  if (items > 0x3fffffffLL) return false;
  p->n_items = static_cast<int>(items);
  // as many units in a run as keep their q, dout, k and v within 64 MB of L2
  long long run = (64LL << 20) / (512LL * (static_cast<long long>(Sq) * p->group + Sk));
  if (run < 1) run = 1;
  if (run > 64) run = 64;
  if (run > units) run = units;
  // runs of nearly equal size, so that the last one is not a small remainder
  const int runs = static_cast<int>((units + run - 1) / run);
  const int base = static_cast<int>(units) / runs, extra = static_cast<int>(units) % runs;
  p->run = extra == 0 ? base : base + 1;
  p->run_extra = extra == 0 ? runs : extra;
  return true;
}

// Row statistics, then the partial sums of dq, dk and dv; every part is a multiple of 512 bytes.
size_t bwd_workspace_bytes(const BwdParams& p) {
  return 2 * bwd_stat_bytes(p.B, p.Hq, p.Sq) + bwd_part_bytes(p.qry_splits, p.B, p.Hq, p.n_qt) +
         2 * bwd_part_bytes(p.key_splits, p.B, p.Hkv, p.n_kt);
}

struct BwdTensors {
  const void *dout, *q, *k, *v, *o;
  const float *lse, *dlse;
  void *dq, *dk, *dv;
};
struct BwdStrides {
  Strides3 dout, q, k, v, o, dq, dk, dv;
};

attn_status_t bwd_device(const BwdTensors& t, int B, int Hq, int Hkv, int Sq, int Sk, int D, const BwdStrides& ts,
                         int causal, float scale, void* workspace, size_t workspace_bytes, void* stream) {
  if (t.dout == nullptr || t.lse == nullptr || t.dq == nullptr || t.dk == nullptr || t.dv == nullptr ||
      workspace == nullptr)
    return ATTN_ERR_NULL;
  attn_status_t st = check_args(t.q, t.k, t.v, const_cast<void*>(t.o), t.lse, B, Hq, Hkv, Sq, Sk, D, causal, scale, true);
  if (st != ATTN_OK) return st;
  BwdParams p;
  if (!fill_bwd_plan(&p, B, Hq, Hkv, Sq, Sk, causal)) return ATTN_ERR_UNSUPPORTED;
  const void* aligned[] = {t.dout, t.dq, t.dk, t.dv, workspace};
  for (const void* a : aligned) {
    if (reinterpret_cast<uintptr_t>(a) & 15) return ATTN_ERR_ALIGN;
  }
  if (t.dlse != nullptr && (reinterpret_cast<uintptr_t>(t.dlse) & 3)) return ATTN_ERR_ALIGN;
  // an output in the place of an input or of another output (slices of one buffer have addresses of their own)
  const void* out[] = {t.dq, t.dk, t.dv, workspace};
  const void* in[] = {t.dout, t.q, t.k, t.v, t.o, t.lse, t.dlse};
  for (int i = 0; i < 4; ++i) {
    for (const void* x : in) {
      if (out[i] == x) return ATTN_ERR_UNSUPPORTED;
    }
    for (int j = 0; j < i; ++j) {
      if (out[i] == out[j]) return ATTN_ERR_UNSUPPORTED;
    }
  }
  if (workspace_bytes < bwd_workspace_bytes(p)) return ATTN_ERR_TOO_LARGE;
  DeviceState* dev = device_state(&st);
  if (dev == nullptr) return st;

  CUtensorMap tm_q, tm_k, tm_v, tm_do, tm_dq, tm_dk, tm_dv;
  if (!make_tensor_map(&tm_q, t.q, B, Sq, Hq, ts.q) || !make_tensor_map(&tm_k, t.k, B, Sk, Hkv, ts.k) ||
      !make_tensor_map(&tm_v, t.v, B, Sk, Hkv, ts.v) || !make_tensor_map(&tm_do, t.dout, B, Sq, Hq, ts.dout) ||
      !make_tensor_map(&tm_dq, t.dq, B, Sq, Hq, ts.dq) || !make_tensor_map(&tm_dk, t.dk, B, Sk, Hkv, ts.dk) ||
      !make_tensor_map(&tm_dv, t.dv, B, Sk, Hkv, ts.dv))
    return ATTN_ERR_CUDA;

  uint8_t* ws = static_cast<uint8_t*>(workspace);
  float* neg_lse2 = reinterpret_cast<float*>(ws);
  float* neg_delta = reinterpret_cast<float*>(ws + bwd_stat_bytes(B, Hq, Sq));
  const size_t dq_bytes = bwd_part_bytes(p.qry_splits, B, Hq, p.n_qt), dk_bytes = bwd_part_bytes(p.key_splits, B, Hkv, p.n_kt);
  p.dq_part = reinterpret_cast<float*>(ws + 2 * bwd_stat_bytes(B, Hq, Sq));
  p.dk_part = p.dq_part + dq_bytes / sizeof(float);
  p.dv_part = p.dk_part + dk_bytes / sizeof(float);
  p.scale = scale;
  p.scale_log2 = scale * 1.4426950408889634f;
  p.neg_lse2 = neg_lse2;
  p.neg_delta = neg_delta;
  p.status = dev->status;
  cudaStream_t s = static_cast<cudaStream_t>(stream);
  const int padded = p.n_qt * attn::kTile;
  int heads_log2 = 0;  // heads of a block: up to 8, so that 256 rows are 32 positions or more
  while (heads_log2 < 3 && (2 << heads_log2) <= Hq) ++heads_log2;
  const int prep_rows = attn::bwd::kPrepThreads >> heads_log2;
  const long long prep_blocks = static_cast<long long>(B) * ((padded + prep_rows - 1) / prep_rows) *
                                ((Hq + (1 << heads_log2) - 1) >> heads_log2);
  const int cap = dev->sm_count * 8;
  attn::bwd::attn_bwd_prep_kernel<<<static_cast<int>(prep_blocks < cap ? prep_blocks : cap), attn::bwd::kPrepThreads, 0, s>>>(
      static_cast<const uint16_t*>(t.o), static_cast<const uint16_t*>(t.dout),
      attn::bwd::RowStrides{ts.o.b, ts.o.s, ts.o.h}, attn::bwd::RowStrides{ts.dout.b, ts.dout.s, ts.dout.h}, t.lse, t.dlse,
      neg_lse2, neg_delta, Hq, Sq, padded, heads_log2, static_cast<int>(prep_blocks));
  if (cudaGetLastError() != cudaSuccess) return ATTN_ERR_CUDA;
  const int grid = p.n_items;
  attn::bwd::attn_bwd_kernel<<<grid, attn::bwd::kBwdThreads, attn::bwd::kSmemBwdBytes, s>>>(tm_q, tm_k, tm_v, tm_do, tm_dq,
                                                                                       tm_dk, tm_dv, p);
  if (cudaGetLastError() != cudaSuccess) return ATTN_ERR_CUDA;
  if (p.key_splits == 1 && p.qry_splits == 1) return ATTN_OK;
  attn::bwd::JoinParams jp = {};
  int n_out = 0;
  long long most = 0;
  auto join = [&](const float* part, void* out, Strides3 st3, int splits, int H, int S, int tiles) {
    const long long padded_rows = static_cast<long long>(tiles) * attn::kTile;
    attn::bwd::JoinOut& j = jp.o[n_out++];
    j.part = part;
    j.out = static_cast<uint16_t*>(out);
    j.strides = attn::bwd::RowStrides{st3.b, st3.s, st3.h};
    j.splits = splits;
    j.H = H;
    j.S = S;
    j.padded = tiles * attn::kTile;
    j.n_rows = static_cast<long long>(B) * H * S;
    j.part_stride = static_cast<long long>(B) * H * padded_rows * attn::kHeadDim;
    if (j.n_rows > most) most = j.n_rows;
  };
  if (p.qry_splits > 1) join(p.dq_part, t.dq, ts.dq, p.qry_splits, Hq, Sq, p.n_qt);
  if (p.key_splits > 1) {
    join(p.dk_part, t.dk, ts.dk, p.key_splits, Hkv, Sk, p.n_kt);
    join(p.dv_part, t.dv, ts.dv, p.key_splits, Hkv, Sk, p.n_kt);
  }
  long long join_blocks = (most + attn::bwd::kJoinThreads / 32 - 1) / (attn::bwd::kJoinThreads / 32);
  if (join_blocks > cap) join_blocks = cap;
  attn::bwd::attn_bwd_join_kernel<<<dim3(static_cast<unsigned>(join_blocks), n_out), attn::bwd::kJoinThreads, 0, s>>>(jp);
  return cudaGetLastError() == cudaSuccess ? ATTN_OK : ATTN_ERR_CUDA;
}

}  // namespace

extern "C" {

size_t attn_bwd_workspace_bytes(int B, int Hq, int Hkv, int Sq, int Sk, int D, int causal) {
  int dummy = 0;
  if (check_args(&dummy, &dummy, &dummy, &dummy, nullptr, B, Hq, Hkv, Sq, Sk, D, causal, 1.0f, false) != ATTN_OK) return 0;
  BwdParams p;
  return fill_bwd_plan(&p, B, Hq, Hkv, Sq, Sk, causal) ? bwd_workspace_bytes(p) : 0;
}

attn_status_t attn_bwd(const void* dout, const void* q, const void* k, const void* v, const void* o, const float* lse,
                       const float* dlse, void* dq, void* dk, void* dv, int B, int Hq, int Hkv, int Sq, int Sk, int D,
                       int causal, float scale, void* workspace, size_t workspace_bytes, void* stream) {
  const Strides3 sq = contiguous_strides(Sq, Hq), sk = contiguous_strides(Sk, Hkv);
  return bwd_device(BwdTensors{dout, q, k, v, o, lse, dlse, dq, dk, dv}, B, Hq, Hkv, Sq, Sk, D,
                    BwdStrides{sq, sq, sk, sk, sq, sq, sk, sk}, causal, scale, workspace, workspace_bytes, stream);
}

attn_status_t attn_bwd_strided(const void* dout, const void* q, const void* k, const void* v, const void* o,
                               const float* lse, const float* dlse, void* dq, void* dk, void* dv, int B, int Hq, int Hkv,
                               int Sq, int Sk, int D, const long long* dout_strides, const long long* q_strides,
                               const long long* k_strides, const long long* v_strides, const long long* o_strides,
                               const long long* dq_strides, const long long* dk_strides, const long long* dv_strides,
                               int causal, float scale, void* workspace, size_t workspace_bytes, void* stream) {
  const long long* all[8] = {dout_strides, q_strides, k_strides, v_strides, o_strides, dq_strides, dk_strides, dv_strides};
  Strides3 s[8];
  for (int i = 0; i < 8; ++i) {
    const attn_status_t st = check_strides(all[i]);
    if (st != ATTN_OK) return st;
    s[i] = Strides3{all[i][0], all[i][1], all[i][2]};
  }
  return bwd_device(BwdTensors{dout, q, k, v, o, lse, dlse, dq, dk, dv}, B, Hq, Hkv, Sq, Sk, D,
                    BwdStrides{s[0], s[1], s[2], s[3], s[4], s[5], s[6], s[7]}, causal, scale, workspace, workspace_bytes,
                    stream);
}

}  // extern "C"
