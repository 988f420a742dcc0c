// Host side of the backward entry points: argument checks, plan, TMA descriptors, launches.
// Included by attn_api.cu (uses its device state and descriptor helpers).
#pragma once

namespace {

using attn::bwd::BwdParams;

// Bytes of one row-statistics array: fp32 [B * Hq][n_qt * 128].
size_t bwd_stat_bytes(const BwdParams& p) { return static_cast<size_t>(p.B) * p.Hq * p.n_qt * attn::kTile * sizeof(float); }

constexpr int kPlanSms = 148;  // the plan, and with it the workspace, does not depend on the device
constexpr int kMaxParts = 32;

// Bytes of the partial sums of `splits` parts: fp32 [splits][B][H][tiles * 128][128]; none without a split.
size_t bwd_part_bytes(int splits, int B, int H, int tiles) {
  return splits > 1 ? static_cast<size_t>(splits) * B * H * tiles * attn::kTile * attn::kHeadDim * sizeof(float) : 0;
}

// Estimate of a launch, in SM clocks: the kind of item with the longer streams goes first, the other fills up behind it.
// Measured on B200: a tile pair takes 2650 (key) or 2450 (query) clocks, the start and end of an item 3500, an fp32
// partial result 8000 / 4000 more, and the join a launch and the reading of the partial sums.
struct BwdCost {
  double total, longest, average;
  int queries_first;
};
BwdCost bwd_cost(const BwdParams& p, long long key_tiles, long long key_len, int ks, long long qry_tiles, long long qry_len, int qs,
                 double seen) {
  const double key_item = 3500 + (ks > 1 ? 8000 : 0), qry_item = 3500 + (qs > 1 ? 4000 : 0);
  const double key_max = key_item + 2650.0 * key_len / ks, qry_max = qry_item + 2450.0 * qry_len / qs;
  const double key_avg = key_item + 2650.0 * seen * key_len / ks, qry_avg = qry_item + 2450.0 * seen * qry_len / qs;
  const double n_key = static_cast<double>(key_tiles) * ks, n_qry = static_cast<double>(qry_tiles) * qs;
  BwdCost c;
  c.queries_first = qry_max > key_max ? 1 : 0;
  c.average = (n_key * key_avg + n_qry * qry_avg) / kPlanSms;
  c.longest = std::fmax(key_max, qry_max);
  const double n1 = c.queries_first ? n_qry : n_key, avg1 = c.queries_first ? qry_avg : key_avg;
  const double max2 = std::fmin(key_max, qry_max), avg2 = c.queries_first ? key_avg : qry_avg;
  const double first = n1 <= kPlanSms ? c.longest : std::ceil(n1 / kPlanSms) * avg1;  // the first kind by itself
  const double second = std::floor(n1 / kPlanSms) * avg1 + max2;                      // the first free SM takes one of the second
  const double tail = n_key + n_qry > kPlanSms ? 0.5 * avg2 : 0.0;
  c.total = std::fmax(c.average + tail, std::fmax(first, second));
  if (ks > 1 || qs > 1) {
    const double parts = (ks > 1 ? 2 * n_key : 0) + (qs > 1 ? n_qry : 0);  // tiles of 64 KB
    c.total += 7000 + parts * 65536 / 3500;
  }
  return c;
}

// Problem geometry and launch order (no device access).  False if the launch grid cannot hold the items.
bool fill_bwd_plan(BwdParams* p, int B, int Hq, int Hkv, int Sq, int Sk, int causal) {
  std::memset(p, 0, sizeof(*p));
  p->B = B; p->Hq = Hq; p->Hkv = Hkv; p->Sq = Sq; p->Sk = Sk;
  p->group = Hq / Hkv;
  p->causal = causal ? 1 : 0;
  p->off = Sk - Sq;
  p->n_qt = (Sq + attn::kTile - 1) / attn::kTile;
  // Pack a group's heads into the rows of a tile where that saves an eighth of the query tiles or more (one row of 4
  // heads for each of 8 key heads, 4 sequences of 32768 keys: 0.73 -> 0.40 ms).
  const int group = p->group;
  if (group >= 2 && group <= 16 && (group & (group - 1)) == 0 && static_cast<long long>(Sq) * group <= 0x3fffff00) {
    const int packed = (Sq * group + attn::kTile - 1) / attn::kTile;
    if (8LL * packed <= 7LL * group * p->n_qt) {
      while ((1 << p->pack_log2) < group) ++p->pack_log2;
      p->Hq = Hkv;
      p->group = 1;
      p->Sq = Sq = Sq * group;
      p->n_qt = packed;
    }
  }
  p->n_kt = (Sk + attn::kTile - 1) / attn::kTile;
  const long long units = static_cast<long long>(B) * Hkv;
  const long long key_tiles = units * p->n_kt, qry_tiles = units * p->group * p->n_qt;
  const long long key_len = static_cast<long long>(p->group) * p->n_qt, qry_len = p->n_kt;  // longest streams
  const double rows = Sq >> p->pack_log2;
  const double seen = !causal ? 1.0 : Sk >= rows ? 1.0 - 0.5 * rows / Sk : 0.5 * Sk / rows;  // share of visible tile pairs
  const BwdCost one = bwd_cost(*p, key_tiles, key_len, 1, qry_tiles, qry_len, 1, seen);
  p->key_splits = p->qry_splits = 1;
  p->queries_first = one.queries_first;
  // With many more items than SMs the order alone balances them; else the streams may be worth cutting.
  const bool few = one.longest > 0.25 * one.average;
  if (few) {
    double best = one.total;
    for (int ks = 1; ks <= kMaxParts; ks *= 2) {
      for (int qs = 1; qs <= kMaxParts; qs *= 2) {
        if ((ks > 1 && key_len < 2 * ks) || (qs > 1 && qry_len < 2 * qs)) continue;
        const BwdCost c = bwd_cost(*p, key_tiles, key_len, ks, qry_tiles, qry_len, qs, seen);
        if (c.total < best) {
          best = c.total;
          p->key_splits = ks;
          p->qry_splits = qs;
          p->queries_first = c.queries_first;
        }
      }
    }
  }
  const long long items = key_tiles * p->key_splits + qry_tiles * p->qry_splits;
  if (items > 0x3fffffffLL) return false;
  p->n_items = static_cast<int>(items);
  // as many units in a run as keep their q, dout, k and v within 64 MB of L2; all where the order has to balance the
  // SMs (512 rows on 65536 keys, 16 heads: 1.17 -> 0.81 ms)
  long long run = few ? units : (64LL << 20) / (512LL * (static_cast<long long>(Sq) * p->group + Sk));
  if (run < 1) run = 1;
  if (!few && run > 64) run = 64;
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
  return 2 * bwd_stat_bytes(p) + bwd_part_bytes(p.qry_splits, p.B, p.Hq, p.n_qt) +
         2 * bwd_part_bytes(p.key_splits, p.B, p.Hkv, p.n_kt);
}

// Whether the gradients are sums of so few terms that P and dS are kept as two BF16 numbers (see attn_bwd_kernel.cuh).
// With one, results with at most 64 rows or keys were up to 2.3 times as far off as a rounding of their own leaves them;
// with two 1.00 times, in 7 to 15 % more time (16 sequences of 64 rows, 32 heads: 48 -> 55 us;
// one row, 32 heads on 8, 4 sequences of 32768 keys: 382 -> 415 us).  The rule is one for whole calls: short sums inside a
// longer call (first rows and last keys under the causal mask) keep one number, and a long dq of one row gets two.
constexpr int kFineRows = 64;
bool fine_bwd(int Sq, int Sk) { return Sq <= kFineRows || Sk <= kFineRows; }

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
  if (!make_tensor_map(&tm_q, t.q, B, Sq, Hq, ts.q, p.pack_log2) || !make_tensor_map(&tm_k, t.k, B, Sk, Hkv, ts.k) ||
      !make_tensor_map(&tm_v, t.v, B, Sk, Hkv, ts.v) || !make_tensor_map(&tm_do, t.dout, B, Sq, Hq, ts.dout, p.pack_log2) ||
      !make_tensor_map(&tm_dq, t.dq, B, Sq, Hq, ts.dq, p.pack_log2) || !make_tensor_map(&tm_dk, t.dk, B, Sk, Hkv, ts.dk) ||
      !make_tensor_map(&tm_dv, t.dv, B, Sk, Hkv, ts.dv))
    return ATTN_ERR_CUDA;

  uint8_t* ws = static_cast<uint8_t*>(workspace);
  float* neg_lse2 = reinterpret_cast<float*>(ws);
  float* neg_delta = reinterpret_cast<float*>(ws + bwd_stat_bytes(p));
  const size_t dq_bytes = bwd_part_bytes(p.qry_splits, B, p.Hq, p.n_qt), dk_bytes = bwd_part_bytes(p.key_splits, B, Hkv, p.n_kt);
  p.dq_part = reinterpret_cast<float*>(ws + 2 * bwd_stat_bytes(p));
  p.dk_part = p.dq_part + dq_bytes / sizeof(float);
  p.dv_part = p.dk_part + dk_bytes / sizeof(float);
  p.scale = scale;
  p.scale_log2 = scale * 1.4426950408889634f;
  p.neg_lse2 = neg_lse2;
  p.neg_delta = neg_delta;
  p.status = dev->status;
  cudaStream_t s = static_cast<cudaStream_t>(stream);
  const int padded = (p.n_qt * attn::kTile) >> p.pack_log2;  // query rows of a head, to whole tiles
  int heads_log2 = 0;  // heads of a block: up to 8, so that 256 rows are 32 positions or more
  while (heads_log2 < 3 && (2 << heads_log2) <= Hq) ++heads_log2;
  const int prep_rows = attn::bwd::kPrepThreads >> heads_log2;
  const long long prep_blocks = static_cast<long long>(B) * ((padded + prep_rows - 1) / prep_rows) *
                                ((Hq + (1 << heads_log2) - 1) >> heads_log2);
  const int cap = dev->sm_count * 8;
  attn::bwd::attn_bwd_prep_kernel<<<static_cast<int>(prep_blocks < cap ? prep_blocks : cap), attn::bwd::kPrepThreads, 0, s>>>(
      static_cast<const uint16_t*>(t.o), static_cast<const uint16_t*>(t.dout),
      attn::bwd::RowStrides{ts.o.b, ts.o.s, ts.o.h}, attn::bwd::RowStrides{ts.dout.b, ts.dout.s, ts.dout.h}, t.lse, t.dlse,
      neg_lse2, neg_delta, Hq, Sq, padded, p.pack_log2, heads_log2, static_cast<int>(prep_blocks));
  if (cudaGetLastError() != cudaSuccess) return ATTN_ERR_CUDA;
  const int grid = p.n_items;
  const auto kernel = fine_bwd(Sq, Sk) ? attn::bwd::attn_bwd_kernel<true> : attn::bwd::attn_bwd_kernel<false>;
  kernel<<<grid, attn::bwd::kBwdThreads, attn::bwd::kSmemBwdBytes, s>>>(tm_q, tm_k, tm_v, tm_do, tm_dq, tm_dk, tm_dv, p);
  if (cudaGetLastError() != cudaSuccess) return ATTN_ERR_CUDA;
  if (p.key_splits == 1 && p.qry_splits == 1) return ATTN_OK;
  attn::bwd::JoinParams jp = {};
  int n_out = 0;
  long long most = 0;
  auto join = [&](const float* part, void* out, Strides3 st3, int splits, int H, int S, int tiles, int pack_log2) {
    const long long padded_rows = static_cast<long long>(tiles) * attn::kTile;
    attn::bwd::JoinOut& j = jp.o[n_out++];
    j.part = part;
    j.out = static_cast<uint16_t*>(out);
    j.strides = attn::bwd::RowStrides{st3.b, st3.s, st3.h};
    j.splits = splits;
    j.H = H;
    j.S = S;
    j.padded = tiles * attn::kTile;
    j.pack_log2 = pack_log2;
    j.n_rows = static_cast<long long>(B) * H * S;
    j.part_stride = static_cast<long long>(B) * H * padded_rows * attn::kHeadDim;
    if (j.n_rows > most) most = j.n_rows;
  };
  if (p.qry_splits > 1) join(p.dq_part, t.dq, ts.dq, p.qry_splits, p.Hq, p.Sq, p.n_qt, p.pack_log2);
  if (p.key_splits > 1) {
    join(p.dk_part, t.dk, ts.dk, p.key_splits, Hkv, Sk, p.n_kt, 0);
    join(p.dv_part, t.dv, ts.dv, p.key_splits, Hkv, Sk, p.n_kt, 0);
  }
  long long join_blocks = (most + attn::bwd::kJoinThreads / 32 - 1) / (attn::bwd::kJoinThreads / 32);
  if (join_blocks > cap) join_blocks = cap;
  attn::bwd::attn_bwd_join_kernel<<<dim3(static_cast<unsigned>(join_blocks), n_out), attn::bwd::kJoinThreads, 0, s>>>(jp);
  return cudaGetLastError() == cudaSuccess ? ATTN_OK : ATTN_ERR_CUDA;
}

// The plan for sizes alone, checked as a call checks them.
attn_status_t bwd_plan_of(BwdParams* p, int B, int Hq, int Hkv, int Sq, int Sk, int D, int causal) {
  int dummy = 0;
  const attn_status_t st = check_args(&dummy, &dummy, &dummy, &dummy, nullptr, B, Hq, Hkv, Sq, Sk, D, causal, 1.0f, false);
  if (st != ATTN_OK) return st;
  return fill_bwd_plan(p, B, Hq, Hkv, Sq, Sk, causal) ? ATTN_OK : ATTN_ERR_UNSUPPORTED;
}

}  // namespace

extern "C" {

size_t attn_bwd_workspace_bytes(int B, int Hq, int Hkv, int Sq, int Sk, int D, int causal) {
  BwdParams p;
  return bwd_plan_of(&p, B, Hq, Hkv, Sq, Sk, D, causal) == ATTN_OK ? bwd_workspace_bytes(p) : 0;
}

attn_status_t attn_bwd_plan(int B, int Hq, int Hkv, int Sq, int Sk, int D, int causal, int* plan) {
  if (plan == nullptr) return ATTN_ERR_NULL;
  BwdParams p;
  const attn_status_t st = bwd_plan_of(&p, B, Hq, Hkv, Sq, Sk, D, causal);
  if (st != ATTN_OK) return st;
  const int out[] = {p.n_items, p.Hq, p.pack_log2, p.n_qt, p.n_kt, p.key_splits, p.qry_splits, p.run, p.run_extra};
  std::memcpy(plan, out, sizeof(out));
  return ATTN_OK;
}

attn_status_t attn_bwd_plan_item(int B, int Hq, int Hkv, int Sq, int Sk, int D, int causal, int w, int* item) {
  if (item == nullptr) return ATTN_ERR_NULL;
  BwdParams p;
  const attn_status_t st = bwd_plan_of(&p, B, Hq, Hkv, Sq, Sk, D, causal);
  if (st != ATTN_OK) return st;
  if (w < 0 || w >= p.n_items) return ATTN_ERR_SHAPE;
  const attn::bwd::BwdItem it = attn::bwd::decode_item(p, w);
  const int out[] = {it.keys, it.b, it.h, it.row0, it.first, it.per_head, it.t0, it.n, it.split};
  std::memcpy(item, out, sizeof(out));
  return ATTN_OK;
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
