// Host side of attn_qk_norm_rope and its gradient.  Included by attn_api.cu.
#pragma once

namespace {

using attn::rope::RopeParams;

struct RopeArgs {
  const void *q, *k, *q_weight, *k_weight;
  int weight_type;
  const float *cos_table, *sin_table;
  const void* positions;
  int position_type;
  const long long* position_strides;
  int B, S, Hq, Hkv, D, rot_dim, n_positions, interleaved;
  float eps;
};

// Strides of one tensor: null means contiguous.
attn_status_t rope_strides(const long long* s, int S, int H, attn::rope::RopeStrides* out) {
  if (s == nullptr) {
    const Strides3 c = contiguous_strides(S, H);
    *out = attn::rope::RopeStrides{c.b, c.s, c.h};
    return ATTN_OK;
  }
  const attn_status_t st = check_strides(s);
  if (st == ATTN_OK) *out = attn::rope::RopeStrides{s[0], s[1], s[2]};
  return st;
}

bool misaligned(const void* p, uintptr_t mask) { return (reinterpret_cast<uintptr_t>(p) & mask) != 0; }

bool same_strides(const attn::rope::RopeStrides& a, const attn::rope::RopeStrides& b) {
  return a.b == b.b && a.s == b.s && a.h == b.h;
}

// Checks the arguments both directions share and fills the parameters from them (strides: q, k).
attn_status_t rope_params(const RopeArgs& a, const long long* const* in_strides, RopeParams* p) {
  std::memset(p, 0, sizeof(*p));
  if (a.q == nullptr || a.k == nullptr || a.cos_table == nullptr || a.sin_table == nullptr) return ATTN_ERR_NULL;
  if (a.B <= 0 || a.S <= 0 || a.Hq <= 0 || a.Hkv <= 0 || a.D <= 0 || a.n_positions <= 0) return ATTN_ERR_SHAPE;
  if (a.positions == nullptr && a.S > a.n_positions) return ATTN_ERR_SHAPE;
  if (a.D != attn::rope::kRopeDim) return ATTN_ERR_UNSUPPORTED;
  if (a.rot_dim < 16 || a.rot_dim > attn::rope::kRopeDim || a.rot_dim % 16 != 0) return ATTN_ERR_UNSUPPORTED;
  if (!std::isfinite(a.eps) || !(a.eps > 0.f)) return ATTN_ERR_UNSUPPORTED;
  if (a.weight_type < 0 || a.weight_type > 1 || a.position_type < 0 || a.position_type > 1) return ATTN_ERR_UNSUPPORTED;
  if (misaligned(a.q, 15) || misaligned(a.k, 15) || misaligned(a.q_weight, 15) || misaligned(a.k_weight, 15) ||
      misaligned(a.cos_table, 15) || misaligned(a.sin_table, 15) || misaligned(a.positions, a.position_type ? 7 : 3))
    return ATTN_ERR_ALIGN;
  p->x[0] = static_cast<const uint16_t*>(a.q);
  p->x[1] = static_cast<const uint16_t*>(a.k);
  p->heads[0] = a.Hq;
  p->heads[1] = a.Hkv;
  for (int t = 0; t < 2; ++t) {
    const attn_status_t st = rope_strides(in_strides[t], a.S, p->heads[t], &p->sx[t]);
    if (st != ATTN_OK) return st;
    p->units[t] = (p->heads[t] - 1) / attn::rope::kUnitRows + 1;
  }
  p->w[0] = a.q_weight;
  p->w[1] = a.k_weight;
  p->w_bf16 = a.weight_type;
  p->cos_tab = a.cos_table;
  p->sin_tab = a.sin_table;
  p->positions = a.positions;
  p->positions_64 = a.position_type;
  p->pos_b = a.position_strides != nullptr ? a.position_strides[0] : a.S;
  p->pos_s = a.position_strides != nullptr ? a.position_strides[1] : 1;
  p->n_positions = a.n_positions;
  p->S = a.S;
  p->rot = a.rot_dim;
  p->eps = a.eps;
  // the kernels count units in 32 bits (2^30 units are 2 TB of rows)
  if (static_cast<long long>(a.B) * a.S > 0x3fffffffLL / (static_cast<long long>(p->units[0]) + p->units[1])) return ATTN_ERR_UNSUPPORTED;
  for (int t = 0; t < 2; ++t) p->n_units[t] = static_cast<uint32_t>(a.B) * a.S * p->units[t];
  return ATTN_OK;
}

// An output, which may be one of `in` itself (same address and strides).
attn_status_t rope_output(void* out, const long long* strides, const RopeParams& p, int t, RopeParams* dst) {
  if (out == nullptr) return ATTN_ERR_NULL;
  if (misaligned(out, 15)) return ATTN_ERR_ALIGN;
  const attn_status_t st = rope_strides(strides, p.S, p.heads[t], &dst->sout[t]);
  if (st != ATTN_OK) return st;
  dst->out[t] = static_cast<uint16_t*>(out);
  const int other = 1 - t;  // in the place of the other tensor's data
  if (out == p.x[other] || out == p.dy[other] || out == dst->out[other]) return ATTN_ERR_UNSUPPORTED;
  if ((out == p.x[t] && !same_strides(dst->sout[t], p.sx[t])) || (out == p.dy[t] && !same_strides(dst->sout[t], p.sdy[t])))
    return ATTN_ERR_UNSUPPORTED;
  return ATTN_OK;
}

int rope_grid(const RopeParams& p, int cap) {
  const int ctas = static_cast<int>((p.n_units[0] + p.n_units[1] + attn::rope::kRopeWarps - 1) / attn::rope::kRopeWarps);
  return ctas < cap ? ctas : cap;
}

}  // namespace

extern "C" {

attn_status_t attn_qk_norm_rope(const void* q, const void* k, const void* q_weight, const void* k_weight, int weight_type,
                                const float* cos_table, const float* sin_table, const void* positions, int position_type,
                                const long long* position_strides, void* q_out, void* k_out, int B, int S, int Hq, int Hkv,
                                int D, int rot_dim, int n_positions, int interleaved, float eps, const long long* q_strides,
                                const long long* k_strides, const long long* q_out_strides, const long long* k_out_strides,
                                void* stream) {
  RopeParams p;
  const long long* in[2] = {q_strides, k_strides};
  attn_status_t st = rope_params(RopeArgs{q, k, q_weight, k_weight, weight_type, cos_table, sin_table, positions, position_type,
                                          position_strides, B, S, Hq, Hkv, D, rot_dim, n_positions, interleaved, eps},
                                 in, &p);
  if (st == ATTN_OK) st = rope_output(q_out, q_out_strides, p, 0, &p);
  if (st == ATTN_OK) st = rope_output(k_out, k_out_strides, p, 1, &p);
  if (st != ATTN_OK) return st;
  DeviceState* dev = device_state(&st);
  if (dev == nullptr) return st;
  const int grid = rope_grid(p, dev->sm_count * 3);  // as many CTAs as are resident
  cudaStream_t s = static_cast<cudaStream_t>(stream);
  if (interleaved) {
    attn::rope::qk_norm_rope_kernel<true><<<grid, attn::rope::kRopeThreads, 0, s>>>(p);
  } else {
    attn::rope::qk_norm_rope_kernel<false><<<grid, attn::rope::kRopeThreads, 0, s>>>(p);
  }
  return cudaGetLastError() == cudaSuccess ? ATTN_OK : ATTN_ERR_CUDA;
}

size_t attn_qk_norm_rope_bwd_workspace_bytes(void) {
  return static_cast<size_t>(attn::rope::kDwCtas) * 2 * attn::rope::kRopeDim * sizeof(float);
}

attn_status_t attn_qk_norm_rope_bwd(const void* dq_out, const void* dk_out, const void* q, const void* k, const void* q_weight,
                                    const void* k_weight, int weight_type, const float* cos_table, const float* sin_table,
                                    const void* positions, int position_type, const long long* position_strides, void* dq,
                                    void* dk, float* dq_weight, float* dk_weight, int B, int S, int Hq, int Hkv, int D,
                                    int rot_dim, int n_positions, int interleaved, float eps, const long long* dq_out_strides,
                                    const long long* dk_out_strides, const long long* q_strides, const long long* k_strides,
                                    const long long* dq_strides, const long long* dk_strides, void* workspace,
                                    size_t workspace_bytes, void* stream) {
  if (dq_out == nullptr || dk_out == nullptr) return ATTN_ERR_NULL;
  RopeParams p;
  const long long* in[2] = {q_strides, k_strides};
  attn_status_t st = rope_params(RopeArgs{q, k, q_weight, k_weight, weight_type, cos_table, sin_table, positions, position_type,
                                          position_strides, B, S, Hq, Hkv, D, rot_dim, n_positions, interleaved, eps},
                                 in, &p);
  if (st != ATTN_OK) return st;
  if (misaligned(dq_out, 15) || misaligned(dk_out, 15) || misaligned(dq_weight, 3) || misaligned(dk_weight, 3))
    return ATTN_ERR_ALIGN;
  p.dy[0] = static_cast<const uint16_t*>(dq_out);
  p.dy[1] = static_cast<const uint16_t*>(dk_out);
  st = rope_strides(dq_out_strides, S, Hq, &p.sdy[0]);
  if (st == ATTN_OK) st = rope_strides(dk_out_strides, S, Hkv, &p.sdy[1]);
  if (st == ATTN_OK) st = rope_output(dq, dq_strides, p, 0, &p);
  if (st == ATTN_OK) st = rope_output(dk, dk_strides, p, 1, &p);
  if (st != ATTN_OK) return st;
  const bool want_dw = dq_weight != nullptr || dk_weight != nullptr;
  if (want_dw) {
    if (workspace == nullptr) return ATTN_ERR_NULL;
    if (misaligned(workspace, 15)) return ATTN_ERR_ALIGN;
    if (workspace_bytes < attn_qk_norm_rope_bwd_workspace_bytes()) return ATTN_ERR_TOO_LARGE;
    p.partials = static_cast<float*>(workspace);
  }
  DeviceState* dev = device_state(&st);
  if (dev == nullptr) return st;
  const int grid = rope_grid(p, attn::rope::kDwCtas);
  cudaStream_t s = static_cast<cudaStream_t>(stream);
  if (interleaved) {
    attn::rope::qk_norm_rope_bwd_kernel<true><<<grid, attn::rope::kRopeThreads, 0, s>>>(p);
  } else {
    attn::rope::qk_norm_rope_bwd_kernel<false><<<grid, attn::rope::kRopeThreads, 0, s>>>(p);
  }
  if (cudaGetLastError() != cudaSuccess) return ATTN_ERR_CUDA;
  if (want_dw) {
    attn::rope::qk_norm_rope_dw_kernel<<<2 * attn::rope::kRopeDim / 8, 256, 0, s>>>(p.partials, grid, dq_weight, dk_weight);
    if (cudaGetLastError() != cudaSuccess) return ATTN_ERR_CUDA;
  }
  return ATTN_OK;
}

}  // extern "C"
