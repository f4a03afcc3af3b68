// Host side of the C ABI for attention to an encoder's states and attention with a relative position bias: argument checks, sizes, dispatch.
#include <math.h>
#include "dense_attn.h"

using namespace da;

namespace {

const long long kMaxRows = 1LL << 29;   // sums of three of them stay below 2^31

inline bool misaligned(const void* p) { return ((uintptr_t)p & 15u) != 0; }
inline int hip_status(hipError_t e) { return e == hipSuccess ? DA_OK : DA_ERR_HIP; }

// An extent of 1 has no stride.  Outputs: no two elements at one place (each stride beyond all that the smaller ones reach).
int set_rows(const da_layout* l, long long per, int B, int heads, long long rows, int d, bool output, Rows* out) {
  if (!l || (l->stride_b == 0 && l->stride_h == 0 && l->stride_n == 0)) {
    out->sn = d; out->sh = rows * d; out->sb = heads * rows * d;
    return DA_OK;
  }
  const long long extent[3] = {B, heads, rows};
  const long long stride[3] = {l->stride_b, l->stride_h, l->stride_n};
  double reach = d;
  for (int i = 0; i < 3; ++i) {
    if (extent[i] == 1) continue;
    if (stride[i] < (i == 2 ? d : 1)) return DA_ERR_DIM;
    if (stride[i] % per) return DA_ERR_ALIGN;
    reach += (double)stride[i] * (double)(extent[i] - 1);
  }
  if (reach > 4.0e15) return DA_ERR_DIM;
  if (output) {
    long long beyond = d;
    bool done[3] = {extent[0] == 1, extent[1] == 1, extent[2] == 1};
    for (int n = 0; n < 3; ++n) {
      int at = -1;
      for (int i = 0; i < 3; ++i)
        if (!done[i] && (at < 0 || stride[i] < stride[at])) at = i;
      if (at < 0) break;
      if (stride[at] < beyond) return DA_ERR_DIM;
      beyond += stride[at] * (extent[at] - 1);
      done[at] = true;
    }
  }
  out->sb = extent[0] == 1 ? 0 : stride[0];
  out->sh = extent[1] == 1 ? 0 : stride[1];
  out->sn = extent[2] == 1 ? d : stride[2];
  return DA_OK;
}

int check_attn(const da_attn_problem* p, const da_rel_bias* bias, const da_attn_layouts* l, DenseGeo* out) {
  if (!p) return DA_ERR_NULL;
  if (p->B < 1 || p->H < 1 || p->Hk < 1 || p->N < 1 || p->M < 1 || p->d < 1 || p->H % p->Hk != 0) return DA_ERR_DIM;
  if (p->dtype != DA_F32 && p->dtype != DA_BF16) return DA_ERR_DIM;
  if (p->scale != 0.0 && !(p->scale >= 1.0e-30 && p->scale <= 1.0e30)) return DA_ERR_DIM;   // also rejects NaN
  DenseGeo q;
  q.B = p->B; q.H = p->H; q.Hk = p->Hk; q.group = p->H / p->Hk; q.N = p->N; q.M = p->M; q.d = p->d; q.dtype = p->dtype;
  if (q.N > kMaxRows || q.M > kMaxRows || (long long)q.group * q.N > kMaxRows || (long long)q.B * q.H > 2147483647LL) return DA_ERR_DIM;
  if ((double)q.B * q.H * ((double)q.N + q.M) * q.d > 4.0e15) return DA_ERR_DIM;
  const double scale = p->scale > 0.0 ? p->scale : 1.0 / sqrt((double)p->d);
  q.scale = (float)scale;
  q.c2 = (float)(scale * 1.4426950408889634);
  q.c2_lo = (float)(scale * 1.4426950408889634 - (double)q.c2);
  q.s_low = -(float)fmin(3.4e38, q.c2_lo == 0.f ? 3.4e38 : 3.4e38 / fabs((double)q.c2_lo));
  q.kv_len = nullptr;
  q.bias = 0; q.buckets = 0; q.q_pos = 0;
  q.rule = RelRule();
  if (bias) {
    if (!make_rel_rule(bias->buckets, bias->max_distance, bias->bidirectional, &q.rule)) return DA_ERR_DIM;
    if (bias->q_pos < -kMaxRows || bias->q_pos > kMaxRows) return DA_ERR_DIM;
    q.bias = 1; q.buckets = bias->buckets; q.q_pos = bias->q_pos;
  }
  const long long per = q.dtype == DA_BF16 ? 8 : 4;
  int st;
  if ((st = set_rows(l ? &l->q : nullptr, per, q.B, q.H, q.N, q.d, false, &q.q)) != DA_OK) return st;
  if ((st = set_rows(l ? &l->k : nullptr, per, q.B, q.Hk, q.M, q.d, false, &q.k)) != DA_OK) return st;
  if ((st = set_rows(l ? &l->v : nullptr, per, q.B, q.Hk, q.M, q.d, false, &q.v)) != DA_OK) return st;
  if ((st = set_rows(l ? &l->o : nullptr, per, q.B, q.H, q.N, q.d, true, &q.o)) != DA_OK) return st;
  if ((st = set_rows(l ? &l->dout : nullptr, per, q.B, q.H, q.N, q.d, false, &q.dout)) != DA_OK) return st;
  if ((st = set_rows(l ? &l->dq : nullptr, per, q.B, q.H, q.N, q.d, true, &q.dq)) != DA_OK) return st;
  if ((st = set_rows(l ? &l->dk : nullptr, per, q.B, q.Hk, q.M, q.d, true, &q.dk)) != DA_OK) return st;
  if ((st = set_rows(l ? &l->dv : nullptr, per, q.B, q.Hk, q.M, q.d, true, &q.dv)) != DA_OK) return st;
  if (q.d != 64 && q.d != 128) return DA_ERR_UNSUPPORTED;
  *out = q;
  return DA_OK;
}

int check_ws(const void* ws, size_t have, size_t need) {
  if (need == 0) return DA_OK;
  if (!ws) return DA_ERR_NULL;
  if (((uintptr_t)ws & 255u) != 0) return DA_ERR_ALIGN;
  return have < need ? DA_ERR_WORKSPACE : DA_OK;
}

int forward(const da_attn_problem* p, const da_rel_bias* bias, const da_attn_layouts* l, const void* Q, const void* K, const void* V,
            const void* table, const int32_t* kv_len, void* O, float* lse, void* ws, size_t ws_bytes, void* stream) {
  DenseGeo q;
  int st = check_attn(p, bias, l, &q);
  if (st != DA_OK) return st;
  if (!Q || !K || !V || !O || (bias && !table)) return DA_ERR_NULL;
  if (misaligned(Q) || misaligned(K) || misaligned(V) || misaligned(O) || misaligned(table) || misaligned(kv_len) || misaligned(lse))
    return DA_ERR_ALIGN;
  if ((st = check_ws(ws, ws_bytes, dense_fwd_workspace(q))) != DA_OK) return st;
  q.kv_len = kv_len;
  return hip_status(launch_dense_fwd(q, Q, K, V, table, O, lse, ws, (hipStream_t)stream));
}

int backward(const da_attn_problem* p, const da_rel_bias* bias, const da_attn_layouts* l, const void* Q, const void* K, const void* V,
             const void* table, const int32_t* kv_len, const void* O, const float* lse, const void* dO, void* dQ, void* dK, void* dV,
             void* dtable, void* ws, size_t ws_bytes, void* stream) {
  DenseGeo q;
  int st = check_attn(p, bias, l, &q);
  if (st != DA_OK) return st;
  if (!Q || !K || !V || !O || !lse || !dO || !dQ || !dK || !dV || (bias && (!table || !dtable))) return DA_ERR_NULL;
  if (misaligned(Q) || misaligned(K) || misaligned(V) || misaligned(O) || misaligned(lse) || misaligned(dO) || misaligned(dQ) ||
      misaligned(dK) || misaligned(dV) || misaligned(table) || misaligned(dtable) || misaligned(kv_len))
    return DA_ERR_ALIGN;
  if ((st = check_ws(ws, ws_bytes, dense_bwd_workspace(q))) != DA_OK) return st;
  q.kv_len = kv_len;
  return hip_status(launch_dense_bwd(q, Q, K, V, table, O, lse, dO, dQ, dK, dV, dtable, ws, (hipStream_t)stream));
}

}  // namespace

extern "C" {

int da_attn_sizes(const da_attn_problem* p, const da_rel_bias* bias, da_attn_dims* out) {
  if (!out) return DA_ERR_NULL;
  DenseGeo q;
  int st = check_attn(p, bias, nullptr, &q);
  if (st != DA_OK) return st;
  out->forward_ws = dense_fwd_workspace(q);
  out->backward_ws = dense_bwd_workspace(q);
  return DA_OK;
}

int da_cross_attn(const da_attn_problem* p, const da_attn_layouts* layouts, const void* Q, const void* K, const void* V,
                  const int32_t* kv_len, void* O, float* lse, void* ws, size_t ws_bytes, void* stream) {
  return forward(p, nullptr, layouts, Q, K, V, nullptr, kv_len, O, lse, ws, ws_bytes, stream);
}

int da_cross_attn_bwd(const da_attn_problem* p, const da_attn_layouts* layouts, const void* Q, const void* K, const void* V,
                      const int32_t* kv_len, const void* O, const float* lse, const void* dO, void* dQ, void* dK, void* dV, void* ws,
                      size_t ws_bytes, void* stream) {
  return backward(p, nullptr, layouts, Q, K, V, nullptr, kv_len, O, lse, dO, dQ, dK, dV, nullptr, ws, ws_bytes, stream);
}

int da_bias_attn(const da_attn_problem* p, const da_rel_bias* bias, const da_attn_layouts* layouts, const void* Q, const void* K,
                 const void* V, const void* table, const int32_t* kv_len, void* O, float* lse, void* ws, size_t ws_bytes, void* stream) {
  if (!bias) return DA_ERR_NULL;
  return forward(p, bias, layouts, Q, K, V, table, kv_len, O, lse, ws, ws_bytes, stream);
}

int da_bias_attn_bwd(const da_attn_problem* p, const da_rel_bias* bias, const da_attn_layouts* layouts, const void* Q, const void* K,
                     const void* V, const void* table, const int32_t* kv_len, const void* O, const float* lse, const void* dO, void* dQ,
                     void* dK, void* dV, void* dtable, void* ws, size_t ws_bytes, void* stream) {
  if (!bias) return DA_ERR_NULL;
  return backward(p, bias, layouts, Q, K, V, table, kv_len, O, lse, dO, dQ, dK, dV, dtable, ws, ws_bytes, stream);
}

}  // extern "C"
