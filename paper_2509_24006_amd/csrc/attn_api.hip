// C ABI of the softmax attention (sla_attn_*): argument checks.  Host code only.
#include <math.h>

#include "attn.h"

using namespace sla;

namespace {

constexpr int kMaxRows = 1 << 28;          // positions and their differences stay far inside an int
constexpr long long kMaxPitch = 1 << 24;   // bytes between rows: offsets inside a tile of 64 stay below 2^30
constexpr float kMinScale = 1e-20f;        // L / scale stays a float, and -1e30 scale (an empty row) is far below any exponent

inline bool off(const void* p, size_t a) { return ((uintptr_t)p & (a - 1)) != 0; }

int make_attn(const sla_attn_params* p, Attn* a) {
  if (!p) return SLA_EINVAL;
  if (p->B <= 0 || p->H <= 0 || p->Hkv <= 0 || p->Nq <= 0 || p->Nk < 0 || p->Np < 0 || p->H % p->Hkv) return SLA_EINVAL;
  if (!(p->scale > 0.0f) || !isfinite(p->scale)) return SLA_EINVAL;
  if (p->scale < kMinScale || p->scale > 1.0f / kMinScale) return SLA_EUNSUPPORTED;
  if (p->d != 64 && p->d != 128) return SLA_EUNSUPPORTED;
  if (p->dtype != SLA_F32 && p->dtype != SLA_BF16) return SLA_EUNSUPPORTED;
  if (p->table_dtype != SLA_F32 && p->table_dtype != SLA_BF16) return SLA_EUNSUPPORTED;
  if ((long long)p->B * p->H > 65535) return SLA_EUNSUPPORTED;
  if (p->Nq > kMaxRows || p->Nk > kMaxRows || p->Np > kMaxRows || p->q_pos > kMaxRows || p->q_pos < -kMaxRows)
    return SLA_EUNSUPPORTED;
  if ((long long)p->B * p->H * ((p->Nq + 63) / 64) >= (1 << 28) || (long long)p->B * p->Hkv * ((p->Nk + 63) / 64) >= (1 << 28))
    return SLA_EUNSUPPORTED;   // workgroups of a launch
  a->B = p->B; a->H = p->H; a->Hkv = p->Hkv; a->G = p->H / p->Hkv;
  a->Nq = p->Nq; a->Nk = p->Nk; a->Np = p->Np;
  a->d = p->d;
  a->dtype = p->dtype;
  a->causal = p->causal != 0;
  a->q_pos = p->q_pos;
  a->q_from_end = p->q_from_end != 0;
  a->table16 = p->table_dtype == SLA_BF16;
  a->scale = p->scale;
  const sla_buckets& bk = p->buckets;
  const int sides = bk.two_sided ? 2 : 1, nb = bk.n_buckets;
  if (nb < 0 || nb % sides || nb / sides > SLA_ATTN_BORDERS + 1) return SLA_EINVAL;
  a->bias.n_borders = nb / sides - 1;   // -1: no bias
  a->bias.two_sided = sides == 2;
  a->bias.far = 1;
  for (int i = 0; i < a->bias.n_borders; ++i) {
    const int v = bk.borders[i];
    if (v < (i ? bk.borders[i - 1] : 1) || v > SLA_ATTN_MAX_DISTANCE) return SLA_EINVAL;
    a->bias.borders[i] = v;
    a->bias.far = v;
  }
  return SLA_OK;
}

// one tensor of `heads` heads of n rows for each of `batch` sequences
int view(const Attn& a, const sla_tensor* t, int batch, int heads, int n, View* v) {
  if (!t) return SLA_EINVAL;
  const long long esz = a.dtype == SLA_F32 ? 4 : 2, q = 16 / esz;
  const long long sb = batch > 1 ? t->stride_b : 0, sh = heads > 1 ? t->stride_h : 0, sn = n > 1 ? t->stride_n : a.d;
  if (sb < 0 || sh < 0 || sn < a.d || sb % q || sh % q || sn % q) return SLA_EINVAL;
  if (n > 0 && (!t->data || off(t->data, 16))) return SLA_EINVAL;
  if (sn * esz > kMaxPitch) return SLA_EUNSUPPORTED;
  *v = View{t->data, sb, sh, (int)sn};
  return SLA_OK;
}

#define ATTN_VIEW(t, batch, heads, n, v)                              \
  do {                                                                \
    const int rc_ = view(a, t, batch, heads, n, v);                   \
    if (rc_ != SLA_OK) return rc_;                                    \
  } while (0)

int lengths_and_table(Attn& a, const void* table, const int32_t* q_len, const int32_t* k_len) {
  if (off(q_len, 4) || off(k_len, 4)) return SLA_EINVAL;
  if ((table != nullptr) != a.has_bias() || off(table, a.table16 ? 2 : 4)) return SLA_EINVAL;
  a.table = table;
  a.q_len = q_len;
  a.k_len = k_len;
  return SLA_OK;
}

int hip_status(hipError_t e) { return e == hipSuccess ? SLA_OK : SLA_EHIP; }

}  // namespace

extern "C" {

int sla_attn_sizes(const sla_attn_params* p, uint64_t* forward_bytes, uint64_t* backward_bytes) {
  Attn a = {};
  if (!forward_bytes || !backward_bytes) return SLA_EINVAL;
  const int rc = make_attn(p, &a);
  if (rc != SLA_OK) return rc;
  *forward_bytes = attn_forward_ws(a);
  *backward_bytes = a.Np ? 0 : attn_backward_ws(a);
  return SLA_OK;
}

int sla_attn_forward(const sla_attn_params* p, const sla_tensor* Q, const sla_tensor* K, const sla_tensor* V,
                     const sla_tensor* Kp, const sla_tensor* Vp, const void* table, const int32_t* q_len,
                     const int32_t* k_len, const sla_tensor* O, float* L, void* workspace, size_t workspace_bytes,
                     void* stream) {
  Attn a = {};
  int rc = make_attn(p, &a);
  if (rc != SLA_OK) return rc;
  ATTN_VIEW(Q, a.B, a.H, a.Nq, &a.Q);
  ATTN_VIEW(K, a.B, a.Hkv, a.Nk, &a.K);
  ATTN_VIEW(V, a.B, a.Hkv, a.Nk, &a.V);
  ATTN_VIEW(O, a.B, a.H, a.Nq, &a.O);
  if (a.Np) {
    ATTN_VIEW(Kp, 1, a.Hkv, a.Np, &a.Kp);
    ATTN_VIEW(Vp, 1, a.Hkv, a.Np, &a.Vp);
  }
  rc = lengths_and_table(a, table, q_len, k_len);
  if (rc != SLA_OK) return rc;
  if (off(L, 4) || off(workspace, 16)) return SLA_EINVAL;
  a.L = L;
  if (!attn_forward_fits(a)) return SLA_EUNSUPPORTED;
  const size_t need = attn_forward_ws(a);
  if (need && !workspace) return SLA_EINVAL;
  if (workspace_bytes < need) return SLA_ENOSPACE;
  return hip_status(attn_forward(a, (char*)workspace, (hipStream_t)stream));
}

int sla_attn_backward(const sla_attn_params* p, const sla_tensor* Q, const sla_tensor* K, const sla_tensor* V,
                      const sla_tensor* O, const sla_tensor* dO, const float* L, const void* table,
                      const int32_t* q_len, const int32_t* k_len, const sla_tensor* dQ, const sla_tensor* dK,
                      const sla_tensor* dV, void* dtable, void* workspace, size_t workspace_bytes, void* stream) {
  Attn a = {};
  AttnGrads g = {};
  int rc = make_attn(p, &a);
  if (rc != SLA_OK) return rc;
  if (a.Np) return SLA_EUNSUPPORTED;
  ATTN_VIEW(Q, a.B, a.H, a.Nq, &a.Q);
  ATTN_VIEW(K, a.B, a.Hkv, a.Nk, &a.K);
  ATTN_VIEW(V, a.B, a.Hkv, a.Nk, &a.V);
  ATTN_VIEW(O, a.B, a.H, a.Nq, &a.O);
  ATTN_VIEW(dO, a.B, a.H, a.Nq, &g.dO);
  ATTN_VIEW(dQ, a.B, a.H, a.Nq, &g.dQ);
  ATTN_VIEW(dK, a.B, a.Hkv, a.Nk, &g.dK);
  ATTN_VIEW(dV, a.B, a.Hkv, a.Nk, &g.dV);
  const long long esz = a.dtype == SLA_F32 ? 4 : 2;
  for (const View* v : {&a.Q, &a.O, &g.dO, &g.dQ})
    if (a.Nq * (long long)v->sn * esz >= (1ll << 31)) return SLA_EUNSUPPORTED;
  for (const View* v : {&a.K, &a.V, &g.dK, &g.dV})
    if (a.Nk * (long long)v->sn * esz >= (1ll << 31)) return SLA_EUNSUPPORTED;
  rc = lengths_and_table(a, table, q_len, k_len);
  if (rc != SLA_OK) return rc;
  if (!L || off(L, 4) || off(workspace, 16)) return SLA_EINVAL;
  if (dtable && (!a.has_bias() || off(dtable, a.table16 ? 2 : 4))) return SLA_EINVAL;
  a.L = const_cast<float*>(L);
  g.dtable = dtable;
  const size_t need = attn_backward_ws(a);
  if (need && !workspace) return SLA_EINVAL;
  if (workspace_bytes < need) return SLA_ENOSPACE;
  return hip_status(attn_backward(a, g, (char*)workspace, (hipStream_t)stream));
}

}  // extern "C"
