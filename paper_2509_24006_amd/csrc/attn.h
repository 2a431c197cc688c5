// Softmax attention of a transformer's other layers (sla_attn_forward, sla_attn_backward): what its translation
// units share.
#ifndef SLA_ATTN_H_
#define SLA_ATTN_H_

#include "../../include/sla.h"
#include "sla_internal.h"

namespace sla {

// A caller's tensor: element (b, h, n, c) at p[b sb + h sh + n sn + c].
struct View {
  void* p;
  long long sb, sh;
  int sn;
};

// Buckets of the position bias; n_borders < 0: no bias.  Distances from `far` on share the last bucket of their side.
struct Buckets {
  int n_borders, two_sided, far;
  int borders[SLA_ATTN_BORDERS];
};

// One call.  Query head h reads K, V head h / G.
struct Attn {
  int B, H, Hkv, G, Nq, Nk, Np, d, dtype, causal, q_pos, q_from_end, table16;
  float scale;
  Buckets bias;
  const void* table;
  const int32_t *q_len, *k_len;
  View Q, K, V, Kp, Vp, O;   // (Kp, Vp: no batch stride)
  float* L;
  bool has_bias() const { return bias.n_borders >= 0; }
};
struct AttnGrads {
  View dO, dQ, dK, dV;
  void* dtable;
};

// Queries, own keys and position of the first query of one sequence.  A length outside its tensor is cut to it.
struct Seq {
  int nq, nk, pos;
};
__device__ __forceinline__ Seq seq_of(const Attn& a, int b) {
  Seq s;
  s.nq = a.q_len ? min(max(a.q_len[b], 0), a.Nq) : a.Nq;
  s.nk = a.k_len ? min(max(a.k_len[b], 0), a.Nk) : a.Nk;
  s.pos = a.q_pos + (a.q_from_end ? a.Np + s.nk : 0);
  return s;
}

// bucket of a key at distance rel = key position - query position
__device__ __forceinline__ int bucket_of(const Buckets& bk, int rel) {
  const int n = bk.two_sided ? abs(rel) : max(-rel, 0);
  int u = 0;
  for (int i = 0; i < bk.n_borders; ++i) u += n >= bk.borders[i];
  return bk.two_sided && rel > 0 ? u + bk.n_borders + 1 : u;
}
__host__ __device__ inline int bucket_count(const Buckets& bk) { return (bk.n_borders + 1) * (bk.two_sided ? 2 : 1); }

__device__ __forceinline__ float table_at(const Attn& a, int bucket, int h) {
  const size_t i = (size_t)bucket * a.H + h;
  return a.table16 ? to_f32(reinterpret_cast<const __hip_bfloat16*>(a.table)[i]) : reinterpret_cast<const float*>(a.table)[i];
}

size_t attn_forward_ws(const Attn& a);
size_t attn_backward_ws(const Attn& a);
bool attn_forward_fits(const Attn& a);   // whether offsets inside the tensors fit the kernels' 32 bits
hipError_t attn_forward(const Attn& a, char* ws, hipStream_t st);
hipError_t attn_backward(const Attn& a, const AttnGrads& g, char* ws, hipStream_t st);

// the backward pass by storage type
hipError_t attn_backward_f32(const Attn& a, const AttnGrads& g, char* ws, hipStream_t st);
hipError_t attn_backward_bf16(const Attn& a, const AttnGrads& g, char* ws, hipStream_t st);

}  // namespace sla
#endif
