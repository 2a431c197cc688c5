// Softmax attention of a transformer's other layers (sla_attn_forward, sla_attn_backward): what its translation
// units share.
#ifndef SLA_ATTN_H_
#define SLA_ATTN_H_

#include "../../include/sla.h"
#include "mfma_common.h"

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

// A bias by distance lies in LDS for the distances -far .. far and a margin on both sides: a tile of 32 keys and 32
// neighbouring queries that reaches into -far .. far reaches no further than 62 beyond, so that a value is found at its
// distance without a comparison.
constexpr int kBiasPad = 64;
__host__ __device__ inline int bias_width(int far) { return 2 * (far + kBiasPad) + 1; }

// An entry of -1e30 and below is a mask, a type's lowest value among them: beside it a score has no bits left, and its
// logarithm to base 2 may not be finite.
__device__ __forceinline__ float table_at(const Attn& a, int bucket, int h) {
  const size_t i = (size_t)bucket * a.H + h;
  const float x = a.table16 ? to_f32(reinterpret_cast<const __hip_bfloat16*>(a.table)[i]) : reinterpret_cast<const float*>(a.table)[i];
  return x <= -1e30f ? -INFINITY : x;
}

// Which head and tile a workgroup of a launch over BH heads of nb tiles owns.  Workgroups are dealt to the 8 XCDs (each with
// its own L2) round robin, and what a tile reads beside its own rows is read by all tiles of its head and group.  Where
// the heads can be dealt out evenly, all with the same work, an XCD takes whole heads: one after the other, or under a causal
// mask, where a tile's work falls with its index, their tiles in turn, the longest first.  Else the XCDs share every head:
// in ranges (block_of) or, causal, tile by tile across all heads, the longest first.
// (Forward / query side / key side, us, ranges of every head -> whole heads: 256 heads x 16 tiles, d = 64, 120 / 139 / 195
// -> 113 / 134 / 187; causal 32 x 64 over 8 K, V heads, d = 128, 193 / 254 / 306 -> 159 / 212 / 300; of two sequences of
// different lengths, 24 x 512, 239 / 340 / 371 -> 296 / 391 / 415, hence the condition.  Causal 12 x 79 with a bias, d = 64:
// ranges 103, tile by tile 84.)
struct TileOf {
  int bh, i;   // i < 0: a padding workgroup
};
struct TileMap {
  int BH, nb, whole, falling;
  __device__ __forceinline__ TileOf at(int index) const {
    if (whole) {
      const int x = index & 7, m = index >> 3, hp = BH >> 3;
      return falling ? TileOf{x * hp + m % hp, m / hp} : TileOf{x * hp + m / nb, m % nb};
    }
    if (falling) return TileOf{index % BH, index / BH};
    const int row = block_row(nb), y = index / row;
    const BlockOf o = block_of(y, index - y * row, BH, nb);
    return TileOf{o.bh, o.i};
  }
  int blocks() const { return nb == 0 ? 0 : whole || falling ? BH * nb : block_row(nb) * block_rows(BH, nb); }
};
inline TileMap tile_map(const Attn& a, int BH, int nb) { return TileMap{BH, nb, BH % 8 == 0 && !a.q_len && !a.k_len, a.causal}; }

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
