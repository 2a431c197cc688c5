// What the two backward paths of the softmax attention share: the cut of the key side, and the bias table's gradient.
#ifndef SLA_ATTN_BWD_H_
#define SLA_ATTN_BWD_H_

#include "attn.h"

namespace sla {

// The steps of a key tile run over the query tiles from the first that sees it, head by head.  Above `piece` of them they
// are cut: piece p leaves its sums in slot unit * pieces + p, and a second launch adds them.
struct KeyPlan {
  int tiles, pieces, piece;   // key tiles; most pieces of one, steps in a piece
  int quarters;               // float: workgroups per key tile
  TileMap map;                // (bf16)
  int blocks;                 // workgroups of one piece index
  float* part;                // [B Hkv tiles][pieces] slots of 2 x 64 x d floats
};
struct KeySteps {
  int i0, per_head, total;    // first query tile, tiles per head, steps
};
__device__ __forceinline__ KeySteps key_steps(const Attn& a, const Seq& s, int j) {
  KeySteps k;
  k.i0 = a.causal ? max(0, j * kBlk - s.pos) / kBlk : 0;
  k.per_head = j * kBlk < s.nk ? max(0, (s.nq + kBlk - 1) / kBlk - k.i0) : 0;
  k.total = k.per_head * a.G;
  return k;
}

// A softmax over one key is 1 whatever the score is: nothing flows back through it.  What the formula P (dP - D) leaves of
// such a row is a rounding, so the query side takes P = 0 there and the key side of a sequence of one key drops dK.
__device__ __forceinline__ float dk_scale(const Attn& a, const Seq& s) { return s.nk == 1 ? 0.0f : a.scale; }

struct BwdPlan {
  KeyPlan key;
  int shares;          // float: workgroups per query tile
  int qparts;          // workgroups of the query side per head
  TileMap map;         // of the query side
  float* stat;         // what the key side needs of every query: float D, bf16 L and D as an operand (16 bytes)
  float* tpart;        // parts of the table's gradient, [B][H][qparts][buckets]
  size_t bytes;
};
BwdPlan attn_bwd_plan(const Attn& a, char* ws);

// One workgroup's part of its head's column of the table's gradient.  dist: NA arrays of sums by distance (`width` floats
// each) in LDS, behind them room for eight floats; sumL, sumR: this lane's sums at distances of -far and less, far
// and more.  Called by the whole workgroup, behind its last addition.
template <int NA>
__device__ __forceinline__ void table_part(const Attn& a, float* dist, int width, float sumL, float sumR, float* out) {
  const int tid = threadIdx.x, w = tid >> 6, far = a.bias.far;
  float* const ends = dist + NA * width;   // left sums of the waves, right sums
#pragma unroll
  for (int o = 32; o; o >>= 1) {
    sumL += __shfl_xor(sumL, o);
    sumR += __shfl_xor(sumR, o);
  }
  if ((tid & 63) == 0) {
    ends[w] = sumL;
    ends[4 + w] = sumR;
  }
  __syncthreads();
  for (int x = tid; x < width; x += 256) {
    float t = dist[x];
#pragma unroll
    for (int e = 1; e < NA; ++e) t += dist[e * width + x];
    dist[x] = t;
  }
  __syncthreads();
  // bucket by bucket, a power of two of neighbouring lanes each: the distances [n0, n1) of a side, the last bucket with the
  // far sums
  const int nb = bucket_count(a.bias), side = a.bias.n_borders + 1;
  int share = 64;
  while (share * nb > 256) share >>= 1;
  const int u = tid / share, sub = tid & (share - 1);
  float t = 0.0f;
  if (u < nb) {
    const bool right = u >= side, first = u == 0 && !a.bias.two_sided;   // (one-sided: bucket 0 has the keys behind the query too)
    const int v = right ? u - side : u;
    const int n0 = v ? a.bias.borders[v - 1] : 0, n1 = v < side - 1 ? a.bias.borders[v] : far;
    for (int x = (right ? max(n0, 1) : n0) + sub; x < n1; x += share) t += dist[right ? far + x : far - x];
    if (first)
      for (int x = 1 + sub; x < far; x += share) t += dist[far + x];
    const float el = (ends[0] + ends[1]) + (ends[2] + ends[3]), er = (ends[4] + ends[5]) + (ends[6] + ends[7]);
    if (sub == 0) t += (v == side - 1 ? (right ? er : el) : 0.0f) + (first ? er : 0.0f);
  }
  for (int o = share >> 1; o; o >>= 1) t += __shfl_xor(t, o);
  if (u < nb && sub == 0) out[u] = t;
}

// The gradient of one head's column of the table: the sum of the parts [b][tile], in an order fixed by their number.
__device__ __forceinline__ void table_sum(const Attn& a, const AttnGrads& gr, const float* tpart, int tiles, int h,
                                          unsigned char* smem) {
  float* red = reinterpret_cast<float*>(smem);   // [slice][nb]
  const int nb = bucket_count(a.bias), slices = 256 / nb, u = threadIdx.x % nb, sl = threadIdx.x / nb;
  const int total = a.B * tiles;
  if (sl < slices) {
    float s = 0.0f;
#pragma unroll 4
    for (int x = sl; x < total; x += slices) {
      const int b = x / tiles, t = x - b * tiles;
      s += tpart[(((size_t)b * a.H + h) * tiles + t) * nb + u];
    }
    red[sl * nb + u] = s;
  }
  __syncthreads();
  if ((int)threadIdx.x < nb) {
    float s = 0.0f;
    for (int x = 0; x < slices; ++x) s += red[x * nb + threadIdx.x];
    const size_t at = (size_t)threadIdx.x * a.H + h;
    if (a.table16) reinterpret_cast<__hip_bfloat16*>(gr.dtable)[at] = __float2bfloat16(s);
    else reinterpret_cast<float*>(gr.dtable)[at] = s;
  }
}

}  // namespace sla
#endif
