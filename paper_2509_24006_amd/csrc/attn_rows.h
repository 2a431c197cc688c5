// Which rows and keys a workgroup of a forward pass owns, and what one of its rows sees (see AttnPlan).
#ifndef SLA_ATTN_ROWS_H_
#define SLA_ATTN_ROWS_H_

#include "attn_plan.h"
#include "mfma_common.h"

namespace sla {

// The query of a row, from its index in the unit's rows.
struct RowOf {
  int b, g, n;   // sequence, head of the unit, query
  bool in;
};

struct FwdTile {
  bool pre;              // keys of the shared prefix
  int unit, tile, part;
  int ub;                // sequence, -1: rows of all of them
  int h0, hk;            // first query head, K, V head
  int r0;                // first row
  int limmax;            // keys that any of the rows may see
  int t0, steps;         // first key tile of this part, number of them

  // false: nothing to do
  template <bool PART>
  __device__ __forceinline__ bool open(const Attn& a, const AttnPlan& plan) {
    pre = PART && (int)blockIdx.x < plan.prefix.blocks;
    const AttnPart& pt = pre ? plan.prefix : plan.own;
    part = 0;
    if constexpr (PART) {
      // The row tiles that read the same keys follow each other eight blocks apart: on one XCD, whose L2 fetches them once.
      // (Prefix of 16384, 32 sequences: 16 heads over 4, two row tiles 19.5 -> 18.8 us; 32 heads of 8 new tokens, sixteen, 120 -> 108.)
      const int x = blockIdx.x - (pre ? 0 : plan.prefix.blocks), cuts = pt.units * pt.splits;
      const int first = x / (8 * pt.tiles) * 8, m = min(8, cuts - first), r = x - first * pt.tiles, c = first + r % m;
      tile = r / m;
      part = c % pt.splits;
      unit = c / pt.splits;
    } else {
      const TileOf own = plan.map.at(blockIdx.x);
      if (own.i < 0) return false;
      unit = own.bh;
      tile = a.causal ? plan.own.tiles - 1 - own.i : own.i;   // (longest rows first)
    }
    if (PART && a.causal && !pt.packed) tile = pt.tiles - 1 - tile;   // (longest rows first)
    unit = wave_uniform(unit);
    tile = wave_uniform(tile);
    const int per_b = a.H / pt.heads;   // units per sequence (prefix: units in all)
    ub = pre ? -1 : unit / per_b;
    h0 = (pre ? unit : unit - ub * per_b) * pt.heads;
    hk = h0 / a.G;
    r0 = tile * kBlk;
    if (pre) {
      limmax = a.Np;
    } else {
      const Seq s = seq_of(a, ub);
      const int last = pt.packed ? s.nq : min(r0 + kBlk, s.nq);   // one behind the last query
      limmax = (pt.packed ? s.nq > 0 : last > r0) ? s.nk : 0;
      if (a.causal) limmax = max(0, min(limmax, s.pos + last - a.Np));
    }
    const int T_all = (limmax + kBlk - 1) / kBlk;
    t0 = PART ? (int)((long long)T_all * part / pt.splits) : 0;
    const int t1 = PART ? (int)((long long)T_all * (part + 1) / pt.splits) : T_all;
    steps = wave_uniform(t1 - t0);
    return true;
  }
  __device__ __forceinline__ RowOf row(const Attn& a, const AttnPart& pt, int i) const {   // i: 0 .. 63
    RowOf o;
    const int r = r0 + i;
    o.in = r < pt.rows;
    o.b = ub;
    o.g = 0;
    o.n = r;
    if (pt.packed) {
      const int rg = r / a.Nq;
      o.n = r - rg * a.Nq;
      o.g = rg;
      if (ub < 0) {   // rows of all sequences
        o.b = rg / pt.heads;
        o.g = rg - o.b * pt.heads;
      }
    }
    if (!o.in) {   // (behind the last row of a head: a position next to the others', for the bias)
      o.b = max(ub, 0);
      o.g = 0;
      o.n = pt.packed ? 0 : r;
    }
    return o;
  }
  __device__ __forceinline__ size_t slot(const AttnPart& pt) const {
    return (size_t)pt.slot0 + ((size_t)unit * pt.tiles + tile) * pt.splits + part;
  }
  // elements from a tensor's start to row n of head g of the unit in sequence b
  __device__ __forceinline__ long long at(const View& v, const RowOf& x) const {
    return (long long)x.b * v.sb + (long long)(h0 + x.g) * v.sh + (long long)x.n * v.sn;
  }
  // first key of this part
  __device__ __forceinline__ long long key_at(const View& v) const {
    return (long long)(pre ? 0 : ub) * v.sb + (long long)hk * v.sh + (long long)t0 * kBlk * v.sn;
  }
  __device__ __forceinline__ int keys() const { return max(1, min(limmax - t0 * kBlk, steps * kBlk)); }   // up to the last valid one
};

// What a row sees of the keys of its workgroup's part.
struct RowKeys {
  bool live;   // a query within its sequence's length
  int pos;     // its position, counted in these keys
  int lim;     // number of keys; a row that is not live sees all it comes across, and is written as zeros
};
__device__ __forceinline__ RowKeys row_keys(const Attn& a, const FwdTile& x, const RowOf& row) {
  RowKeys k;
  const Seq s = seq_of(a, row.b);
  k.live = row.in && row.n < s.nq;
  k.pos = s.pos + row.n - (x.pre ? 0 : a.Np);
  k.lim = 0x7fffffff;
  if (k.live) {
    k.lim = x.pre ? a.Np : s.nk;
    if (a.causal) k.lim = max(0, min(k.lim, k.pos + 1));
  }
  return k;
}

}  // namespace sla
#endif
