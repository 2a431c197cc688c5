// How the passes are cut into workgroups, and the kernel that joins the forward pass's sums of keys that were cut.
#include "attn_plan.h"

#include <math.h>

#include <algorithm>

#include "attn_bwd.h"
#include "mfma_common.h"

namespace sla {

namespace {

// Workgroups that the forward plan has room for: two per CU, as the bf16 kernels run at d = 128 and with a bias.  (Those at d = 64
// without one run three per CU and the float ones three or four: there keys are cut into fewer parts than would run at a time.)
constexpr int kSlots = 512;

long long ceil_div(long long a, long long b) { return (a + b - 1) / b; }

AttnPart part_of(int units, int heads, long long rows, bool packed) {
  AttnPart p = {};
  p.units = units;
  p.heads = heads;
  p.rows = (int)rows;
  p.tiles = (int)ceil_div(rows, kBlk);
  p.splits = 1;
  p.packed = packed;
  return p;
}

}  // namespace

AttnPlan attn_plan(const Attn& a, char* ws) {
  AttnPlan p = {};
  // The heads of a group share a row tile where one head's queries would leave most of it empty.  (Their bias takes
  // LDS per head: as many as leave room for two workgroups on a CU, else one.)
  const long long bias = a.has_bias() ? a.G * 4ll * bias_width(a.bias.far) : 0;
  const bool packed = (a.Nq < kBlk || a.Np > 0) && bias <= 12 * 1024;
  const int heads = packed ? a.G : 1;
  p.own = part_of(a.B * a.H / heads, heads, (long long)heads * a.Nq, packed);
  const long long T = ceil_div(a.Nk, kBlk), Tp = ceil_div(a.Np, kBlk);
  if (a.Np > 0) p.prefix = part_of(a.H / heads, heads, (long long)a.B * heads * a.Nq, true);
  // Parts of about equal length, two key tiles or more each (less does not pay for a part's fixed cost and its sums),
  // kSlots of them at most: one more would wait for a whole round.  They are counted by the capacities Nk and Np, and every sequence's own
  // keys are then cut into as many: from kSlots row tiles on nothing is cut, and a long sequence among short ones is read by one
  // workgroup per row tile.
  const long long tiles = (long long)p.own.units * p.own.tiles, ptiles = (long long)p.prefix.units * p.prefix.tiles;
  long long len = std::max(2ll, ceil_div(tiles * T + ptiles * Tp, kSlots));
  while (tiles * ceil_div(T, len) + ptiles * ceil_div(Tp, len) > kSlots && len < std::max(T, Tp)) ++len;
  p.own.splits = (int)std::max(1ll, std::min(ceil_div(T, len), 256ll));
  // Under a causal mask row tiles have from few steps to T of them, and the longest parts decide: cut finer, down to where the load
  // of a workgroup's place is more than a part.  The load in steps has a part's costs beside its own (as on the key side, see
  // attn_bwd_plan).  Float, d = 128: 9 heads of 1692 122 -> 105 us, 4 of 2900 152 -> 102.  Rows that were whole stay so: two parts gain
  // less than the joining launch takes (bf16, 8 heads of 4000 56 -> 54 + 30, float, 16 of 1500 151 -> 137 + 24).
  if (a.causal && !packed && !a.Np && p.own.splits > 1) {
    const double load = T - 0.5 * std::min(T, (long long)p.own.tiles);
    double best = 1e300;
    for (int n = 2; n <= 16 && 2 * n <= T; ++n) {
      const double extra = (0.5 * n + 0.5) * (a.dtype == SLA_F32 ? 4.0 : 10.0);
      const double t = std::max((double)ceil_div(T, n), tiles * (load + extra) / kSlots);
      if (t < 0.95 * best) {
        best = t;
        p.own.splits = n;
      }
    }
  }
  p.prefix.splits = (int)std::max(1ll, std::min(ceil_div(Tp, len), 256ll));
  p.parts = a.Np > 0 || p.own.splits > 1;
  p.map = tile_map(a, p.own.units, p.own.tiles);
  if (p.parts) {
    p.own.blocks = (int)(tiles * p.own.splits);
    p.prefix.blocks = (int)(ptiles * p.prefix.splits);
    p.own.slot0 = p.prefix.blocks;
    p.slots = p.own.slot0 + p.own.blocks;
    p.part = reinterpret_cast<float*>(ws);
    p.stat = reinterpret_cast<float*>(ws + align_up((size_t)p.slots * kBlk * a.d * 4));
  }
  return p;
}

size_t attn_plan_ws(const Attn& a, const AttnPlan& p) {
  return p.parts ? align_up((size_t)p.slots * kBlk * a.d * 4) + align_up((size_t)p.slots * kBlk * 8) : 0;
}

bool attn_forward_fits(const Attn& a) {
  const AttnPlan p = attn_plan(a, nullptr);
  constexpr long long lim = (1ll << 31) - (1 << 17);
  const long long esz = a.dtype == SLA_F32 ? 4 : 2;
  // keys of one workgroup behind one descriptor
  auto span = [&](const View& v, long long n, long long tiles, int splits) {
    return std::min(n, (ceil_div(tiles, splits) + 1) * kBlk) * v.sn * esz;
  };
  const long long T = ceil_div(a.Nk, kBlk), Tp = ceil_div(a.Np, kBlk);
  if (span(a.K, a.Nk, T, p.own.splits) >= lim || span(a.V, a.Nk, T, p.own.splits) >= lim) return false;
  if (a.Np && (span(a.Kp, a.Np, Tp, p.prefix.splits) >= lim || span(a.Vp, a.Np, Tp, p.prefix.splits) >= lim)) return false;
  if ((long long)(a.Np ? a.B : 1) * p.own.heads * a.Nq >= lim) return false;   // rows of a unit
  // rows of a packed unit (those of one head are counted from their tile)
  if (p.own.packed || a.Np) {
    auto rows = [&](const View& v) { return ((a.Np ? a.B - 1 : 0) * v.sb + (p.own.heads - 1) * v.sh + (long long)(a.Nq - 1) * v.sn + a.d) * esz; };
    if (rows(a.Q) >= lim || rows(a.O) >= lim) return false;
  }
  return true;
}

namespace {

__device__ __forceinline__ void put_pair(float* p, float x, float y) { *reinterpret_cast<float2*>(p) = float2{x, y}; }
__device__ __forceinline__ void put_pair(bf16* p, float x, float y) {
  bf16x2 v;
  v[0] = (__bf16)x;
  v[1] = (__bf16)y;
  *reinterpret_cast<bf16x2*>(p) = v;
}
__device__ __forceinline__ void put_one(float* p, float x) { *p = x; }
__device__ __forceinline__ void put_one(bf16* p, float x) { *reinterpret_cast<__bf16*>(p) = (__bf16)x; }

// O = sum_i 2^(m_i - M) o_i / sum_i 2^(m_i - M) l_i over the parts of a row.  W waves share a row (each takes every W-th
// part, eight loads in flight) and meet in LDS; the order of the sums follows from the number of parts.  Bound by the
// latency of its two rounds of loads.
template <class E, int D, int W>
__global__ __launch_bounds__(256) void attn_join_kernel(Attn a, AttnPlan plan) {
  __shared__ float red[W > 1 ? 4 : 1][D];
  const int l = threadIdx.x & 63, w = wave_uniform(threadIdx.x >> 6), sub = w % W;
  const long long row = (long long)blockIdx.x * (4 / W) + w / W;
  const bool in = row < (long long)a.B * a.H * a.Nq;
  const int n = in ? row % a.Nq : 0, bh = in ? row / a.Nq : 0, b = bh / a.H, h = bh - b * a.H;
  const AttnPart &ow = plan.own, &pp = plan.prefix;
  const int u = h / ow.heads, hg = h - u * ow.heads;
  // first slot and row of this query among the prefix's and its own sums
  const int pr = (b * ow.heads + hg) * a.Nq + n, orow = ow.packed ? hg * a.Nq + n : n;
  const size_t ps = pp.blocks ? ((size_t)u * pp.tiles + pr / kBlk) * pp.splits : 0;
  const size_t os = ow.slot0 + ((size_t)(b * (a.H / ow.heads) + u) * ow.tiles + orow / kBlk) * ow.splits;
  const int np = pp.blocks ? pp.splits : 0, total = np + ow.splits;
  auto at = [&](int i) { return i < np ? (ps + i) * kBlk + pr % kBlk : (os + i - np) * kBlk + orow % kBlk; };
  // statistics: part i in lane i % 64
  float M = -INFINITY;
  for (int i = l; i < total; i += 64) {
    const float2 x = *reinterpret_cast<const float2*>(plan.stat + 2 * at(i));
    if (x.y != 0.0f) M = fmaxf(M, x.x);
  }
#pragma unroll
  for (int o = 32; o; o >>= 1) M = fmaxf(M, __shfl_xor(M, o));
  float lsum = 0.0f, acc[D / 64] = {};
  for (int i0 = 0; i0 < total; i0 += 64) {
    float2 x = {0.0f, 0.0f};
    if (i0 + l < total) x = *reinterpret_cast<const float2*>(plan.stat + 2 * at(i0 + l));
    const float wt = x.y != 0.0f ? fast_exp2(x.x - M) : 0.0f;   // (a sum that is no number stays one)
    float s = wt * x.y;
#pragma unroll
    for (int o = 32; o; o >>= 1) s += __shfl_xor(s, o);
    lsum += s;
    const int cnt = min(64, total - i0);
    for (int i = sub; i < cnt; i += 8 * W) {
      float y[8][D / 64], wi[8];
#pragma unroll
      for (int k = 0; k < 8; ++k) {   // (past the end, and parts without a key, whose sums are not written: nothing is read)
        wi[k] = i + k * W < cnt ? __shfl(wt, (i + k * W) & 63) : 0.0f;
        const float* p = plan.part + at(i0 + min(i + k * W, cnt - 1)) * D + (D / 64) * l;
#pragma unroll
        for (int e = 0; e < D / 64; ++e) y[k][e] = wi[k] != 0.0f ? p[e] : 0.0f;
      }
#pragma unroll
      for (int k = 0; k < 8; ++k)
#pragma unroll
        for (int e = 0; e < D / 64; ++e) acc[e] = fmaf(wi[k], y[k][e], acc[e]);
    }
  }
  if constexpr (W > 1) {
#pragma unroll
    for (int e = 0; e < D / 64; ++e) red[w][(D / 64) * l + e] = acc[e];
    __syncthreads();
    if (sub) return;
#pragma unroll
    for (int x = 1; x < W; ++x)
#pragma unroll
      for (int e = 0; e < D / 64; ++e) acc[e] += red[w + x][(D / 64) * l + e];
  }
  if (!in) return;
  const float inv = lsum != 0.0f ? 1.0f / lsum : 0.0f;
  E* o = reinterpret_cast<E*>(a.O.p) + b * a.O.sb + h * a.O.sh + (long long)n * a.O.sn + (D / 64) * l;
  if constexpr (D == 128) put_pair(o, acc[0] * inv, acc[1] * inv);
  else put_one(o, acc[0] * inv);
  if (a.L && l == 0) a.L[row] = lsum != 0.0f ? M * kLn2 + logf(lsum) : -INFINITY;
}

template <class E, int D>
hipError_t join_impl(const Attn& a, const AttnPlan& plan, hipStream_t st) {
  const long long rows = (long long)a.B * a.H * a.Nq;
  const int parts = plan.own.splits + (plan.prefix.blocks ? plan.prefix.splits : 0);
  KernelTimer kt("attn_join", st);
  // four waves a row where a wave alone would take a third round of loads
  if (parts > 8) attn_join_kernel<E, D, 4><<<(unsigned)rows, 256, 0, st>>>(a, plan);
  else attn_join_kernel<E, D, 1><<<(unsigned)((rows + 3) / 4), 256, 0, st>>>(a, plan);
  return hipGetLastError();
}

}  // namespace

hipError_t attn_join(const Attn& a, const AttnPlan& plan, hipStream_t st) {
  if (a.dtype == SLA_F32) return a.d == 64 ? join_impl<float, 64>(a, plan, st) : join_impl<float, 128>(a, plan, st);
  return a.d == 64 ? join_impl<bf16, 64>(a, plan, st) : join_impl<bf16, 128>(a, plan, st);
}

// Key tiles alone may not fill the chip (text of a few hundred tokens under a long video), and under a causal mask the
// first one has all queries and the last one few.  A piece costs about ten steps beside its own (operands, sums out and
// back, the joining launch; float steps are longer, there it is three); among the numbers of pieces the least estimated
// time is taken, in steps: full rounds of the chip's workgroups where all tiles are alike, average and one last
// piece where they are not.
BwdPlan attn_bwd_plan(const Attn& a, char* ws) {
  BwdPlan p = {};
  size_t off = 0;
  auto take = [&](size_t n) {
    float* x = reinterpret_cast<float*>(ws + off);
    off += align_up(n * sizeof(float));
    return x;
  };
  const bool f32 = a.dtype == SLA_F32;
  const int qtiles = (a.Nq + kBlk - 1) / kBlk;
  // float query side: as many parts of a tile as fill the chip's 512 places
  const long long qunits = (long long)a.B * a.H * qtiles;
  // (under a causal mask half of the steps are empty and the longest rows decide, twice as many places count: d = 128, 9 heads of 1692
  // 140 -> 111 us, 16 of 1500 206 -> 139)
  const long long places = a.causal ? 512 : 256;
  p.shares = !f32 || qunits > places ? 1 : qunits > places / 2 ? 2 : 4;
  p.qparts = (a.Nq + kBlk / p.shares - 1) / (kBlk / p.shares);
  p.map = tile_map(a, a.B * a.H, p.qparts);
  KeyPlan& k = p.key;
  k.tiles = (a.Nk + kBlk - 1) / kBlk;
  const long long units = (long long)a.B * a.Hkv * k.tiles;
  k.quarters = f32 ? (units < 384 ? 4 : 2) : 1;
  k.map = tile_map(a, a.B * a.Hkv, k.tiles);
  k.blocks = f32 ? (int)units * k.quarters : k.map.blocks();
  // (workgroups at a time; d = 128 with a bias runs one per CU, see DkLds, and is counted as two)
  const double slots = !f32 && a.d == 64 ? 768 : 512, wgs = (double)units * k.quarters, steps = (double)a.G * qtiles;
  double best = 1e300;
  k.pieces = 1;
  for (int n = 1; n <= 64 && n <= steps && k.tiles > 0; ++n) {   // (without keys there is nothing to cut, nor to join)
    const double len = ceil(steps / n), extra = n == 1 ? 3.0 : f32 ? 4.0 : 10.0;
    const double t = a.causal ? (0.5 * wgs * steps + (n > 1 ? 0.5 * n + 0.5 : 1.0) * wgs * extra) / slots + len
                              : ceil(wgs * n / slots) * (len + extra);
    if (t < 0.95 * best) {
      best = t;
      k.pieces = n;
    }
  }
  k.piece = k.pieces > 1 ? (int)ceil(steps / k.pieces) : 0x7fffffff;
  p.stat = take((size_t)a.B * a.H * a.Nq * (f32 ? 1 : 4));
  p.tpart = take(a.has_bias() ? (size_t)a.B * a.H * p.qparts * bucket_count(a.bias) : 0);
  k.part = take(k.pieces > 1 ? (size_t)units * k.pieces * 2 * kBlk * a.d : 0);
  p.bytes = off;
  return p;
}

size_t attn_forward_ws(const Attn& a) { return attn_plan_ws(a, attn_plan(a, nullptr)); }
size_t attn_backward_ws(const Attn& a) { return attn_bwd_plan(a, nullptr).bytes; }

hipError_t attn_forward(const Attn& a, char* ws, hipStream_t st) {
  const AttnPlan p = attn_plan(a, ws);
  return a.dtype == SLA_F32 ? attn_forward_f32(a, p, st) : attn_forward_bf16(a, p, st);
}
hipError_t attn_backward(const Attn& a, const AttnGrads& g, char* ws, hipStream_t st) {
  return a.dtype == SLA_F32 ? attn_backward_f32(a, g, ws, st) : attn_backward_bf16(a, g, ws, st);
}

}  // namespace sla
