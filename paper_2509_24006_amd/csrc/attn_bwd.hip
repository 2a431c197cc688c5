// bf16 softmax attention, backward pass on the matrix cores.  The probabilities are formed again from the scores and L.
//   attn_dq_kernel   one workgroup per 64 queries of a head: D = rowsum(dO O), dQ, and its part of the bias table's gradient
//   attn_dkdv_kernel one workgroup per 64 keys (and piece of the queries): dK, dV summed over the queries of all heads
//                    that read them; its last workgroups add up the table's gradient
//   attn_kv_join     adds the pieces
// S and dP are formed in both kernels (seven products instead of five): dQ summed where dK and dV are would need float
// atomics of a 64 x d tile per pair, whose order changes the result and whose traffic costs more than the two products.
// P and dS enter their second products rounded to bf16, the matrix cores' operand type; all sums are in float.
#include <type_traits>

#include "attn_bwd.h"
#include "mfma_common.h"

namespace sla {
namespace {

template <int D>
__device__ __forceinline__ BufDesc rows_rsrc(const View& v, int b, int h, int n) {
  const bf16* p = reinterpret_cast<const bf16*>(v.p) + (size_t)b * v.sb + (size_t)h * v.sh;
  return tile_rsrc(p, (max(n, 1) - 1) * 2 * v.sn + 2 * D);
}

// bias in log2 units by distance
__device__ __forceinline__ void expand_bias(const Attn& a, int h, float* out) {
  const int mid = a.bias.far + kBiasPad;
  for (int i = threadIdx.x; i <= 2 * mid; i += 256) out[i] = table_at(a, bucket_of(a.bias, i - mid), h) * kLog2e;
}

// A query's L / scale and D, each as three bf16 terms (24 bits): the A operand of one more k-step of the key side's first
// products, whose B operands hold -1 at the places of one or the other, so that the accumulators come out as
// S - L / scale and dP - D.
typedef bf16x8 RowStat;
__device__ __forceinline__ RowStat row_stat(float L, float D, float rscale) {
  const float l = L == -INFINITY ? 1e30f : L * rscale;   // (a row without a key: P = 0)
  RowStat r = zero_bf16x8();
  float x = l, y = D;
#pragma unroll
  for (int e = 0; e < 3; ++e) {
    r[e] = (__bf16)x;
    r[4 + e] = (__bf16)y;
    x -= (float)r[e];
    y -= (float)r[4 + e];
  }
  return r;
}

// ------------------------------------------------------------------ dQ
// (d = 128 with a bias: 74804 + 40 far bytes in all, two workgroups per CU up to far = 177 and one beyond.)
template <int D>
struct DqLds {
  static constexpr int TILE = SwzTile<D>::BYTES;
  static constexpr int BUF = 2 * TILE;             // K_j and V_j
  static constexpr int SP = D + 4;                 // floats per row of the output staging
  static constexpr int FIXED = 2 * BUF > kBlk * SP * 4 ? 2 * BUF : kBlk * SP * 4;
  static constexpr int STAT = FIXED;               // a sum of each of the 64 queries and two key halves
  // with a bias: 16 x 32 floats per wave, the bias by distance, the sums of dS by distance (an array per wave)
  static constexpr int SKEW = STAT + 512;
  static constexpr int BIAS = SKEW + 4 * 2048;
};
template <int D>
int dq_lds(const Attn& a) {
  return a.has_bias() ? DqLds<D>::BIAS + bias_width(a.bias.far) * 4 + 4 * (2 * a.bias.far + 1) * 4 + 32 : DqLds<D>::SKEW;
}

// Wave (qh, kh): S^T and dP^T are [key][query], one query per lane, so L and D are per-lane scalars and dS^T feeds
// dQ^T = K^T dS^T from registers.  The two kh waves hold sums over their keys and are added at the end.
//
// D: rowsum(dO O) has the rounding of O in it, which a sum of dS over many keys of a row (the last bucket of a bias) does not
// average out, nor a row with few keys.  The sum of P (dP - D') over all keys is D - D' whatever D' is: the key side gets the
// D that is corrected by it, and the last buckets' sums are corrected too.  dQ takes D' = rowsum(dO O) where there are
// many keys, and otherwise D from a pass over them before: one tile of them, or two where a bias makes probabilities less even
// (with even scores its relative error from the rounding is 2^-9 over the root of the number of keys).
//
// The table's gradient is a sum of dS by distance.  Away from the diagonal a lane's values all belong to the last bucket
// of a side, and stay in registers.  Near it the wave's 32 x 32 values are summed along their diagonals through LDS, 16 keys
// at a time: lane e reads the values of the diagonals e and e - 32.  A wave meets a distance in one step only (its
// distances move on by 64 and span 63), so that the sum is stored, not added: no atomics, which take a cycle per lane.
// (768 workgroups of up to 8 steps: 64 us with LDS atomics, 32 this way.)
template <int D, bool BIAS>
__global__ __launch_bounds__(256, D == 64 && !BIAS ? 3 : 2) void attn_dq_kernel(Attn a, AttnGrads gr, RowStat* __restrict__ stats,
                                                                                float* __restrict__ tpart, TileMap map) {
  using Lds = DqLds<D>;
  using T = SwzTile<D>;
  constexpr int NT = D / 32, KT = D / 16, RB = 16 * T::ROW_BYTES;
  extern __shared__ __attribute__((aligned(16))) unsigned char smem[];
  const int tid = threadIdx.x, w = tid >> 6, l = tid & 63, g = l >> 5, ln = l & 31;
  const int qh = w & 1, kh = w >> 1;
  const TileOf own = map.at(blockIdx.x);
  if (own.i < 0) return;
  const int tiles = map.nb;
  const int bh = wave_uniform(own.bh), i = wave_uniform(a.causal ? tiles - 1 - own.i : own.i);   // (longest rows first)
  const int b = bh / a.H, h = bh - b * a.H, hk = h / a.G;
  const Seq s = seq_of(a, b);
  const int q0 = i * kBlk, rows = min(kBlk, a.Nq - q0), n = q0 + qh * 32 + ln;
  const bool live = n < s.nq;
  const int pos = s.pos + n;
  int limmax = q0 < s.nq ? s.nk : 0;
  if (a.causal) limmax = max(0, min(limmax, s.pos + min(q0 + kBlk, s.nq)));
  const int steps = wave_uniform((limmax + kBlk - 1) / kBlk);
  const int lim = !live ? 0x7fffffff : a.causal ? max(0, min(s.nk, pos + 1)) : s.nk;   // (rows that are not live: dO = 0)
  const float sl2 = a.scale * kLog2e;

  TileLoader<D> tq, tg;
  RunLoader<D> tk, tv;
  tq.init(lds_base(smem), w, l, 2 * a.Q.sn);
  tg.init(lds_base(smem), w, l, 2 * gr.dO.sn);
  tk.init(lds_base(smem), w, l, 2 * a.K.sn, kBlk);
  tv.init(lds_base(smem), w, l, 2 * a.V.sn, kBlk);
  tq.load(rows_rsrc<D>(a.Q, b, h, s.nq), i, Lds::BUF);
  tg.load(rows_rsrc<D>(gr.dO, b, h, s.nq), i, Lds::BUF + Lds::TILE);
  const size_t li = (size_t)bh * a.Nq + n;
  float Lq = live ? a.L[li] * kLog2e : INFINITY;
  if (Lq == -INFINITY) Lq = INFINITY;   // (a row without a key: P = 0)
  bf16x8 of[KT];
  {
    const bf16* o = reinterpret_cast<const bf16*>(a.O.p) + (size_t)b * a.O.sb + (size_t)h * a.O.sh + (size_t)min(n, a.Nq - 1) * a.O.sn;
#pragma unroll
    for (int t = 0; t < KT; ++t) of[t] = *reinterpret_cast<const bf16x8*>(o + 16 * t + 8 * g);
  }
  const BufDesc descK = rows_rsrc<D>(a.K, b, hk, s.nk), descV = rows_rsrc<D>(a.V, b, hk, s.nk);
  const std::integral_constant<int, 0> b0;   // the two pair buffers
  const std::integral_constant<int, 1> b1;
  auto issue = [&](int j, auto Buf) __attribute__((always_inline)) {
    constexpr int O = decltype(Buf)::value * Lds::BUF;
    tk.template load<O>(descK, j * tk.tile_step);
    tv.template load<O + Lds::TILE>(descV, j * tv.tile_step);
  };
  if (steps > 0) issue(0, b0);
  tk.pin();
  tv.pin();
  float* const bias = reinterpret_cast<float*>(smem + Lds::BIAS);
  const int far = a.bias.far, width = 2 * far + 1;
  float* const dist = bias + bias_width(far);          // [wave][width]
  const float* const bmid = bias + far + kBiasPad;     // at distance 0
  float* const skew = reinterpret_cast<float*>(smem + Lds::SKEW) + 512 * w;
  float* const stat = reinterpret_cast<float*>(smem + Lds::STAT);   // [kh][64]
  if constexpr (BIAS) {
    expand_bias(a, h, bias);
    for (int x = tid; x < 4 * width; x += 256) dist[x] = 0.0f;
  }
  wait_vm0_known();
  __syncthreads();
  bf16x8 qf[KT], gf[KT];
  {
    TileAddr<D> qa;
    qa.init(32 * qh, l);
#pragma unroll
    for (int t = 0; t < KT; ++t) {
      qf[t] = lds_row(smem, qa.row(t) + Lds::BUF);
      gf[t] = lds_row(smem, qa.row(t) + Lds::BUF + Lds::TILE);
    }
  }
  float dsum = 0.0f;
#pragma unroll
  for (int t = 0; t < KT; ++t) {
    pin_loaded(qf[t]);
    pin_loaded(gf[t]);
#pragma unroll
    for (int e = 0; e < 8; ++e) dsum = fmaf((float)gf[t][e], (float)of[t][e], dsum);
  }
  dsum = live ? half_sum(dsum) : 0.0f;
  float nDq = -dsum, drow = 0.0f;   // drow: sum of P (dP - D') over this lane's keys
  f32x16 dqT[NT];
#pragma unroll
  for (int t = 0; t < NT; ++t) dqT[t] = zero_f32x16();
  float sumL = 0.0f, sumR = 0.0f;   // dS at distances of -far and less, far and more
  float pL = 0.0f, pR = 0.0f;       // P there (in tiles that lie there as a whole)
  TileAddr<D> ad;   // this wave reads rows 32 kh .. of K_j and V_j
  ad.init(32 * kh, l);
  // MAIN: the step proper; else only drow
  auto step = [&](auto Main, int j, auto Buf) __attribute__((always_inline)) {
    constexpr bool MAIN = decltype(Main)::value;
    constexpr int buf = decltype(Buf)::value, KO = buf * Lds::BUF, VO = KO + Lds::TILE;
    // (registers: with a bias and 128 features K_j^T comes after the table's sums, and fewer operands run ahead; left as in the
    // other kernels 43 of them spill: 12 heads of 4000 269 -> 194 us, causal 131 -> 102)
    constexpr bool LATE = BIAS && D == 128;
    const int key0 = j * kBlk + 32 * wave_uniform(kh);
    ad.refresh();
    wait_vm0();
    __syncthreads();   // tiles of step j have landed for every wave; step j - 1 is fully consumed
    if (j + 1 < steps) issue(j + 1, std::integral_constant<int, buf ^ 1>());
    constexpr int PF = LATE ? 3 : 4;   // LDS reads run PF operand pairs ahead of the products
    bf16x8 ka[PF], va[PF], ta[2][NT];
    auto read_s = [&](int t) __attribute__((always_inline)) {
      ka[t % PF] = lds_row(smem, ad.row(t) + KO);
      va[t % PF] = lds_row(smem, ad.row(t) + VO);
    };
#pragma unroll
    for (int t = 0; t < PF; ++t) read_s(t);
    sched_fence();
    f32x16 sT = zero_f32x16(), dpT;   // (dP starts at -D' of the lane's query)
#pragma unroll
    for (int r = 0; r < 16; ++r) dpT[r] = nDq;
#pragma unroll
    for (int t = 0; t < KT; ++t) {
      sT = mfma32(ka[t % PF], qf[t], sT);
      dpT = mfma32(va[t % PF], gf[t], dpT);
      if (t + PF < KT) read_s(t + PF);
      sched_fence();
    }
    // K_j^T for the third product arrives under the exponentials
    auto read_k = [&]() __attribute__((always_inline)) {
#pragma unroll
      for (int u = 0; u < 2; ++u)
#pragma unroll
        for (int dt = 0; dt < NT; ++dt)
          ta[u][dt] = lds_tr<D>(smem, ad.tr(0, dt) + KO + u * RB, ad.tr(1, dt) + KO + u * RB);
    };
    if constexpr (MAIN && !LATE) read_k();
    sched_fence();
    const int d0 = key0 - pos;   // distance of this wave's first key
    bool near = false;
    if constexpr (BIAS) {
      near = __any(d0 + 31 > -far && d0 < far);
      if (near) {
#pragma unroll
        for (int r = 0; r < 16; ++r) sT[r] = fast_exp2(fmaf(sT[r], sl2, bmid[d0 + 4 * g + c_row(r, 0)] - Lq));
      } else {
        const float bc = bmid[d0 < 0 ? -far : far] - Lq;
#pragma unroll
        for (int r = 0; r < 16; ++r) sT[r] = fast_exp2(fmaf(sT[r], sl2, bc));
      }
    } else {
#pragma unroll
      for (int r = 0; r < 16; ++r) sT[r] = fast_exp2(fmaf(sT[r], sl2, -Lq));
    }
    if (__any(lim < key0 + 32)) {
      int first = lim - key0;
      asm volatile("" : "+v"(first));   // (the comparisons stay inside the branch)
#pragma unroll
      for (int r = 0; r < 16; ++r)
        if (c_row(r, g) >= first) sT[r] = 0.0f;
    }
    float ds = 0.0f;
#pragma unroll
    for (int r = 0; r < 16; ++r) {
      dpT[r] = sT[r] * dpT[r];
      ds += dpT[r];
    }
    drow += ds;
    if constexpr (!MAIN) return;
    if constexpr (BIAS) {
      if (near) {
        float da = 0.0f, db = 0.0f;   // diagonals ln and ln - 32
        const int eg = ln - 8 * g;
#pragma unroll
        for (int u = 0; u < 2; ++u) {
#pragma unroll
          for (int r = 0; r < 8; ++r) skew[32 * (c_row(8 * u + r, g) - 16 * u) + ln] = dpT[8 * u + r];
          asm volatile("" ::: "memory");
#pragma unroll
          for (int k = 0; k < 8; ++k) {   // key 16 u + 8 g + k
            const float v = skew[32 * (8 * g + k) + ((16 * u + k - eg) & 31)];
            da += eg <= 16 * u + k ? v : 0.0f;
            db += eg <= 16 * u + k ? 0.0f : v;
          }
          asm volatile("" ::: "memory");
        }
        da = half_sum(da);
        db = half_sum(db);
        const int d = key0 - (s.pos + q0 + 32 * wave_uniform(qh)) + ln - 32 * g;
        const float v = g ? db : da;
        if (d <= -far) sumL += v;
        else if (d >= far) sumR += v;
        else dist[w * width + d + far] = v;
      } else {
        float ps = 0.0f;
#pragma unroll
        for (int r = 0; r < 16; ++r) ps += sT[r];
        sumL += d0 < 0 ? ds : 0.0f;
        sumR += d0 < 0 ? 0.0f : ds;
        pL += d0 < 0 ? ps : 0.0f;
        pR += d0 < 0 ? 0.0f : ps;
      }
    }
    if constexpr (LATE) read_k();
#pragma unroll
    for (int u = 0; u < 2; ++u) {
      const bf16x8 sb = c_to_operand(dpT, u);
#pragma unroll
      for (int dt = 0; dt < NT; ++dt) dqT[dt] = mfma32(ta[u][dt], sb, dqT[dt]);   // K_j^T dS^T
    }
  };
  // the two key halves' sums of a query
  auto both = [&](float x) {
    x = half_sum(x);
    __syncthreads();
    if (g == 0) stat[kh * kBlk + qh * 32 + ln] = x;
    __syncthreads();
    return stat[qh * 32 + ln] + stat[kBlk + qh * 32 + ln];
  };
  const std::integral_constant<bool, true> main;
  if (steps > 0 && steps <= (BIAS ? 2 : 1)) {
    const std::integral_constant<bool, false> probe;
    nDq = 0.0f;
    step(probe, 0, b0);
    if (BIAS && steps > 1) step(probe, 1, b1);
    dsum = both(drow);
    nDq = -dsum;
    drow = 0.0f;
    if (lim == 1) Lq = INFINITY;   // (a single key, see dk_scale; the other rows of its tile see 64 keys at most)
    issue(0, b0);
  }
  for (int j = 0; j < steps; j += 2) {
    step(main, j, b0);
    if (j + 1 < steps) step(main, j + 1, b1);
  }
  {
    const float dd = both(drow);
    if (kh == 0 && g == 0 && live) stats[li] = row_stat(a.L[li], dsum + dd, 1.0f / a.scale);
    sumL -= dd * pL;
    sumR -= dd * pR;
  }
  if constexpr (BIAS) table_part<4>(a, dist, width, sumL, sumR, tpart + ((size_t)bh * tiles + i) * bucket_count(a.bias));
  // ---- add the two key halves in a row-major staging area, then every thread stores 8-byte pieces of whole rows
  __syncthreads();   // every wave is done with the tiles
  constexpr int C4 = D / 4, NIT = kBlk * C4 / 256, SP = Lds::SP;
  float* stg = reinterpret_cast<float*>(smem);   // [64 queries][SP]
  const int srow = (qh * 32 + ln) * SP + 4 * g;
  if (kh == 1) {
#pragma unroll
    for (int dt = 0; dt < NT; ++dt)
#pragma unroll
      for (int r4 = 0; r4 < 4; ++r4)
        *reinterpret_cast<f32x4*>(stg + srow + 32 * dt + 8 * r4) =
            f32x4{dqT[dt][4 * r4], dqT[dt][4 * r4 + 1], dqT[dt][4 * r4 + 2], dqT[dt][4 * r4 + 3]};
  }
  __syncthreads();
  if (kh == 0) {
#pragma unroll
    for (int dt = 0; dt < NT; ++dt)
#pragma unroll
      for (int r4 = 0; r4 < 4; ++r4) {
        f32x4 x = *reinterpret_cast<const f32x4*>(stg + srow + 32 * dt + 8 * r4);
#pragma unroll
        for (int r = 0; r < 4; ++r) x[r] = live ? x[r] + dqT[dt][4 * r4 + r] : 0.0f;
        *reinterpret_cast<f32x4*>(stg + srow + 32 * dt + 8 * r4) = x;
      }
  }
  __syncthreads();
  bf16* const dQ = reinterpret_cast<bf16*>(gr.dQ.p) + (size_t)b * gr.dQ.sb + (size_t)h * gr.dQ.sh + (size_t)q0 * gr.dQ.sn;
#pragma unroll
  for (int it = 0; it < NIT; ++it) {
    const int idx = it * 256 + tid, row = idx / C4, c4 = idx % C4;
    if (row < rows) {
      const f32x4 sv = *reinterpret_cast<const f32x4*>(stg + row * SP + 4 * c4);
      bf16x4 pk;
#pragma unroll
      for (int r = 0; r < 4; ++r) pk[r] = (__bf16)(sv[r] * a.scale);
      *reinterpret_cast<bf16x4*>(dQ + (size_t)row * gr.dQ.sn + 4 * c4) = pk;
    }
  }
}

// ------------------------------------------------------------------ dK, dV
// First products (S, dP): wave (kh, x) takes keys 32 kh .., queries 32 x .. of the pair; S and dP are [query][key], one
// key per lane.  Second products (dV^T = dO^T P, dK^T = Q^T dS): the same wave takes keys 32 kh .. and the
// feature half x, over all 64 queries.  P and dS cross between the two waves of a key half through LDS in operand layout.
// L and D of a query enter the first products as one more k-step (row_stat).  What counts is the number of instructions
// (a wave issues one in five cycles or more): loads with one M0 a tile, descriptors that change with the head only, L and
// D as a ready operand.  (Instructions of a step 414 -> 290 at d = 128, 337 -> 240 at d = 64; key side of 256 heads x 1024,
// d = 64, 221 -> 195 us, of 12 x 32760, d = 128, 12.58 -> 12.19 ms.)
// LDS at d = 128 is half of a CU's without a bias; any bias beside it leaves one workgroup per CU.
template <int D>
struct DkLds {
  static constexpr int TILE = SwzTile<D>::BYTES;
  static constexpr int BUF = 2 * TILE;                   // Q_i and dO_i of a pair
  static constexpr int XOFF = 2 * BUF;                   // exchange: [kh][k-step 0..3][P | dS][lane] x 16 bytes
  static constexpr int XBYTES = 2 * 4 * 2 * 64 * 16;
  static constexpr int BIAS = XOFF + XBYTES;
  static constexpr int STG = 32 * (64 * (D / 64) + 16);  // output staging of one wave, laid over the tiles
};

template <int D>
__device__ __forceinline__ f32x4* key_slot(const KeyPlan& kp, size_t slot, int w, int l) {
  return reinterpret_cast<f32x4*>(kp.part + slot * (2 * kBlk * D)) + w * (D / 8 * 64) + l;
}
template <int D>
__device__ __forceinline__ void store_keys(const Attn& a, const AttnGrads& gr, unsigned char* stage, f32x16 (&dvT)[D / 64],
                                           f32x16 (&dkT)[D / 64], int b, int hk, int j, int kh, int xh, bool ok, float scale, int l) {
  const int rows = a.Nk - j * kBlk - 32 * kh;
#pragma unroll
  for (int dt = 0; dt < D / 64; ++dt)
#pragma unroll
    for (int r = 0; r < 16; ++r) {
      dvT[dt][r] = ok ? dvT[dt][r] : 0.0f;
      dkT[dt][r] = ok ? dkT[dt][r] * scale : 0.0f;
    }
  auto at = [&](const View& v) {
    return reinterpret_cast<bf16*>(v.p) + (size_t)b * v.sb + (size_t)hk * v.sh + (size_t)(j * kBlk + 32 * kh) * v.sn + (D / 2) * xh;
  };
  store_rows_bf16<D / 64>(stage, dvT, at(gr.dV), gr.dV.sn, rows, l);
  store_rows_bf16<D / 64>(stage, dkT, at(gr.dK), gr.dK.sn, rows, l);
}

// (d = 64 with a bias: 19 registers spill at three workgroups per CU, and still 157 -> 136 us at 12 heads of 4000)
template <int D, bool BIAS>
__global__ __launch_bounds__(256, D == 64 ? 3 : 2) void attn_dkdv_kernel(Attn a, AttnGrads gr, const RowStat* __restrict__ stats, KeyPlan kp,
                                                            const float* __restrict__ tpart, int qparts) {
  using Lds = DkLds<D>;
  using T = SwzTile<D>;
  constexpr int NT = D / 32, KT = D / 16, HT = NT / 2;
  constexpr int RB = 16 * T::ROW_BYTES;
  extern __shared__ __attribute__((aligned(16))) unsigned char smem[];
  if ((int)blockIdx.x >= kp.blocks * kp.pieces) {
    if constexpr (BIAS) table_sum(a, gr, tpart, qparts, blockIdx.x - kp.blocks * kp.pieces, smem);
    return;
  }
  const int tid = threadIdx.x, w = tid >> 6, l = tid & 63, g = l >> 5, ln = l & 31;
  const int kh = w & 1, xh = w >> 1;
  const int p = blockIdx.x / kp.blocks, bx = blockIdx.x - p * kp.blocks;
  const TileOf own = kp.map.at(bx);
  if (own.i < 0) return;
  const int bh = wave_uniform(own.bh), j = wave_uniform(own.i);
  const int b = bh / a.Hkv, hk = bh - b * a.Hkv;
  const Seq sq = seq_of(a, b);
  const KeySteps ks_ = key_steps(a, sq, j);
  const int s_beg = wave_uniform(p * kp.piece), s_end = wave_uniform(min(ks_.total, s_beg + kp.piece));
  if (p > 0 && s_beg >= s_end) return;
  const bool cut = ks_.total > kp.piece;
  const int cnt = s_end - s_beg;
  const int k0 = j * kBlk, key = k0 + kh * 32 + ln;
  const bool kok = key < sq.nk;
  bf16x8 kf[KT], vf[KT];
  f32x16 dvT[HT], dkT[HT];
#pragma unroll
  for (int t = 0; t < HT; ++t) {
    dvT[t] = zero_f32x16();
    dkT[t] = zero_f32x16();
  }
  const float sl2 = a.scale * kLog2e;
  const int wu = wave_uniform(w);
  RunLoader<D> tq, tg;
  tq.init(lds_base(smem), w, l, 2 * a.Q.sn, kBlk);
  tg.init(lds_base(smem), w, l, 2 * gr.dO.sn, kBlk);
  // head and query tile of the step in flight or in use, and where they lie
  const int i_end = ks_.i0 + ks_.per_head;
  int ch = hk * a.G, ci = ks_.i0;
  if (cnt > 0) {
    const int hh = s_beg / ks_.per_head;
    ch = wave_uniform(ch + hh);
    ci = wave_uniform(ks_.i0 + s_beg - hh * ks_.per_head);
  }
  BufDesc descQ, descG, descS;
  auto turn = [&]() __attribute__((always_inline)) {
    const int h = min(ch, a.H - 1);   // (behind the last step of the last head: not read)
    descQ = rows_rsrc<D>(a.Q, b, h, sq.nq);
    descG = rows_rsrc<D>(gr.dO, b, h, sq.nq);
    descS = tile_rsrc(stats + ((size_t)b * a.H + h) * a.Nq, sq.nq * 16);
  };
  turn();
  auto issue = [&](auto Buf) __attribute__((always_inline)) {
    constexpr int O = decltype(Buf)::value * Lds::BUF;
    tq.template load<O>(descQ, ci * tq.tile_step);
    tg.template load<O + Lds::TILE>(descG, ci * tg.tile_step);
  };
  {
    TileLoader<D> t;
    t.init(lds_base(smem), w, l, 2 * a.K.sn);
    t.load(rows_rsrc<D>(a.K, b, hk, sq.nk), j, Lds::BUF);
    t.init(lds_base(smem), w, l, 2 * a.V.sn);
    t.load(rows_rsrc<D>(a.V, b, hk, sq.nk), j, Lds::BUF + Lds::TILE);
  }
  const std::integral_constant<int, 0> b0;
  const std::integral_constant<int, 1> b1;
  if (cnt > 0) issue(b0);
  float* const bias = reinterpret_cast<float*>(smem + Lds::BIAS);
  const int far = a.bias.far;
  const float* const bmid = bias + far + kBiasPad;   // at distance 0
  if constexpr (BIAS) expand_bias(a, ch, bias);
  wait_vm0_known();
  __syncthreads();
  {
    TileAddr<D> ka;
    ka.init(32 * kh, l);
#pragma unroll
    for (int t = 0; t < KT; ++t) {
      kf[t] = lds_row(smem, ka.row(t) + Lds::BUF);
      vf[t] = lds_row(smem, ka.row(t) + Lds::BUF + Lds::TILE);
    }
  }
#pragma unroll
  for (int t = 0; t < KT; ++t) {
    pin_loaded(kf[t]);
    pin_loaded(vf[t]);
  }
  TileAddr<D> ad;   // first products: rows 32 x .. of Q_i, dO_i by rows
  ad.init(32 * xh, l);
  TileAddr<D> at;   // second products: transposing reads, feature tiles x HT ..
  at.init(0, l);
  bf16x8 bL, bD;    // B operands of the extra k-step
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    bL[e] = (__bf16)((g == 0 && e < 3) ? -1.0f : 0.0f);
    bD[e] = (__bf16)((g == 0 && e >= 4 && e < 7) ? -1.0f : 0.0f);
  }
  tq.pin();
  tg.pin();
  const int xw = Lds::XOFF + ((kh * 4 + 2 * xh) * 2 * 64 + l) * 16;   // this wave's exchange writes
  const int xr = Lds::XOFF + (kh * 4 * 2 * 64 + l) * 16;              // ... and reads
  const int xwave = Lds::XOFF + (kh * 4 + 2 * xh) * 2 * 64 * 16;      // start of this wave's part (uniform)
  const unsigned xstat = lds_base(smem) + wave_uniform(xwave);
  auto step = [&](int s, auto Buf) __attribute__((always_inline)) {
    constexpr int buf = decltype(Buf)::value, QO = buf * Lds::BUF, GO = QO + Lds::TILE;
    ad.refresh();
    at.refresh();
    wait_vm0_known();
    __syncthreads();   // tiles of step s have landed for every wave; step s-1 is fully consumed
    // L and D of this step's 64 queries are requested ahead of the next pair's tiles (loads return in order) and picked
    // up after the first products.  They go global -> LDS into the first KB of this wave's own part of the exchange
    // area, which it overwrites with P and dS only after it has read them back.  Rows past the end read as 0; their Q
    // and dO rows are zero too, so the finite P they get adds nothing (with a bias: P = 0).
    load_to_lds16(descS, lane_id() * 16, ci * (kBlk * 16), xstat);
    const int qt = ci;
    // (the last step requests its own pair once more, into the other buffer, where nobody reads it: every step then
    // has the same number of loads in flight and one wait serves all)
    const bool turned = s + 1 < s_end && ci + 1 == i_end;
    if (turned) {
      ++ch;
      ci = ks_.i0;
      turn();
    } else if (s + 1 < s_end) {
      ++ci;
    }
    issue(std::integral_constant<int, buf ^ 1>());
    constexpr int PF = 4;   // LDS reads run PF operand pairs ahead of the products
    bf16x8 qa[PF], ga[PF];
    auto read_s = [&](int t) __attribute__((always_inline)) {
      qa[t % PF] = lds_row(smem, ad.row(t) + QO);
      ga[t % PF] = lds_row(smem, ad.row(t) + GO);
    };
#pragma unroll
    for (int t = 0; t < PF; ++t) read_s(t);
    sched_fence();
    f32x16 sm = zero_f32x16(), dp = zero_f32x16();
#pragma unroll
    for (int t = 0; t < KT; ++t) {
      sm = mfma32(qa[t % PF], kf[t], sm);
      dp = mfma32(ga[t % PF], vf[t], dp);
      if (t + PF < KT) read_s(t + PF);
      sched_fence();
    }
    wait_vm<2 * T::IPW>();   // the statistics are there, the tile loads may still fly
    {
      const RowStat st = *reinterpret_cast<const RowStat*>(smem + xwave + (32 * xh + (lane_id() & 31)) * 16);
      sm = mfma32(st, bL, sm);
      dp = mfma32(st, bD, dp);
    }
    // operand i of the second products: i = 2 HT ks + 2 dt + which; which 0: dO^T rows of feature tile x HT + dt (for
    // dV), which 1: Q^T (for dK); k = pair rows 16 ks ..
    constexpr int PT = 6, NOP = 8 * HT;
    bf16x8 ta[PT];
    auto read_t = [&](int i) __attribute__((always_inline)) {
      const int ks = i / (2 * HT), et = xh * HT + (i % (2 * HT)) / 2, base = (i % 2 ? QO : GO) + ks * RB;
      ta[i % PT] = lds_tr<D>(smem, at.tr(0, et) + base, at.tr(1, et) + base);
    };
#pragma unroll
    for (int i = 0; i < PT; ++i) read_t(i);
    sched_fence();
    // P = exp(S - L), dS = P (dP - D).  A lane past the end of the keys (its K and V rows are zero) computes values that
    // stay in its own columns of dK^T and dV^T, which are written as zeros.
    const int e0 = key - sq.pos - qt * kBlk - 32 * xh;   // distance of this wave's first query
    if constexpr (BIAS) {
      if (__any(e0 > -far && e0 - 31 < far)) {
#pragma unroll
        for (int r = 0; r < 16; ++r) sm[r] = fast_exp2(fmaf(sm[r], sl2, bmid[e0 - 4 * g - 27 + (27 - c_row(r, 0))]));
      } else {
        const float bc = bmid[e0 < 0 ? -far : far];
#pragma unroll
        for (int r = 0; r < 16; ++r) sm[r] = fast_exp2(fmaf(sm[r], sl2, bc));
      }
      int last = sq.nq - qt * kBlk - 32 * xh;   // rows past the end: a large bias may be infinity there
      if (last < 32) {
        asm volatile("" : "+v"(last));
#pragma unroll
        for (int r = 0; r < 16; ++r)
          if (c_row(r, g) >= last) sm[r] = 0.0f;
      }
    } else {
#pragma unroll
      for (int r = 0; r < 16; ++r) sm[r] = fast_exp2(sm[r] * sl2);
    }
    if (a.causal && __any(e0 > 0)) {   // queries before the key
      int first = e0;
      asm volatile("" : "+v"(first));
#pragma unroll
      for (int r = 0; r < 16; ++r)
        if (c_row(r, g) < first) sm[r] = 0.0f;
    }
#pragma unroll
    for (int r = 0; r < 16; ++r) dp[r] *= sm[r];
#pragma unroll
    for (int u = 0; u < 2; ++u) {
      *reinterpret_cast<bf16x8*>(smem + xw + (2 * u) * 1024) = c_to_operand(sm, u);
      *reinterpret_cast<bf16x8*>(smem + xw + (2 * u + 1) * 1024) = c_to_operand(dp, u);
    }
    __syncthreads();   // P and dS of all 64 queries are there for both waves of the key half
    bf16x8 pb[4], sb[4];
#pragma unroll
    for (int ks = 0; ks < 4; ++ks) {
      pb[ks] = lds_row(smem, xr + (2 * ks) * 1024);
      sb[ks] = lds_row(smem, xr + (2 * ks + 1) * 1024);
    }
    sched_fence();
#pragma unroll
    for (int i = 0; i < NOP; ++i) {
      const int ks = i / (2 * HT), dt = (i % (2 * HT)) / 2;
      if (i % 2 == 0) dvT[dt] = mfma32(ta[i % PT], pb[ks], dvT[dt]);   // dO_i^T P
      else dkT[dt] = mfma32(ta[i % PT], sb[ks], dkT[dt]);              // Q_i^T dS
      if (i + PT < NOP) read_t(i + PT);
      sched_fence();
    }
    if constexpr (BIAS) {
      if (turned) {   // the next step is of another head (its bias is read behind the next barrier)
        __syncthreads();
        expand_bias(a, ch, bias);
      }
    }
  };
  for (int s = s_beg; s < s_end; s += 2) {
    step(s, b0);
    if (s + 1 < s_end) step(s + 1, b1);
  }
  wait_vm0_known();        // the last step's surplus request has landed
  if (cut) {
    f32x4* o = key_slot<D>(kp, ((size_t)bh * kp.tiles + j) * kp.pieces + p, wu, l);
#pragma unroll
    for (int dt = 0; dt < HT; ++dt)
#pragma unroll
      for (int r4 = 0; r4 < 4; ++r4) {
        o[(4 * dt + r4) * 64] = f32x4{dvT[dt][4 * r4], dvT[dt][4 * r4 + 1], dvT[dt][4 * r4 + 2], dvT[dt][4 * r4 + 3]};
        o[(4 * (HT + dt) + r4) * 64] = f32x4{dkT[dt][4 * r4], dkT[dt][4 * r4 + 1], dkT[dt][4 * r4 + 2], dkT[dt][4 * r4 + 3]};
      }
    return;
  }
  __syncthreads();   // every wave is done with the tiles
  store_keys<D>(a, gr, smem + wu * Lds::STG, dvT, dkT, b, hk, j, kh, xh, kok, dk_scale(a, sq), l);
}

// dK, dV of the key tiles whose steps were cut: the sums of the pieces in order.  Bound by its traffic.
template <int D>
__global__ __launch_bounds__(256) void attn_kv_join_kernel(Attn a, AttnGrads gr, KeyPlan kp) {
  constexpr int HT = D / 64, NQ = 2 * HT * 4;
  extern __shared__ __attribute__((aligned(16))) unsigned char smem[];
  const int tid = threadIdx.x, w = tid >> 6, l = tid & 63, kh = w & 1, xh = w >> 1;
  const int bh = blockIdx.x / kp.tiles, j = blockIdx.x - bh * kp.tiles, b = bh / a.Hkv, hk = bh - b * a.Hkv;
  const Seq sq = seq_of(a, b);
  const int total = key_steps(a, sq, j).total;
  if (total <= kp.piece) return;
  const int np = (total + kp.piece - 1) / kp.piece;
  f32x4 s[NQ];
  const size_t slot = (size_t)blockIdx.x * kp.pieces;
#pragma unroll
  for (int q = 0; q < NQ; ++q) s[q] = key_slot<D>(kp, slot, w, l)[q * 64];
  for (int e = 1; e < np; e += 2) {   // (two in flight; past the end: the last again, not added)
    f32x4 x[2][NQ];
#pragma unroll
    for (int k = 0; k < 2; ++k) {
      const f32x4* y = key_slot<D>(kp, slot + min(e + k, np - 1), w, l);
#pragma unroll
      for (int q = 0; q < NQ; ++q) x[k][q] = y[q * 64];
    }
    const bool two = e + 1 < np;
#pragma unroll
    for (int q = 0; q < NQ; ++q) {
      s[q] += x[0][q];
      if (two) s[q] += x[1][q];
    }
  }
  f32x16 dvT[HT], dkT[HT];
#pragma unroll
  for (int dt = 0; dt < HT; ++dt)
#pragma unroll
    for (int r = 0; r < 16; ++r) {
      dvT[dt][r] = s[4 * dt + r / 4][r % 4];
      dkT[dt][r] = s[4 * (HT + dt) + r / 4][r % 4];
    }
  store_keys<D>(a, gr, smem + wave_uniform(w) * DkLds<D>::STG, dvT, dkT, b, hk, j, kh, xh,
                j * kBlk + kh * 32 + (l & 31) < sq.nk, dk_scale(a, sq), l);
}

template <int D>
hipError_t backward_impl(const Attn& a, const AttnGrads& g, char* ws, hipStream_t st) {
  const BwdPlan p = attn_bwd_plan(a, ws);
  {
    const int lds = dq_lds<D>(a);
    auto kern = a.has_bias() ? attn_dq_kernel<D, true> : attn_dq_kernel<D, false>;
    SLA_TRY(ensure_dyn_lds(kern, lds));
    KernelTimer kt("attn_dq", st);
    kern<<<p.map.blocks(), 256, lds, st>>>(a, g, (RowStat*)p.stat, p.tpart, p.map);
  }
  const int tables = g.dtable ? a.H : 0, grid = p.key.blocks * p.key.pieces + tables;
  if (grid == 0) return hipGetLastError();
  {
    const int lds = DkLds<D>::BIAS + (a.has_bias() ? bias_width(a.bias.far) * 4 : 0);
    auto kern = a.has_bias() ? attn_dkdv_kernel<D, true> : attn_dkdv_kernel<D, false>;
    SLA_TRY(ensure_dyn_lds(kern, lds));
    KernelTimer kt("attn_dkdv", st);
    kern<<<grid, 256, lds, st>>>(a, g, (const RowStat*)p.stat, p.key, p.tpart, p.qparts);
  }
  if (p.key.pieces > 1) {
    KernelTimer kt("attn_kv_join", st);
    attn_kv_join_kernel<D><<<a.B * a.Hkv * p.key.tiles, 256, 4 * DkLds<D>::STG, st>>>(a, g, p.key);
  }
  return hipGetLastError();
}

}  // namespace

hipError_t attn_backward_bf16(const Attn& a, const AttnGrads& g, char* ws, hipStream_t st) {
  return a.d == 64 ? backward_impl<64>(a, g, ws, st) : backward_impl<128>(a, g, ws, st);
}

}  // namespace sla
