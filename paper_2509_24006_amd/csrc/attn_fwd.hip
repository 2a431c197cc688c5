// bf16 softmax attention, forward pass on the matrix cores: online softmax over tiles of 64 keys.
//
// Work is cut into row tiles of 64 queries.  With many queries the rows of a tile are consecutive queries of one head.
// With few (fewer than 64, or behind a shared prefix) they are packed: the queries of all heads that share a K, V
// head, and for the prefix those of all sequences too, so that a key is fetched once for everything that reads it.
// Where row tiles alone would not fill the chip the keys are cut as well (parts): every workgroup leaves unnormalised
// float sums with its maximum and sum, and attn_join_kernel weighs and adds them.
//
// A workgroup is four waves: wave (qh, par) takes 32 of the 64 rows and 32 of a tile's 64 keys.  Everything is held
// transposed (S^T = K Q^T, O^T = V^T P^T), so that a lane owns one row: its statistics, its position, its number
// of keys and its head are per-lane scalars, and P goes from C registers straight into the second product.  Each wave runs
// its own online softmax over its keys; the two streams of a row meet at the end.  P enters the second product
// rounded to bf16 (the matrix cores' operand); its sum is taken before the rounding, in float.
#include <type_traits>

#include "attn_rows.h"

namespace sla {
namespace {

template <int D>
struct AttnLds {
  // Slot 2p holds the K tile and slot 2p + 1 the V tile of the steps of parity p; Q comes in through V_1's slot.
  static constexpr int TILE = SwzTile<D>::BYTES;
  static constexpr int STAT = 4 * TILE;         // statistics of the four waves (1 KB)
  static constexpr int ROWQ = STAT + 1024;      // byte offsets of the 64 rows of Q (-1: none)
  static constexpr int ROWO = ROWQ + 256;       // offsets of the 64 rows of O in 16-byte units (-1: none)
  static constexpr int BIAS = ROWO + 256;       // per head of the tile: bias in log2 units by distance (bias_width floats)
};

// PART: the workgroup leaves sums for attn_join_kernel.  (d = 128 with a bias: 13 registers spill at two workgroups per CU, 17 with PART.)
template <int D, bool BIAS, bool PART>
__global__ __launch_bounds__(256, 2) void attn_fwd_kernel(Attn a, AttnPlan plan, float c2) {
  using Lds = AttnLds<D>;
  using T = SwzTile<D>;
  constexpr int NT = D / 32, KT = D / 16, HT = NT / 2;
  extern __shared__ __attribute__((aligned(16))) unsigned char smem[];
  const int tid = threadIdx.x, w = tid >> 6, l = tid & 63, g = l >> 5, ln = l & 31;
  const int qh = w & 1, par = w >> 1;

  FwdTile x;
  if (!x.template open<PART>(a, plan)) return;
  const AttnPart& pt = x.pre ? plan.prefix : plan.own;
  const int steps = x.steps, h0 = x.h0;
  const RowOf row = x.row(a, pt, qh * 32 + ln);   // this lane's
  const RowKeys rk = row_keys(a, x, row);
  const bool live = rk.live;
  const int posk = rk.pos, lim = rk.lim;
  // 32-bit offsets of the tile's rows, from the unit's first row or, where a unit is one head, the tile's
  const RowOf first = {max(x.ub, 0), 0, pt.packed ? 0 : x.r0, true};
  const long long qbase = x.at(a.Q, first), obase = x.at(a.O, first);
  int* const rowq = reinterpret_cast<int*>(smem + Lds::ROWQ);
  int* const rowo = reinterpret_cast<int*>(smem + Lds::ROWO);
  if (tid < kBlk) {
    const RowOf r = x.row(a, pt, tid);
    rowq[tid] = r.in && r.n < seq_of(a, r.b).nq ? (int)(2 * (x.at(a.Q, r) - qbase)) : -1;
    rowo[tid] = r.in ? (int)((x.at(a.O, r) - obase) >> 3) : -1;
  }
  float* const bias = reinterpret_cast<float*>(smem + Lds::BIAS);
  const int far = a.bias.far, width = bias_width(far);
  if constexpr (BIAS) {
    for (int i = tid; i < pt.heads * width; i += 256) {
      const int hg = i / width;
      bias[i] = table_at(a, bucket_of(a.bias, i - hg * width - far - kBiasPad), h0 + hg) * kLog2e;
    }
  }
  __syncthreads();

  f32x16 oT[NT];
#pragma unroll
  for (int et = 0; et < NT; ++et) oT[et] = zero_f32x16();
  float m = -INFINITY, lsum = 0.0f;
  const View &VK = x.pre ? a.Kp : a.K, &VV = x.pre ? a.Vp : a.V;
  RunLoader<D> tk, tv;
  tk.init(lds_base(smem), w, l, 2 * VK.sn, kBlk);
  tv.init(lds_base(smem), w, l, 2 * VV.sn, kBlk);
  constexpr int IPW = RunLoader<D>::IPW, QSLOT = 3 * Lds::TILE;
  // the descriptors span this workgroup's keys up to the last valid one: rows behind it read as zeros
  auto rsrc = [&](const View& v) {
    return tile_rsrc(reinterpret_cast<const bf16*>(v.p) + x.key_at(v), (x.keys() - 1) * 2 * v.sn + 2 * D);
  };
  const BufDesc descK = rsrc(VK), descV = rsrc(VV);
  {
    const BufDesc dq = tile_rsrc(reinterpret_cast<const bf16*>(a.Q.p) + qbase, 0x7fff0000);
    const int qr = T::RPI * w + l / T::CPR, chunk = ((l % T::CPR) ^ swz<D>(qr)) << 4;
#pragma unroll
    for (int k = 0; k < IPW; ++k) {   // (16 rows or a multiple of it further each time: the same swizzle)
      const int o = rowq[qr + 4 * T::RPI * k];
      load_to_lds16(dq, o < 0 ? (int)kPastEnd : o + chunk, 0, lds_base(smem) + QSLOT + wave_uniform(w) * 1024 + 4096 * k);
    }
  }
  if (steps > 0) {
    tk.template load<0>(descK, 0);
    tv.template load<Lds::TILE>(descV, 0);
    if (steps > 1) tk.template load<2 * Lds::TILE>(descK, tk.tile_step);
  }
  // per-lane LDS offsets of the operand reads inside a tile; accumulator tile et holds feature tile et ^ rot: the half
  // of the features that the wave finishes by itself comes first
  const int rot = wave_uniform(par) * HT;
  int kaddr[KT], vaddr[2][NT];
  {
    TileAddr<D> ad;
    ad.init(32 * par, l);
#pragma unroll
    for (int t = 0; t < KT; ++t) {
      kaddr[t] = ad.row(t);
      asm volatile("" : "+v"(kaddr[t]));
    }
#pragma unroll
    for (int h = 0; h < 2; ++h)
#pragma unroll
      for (int et = 0; et < NT; ++et) {
        vaddr[h][et] = ad.tr(h, et ^ rot);
        asm volatile("" : "+v"(vaddr[h][et]));
      }
  }
  tk.pin();
  tv.pin();
  // The scores of a step are formed one step ahead: their products run under the exponentials of the current step.
  f32x16 sT = zero_f32x16();
  bf16x8 qf[KT], k0[KT];
  if (steps > 1) wait_vm<2 * IPW>();   // Q and K_0 have landed; V_0 and K_1 may stay in flight
  else wait_vm0();
  __syncthreads();
  {
    TileAddr<D> qa;
    qa.init(32 * qh, l);
#pragma unroll
    for (int t = 0; t < KT; ++t) qf[t] = lds_row(smem, qa.row(t) + QSLOT);
#pragma unroll
    for (int t = 0; t < KT; ++t) k0[t] = lds_row(smem, kaddr[t]);   // (without steps: not used)
  }
#pragma unroll
  for (int t = 0; t < KT; ++t) pin_loaded(qf[t]);
#pragma unroll
  for (int t = 0; t < KT; ++t) pin_loaded(k0[t]);
  __syncthreads();                     // every wave holds its rows of both: the slots take V_1 and K_2
  if (steps > 1) {
    tv.template load<3 * Lds::TILE>(descV, tv.tile_step);
    if (steps > 2) tk.template load<0>(descK, 2 * tk.tile_step);
  }
  if (steps > 0) {
#pragma unroll
    for (int t = 0; t < KT; ++t) sT = mfma32(k0[t], qf[t], sT);
    if (steps > 2) wait_vm<2 * IPW>();    // V_0 and K_1 have landed
    else wait_vm0();
    __syncthreads();
  }
  const float cs = BIAS ? 1.0f : c2;              // the scores' factor in the exponent of 2
  const float* const brow = bias + (BIAS ? row.g * width + far + kBiasPad : 0);   // at distance 0
  int key0 = x.t0 * kBlk + 32 * wave_uniform(par);  // first key of this wave in the current tile
  unsigned koff = 3u * (unsigned)tk.tile_step, voff = 2u * (unsigned)tv.tile_step;
  // One step; P = parity of s.  On entry K_{s+1} and V_s are in their slots for every wave and sT holds S_s; sN
  // receives S_{s+1}.  The wave copies its operands to registers first; a second barrier then frees both slots for
  // K_{s+3} and V_{s+2}.  MID: s + 3 < steps, where every condition holds.
  auto step = [&](auto Pc, auto Mid, int s, f32x16& sT, f32x16& sN) __attribute__((always_inline)) {
    constexpr int P = decltype(Pc)::value;
    constexpr bool MID = decltype(Mid)::value;
    constexpr int VS = (2 * P + 1) * Lds::TILE;    // V_s, then V_{s+2}
    constexpr int KN = 2 * (1 - P) * Lds::TILE;    // K_{s+1}, then K_{s+3}
    bf16x8 ka[KT], va[2][NT];
#pragma unroll
    for (int t = 0; t < KT; ++t) ka[t] = lds_row(smem, kaddr[t] + KN);
#pragma unroll
    for (int u = 0; u < 2; ++u)
#pragma unroll
      for (int et = 0; et < NT; ++et)
        va[u][et] = lds_tr<D>(smem, vaddr[0][et] + VS + u * 16 * T::ROW_BYTES, vaddr[1][et] + VS + u * 16 * T::ROW_BYTES);
    if constexpr (BIAS) {
      // Distances of far and more share a bucket: away from the diagonal the bias is one value per row.
      const int d0 = key0 - posk;   // distance of this wave's first key
      if (__any(d0 + 31 > -far && d0 < far)) {
        // (queries of a packed tile may be far apart; those of others are neighbours, within the padding)
        const float* const b0 = brow + (PART || pt.packed ? min(max(d0, -far - 31), far) : d0) + 4 * g;
#pragma unroll
        for (int r = 0; r < 16; ++r) sT[r] = fmaf(sT[r], c2, b0[c_row(r, 0)]);
      } else {
        const float bc = brow[d0 < 0 ? -far : far];
#pragma unroll
        for (int r = 0; r < 16; ++r) sT[r] = fmaf(sT[r], c2, bc);
      }
    }
    if (__any(lim < key0 + 32)) {
      int first = lim - key0;
      asm volatile("" : "+v"(first));   // (the comparisons stay inside the branch)
#pragma unroll
      for (int r = 0; r < 16; ++r)
        if (c_row(r, g) >= first) sT[r] = -INFINITY;
    }
    float mx = sT[0];
#pragma unroll
    for (int r = 1; r < 16; ++r) mx = fmaxf(mx, sT[r]);
    mx = half_max(mx);
    const float mnew = fmaxf(m, mx);
    // The reference point of the exponentials follows the running maximum lazily (P is then at most 2^kLazy instead
    // of 1), so that the accumulators are rescaled on few steps.
    constexpr float kLazy = 8.0f;
    if (__any((mnew - m) * cs > kLazy)) {
      const float alpha = mnew == -INFINITY ? 1.0f : fast_exp2((m - mnew) * cs);   // (no key yet: nothing to scale)
      lsum *= alpha;
#pragma unroll
      for (int et = 0; et < NT; ++et)
#pragma unroll
        for (int r = 0; r < 16; ++r) oT[et][r] *= alpha;
      m = mnew;
    }
    const float moff = m == -INFINITY ? 0.0f : -m * cs;
    __syncthreads();   // every wave holds its operands of this step: both slots are refilled
    if (MID || s + 3 < steps) tk.template load<KN>(descK, (int)koff);
    if (MID || s + 2 < steps) tv.template load<VS>(descV, (int)voff);
    koff += tk.tile_step;
    voff += tv.tile_step;
    key0 += kBlk;
    sched_fence();
    sN = zero_f32x16();
#pragma unroll
    for (int t = 0; t < KT; ++t) {
      sN = mfma32(ka[t], qf[t], sN);   // (in the last step: of a slot that holds no tile, unused)
#pragma unroll
      for (int r = t * (16 / KT); r < (t + 1) * (16 / KT); ++r) sT[r] = fast_exp2(fmaf(sT[r], cs, moff));
    }
    float psum = 0.0f;
#pragma unroll
    for (int u = 0; u < 2; ++u) {
      const bf16x8 pf = c_to_operand(sT, u);
#pragma unroll
      for (int e = 0; e < 8; ++e) psum += sT[8 * u + e];
#pragma unroll
      for (int et = 0; et < NT; ++et) oT[et] = mfma32(va[u][et], pf, oT[et]);
    }
    lsum += psum;
    sched_fence();     // (the products above are issued before this wait)
    // K_{s+2} and V_{s+1} have landed; what this step requested may stay in flight
    if (MID || s + 1 < steps) {
      if (MID || s + 3 < steps) wait_vm<2 * IPW>();
      else if (s + 2 < steps) wait_vm<IPW>();
      else wait_vm0();
      __syncthreads();
    }
  };
  {
    const std::integral_constant<int, 0> p0;
    const std::integral_constant<int, 1> p1;
    const std::integral_constant<bool, true> mid;
    const std::integral_constant<bool, false> any;
    f32x16 sU = zero_f32x16();
    int s = 0;
    for (; s + 4 < steps; s += 2) {
      step(p0, mid, s, sT, sU);
      step(p1, mid, s + 1, sU, sT);
    }
    for (; s < steps; s += 2) {
      step(p0, any, s, sT, sU);
      if (s + 1 < steps) step(p1, any, s + 1, sU, sT);
    }
  }
  // ---- the two waves of a row hold sums over different keys of all features; each finishes half of the features
  lsum = half_sum(lsum);
  float* const ml = reinterpret_cast<float*>(smem + Lds::STAT);   // [par][qh][32][2]
  if (g == 0) {
    ml[((par * 2 + qh) * 32 + ln) * 2 + 0] = m;
    ml[((par * 2 + qh) * 32 + ln) * 2 + 1] = lsum;
  }
  __syncthreads();   // also: all waves are done with the K, V tiles
  const float m_o = ml[(((par ^ 1) * 2 + qh) * 32 + ln) * 2 + 0];
  const float l_o = ml[(((par ^ 1) * 2 + qh) * 32 + ln) * 2 + 1];
  const float mstar = fmaxf(m, m_o);
  // the row has seen a key, or scores that are no numbers, which a maximum passes over
  const bool some = live && (mstar != -INFINITY || __builtin_isnan(lsum + l_o));
  const float a_me = some ? fast_exp2((m - mstar) * cs) : 0.0f, a_ot = some ? fast_exp2((m_o - mstar) * cs) : 0.0f;
  const float ltot = lsum * a_me + l_o * a_ot;
  const float cw = PART ? a_me : some ? a_me / ltot : 0.0f;
#pragma unroll
  for (int et = 0; et < NT; ++et)
#pragma unroll
    for (int r = 0; r < 16; ++r) oT[et][r] = some ? oT[et][r] * cw : 0.0f;
  float* const xch = reinterpret_cast<float*>(smem + qh * Lds::TILE);
#pragma unroll
  for (int h2 = 0; h2 < HT; ++h2)
#pragma unroll
    for (int r4 = 0; r4 < 4; ++r4)
      *reinterpret_cast<f32x4*>(xch + par * (Lds::TILE / 8) + ((h2 * 4 + r4) * 64 + l) * 4) =
          f32x4{oT[HT + h2][4 * r4], oT[HT + h2][4 * r4 + 1], oT[HT + h2][4 * r4 + 2], oT[HT + h2][4 * r4 + 3]};
  __syncthreads();
#pragma unroll
  for (int h2 = 0; h2 < HT; ++h2)
#pragma unroll
    for (int r4 = 0; r4 < 4; ++r4) {
      const f32x4 xv = *reinterpret_cast<const f32x4*>(xch + (par ^ 1) * (Lds::TILE / 8) + ((h2 * 4 + r4) * 64 + l) * 4);
#pragma unroll
      for (int r = 0; r < 4; ++r) oT[h2][4 * r4 + r] += xv[r];
    }
  f32x16 (&o)[HT] = *reinterpret_cast<f32x16 (*)[HT]>(&oT[0]);
  if constexpr (PART) {
    // rows of D floats, and (maximum in log2 units, sum) of every row; without a key the sum is 0 and the row is not read
    const size_t slot = x.slot(pt);
    if (row.in) {
      const int r = qh * 32 + ln;
      float* const po = plan.part + (slot * kBlk + r) * D + (par ? D / 2 : 0) + 4 * g;
      if (some) {
#pragma unroll
        for (int h2 = 0; h2 < HT; ++h2)
#pragma unroll
          for (int r4 = 0; r4 < 4; ++r4)
            *reinterpret_cast<f32x4*>(po + 32 * h2 + 8 * r4) =
                f32x4{o[h2][4 * r4], o[h2][4 * r4 + 1], o[h2][4 * r4 + 2], o[h2][4 * r4 + 3]};
      }
      if (par == 0 && g == 0) *reinterpret_cast<float2*>(plan.stat + (slot * kBlk + r) * 2) = float2{mstar * cs, some ? ltot : 0.0f};
    }
  } else {
    if (a.L && par == 0 && g == 0 && row.in)
      a.L[((size_t)row.b * a.H + h0 + row.g) * a.Nq + row.n] = some ? mstar * cs * kLn2 + logf(ltot) : -INFINITY;
    // rows of bf16 through LDS, so that they leave in 16-byte pieces of whole rows (the exchange lies in slots 0, 1)
    constexpr int PB = 64 * HT + 16, PPR = 4 * HT;
    unsigned char* const stage = smem + (2 + qh) * Lds::TILE + par * (Lds::TILE / 2);
    static_assert(32 * PB <= Lds::TILE / 2, "staging of two waves fits in a tile slot");
#pragma unroll
    for (int t = 0; t < HT; ++t)
#pragma unroll
      for (int r4 = 0; r4 < 4; ++r4) {
        bf16x4 pk;
#pragma unroll
        for (int r = 0; r < 4; ++r) pk[r] = (__bf16)o[t][4 * r4 + r];
        *reinterpret_cast<bf16x4*>(stage + ln * PB + (32 * t + 8 * r4 + 4 * g) * 2) = pk;
      }
    bf16* const O = reinterpret_cast<bf16*>(a.O.p) + obase + (par ? D / 2 : 0);
#pragma unroll
    for (int it = 0; it < 32 * PPR / 64; ++it) {
      const int idx = it * 64 + l, r = idx / PPR, pc = idx % PPR;
      const u32x4 v = *reinterpret_cast<const u32x4*>(stage + r * PB + pc * 16);
      const int off = rowo[32 * qh + r];
      if (off >= 0) *reinterpret_cast<u32x4*>(O + (size_t)off * 8 + pc * 8) = v;
    }
  }
}

template <int D>
hipError_t forward_impl(const Attn& a, const AttnPlan& plan, hipStream_t st) {
  const float c2 = a.scale * kLog2e;
  const AttnPart& ow = plan.own;
  auto launch = [&](auto kern, dim3 grid, const char* name) -> hipError_t {
    const int lds = AttnLds<D>::BIAS + (a.has_bias() ? ow.heads * bias_width(a.bias.far) * 4 : 0);
    SLA_TRY(ensure_dyn_lds(kern, lds));
    KernelTimer kt(name, st);
    kern<<<grid, 256, lds, st>>>(a, plan, c2);
    return hipGetLastError();
  };
  if (!plan.parts) {
    const dim3 grid(plan.map.blocks());
    return a.has_bias() ? launch(attn_fwd_kernel<D, true, false>, grid, "attn_fwd") : launch(attn_fwd_kernel<D, false, false>, grid, "attn_fwd");
  }
  const dim3 grid(plan.prefix.blocks + ow.blocks);
  return a.has_bias() ? launch(attn_fwd_kernel<D, true, true>, grid, "attn_parts") : launch(attn_fwd_kernel<D, false, true>, grid, "attn_parts");
}

}  // namespace

hipError_t attn_forward_bf16(const Attn& a, const AttnPlan& plan, hipStream_t st) {
  SLA_TRY(a.d == 64 ? forward_impl<64>(a, plan, st) : forward_impl<128>(a, plan, st));
  return plan.parts ? attn_join(a, plan, st) : hipSuccess;
}

}  // namespace sla
