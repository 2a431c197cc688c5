// Float softmax attention on the float matrix instructions: every product and every sum in float.  Operand layouts and
// tiles as in mfma_f32_common.h: a lane owns one token (lane % 16) and a quarter of its features, and a C tile is the
// next product's operand as it stands.  Bound by the float matrix rate and the operand reads from LDS.
#include "attn_bwd.h"
#include "attn_rows.h"
#include "mfma_f32_common.h"

namespace sla {
namespace {

template <int D>
__device__ __forceinline__ BufDesc rows_rsrc(const View& v, int b, int h, int n) {
  return head_rsrc_f32<D>(reinterpret_cast<const float*>(v.p) + (size_t)b * v.sb + (size_t)h * v.sh, max(n, 1), 4 * v.sn);
}
__device__ __forceinline__ float* row_ptr(const View& v, int b, int h, int n) {
  return reinterpret_cast<float*>(v.p) + (size_t)b * v.sb + (size_t)h * v.sh + (size_t)n * v.sn;
}
// bias by distance, 2 far + 1 floats
__device__ __forceinline__ void expand_bias(const Attn& a, int h, float* out) {
  for (int i = threadIdx.x; i <= 2 * a.bias.far; i += 256) out[i] = table_at(a, bucket_of(a.bias, i - a.bias.far), h);
}
__device__ __forceinline__ float bias_at(const float* bias, int far, int d) { return bias[min(max(d, -far), far) + far]; }

// mm_rows and mm_over with the operands of the next group read ahead of the products of this one: left alone, the compiler
// reads a group's operands right before its products, and each group waits an LDS latency.  (2 x 16 heads x 500, d = 64,
// forward / query / key side 31.7 / 40.3 / 51.0 -> 30.7 / 38.9 / 49.9 us; 4 x 1950, d = 128, 92.3 / 131.4 / 168 -> 91.4 / 128 / 168.)
template <int D, int NR, int NT>
__device__ __forceinline__ void rows_ahead(const FAddr<D>& ad, const unsigned char* tile, const f32x4 (&b)[NT], f32x4 (&acc)[NR]) {
  f32x4 x[2][NR];
#pragma unroll
  for (int r = 0; r < NR; ++r) x[0][r] = ad.row(tile, 16 * r, 0);
#pragma unroll
  for (int t = 0; t < NT; ++t) {
    if (t + 1 < NT)
#pragma unroll
      for (int r = 0; r < NR; ++r) x[(t + 1) & 1][r] = ad.row(tile, 16 * r, t + 1);
    sched_fence();
#pragma unroll
    for (int s = 0; s < 4; ++s)
#pragma unroll
      for (int r = 0; r < NR; ++r) acc[r] = mfma16(x[t & 1][r][s], b[t][s], acc[r]);
    sched_fence();
  }
}
template <int D, int NK, int NF>
__device__ __forceinline__ void over_ahead(const FAddr<D>& ad, const unsigned char* tile, const f32x4 (&b)[NK], f32x4 (&acc)[NF]) {
  float x[2][NF];
#pragma unroll
  for (int f = 0; f < NF; ++f) x[0][f] = ad.over(tile, 0, 0, f);
#pragma unroll
  for (int q = 0; q < 4 * NK; ++q) {
    if (q + 1 < 4 * NK)
#pragma unroll
      for (int f = 0; f < NF; ++f) x[(q + 1) & 1][f] = ad.over(tile, 16 * ((q + 1) / 4), (q + 1) % 4, f);
    sched_fence();
#pragma unroll
    for (int f = 0; f < NF; ++f) acc[f] = mfma16(x[q & 1][f], b[q / 4][q % 4], acc[f]);
    sched_fence();
  }
}

// ------------------------------------------------------------------ forward
// A wave takes 16 of the workgroup's 64 rows.  K and V go through one slot each: V_s lands under the scores of step s,
// K_{s+1} under its second product.  PART: sums for attn_join_kernel, as in the bf16 path.
template <int D, bool BIAS, bool PART>
__global__ __launch_bounds__(256, 2) void attn_f32_fwd_kernel(Attn a, AttnPlan plan) {
  constexpr int NT = D / 16, TB = FTile<D>::BYTES;
  extern __shared__ __attribute__((aligned(16))) unsigned char smem[];
  const int tid = threadIdx.x, w = wave_uniform(tid >> 6), l = tid & 63, g = l >> 4, n = l & 15;
  FwdTile x;
  if (!x.template open<PART>(a, plan)) return;
  const AttnPart& pt = x.pre ? plan.prefix : plan.own;
  const RowOf row = x.row(a, pt, 16 * w + n);
  const RowKeys rk = row_keys(a, x, row);
  const View &VK = x.pre ? a.Kp : a.K, &VV = x.pre ? a.Vp : a.V;
  FLoader<D> lk, lv;
  lk.init(lds_base(smem), w, l, 4 * VK.sn);
  lv.init(lds_base(smem), w, l, 4 * VV.sn);
  auto rsrc = [&](const View& v) { return head_rsrc_f32<D>(reinterpret_cast<const float*>(v.p) + x.key_at(v), x.keys(), 4 * v.sn); };
  const BufDesc dK = rsrc(VK), dV = rsrc(VV);
  if (x.steps > 0) {
    lk.load(dK, 0, 0);
    lv.load(dV, 0, TB);
  }
  f32x4 qf[NT], acc[NT];
  load_frag<NT>(reinterpret_cast<const float*>(a.Q.p) + x.at(a.Q, row), rk.live, g, qf);
  float* const bias = reinterpret_cast<float*>(smem + 2 * TB);
  const int far = a.bias.far, width = 2 * far + 1;
  const float* const brow = bias + row.g * width;
  if constexpr (BIAS) {
    for (int i = tid; i < pt.heads * width; i += 256) {
      const int hg = i / width;
      bias[i] = table_at(a, bucket_of(a.bias, i - hg * width - far), x.h0 + hg);
    }
  }
#pragma unroll
  for (int t = 0; t < NT; ++t) acc[t] = zero4();
  float m = -INFINITY, lsum = 0.0f;
  FAddr<D> ad;
  ad.init(l);
  wait_vm0();
  __syncthreads();
  for (int s = 0; s < x.steps; ++s) {
    const int key0 = (x.t0 + s) * kBlk;
    const bool last = s + 1 == x.steps;
    f32x4 p[4];
#pragma unroll
    for (int kt = 0; kt < 4; ++kt) p[kt] = zero4();
    rows_ahead<D, 4, NT>(ad, smem, qf, p);     // S^T: registers = keys 16 kt + 4 g + r, lane = row
    wait_vm0();
    __syncthreads();                        // V_s is there, the K slot is free
    if (!last) lk.load(dK, s + 1, 0);
    float mx = -INFINITY;
#pragma unroll
    for (int kt = 0; kt < 4; ++kt)
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        const int key = key0 + 16 * kt + 4 * g + r;
        float v = p[kt][r] * a.scale;
        if constexpr (BIAS) v += bias_at(brow, far, key - rk.pos);
        p[kt][r] = key < rk.lim ? v : -INFINITY;
        mx = fmaxf(mx, p[kt][r]);
      }
    const float mnew = fmaxf(m, tok_max(mx)), ref = mnew == -INFINITY ? 0.0f : mnew;
    f32x4 sum = zero4();
#pragma unroll
    for (int kt = 0; kt < 4; ++kt)
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        p[kt][r] = expf(p[kt][r] - ref);
        sum[r] += p[kt][r];
      }
    const float alpha = expf(m - ref);
    lsum = alpha * lsum + tok_sum((sum[0] + sum[1]) + (sum[2] + sum[3]));
    m = mnew;
#pragma unroll
    for (int t = 0; t < NT; ++t)
#pragma unroll
      for (int r = 0; r < 4; ++r) acc[t][r] *= alpha;
    over_ahead<D, 4, NT>(ad, smem + TB, p, acc);   // O^T += V^T P^T
    wait_vm0();
    __syncthreads();                        // K_{s+1} is there, the V slot is free
    if (!last) lv.load(dV, s + 1, TB);
  }
  if (!row.in) return;
  const bool some = rk.live && lsum != 0.0f;   // (also where it is no number)
  if constexpr (PART) {
    const size_t at = x.slot(pt) * kBlk + 16 * w + n;
    if (some) store_frag<NT>(plan.part + at * D, g, acc);
    if (g == 0) *reinterpret_cast<float2*>(plan.stat + at * 2) = float2{m * kLog2e, some ? lsum : 0.0f};
    return;
  }
  const float inv = 1.0f / lsum;
#pragma unroll
  for (int t = 0; t < NT; ++t)
#pragma unroll
    for (int r = 0; r < 4; ++r) acc[t][r] = some ? acc[t][r] * inv : 0.0f;
  store_frag<NT>(reinterpret_cast<float*>(a.O.p) + x.at(a.O, row), g, acc);
  if (a.L && g == 0) a.L[((size_t)row.b * a.H + x.h0 + row.g) * a.Nq + row.n] = some ? m + logf(lsum) : -INFINITY;
}

// ------------------------------------------------------------------ dQ
// Lane = query; D = rowsum(dO O).  A workgroup owns 64 / QW queries; the QW waves that share 16 of them split the 64 keys of
// every step, and their sums meet in LDS at the end: parts of a tile fill the chip where there are few tiles.  V_{s+1}
// lands under the scores and dQ of step s, K_{s+1} under dP of step s + 1.  The table's gradient: see
// table_part; the four quarters of a wave hold the same queries, so they add to the wave's array one after the other, which
// keeps the order of the additions fixed.
template <int D>
constexpr int f32_dq_lds(int far) { return 2 * FTile<D>::BYTES + 5 * (2 * far + 1) * 4 + 32; }

// the sums of the QW waves that share 16 tokens; wave wq gets the feature tiles wq, wq + QW, ...  x: [wave][tile][lane]
template <int QW, int NT>
__device__ __forceinline__ void add_shares(f32x4* x, const f32x4 (&part)[NT], int w, int l, f32x4 (&sum)[NT / QW]) {
#pragma unroll
  for (int f = 0; f < NT; ++f) x[(w * NT + f) * 64 + l] = part[f];
  __syncthreads();
#pragma unroll
  for (int m = 0; m < NT / QW; ++m) {
    sum[m] = zero4();
#pragma unroll
    for (int q = 0; q < QW; ++q) sum[m] += x[((w / QW * QW + q) * NT + w % QW + QW * m) * 64 + l];
  }
}

template <int D, int QW, bool BIAS>
__global__ __launch_bounds__(256, 2) void attn_f32_dq_kernel(Attn a, AttnGrads gr, float* __restrict__ Ds,
                                                              float* __restrict__ tpart, TileMap map) {
  constexpr int NT = D / 16, TB = FTile<D>::BYTES, NQ = 4 / QW, NO = NT / QW, ROWS = kBlk / QW;
  extern __shared__ __attribute__((aligned(16))) unsigned char smem[];
  const int tid = threadIdx.x, w = wave_uniform(tid >> 6), l = tid & 63, g = l >> 4, nl = l & 15;
  const int wk = w / QW, wq = w % QW;
  const TileOf own = map.at(blockIdx.x);
  if (own.i < 0) return;
  const int tiles = map.nb;
  const int bh = wave_uniform(own.bh), i = wave_uniform(a.causal ? tiles - 1 - own.i : own.i);
  const int b = bh / a.H, h = bh - b * a.H, hk = h / a.G;
  const Seq s = seq_of(a, b);
  const int q0 = i * ROWS, n = q0 + 16 * wk + nl, pos = s.pos + n;
  const bool in = n < a.Nq, live = n < s.nq;
  int limmax = q0 < s.nq ? s.nk : 0;
  if (a.causal) limmax = max(0, min(limmax, s.pos + min(q0 + ROWS, s.nq)));
  const int steps = wave_uniform((limmax + kBlk - 1) / kBlk);
  const int lim = !live ? 0 : a.causal ? max(0, min(s.nk, pos + 1)) : s.nk;
  FLoader<D> lk, lv;
  lk.init(lds_base(smem), w, l, 4 * a.K.sn);
  lv.init(lds_base(smem), w, l, 4 * a.V.sn);
  const BufDesc dK = rows_rsrc<D>(a.K, b, hk, s.nk), dV = rows_rsrc<D>(a.V, b, hk, s.nk);
  if (steps > 0) {
    lv.load(dV, 0, TB);
    lk.load(dK, 0, 0);
  }
  FAddr<D> ad;
  ad.init(l);
  const int nc = min(n, a.Nq - 1);
  f32x4 qf[NT], gf[NT], dq[NT];
  load_frag<NT>(row_ptr(a.Q, b, h, nc), live, g, qf);
  load_frag<NT>(row_ptr(gr.dO, b, h, nc), live, g, gf);
  float Dr;
  {
    f32x4 of[NT];
    load_frag<NT>(row_ptr(a.O, b, h, nc), live, g, of);
    Dr = dot_frag<NT>(gf, of);
    if (live && g == 0 && wq == 0) Ds[(size_t)bh * a.Nq + n] = Dr;
  }
  float Lr = live ? a.L[(size_t)bh * a.Nq + n] : 0.0f;
  if (Lr == -INFINITY || lim == 1) Lr = INFINITY;   // (P = 0: a row without a key, or with a single one, see dk_scale)
  float* const bias = reinterpret_cast<float*>(smem + 2 * TB);
  const int far = a.bias.far, width = 2 * far + 1;
  float* const dist = bias + width;   // [wave][width], then the far sums of the waves
  if constexpr (BIAS) {
    expand_bias(a, h, bias);
    for (int x = tid; x < 4 * width; x += 256) dist[x] = 0.0f;
  }
  float sumL = 0.0f, sumR = 0.0f;
#pragma unroll
  for (int t = 0; t < NT; ++t) dq[t] = zero4();
  const unsigned char* const Ks = smem + 16 * NQ * wq * FTile<D>::ROWB;   // this wave's keys
  const unsigned char* const Vs = Ks + TB;
  wait_vm0();
  __syncthreads();
  for (int j = 0; j < steps; ++j) {
    const bool more = j + 1 < steps;
    const int key0 = j * kBlk + 16 * NQ * wq;
    f32x4 p[NQ], dp[NQ];
#pragma unroll
    for (int kt = 0; kt < NQ; ++kt) p[kt] = dp[kt] = zero4();
    rows_ahead<D, NQ, NT>(ad, Vs, gf, dp);          // dP^T = V dO^T
    wait_vm0();
    __syncthreads();                             // K_j is there, the V slot is free
    if (more) lv.load(dV, j + 1, TB);
    rows_ahead<D, NQ, NT>(ad, Ks, qf, p);           // S^T = K Q^T
#pragma unroll
    for (int kt = 0; kt < NQ; ++kt)
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        const int key = key0 + 16 * kt + 4 * g + r;
        float v = p[kt][r] * a.scale - Lr;
        if constexpr (BIAS) v += bias_at(bias, far, key - pos);
        dp[kt][r] = key < lim ? expf(v) * (dp[kt][r] - Dr) : 0.0f;
      }
    if constexpr (BIAS) {
      const int d0 = key0 - pos;
      if (__any(d0 + 16 * NQ - 1 > -far && d0 < far)) {
#pragma unroll
        for (int kt = 0; kt < NQ; ++kt)
#pragma unroll
          for (int r = 0; r < 4; ++r) {
            const int d = d0 + 16 * kt + 4 * g + r;
            sumL += d <= -far ? dp[kt][r] : 0.0f;
            sumR += d >= far ? dp[kt][r] : 0.0f;
            const bool near = d > -far && d < far;
#pragma unroll
            for (int q = 0; q < 4; ++q) {
              if (q == g && near) atomicAdd(dist + w * width + d + far, dp[kt][r]);
              __builtin_amdgcn_wave_barrier();
            }
          }
      } else {
        float t = 0.0f;
#pragma unroll
        for (int kt = 0; kt < NQ; ++kt)
#pragma unroll
          for (int r = 0; r < 4; ++r) t += dp[kt][r];
        sumL += d0 < 0 ? t : 0.0f;
        sumR += d0 < 0 ? 0.0f : t;
      }
    }
    over_ahead<D, NQ, NT>(ad, Ks, dp, dq);          // dQ^T += K^T dS^T
    wait_vm0();
    __syncthreads();                             // V_{j+1} is there, the K slot is free
    if (more) lk.load(dK, j + 1, 0);
  }
  if constexpr (BIAS) table_part<4>(a, dist, width, sumL, sumR, tpart + ((size_t)bh * tiles + i) * bucket_count(a.bias));
  f32x4 out[NO];
  add_shares<QW, NT>(reinterpret_cast<f32x4*>(smem), dq, w, l, out);   // (the tiles are consumed)
  if (!in) return;
  float* const o = row_ptr(gr.dQ, b, h, n) + 16 * wq + 4 * g;
#pragma unroll
  for (int m = 0; m < NO; ++m) *reinterpret_cast<f32x4*>(o + 16 * QW * m) = out[m] * a.scale;
}

// ------------------------------------------------------------------ dK, dV
// A workgroup owns 64 / QW keys of a key tile (lane = key); the QW waves that share 16 of them split the 64 queries of every
// step, and their sums meet in LDS at the end.  Q and dO go through one slot each; every load lands under a product that
// reads the other one.  Steps and pieces as in the bf16 path; a piece's sums are rows of its slot.
template <int D>
constexpr int f32_key_lds() { return 2 * FTile<D>::BYTES + 512; }   // + L, D of 64 queries

template <int D, int QW, bool BIAS>
__global__ __launch_bounds__(256, 2) void attn_f32_key_kernel(Attn a, AttnGrads gr, const float* __restrict__ Ds, KeyPlan kp,
                                                               const float* __restrict__ tpart, int qparts) {
  constexpr int NT = D / 16, TB = FTile<D>::BYTES, NQ = 4 / QW, NO = NT / QW;
  extern __shared__ __attribute__((aligned(16))) unsigned char smem[];
  if ((int)blockIdx.x >= kp.blocks * kp.pieces) {
    if constexpr (BIAS) table_sum(a, gr, tpart, qparts, blockIdx.x - kp.blocks * kp.pieces, smem);
    return;
  }
  const unsigned char* stat = smem + 2 * TB;
  const int tid = threadIdx.x, w = wave_uniform(tid >> 6), l = tid & 63, g = l >> 4, n = l & 15;
  const int wk = w / QW, wq = w % QW;
  // (key tiles one after the other across all heads: under a causal mask the longest first)
  const int p = blockIdx.x / kp.blocks, bx = blockIdx.x - p * kp.blocks, BH = a.B * a.Hkv;
  const int bh = wave_uniform(bx % BH), kg = bx / BH % QW, j = wave_uniform(bx / BH / QW), b = bh / a.Hkv, hk = bh - b * a.Hkv;
  const Seq sq = seq_of(a, b);
  const KeySteps st = key_steps(a, sq, j);
  const int s_beg = wave_uniform(p * kp.piece), s_end = wave_uniform(min(st.total, s_beg + kp.piece));
  if (p > 0 && s_beg >= s_end) return;
  const int key = j * kBlk + kg * (kBlk / QW) + 16 * wk + n;
  const bool ok = key < sq.nk;
  f32x4 kf[NT], vf[NT], dk[NT], dv[NT];
  const int kc = min(key, a.Nk - 1);
  load_frag<NT>(row_ptr(a.K, b, hk, kc), ok, g, kf);
  load_frag<NT>(row_ptr(a.V, b, hk, kc), ok, g, vf);
#pragma unroll
  for (int t = 0; t < NT; ++t) dk[t] = dv[t] = zero4();
  FLoader<D> lq, lg;
  lq.init(lds_base(smem), w, l, 4 * a.Q.sn);
  lg.init(lds_base(smem), w, l, 4 * gr.dO.sn);
  FAddr<D> ad;
  ad.init(l);
  const int far = a.bias.far;
  float* const bias = reinterpret_cast<float*>(smem + f32_key_lds<D>());
  auto issue_o = [&](int h, int i) { lg.load(rows_rsrc<D>(gr.dO, b, h, sq.nq), i, TB); };
  // Q_i into slot 0, with L and D of its queries
  auto issue_q = [&](int h, int i) {
    lq.load(rows_rsrc<D>(a.Q, b, h, sq.nq), i, 0);
    const unsigned long long x = reinterpret_cast<unsigned long long>((w == 0 ? a.L : Ds) + ((size_t)b * a.H + h) * a.Nq);
    const void* px = reinterpret_cast<const void*>((unsigned long long)(unsigned)wave_uniform((int)(x >> 32)) << 32 |
                                                   (unsigned)wave_uniform((int)x));   // (in scalar registers)
    if (w < 2) load_to_lds4(tile_rsrc(px, wave_uniform(sq.nq) * 4), (i * kBlk + l) * 4, lds_base(smem) + 2 * TB + 256 * w);
  };
  if (s_beg < s_end) {
    const int hh = wave_uniform(s_beg / st.per_head);
    int i = wave_uniform(st.i0 + s_beg - hh * st.per_head), h = wave_uniform(hk * a.G + hh);
    issue_o(h, i);
    issue_q(h, i);
    if constexpr (BIAS) expand_bias(a, h, bias);
    wait_vm0();
    __syncthreads();
    const unsigned char* Qs = smem + 16 * NQ * wq * FTile<D>::ROWB;         // this wave's queries
    const unsigned char* Gs = Qs + TB;
    const unsigned char* sp = stat + 4 * (16 * NQ * wq + 4 * g);
    for (int s = s_beg; s < s_end; ++s) {
      const bool more = s + 1 < s_end, turn = i + 1 == st.i0 + st.per_head;
      const int in = wave_uniform(turn ? st.i0 : i + 1), hn = wave_uniform(turn ? h + 1 : h);
      f32x4 pr[NQ], dp[NQ];
#pragma unroll
      for (int q = 0; q < NQ; ++q) pr[q] = dp[q] = zero4();
      rows_ahead<D, NQ, NT>(ad, Gs, vf, dp);          // dP = dO V^T: registers = queries, lane = key
      wait_vm0();
      __syncthreads();                             // Q_i is there
      rows_ahead<D, NQ, NT>(ad, Qs, kf, pr);          // S = Q K^T
#pragma unroll
      for (int q = 0; q < NQ; ++q) {
        const f32x4 Lr = *reinterpret_cast<const f32x4*>(sp + 64 * q);
        const f32x4 Dr = *reinterpret_cast<const f32x4*>(sp + 64 * q + 256);
#pragma unroll
        for (int r = 0; r < 4; ++r) {
          const int nq = i * kBlk + 16 * (NQ * wq + q) + 4 * g + r, d = key - (sq.pos + nq);
          float v = pr[q][r] * a.scale - (Lr[r] == -INFINITY ? INFINITY : Lr[r]);
          if constexpr (BIAS) v += bias_at(bias, far, d);
          pr[q][r] = nq < sq.nq && !(a.causal && d > 0) ? expf(v) : 0.0f;
          dp[q][r] = pr[q][r] * (dp[q][r] - Dr[r]);
        }
      }
      over_ahead<D, NQ, NT>(ad, Gs, pr, dv);          // dV^T += dO^T P
      __syncthreads();                             // the dO slot is free, the bias is read
      if (more) {
        issue_o(hn, in);
        if constexpr (BIAS) {
          if (turn) expand_bias(a, hn, bias);
        }
      }
      over_ahead<D, NQ, NT>(ad, Qs, dp, dk);          // dK^T += Q^T dS
      wait_vm0();
      __syncthreads();                             // dO_{i'} is there, the Q slot is free
      if (more) issue_q(hn, in);
      i = in;
      h = hn;
    }
  }
  f32x4 ok_[NO], ov[NO];
  f32x4* const x = reinterpret_cast<f32x4*>(smem);
  add_shares<QW, NT>(x, dk, w, l, ok_);
  add_shares<QW, NT>(x + 4 * NT * 64, dv, w, l, ov);
  float *oK, *oV;
  if (st.total > kp.piece) {
    oK = kp.part + (((size_t)bh * kp.tiles + j) * kp.pieces + p) * (2 * kBlk * D) + (size_t)(key - j * kBlk) * D;
    oV = oK + kBlk * D;
  } else {
    if (key >= a.Nk) return;
    oK = row_ptr(gr.dK, b, hk, key);
    oV = row_ptr(gr.dV, b, hk, key);
  }
  const float scale = st.total > kp.piece ? 1.0f : dk_scale(a, sq);
#pragma unroll
  for (int m = 0; m < NO; ++m) {
#pragma unroll
    for (int r = 0; r < 4; ++r) {
      ok_[m][r] = ok ? ok_[m][r] * scale : 0.0f;
      ov[m][r] = ok ? ov[m][r] : 0.0f;
    }
    *reinterpret_cast<f32x4*>(oK + 16 * (wq + QW * m) + 4 * g) = ok_[m];
    *reinterpret_cast<f32x4*>(oV + 16 * (wq + QW * m) + 4 * g) = ov[m];
  }
}

// dK, dV of the key tiles whose steps were cut: the sums of the pieces in order, 16 of the 128 rows a workgroup
template <int D>
__global__ __launch_bounds__(256) void attn_f32_kv_join_kernel(Attn a, AttnGrads gr, KeyPlan kp) {
  constexpr int C = D / 4;   // 16-byte pieces of a row
  const int bh = blockIdx.x / kp.tiles, j = blockIdx.x - bh * kp.tiles, b = bh / a.Hkv, hk = bh - b * a.Hkv;
  const Seq sq = seq_of(a, b);
  const int total = key_steps(a, sq, j).total;
  if (total <= kp.piece) return;
  const int np = (total + kp.piece - 1) / kp.piece;
  for (int i = blockIdx.y * 16 * C + threadIdx.x; i < (int)(blockIdx.y + 1) * 16 * C; i += 256) {
    const int row = i / C, c = 4 * (i % C), key = j * kBlk + row % kBlk;
    if (key >= a.Nk) continue;
    const float* p = kp.part + (size_t)blockIdx.x * kp.pieces * (2 * kBlk * D) + (size_t)row * D + c;
    f32x4 s = *reinterpret_cast<const f32x4*>(p);
#pragma unroll 4
    for (int e = 1; e < np; ++e) s += *reinterpret_cast<const f32x4*>(p + (size_t)e * (2 * kBlk * D));
    if (row < kBlk) s *= dk_scale(a, sq);
    *reinterpret_cast<f32x4*>(row_ptr(row < kBlk ? gr.dK : gr.dV, b, hk, key) + c) = s;
  }
}

template <int D>
hipError_t forward_impl(const Attn& a, const AttnPlan& plan, hipStream_t st) {
  const AttnPart& ow = plan.own;
  auto launch = [&](auto kern, dim3 grid, const char* name) -> hipError_t {
    const int lds = 2 * FTile<D>::BYTES + (a.has_bias() ? ow.heads * (2 * a.bias.far + 1) * 4 : 0);
    SLA_TRY(ensure_dyn_lds(kern, lds));
    KernelTimer kt(name, st);
    kern<<<grid, 256, lds, st>>>(a, plan);
    return hipGetLastError();
  };
  if (!plan.parts) {
    const dim3 grid(plan.map.blocks());
    return launch(a.has_bias() ? attn_f32_fwd_kernel<D, true, false> : attn_f32_fwd_kernel<D, false, false>, grid, "attn_fwd");
  }
  return launch(a.has_bias() ? attn_f32_fwd_kernel<D, true, true> : attn_f32_fwd_kernel<D, false, true>,
                dim3(plan.prefix.blocks + ow.blocks), "attn_parts");
}

template <int D, int QW>
hipError_t launch_key(const Attn& a, const AttnGrads& g, const BwdPlan& p, hipStream_t st) {
  const int tables = g.dtable ? a.H : 0, grid = p.key.blocks * p.key.pieces + tables;
  if (grid == 0) return hipGetLastError();
  {
    const int lds = f32_key_lds<D>() + (a.has_bias() ? (2 * a.bias.far + 1) * 4 : 0);
    auto kern = a.has_bias() ? attn_f32_key_kernel<D, QW, true> : attn_f32_key_kernel<D, QW, false>;
    SLA_TRY(ensure_dyn_lds(kern, lds));
    KernelTimer kt("attn_dkdv", st);
    kern<<<grid, 256, lds, st>>>(a, g, p.stat, p.key, p.tpart, p.qparts);
  }
  if (p.key.pieces > 1) {
    KernelTimer kt("attn_kv_join", st);
    attn_f32_kv_join_kernel<D><<<dim3(a.B * a.Hkv * p.key.tiles, 8), 256, 0, st>>>(a, g, p.key);
  }
  return hipGetLastError();
}

template <int D, int QW>
hipError_t launch_dq(const Attn& a, const AttnGrads& g, const BwdPlan& p, hipStream_t st) {
  const int lds = a.has_bias() ? f32_dq_lds<D>(a.bias.far) : 2 * FTile<D>::BYTES;
  auto kern = a.has_bias() ? attn_f32_dq_kernel<D, QW, true> : attn_f32_dq_kernel<D, QW, false>;
  SLA_TRY(ensure_dyn_lds(kern, lds));
  KernelTimer kt("attn_dq", st);
  kern<<<p.map.blocks(), 256, lds, st>>>(a, g, p.stat, p.tpart, p.map);
  return hipGetLastError();
}

template <int D>
hipError_t backward_impl(const Attn& a, const AttnGrads& g, char* ws, hipStream_t st) {
  const BwdPlan p = attn_bwd_plan(a, ws);
  SLA_TRY((p.shares == 4 ? launch_dq<D, 4>(a, g, p, st) : p.shares == 2 ? launch_dq<D, 2>(a, g, p, st) : launch_dq<D, 1>(a, g, p, st)));
  return p.key.quarters == 4 ? launch_key<D, 4>(a, g, p, st) : launch_key<D, 2>(a, g, p, st);
}

}  // namespace

hipError_t attn_forward_f32(const Attn& a, const AttnPlan& plan, hipStream_t st) {
  SLA_TRY(a.d == 64 ? forward_impl<64>(a, plan, st) : forward_impl<128>(a, plan, st));
  return plan.parts ? attn_join(a, plan, st) : hipSuccess;
}

hipError_t attn_backward_f32(const Attn& a, const AttnGrads& g, char* ws, hipStream_t st) {
  return a.d == 64 ? backward_impl<64>(a, g, ws, st) : backward_impl<128>(a, g, ws, st);
}

}  // namespace sla
