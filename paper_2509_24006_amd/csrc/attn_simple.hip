// Softmax attention, one wave per row of the result: the scores of 64 keys at a time, a lane each, and every
// product as a sum over them.  Bound by its loads: a row of the result reads all of K and V.
#include "attn.h"

namespace sla {
namespace {

template <class T>
__device__ __forceinline__ const T* row_of(const View& v, int b, int h, int n) {
  return reinterpret_cast<const T*>(v.p) + b * v.sb + h * v.sh + (long long)n * v.sn;
}
template <class T>
__device__ __forceinline__ void put(T* p, float x);
template <>
__device__ __forceinline__ void put<float>(float* p, float x) { *p = x; }
template <>
__device__ __forceinline__ void put<__hip_bfloat16>(__hip_bfloat16* p, float x) { *p = __float2bfloat16(x); }

__device__ __forceinline__ float wave_sum(float x) {
  for (int o = 32; o; o >>= 1) x += __shfl_xor(x, o);
  return x;
}
__device__ __forceinline__ float wave_max(float x) {
  for (int o = 32; o; o >>= 1) x = fmaxf(x, __shfl_xor(x, o));
  return x;
}

template <class T, int D>
__device__ __forceinline__ float dot_row(const float* q, const T* k) {
  float s = 0.0f;
  for (int c = 0; c < D; ++c) s = fmaf(q[c], to_f32(k[c]), s);
  return s;
}

// score of key position kp for a query at position qp
__device__ __forceinline__ float score(const Attn& a, float dot, int kp, int qp, int h) {
  float s = dot * a.scale;
  if (a.bias.n_borders >= 0) s += table_at(a, bucket_of(a.bias, kp - qp), h);
  return s;
}

template <class T, int D>
__global__ __launch_bounds__(256) void simple_forward_kernel(Attn a) {
  __shared__ float qs[4][D];
  const int w = threadIdx.x >> 6, l = threadIdx.x & 63;
  const long long row = (long long)blockIdx.x * 4 + w, rows = (long long)a.B * a.H * a.Nq;
  const bool live = row < rows;
  const int n = live ? row % a.Nq : 0, bh = live ? row / a.Nq : 0, b = bh / a.H, h = bh % a.H, hk = h / a.G;
  const Seq s = seq_of(a, b);
  const bool valid = live && n < s.nq;
  for (int c = l; c < D; c += 64) qs[w][c] = valid ? to_f32(row_of<T>(a.Q, b, h, n)[c]) : 0.0f;
  __syncthreads();
  if (!live) return;
  const int total = a.Np + s.nk, qp = s.pos + n;
  const int lim = !valid ? 0 : a.causal ? max(0, min(total, qp + 1)) : total;
  float m = -INFINITY, lsum = 0.0f, acc[D / 64] = {};
  for (int k0 = 0; k0 < lim; k0 += 64) {
    const int k = k0 + l;
    float x = -INFINITY;
    if (k < lim)
      x = score(a, dot_row<T, D>(qs[w], k < a.Np ? row_of<T>(a.Kp, 0, hk, k) : row_of<T>(a.K, b, hk, k - a.Np)), k, qp, h);
    const float mn = fmaxf(m, wave_max(x)), ref = mn == -INFINITY ? 0.0f : mn;
    const float p = expf(x - ref), alpha = expf(m - ref);
    lsum = lsum * alpha + wave_sum(p);
    m = mn;
    for (int e = 0; e < D / 64; ++e) acc[e] *= alpha;
    for (int i = 0; i < min(64, lim - k0); ++i) {
      const float pi = __shfl(p, i);
      const int ki = k0 + i;
      const T* v = ki < a.Np ? row_of<T>(a.Vp, 0, hk, ki) : row_of<T>(a.V, b, hk, ki - a.Np);
      for (int e = 0; e < D / 64; ++e) acc[e] = fmaf(pi, to_f32(v[l + 64 * e]), acc[e]);
    }
  }
  T* o = const_cast<T*>(row_of<T>(a.O, b, h, n));
  for (int e = 0; e < D / 64; ++e) put(o + l + 64 * e, lsum > 0.0f ? acc[e] / lsum : 0.0f);
  if (a.L && l == 0) a.L[(size_t)bh * a.Nq + n] = lsum > 0.0f ? m + logf(lsum) : -INFINITY;
}

// dQ and D = rowsum(dO * O)
template <class T, int D>
__global__ __launch_bounds__(256) void simple_query_kernel(Attn a, AttnGrads gr, float* __restrict__ Ds) {
  __shared__ float qs[4][2][D];
  const int w = threadIdx.x >> 6, l = threadIdx.x & 63;
  const long long row = (long long)blockIdx.x * 4 + w, rows = (long long)a.B * a.H * a.Nq;
  const bool live = row < rows;
  const int n = live ? row % a.Nq : 0, bh = live ? row / a.Nq : 0, b = bh / a.H, h = bh % a.H, hk = h / a.G;
  const Seq s = seq_of(a, b);
  const bool valid = live && n < s.nq;
  float dsum = 0.0f;
  for (int c = l; c < D; c += 64) {
    qs[w][0][c] = valid ? to_f32(row_of<T>(a.Q, b, h, n)[c]) : 0.0f;
    qs[w][1][c] = valid ? to_f32(row_of<T>(gr.dO, b, h, n)[c]) : 0.0f;
    if (valid) dsum = fmaf(qs[w][1][c], to_f32(row_of<T>(a.O, b, h, n)[c]), dsum);
  }
  dsum = wave_sum(dsum);
  __syncthreads();
  if (!live) return;
  if (l == 0) Ds[(size_t)bh * a.Nq + n] = dsum;
  const int qp = s.pos + n, lim = !valid ? 0 : a.causal ? max(0, min(s.nk, qp + 1)) : s.nk;
  const float Lr = a.L[(size_t)bh * a.Nq + n];
  float acc[D / 64] = {};
  for (int k0 = 0; k0 < lim; k0 += 64) {
    const int k = k0 + l;
    float ds = 0.0f;
    if (k < lim) {
      const float p = expf(score(a, dot_row<T, D>(qs[w][0], row_of<T>(a.K, b, hk, k)), k, qp, h) - Lr);
      ds = p * (dot_row<T, D>(qs[w][1], row_of<T>(a.V, b, hk, k)) - dsum);
    }
    for (int i = 0; i < min(64, lim - k0); ++i) {
      const float di = __shfl(ds, i);
      const T* kr = row_of<T>(a.K, b, hk, k0 + i);
      for (int e = 0; e < D / 64; ++e) acc[e] = fmaf(di, to_f32(kr[l + 64 * e]), acc[e]);
    }
  }
  T* o = const_cast<T*>(row_of<T>(gr.dQ, b, h, n));
  for (int e = 0; e < D / 64; ++e) put(o + l + 64 * e, acc[e] * a.scale);
}

// dK, dV of one key: the queries of all heads that read it
template <class T, int D>
__global__ __launch_bounds__(256) void simple_key_kernel(Attn a, AttnGrads gr, const float* __restrict__ Ds) {
  __shared__ float ks[4][2][D];
  const int w = threadIdx.x >> 6, l = threadIdx.x & 63;
  const long long row = (long long)blockIdx.x * 4 + w, rows = (long long)a.B * a.Hkv * a.Nk;
  const bool live = row < rows;
  const int k = live ? row % a.Nk : 0, bh = live ? row / a.Nk : 0, b = bh / a.Hkv, hk = bh % a.Hkv;
  const Seq s = seq_of(a, b);
  const bool valid = live && k < s.nk;
  for (int c = l; c < D; c += 64) {
    ks[w][0][c] = valid ? to_f32(row_of<T>(a.K, b, hk, k)[c]) : 0.0f;
    ks[w][1][c] = valid ? to_f32(row_of<T>(a.V, b, hk, k)[c]) : 0.0f;
  }
  __syncthreads();
  if (!live) return;
  float dk[D / 64] = {}, dv[D / 64] = {};
  const int n0 = a.causal ? max(0, k - s.pos) : 0;
  for (int h = hk * a.G; valid && h < hk * a.G + a.G; ++h)
    for (int i0 = n0; i0 < s.nq; i0 += 64) {
      const int n = i0 + l;
      float p = 0.0f, ds = 0.0f;
      if (n < s.nq) {
        const size_t at = ((size_t)b * a.H + h) * a.Nq + n;
        p = expf(score(a, dot_row<T, D>(ks[w][0], row_of<T>(a.Q, b, h, n)), k, s.pos + n, h) - a.L[at]);
        ds = p * (dot_row<T, D>(ks[w][1], row_of<T>(gr.dO, b, h, n)) - Ds[at]);
      }
      for (int i = 0; i < min(64, s.nq - i0); ++i) {
        const float pi = __shfl(p, i), di = __shfl(ds, i);
        const T *q = row_of<T>(a.Q, b, h, i0 + i), *g = row_of<T>(gr.dO, b, h, i0 + i);
        for (int e = 0; e < D / 64; ++e) {
          dv[e] = fmaf(pi, to_f32(g[l + 64 * e]), dv[e]);
          dk[e] = fmaf(di, to_f32(q[l + 64 * e]), dk[e]);
        }
      }
    }
  T *ok = const_cast<T*>(row_of<T>(gr.dK, b, hk, k)), *ov = const_cast<T*>(row_of<T>(gr.dV, b, hk, k));
  for (int e = 0; e < D / 64; ++e) {
    put(ok + l + 64 * e, dk[e] * a.scale);
    put(ov + l + 64 * e, dv[e]);
  }
}

// One entry of the table's gradient: the sum of dS over all pairs whose distance falls into its bucket.
template <class T, int D>
__global__ __launch_bounds__(256) void simple_table_kernel(Attn a, AttnGrads gr, const float* __restrict__ Ds) {
  __shared__ float red[4];
  const int w = threadIdx.x >> 6, l = threadIdx.x & 63, u = blockIdx.x, h = blockIdx.y, hk = h / a.G;
  float sum = 0.0f;
  for (int b = 0; b < a.B; ++b) {
    const Seq s = seq_of(a, b);
    for (int n = w; n < s.nq; n += 4) {
      const int qp = s.pos + n, lim = a.causal ? min(s.nk, qp + 1) : s.nk;
      const size_t at = ((size_t)b * a.H + h) * a.Nq + n;
      for (int k = l; k < lim; k += 64) {
        if (bucket_of(a.bias, k - qp) != u) continue;
        float x = 0.0f, y = 0.0f;
        const T *q = row_of<T>(a.Q, b, h, n), *g = row_of<T>(gr.dO, b, h, n), *kr = row_of<T>(a.K, b, hk, k),
                *vr = row_of<T>(a.V, b, hk, k);
        for (int c = 0; c < D; ++c) {
          x = fmaf(to_f32(q[c]), to_f32(kr[c]), x);
          y = fmaf(to_f32(g[c]), to_f32(vr[c]), y);
        }
        sum += expf(score(a, x, k, qp, h) - a.L[at]) * (y - Ds[at]);
      }
    }
  }
  sum = wave_sum(sum);
  if (l == 0) red[w] = sum;
  __syncthreads();
  if (threadIdx.x) return;
  sum = (red[0] + red[1]) + (red[2] + red[3]);
  const size_t at = (size_t)u * a.H + h;
  if (a.table16) put(reinterpret_cast<__hip_bfloat16*>(gr.dtable) + at, sum);
  else put(reinterpret_cast<float*>(gr.dtable) + at, sum);
}

template <class T, int D>
hipError_t forward_impl(const Attn& a, hipStream_t st) {
  KernelTimer kt("attn_forward", st);
  simple_forward_kernel<T, D><<<((long long)a.B * a.H * a.Nq + 3) / 4, 256, 0, st>>>(a);
  return hipGetLastError();
}
template <class T, int D>
hipError_t backward_impl(const Attn& a, const AttnGrads& g, float* Ds, hipStream_t st) {
  KernelTimer kt("attn_backward", st);
  simple_query_kernel<T, D><<<((long long)a.B * a.H * a.Nq + 3) / 4, 256, 0, st>>>(a, g, Ds);
  if (a.Nk > 0) simple_key_kernel<T, D><<<((long long)a.B * a.Hkv * a.Nk + 3) / 4, 256, 0, st>>>(a, g, Ds);
  if (g.dtable) simple_table_kernel<T, D><<<dim3(bucket_count(a.bias), a.H), 256, 0, st>>>(a, g, Ds);
  return hipGetLastError();
}

}  // namespace

size_t attn_backward_ws_f32(const Attn& a) { return align_up((size_t)a.B * a.H * a.Nq * 4); }

hipError_t attn_forward_f32(const Attn& a, hipStream_t st) {
  return a.d == 64 ? forward_impl<float, 64>(a, st) : forward_impl<float, 128>(a, st);
}
hipError_t attn_backward_f32(const Attn& a, const AttnGrads& g, char* ws, hipStream_t st) {
  float* Ds = reinterpret_cast<float*>(ws);
  return a.d == 64 ? backward_impl<float, 64>(a, g, Ds, st) : backward_impl<float, 128>(a, g, Ds, st);
}

}  // namespace sla
