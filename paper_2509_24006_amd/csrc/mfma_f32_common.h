// Device helpers for the float matrix-core kernels on gfx950 (v_mfma_f32_16x16x4_f32: float products, float accumulation).
//
// One instruction multiplies A (16 x 4) by B (4 x 16) into C (16 x 16).  Lane l = 16 g + n:
//   A: row n, k = g        B: column n, k = g        C: column n, rows 4 g + i in registers i
// Any assignment of k-indices to (instruction, g) is right as long as A and B use the same one.
// All kernels take k = 16 t + 4 g + s for instruction s of group t, which gives two things: an
// operand whose k-index runs along a row is read 16 bytes at a time, and a C tile (rows 16 t + 4 g
// + i) is the B operand of the next product as it stands, with no exchange between lanes.  A lane
// therefore owns one token (column n) and the features {16 t + 4 g + s} of it, in every product.
//
// 64 x D tiles lie in LDS row by row, unpadded, filled by direct global -> LDS loads; the 16-byte
// chunk c of row r sits at chunk position c ^ (r % 16).  Both reads are then free of bank
// conflicts: 16 rows at one chunk (operand read by rows) hit 16 different positions, and 4 rows of
// 16 adjacent floats (operand contracted over tile rows) hit four different 64-byte pieces.
#ifndef SLA_MFMA_F32_COMMON_H_
#define SLA_MFMA_F32_COMMON_H_

#include "mfma_common.h"

namespace sla {

__device__ __forceinline__ f32x4 mfma16(float a, float b, f32x4 c) {
  return __builtin_amdgcn_mfma_f32_16x16x4f32(a, b, c, 0, 0, 0);
}
__device__ __forceinline__ f32x4 zero4() { return f32x4{0.0f, 0.0f, 0.0f, 0.0f}; }

template <int D>
struct FTile {
  static constexpr int CPR = D / 4;              // 16-byte chunks per row
  static constexpr int ROWB = 4 * D;
  static constexpr int BYTES = kBlk * ROWB;
  static constexpr int RPI = 1024 / ROWB;        // rows per wave-wide load
  static constexpr int IPW = kBlk / RPI / 4;     // loads per wave and tile (four waves fill a tile)
};

// Direct loads of 64-row tiles whose rows lie tsB bytes apart, behind a descriptor that spans the
// whole head (rows past its end read as zeros: the part of an offset that may pass the end rides on
// the per-lane offset, which the range check covers; the tile's own offset is always inside).
// N tsB is below 2^31, so offsets of rows past the end of a sequence of 62 rows and more stay below
// 2^32.  Shorter ones (a single tile) with rows 64 MB and more apart would come back into range:
// their rows past the end get an offset that is out of range in any case.
template <int D>
struct FLoader {
  using T = FTile<D>;
  static constexpr int kFar = 1 << 26;   // 64 rows of this pitch: 2^32 bytes
  int voff[2];    // this lane's byte offset for even and odd loads (the swizzle has period 16 rows)
  int kend;       // this lane's loads from kend on are of rows past the end (only where rows are far apart)
  int kstep, tile_step;
  unsigned lds0;
  // N: rows of the head (a packed matrix needs none: its rows are near)
  __device__ __forceinline__ void init(unsigned lds_base_addr, int w, int l, int tsB, int N = 0) {
    const int r0 = T::RPI * w + l / T::CPR;
#pragma unroll
    for (int k = 0; k < 2; ++k) {
      const int row = r0 + 4 * T::RPI * k;
      voff[k] = r0 * tsB + (((l % T::CPR) ^ (row & 15)) << 4);
    }
    kend = tsB < kFar ? T::IPW : (N - r0 + 4 * T::RPI - 1) / (4 * T::RPI);
    kstep = 4 * T::RPI * tsB;
    tile_step = kBlk * tsB;
    lds0 = lds_base_addr + wave_uniform(w) * 1024;
  }
  // tile number `tile` of the buffer -> LDS offset `slot`
  __device__ __forceinline__ void load(BufDesc desc, int tile, int slot) const {
#pragma unroll
    for (int k = 0; k < T::IPW; ++k)
      load_to_lds16(desc, k < kend ? voff[k & 1] + k * kstep : 0x7ffffff0, tile * tile_step, lds0 + slot + 4096 * k);
  }
};

template <int D>
__device__ __forceinline__ BufDesc head_rsrc_f32(const float* head_base, int N, int tsB) {
  return tile_rsrc(head_base, (N - 1) * tsB + 4 * D);
}
// a packed matrix of `rows` rows of D floats
template <int D>
__device__ __forceinline__ BufDesc matrix_rsrc_f32(const float* M, int rows) {
  return tile_rsrc(M, rows * 4 * D);
}

// Per-lane addresses of the two operand reads.
template <int D>
struct FAddr {
  int rb, rx;      // by rows: base, swizzle of the chunk index
  int tb[4], tx;   // over rows: base for row 4 g + i, swizzle of the 16-float piece
  __device__ __forceinline__ void init(int l) {
    const int g = l >> 4, n = l & 15;
    rb = n * FTile<D>::ROWB + (((g ^ n) & 3) << 4);
    rx = (n >> 2) << 6;
#pragma unroll
    for (int i = 0; i < 4; ++i)
      tb[i] = (4 * g + i) * FTile<D>::ROWB + ((((n >> 2) ^ i) & 3) << 4) + ((n & 3) << 2);
    tx = g << 6;
  }
  // four k-values (features 16 t + 4 g ..) of tile row r0 + n; r0 a multiple of 16
  __device__ __forceinline__ f32x4 row(const unsigned char* tile, int r0, int t) const {
    return *reinterpret_cast<const f32x4*>(tile + r0 * FTile<D>::ROWB + rb + ((t << 6) ^ rx));
  }
  // feature 16 f + n of tile row r0 + 4 g + i; r0 a multiple of 16
  __device__ __forceinline__ float over(const unsigned char* tile, int r0, int i, int f) const {
    return *reinterpret_cast<const float*>(tile + r0 * FTile<D>::ROWB + tb[i] + ((f << 6) ^ tx));
  }
};

// sum / maximum over the four lanes that hold a token
__device__ __forceinline__ float tok_sum(float x) {
  x += __shfl_xor(x, 16, 64);
  return x + __shfl_xor(x, 32, 64);
}
__device__ __forceinline__ float tok_max(float x) {
  x = fmaxf(x, __shfl_xor(x, 16, 64));
  return fmaxf(x, __shfl_xor(x, 32, 64));
}

// features {16 t + 4 g + s} of one token row (zeros if !ok)
template <int NT>
__device__ __forceinline__ void load_frag(const float* __restrict__ row, bool ok, int g, f32x4 (&x)[NT]) {
#pragma unroll
  for (int t = 0; t < NT; ++t)
    x[t] = ok ? *reinterpret_cast<const f32x4*>(row + 16 * t + 4 * g) : zero4();
}
template <int NT>
__device__ __forceinline__ void store_frag(float* __restrict__ row, int g, const f32x4 (&x)[NT]) {
#pragma unroll
  for (int t = 0; t < NT; ++t) *reinterpret_cast<f32x4*>(row + 16 * t + 4 * g) = x[t];
}
template <int NT>
__device__ __forceinline__ float dot_frag(const f32x4 (&a)[NT], const f32x4 (&b)[NT]) {
  f32x4 s = zero4();
#pragma unroll
  for (int t = 0; t < NT; ++t)
#pragma unroll
    for (int i = 0; i < 4; ++i) s[i] = fmaf(a[t][i], b[t][i], s[i]);
  return tok_sum((s[0] + s[1]) + (s[2] + s[3]));
}

// acc[r] (rows 16 r .. of the result) += tile rows 16 (r0 + r) .. (k along the rows) times the
// fragment b
template <int D, int NR, int NT>
__device__ __forceinline__ void mm_rows(const FAddr<D>& ad, const unsigned char* tile, const f32x4 (&b)[NT],
                                        f32x4 (&acc)[NR]) {
#pragma unroll
  for (int t = 0; t < NT; ++t) {
    f32x4 a[NR];
#pragma unroll
    for (int r = 0; r < NR; ++r) a[r] = ad.row(tile, 16 * r, t);
#pragma unroll
    for (int s = 0; s < 4; ++s)
#pragma unroll
      for (int r = 0; r < NR; ++r) acc[r] = mfma16(a[r][s], b[t][s], acc[r]);
  }
}

// acc[f] (features 16 f .. of the tile) += (tile rows 0 .. 16 NK)^T contracted over the rows with
// the C-layout operand b
template <int D, int NK, int NF>
__device__ __forceinline__ void mm_over(const FAddr<D>& ad, const unsigned char* tile, const f32x4 (&b)[NK],
                                        f32x4 (&acc)[NF]) {
#pragma unroll
  for (int k = 0; k < NK; ++k)
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      float a[NF];
#pragma unroll
      for (int f = 0; f < NF; ++f) a[f] = ad.over(tile, 16 * k, i, f);
#pragma unroll
      for (int f = 0; f < NF; ++f) acc[f] = mfma16(a[f], b[k][i], acc[f]);
    }
}

}  // namespace sla
#endif
