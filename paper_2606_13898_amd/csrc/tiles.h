// Row tiles of the packed sequence and the activation, shared by the projections (gemm.hip) and the int8 product
// of few rows (linear.hip).
#pragma once

#include "common.h"
#include "kernels.h"

namespace hilo {

// tanh-approximated GELU, 0.5 u (1 + tanh(y)) with y = sqrt(2/pi) (u + 0.044715 u^3), evaluated
// through the identity 0.5 (1 + tanh(y)) = 1 / (1 + exp(-2y)): one hardware exp2 and one
// reciprocal (about one ulp each) instead of a full tanh.  Very negative u gives exp2 -> inf and
// the result -0; very positive u gives exp2 -> 0 and the result u.
HILO_DEV float gelu_tanh(float u) {
  constexpr float c = -2.0f * 0.7978845608028654f * 1.4426950408889634f;  // -2 sqrt(2/pi) log2(e)
  const float t = c * u * (1.0f + 0.044715f * u * u);
  return u * __builtin_amdgcn_rcpf(1.0f + __builtin_amdgcn_exp2f(t));
}

// The same of four values with u (a + b u^2) for the polynomial, one operation of five less and rounded elsewhere, and step
// by step through all four: an exponential or a reciprocal cannot be used by the next instruction.  For the int8
// products.  Against gelu_tanh four times on the present tiles the difference is within the noise (codes in, in turn: 22560
// x 12288 x 3072 750 to 758 and 748 to 757 us, 6144 x 12288 x 3072 208 to 211 and 210 to 212, 4708 x 6144 x 1536 58 both).
HILO_DEV void gelu_tanh4(float (&u)[4]) {
  constexpr float a = -2.0f * 0.7978845608028654f * 1.4426950408889634f, b = 0.044715f * a;
  float t[4];
#pragma unroll
  for (int e = 0; e < 4; ++e) t[e] = u[e] * __builtin_fmaf(u[e] * u[e], b, a);
#pragma unroll
  for (int e = 0; e < 4; ++e) t[e] = __builtin_amdgcn_exp2f(t[e]);
#pragma unroll
  for (int e = 0; e < 4; ++e) t[e] = 1.0f + t[e];
#pragma unroll
  for (int e = 0; e < 4; ++e) t[e] = __builtin_amdgcn_rcpf(t[e]);
#pragma unroll
  for (int e = 0; e < 4; ++e) u[e] *= t[e];
}

// Row range of a row tile; tiles of a sample are [image tiles][text tiles].
struct TileRows {
  int s, sigma, row0, nrows;
};

// Active row tiles of the ragged problem: per sample, ceil(image rows / BM) image tiles then
// ceil(L / BM) text tiles.  Only the device knows the row counts, so every workgroup walks the
// (few) segments itself.
HILO_DEV int row_tiles_total(const GemmProblem &p, int BM) {
  int R = 0;
  for (int s = 0; s < p.B; ++s) {
    const int nimg = cu_at(p.cu, s + 1) - p.L - cu_at(p.cu, s);
    R += (nimg + BM - 1) / BM + (p.L + BM - 1) / BM;
  }
  return R;
}

HILO_DEV TileRows decode_row_tile(const GemmProblem &p, int BM, int r) {
  TileRows tr{0, 0, 0, 0};
  for (int s = 0; s < p.B; ++s) {
    const int lo = cu_at(p.cu, s), hi = cu_at(p.cu, s + 1), ts = hi - p.L;
    const int ti = (ts - lo + BM - 1) / BM, tt = (p.L + BM - 1) / BM;
    if (r < ti) {
      tr = TileRows{s, 0, lo + r * BM, min(BM, ts - (lo + r * BM))};
      break;
    }
    r -= ti;
    if (r < tt) {
      tr = TileRows{s, 1, ts + r * BM, min(BM, hi - (ts + r * BM))};
      break;
    }
    r -= tt;
  }
  return tr;
}

// Values that are the same on every lane, restated as such (the compiler otherwise keeps some of
// the stream-K bookkeeping in VGPRs and branches on it with exec masks).
HILO_DEV int uni(int v) { return __builtin_amdgcn_readfirstlane(v); }
HILO_DEV float *uni(float *ptr) {
  const uint64_t v = reinterpret_cast<uint64_t>(ptr);
  const uint32_t lo = __builtin_amdgcn_readfirstlane(uint32_t(v)), hi = __builtin_amdgcn_readfirstlane(uint32_t(v >> 32));
  return reinterpret_cast<float *>((uint64_t(hi) << 32) | lo);
}
HILO_DEV TileRows uni(const TileRows &x) { return TileRows{uni(x.s), uni(x.sigma), uni(x.row0), uni(x.nrows)}; }

}  // namespace hilo
