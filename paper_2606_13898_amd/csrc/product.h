// What the products of a feed-forward share: segments of the packed rows, activations, and the last step of an output.
#pragma once

#include "common.h"
#include "kernels.h"
#include "tiles.h"

namespace hilo {

constexpr uint32_t kBehind = 0x80000000u;  // an offset behind any buffer's end, also with rows of the tile added

// A run of rows of one stream.  Segment 2 s is sample s's image rows, 2 s + 1 its text rows; merged, all rows are one.
struct Segment {
  int lo, n, stream;
};
template <typename P>
HILO_DEV int segments(const P &p) { return p.merged ? 1 : 2 * p.B; }
template <typename P>
HILO_DEV Segment segment(const P &p, int i) {
  if (p.merged) return Segment{0, cu_at(p.cu, p.B), 0};
  const int lo = cu_at(p.cu, i >> 1), hi = cu_at(p.cu, (i >> 1) + 1);
  return (i & 1) ? Segment{hi - p.L, p.L, 1} : Segment{lo, hi - p.L - lo, 0};
}

// Rows of a row tile of BM rows: first row, how many, stream; n = 0 behind the last tile.  Of few samples by scalar loads, one
// after the other, which wait for no load of a tile.  Of many a lane looks at a segment, 64 at a time: the first whose
// tiles, and those of all before, number more than t.  The whole wave calls it with the same t.
struct RowTile {
  int row0, n, stream;
};
template <typename P>
HILO_DEV RowTile find_row_tile(const P &p, int BM, int t) {
  if (p.merged) {
    const int end = cu_at(p.cu, p.B);
    return RowTile{t * BM, max(0, min(BM, end - t * BM)), 0};
  }
  if (p.B <= 32) {
    for (int i = 0; i < 2 * p.B; ++i) {
      const Segment s = segment(p, i);
      const int tiles = (s.n + BM - 1) / BM;
      if (t < tiles) return RowTile{s.lo + t * BM, min(BM, s.n - t * BM), s.stream};
      t -= tiles;
    }
    return RowTile{0, 0, 0};
  }
  const int lane = threadIdx.x & 63, ns = 2 * p.B;
  for (int i0 = 0; i0 < ns; i0 += 64) {
    int tiles = 0;
    if (i0 + lane < ns) {
      const int i = i0 + lane, lo = p.cu[i >> 1], hi = p.cu[(i >> 1) + 1];
      tiles = ((i & 1 ? p.L : hi - p.L - lo) + BM - 1) / BM;
    }
    int upto = tiles;
#pragma unroll
    for (int off = 1; off < 64; off <<= 1) {
      const int o = __shfl_up(upto, off, 64);
      if (lane >= off) upto += o;
    }
    const uint64_t hit = __ballot(t < upto);
    if (hit) {
      const int l = __ffsll((unsigned long long)hit) - 1;
      const int before = __builtin_amdgcn_readlane(upto - tiles, l);
      const Segment s = segment(p, i0 + l);
      const int at = (t - before) * BM;
      return RowTile{uni(s.lo + at), uni(min(BM, s.n - at)), uni(s.stream)};
    }
    t -= __builtin_amdgcn_readlane(upto, 63);
  }
  return RowTile{0, 0, 0};
}
// As many row tiles as the buffers' rows can make: every segment but one may end in a part of one.
template <typename P>
__host__ __device__ __forceinline__ int row_tiles_bound(const P &p, int BM) {
  return (p.rows + BM - 1) / BM + (p.merged ? 0 : 2 * p.B - 1);
}
template <typename P>
HILO_DEV int count_row_tiles(const P &p, int BM) {
  if (p.merged) return (cu_at(p.cu, p.B) + BM - 1) / BM;
  int n = 0;
  for (int i = threadIdx.x & 63; i < 2 * p.B; i += 64) {
    const int lo = p.cu[i >> 1], hi = p.cu[(i >> 1) + 1];
    n += ((i & 1 ? p.L : hi - p.L - lo) + BM - 1) / BM;
  }
#pragma unroll
  for (int off = 32; off > 0; off >>= 1) n += __shfl_xor(n, off, 64);
  return uni(n);
}

// The gate's activation p g with p = 1 / (1 + exp(-z)): z = g for SiLU, and for the tanh form of GELU z = 2 y, y =
// sqrt(2/pi) (g + 0.044715 g^3).  Its derivative is p + g p (1 - p) z'.  EXACT: the library's exponential and a division,
// for float32; otherwise the hardware's exponential and reciprocal, about one ulp each.
template <bool EXACT>
HILO_DEV float gate_p(float g, bool silu) {
  constexpr float c = 2.0f * 0.7978845608028654f;
  const float z = silu ? g : c * g * (1.0f + 0.044715f * g * g);
  if constexpr (EXACT) return 1.0f / (1.0f + expf(-z));
  return __builtin_amdgcn_rcpf(1.0f + __builtin_amdgcn_exp2f(z * -1.4426950408889634f));
}
template <bool EXACT>
HILO_DEV float gate_act(float g, bool silu) { return g * gate_p<EXACT>(g, silu); }
template <bool EXACT>
HILO_DEV void gate_slope(float g, bool silu, float &act, float &slope) {
  constexpr float c = 2.0f * 0.7978845608028654f;
  const float p = gate_p<EXACT>(g, silu), q = p * (1.0f - p);
  act = g * p;
  // far out q is 0 and z' may be infinite
  slope = q == 0.f ? p : p + g * q * (silu ? 1.0f : c * (1.0f + 3.0f * 0.044715f * g * g));
}

// 8 E4M3 codes times their scale as bf16, exact; scale: the bits of a float32 whose exponent is the E8M0 byte.  The conversion
// takes that exponent alone: 0 is 2^-127, and 255 makes every value NaN, a zero's too.
HILO_DEV bf16x8 wide_codes(uint32_t x, uint32_t y, uint32_t scale) {
  typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
  const float s = __uint_as_float(scale);
  const bf16x2 q0 = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(x, s, false), q1 = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(x, s, true);
  const bf16x2 q2 = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(y, s, false), q3 = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(y, s, true);
  return bf16x8{q0[0], q0[1], q1[0], q1[1], q2[0], q2[1], q3[0], q3[1]};
}

// 4 values of a vector of the dtype, or 0 where there is none
HILO_DEV f32x4 load4(const void *v, size_t i, bool bf16) {
  if (!v) return f32x4{0.f, 0.f, 0.f, 0.f};
  if (bf16) {
    const uint2 u = *reinterpret_cast<const uint2 *>(reinterpret_cast<const uint16_t *>(v) + i);
    return f32x4{__uint_as_float(u.x << 16), __uint_as_float(u.x & 0xffff0000u), __uint_as_float(u.y << 16),
                 __uint_as_float(u.y & 0xffff0000u)};
  }
  return *reinterpret_cast<const f32x4 *>(reinterpret_cast<const float *>(v) + i);
}
HILO_DEV void store4(void *o, size_t i, f32x4 v, bool bf16) {
  if (bf16) *reinterpret_cast<uint2 *>(reinterpret_cast<uint16_t *>(o) + i) = make_uint2(bf16_pair(v[0], v[1]), bf16_pair(v[2], v[3]));
  else *reinterpret_cast<f32x4 *>(reinterpret_cast<float *>(o) + i) = v;
}

// Four outputs of a row from the products' sums: biases, pre, activation, rounding.
template <bool GATED>
HILO_DEV void finish_out(const ProductProblem &p, int stream, size_t row, int n, f32x4 g, f32x4 u) {
  u += load4(p.bias[stream][GATED ? 1 : 0], n, p.bf16);
  if constexpr (GATED) {
    g += load4(p.bias[stream][0], n, p.bf16);
    if (p.pre) {
      store4(p.pre, row * 2 * p.N + n, g, p.bf16);
      store4(p.pre, row * 2 * p.N + p.N + n, u, p.bf16);
    }
#pragma unroll
    for (int e = 0; e < 4; ++e) u[e] *= p.bf16 ? gate_act<false>(g[e], p.silu) : gate_act<true>(g[e], p.silu);
  }
  store4(p.out, row * p.N + n, u, p.bf16 && !p.out_f32);
}

}  // namespace hilo
