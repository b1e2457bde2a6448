// Products of at most 64 rows (hilo_linear, hilo_linear_fp8): bound by reading the weights once.
//
// A workgroup has 16 columns of the output (with a gate 16 of either part), its 8 waves an eighth of k each; fragments come
// straight from memory, a lane 32 consecutive bytes of a row of w, so that an instruction pair reads whole 128-byte lines,
// and four steps are on their way while four are multiplied.  The waves' sums meet in LDS.  Rows of a stream need not
// lie side by side: each is looked up.
//
// Measured (us, this and tiles, from weights in memory): 3072 -> 8192 with a gate 1 row 25.3 (101 MB at 4.0 TB/s) and 35.9, 64 rows
// 41.2 and 37.5; 3072 -> 3072 64 rows 17.2 and 21.3; 1024 -> 1024 7.6 and 13.3; of FP8 codes 64 rows 29.7 and 32.4, 11.5 and
// 25.3, 7.5 and 12.7.  So 64 rows stay here, although the widest bf16 weights would gain a tenth on tiles.  Four rows of FP8
// 3072 -> 8192 with a gate, 50 MB: 17.7 us of codes, 21.9 of bf16 rows.
//
// FP8: up to 16 float rows are quantised where they are read, by every workgroup anew: a row's block of 128 is in four lanes, so
// its largest value takes two exchanges, and a launch less is worth more than the arithmetic.  Codes are multiplied as
// bf16, which holds a code times its scale exactly: the FP8 instruction keeps fewer bits, and its rate is of no use here.
#include <algorithm>

#include "product.h"

namespace hilo {

typedef int i32x4 __attribute__((ext_vector_type(4)));
typedef int i32x8 __attribute__((ext_vector_type(8)));

namespace few {

enum Rows { ROWS_BF16, ROWS_CODES, ROWS_QUANTISED };  // x and w bf16; w codes, and x codes; w codes, x bf16

constexpr int kWaves = 8;

// 32 bytes of a row
struct Piece {
  i32x4 lo, hi;
  HILO_DEV void load(const char *at) {
    lo = reinterpret_cast<const i32x4 *>(at)[0];
    hi = reinterpret_cast<const i32x4 *>(at)[1];
  }
  HILO_DEV void load16(const char *at) {
    lo = reinterpret_cast<const i32x4 *>(at)[0];
    hi = i32x4(0);
  }
  // valid: bytes from the first on that belong to the sum
  HILO_DEV void clip(int valid) {
    hi = valid < 32 ? i32x4(0) : hi;
    lo = valid < 16 ? i32x4(0) : lo;
  }
  HILO_DEV bf16x8 half(int h) const { return __builtin_bit_cast(bf16x8, h ? hi : lo); }
  HILO_DEV i32x8 all() const { return __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7); }
  HILO_DEV void values(int h, float (&f)[8]) const { unpack8(__builtin_bit_cast(uint4, h ? hi : lo), f); }
};

// A lane's operands of a step: 64 values of k of bf16, 128 of codes.
template <int ROWS, int PARTS, int MB>
struct Step {
  Piece w[PARTS];
  Piece x[MB][ROWS == ROWS_QUANTISED ? 2 : 1];
  uint32_t sx[ROWS == ROWS_CODES ? MB : 1], sw[PARTS];
};

template <int ROWS, bool GATED, int MB>
__global__ __launch_bounds__(64 * kWaves) void k_product_few(ProductProblem p) {
  constexpr int PARTS = GATED ? 2 : 1, KS = ROWS == ROWS_BF16 ? 64 : 128, ESZ = ROWS == ROWS_BF16 ? 2 : 1;
  constexpr int D = MB == 1 && ROWS != ROWS_QUANTISED ? 4 : MB == 4 ? 1 : 2;  // steps on their way, and as many behind them
  __shared__ f32x4 sums[kWaves][PARTS * MB][64];
  __shared__ int list[64];
  const int lane = threadIdx.x & 63, wid = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int lr = lane & 15, lg = lane >> 4, stream = blockIdx.y, n0 = blockIdx.x * 16;
  // ---- the stream's rows
  int mine = -1;
  if (lane < cu_at(p.cu, p.B)) {
    mine = 0;
    if (!p.merged) mine = lane >= p.cu[sample_of_row(p.cu, p.B, lane) + 1] - p.L;
  }
  const uint64_t mask = __ballot(mine == stream);
  const int rows = __popcll(mask);
  if (rows == 0) return;
  if (wid == 0 && mine == stream) list[__popcll(mask & ((1ull << lane) - 1))] = lane;
  __syncthreads();
  const char *x[MB], *w[PARTS];
  const uint8_t *xs[MB], *ws[PARTS];
#pragma unroll
  for (int i = 0; i < MB; ++i) {
    const size_t row = list[min(16 * i + lr, rows - 1)];
    x[i] = reinterpret_cast<const char *>(p.x) + row * p.K * (ROWS == ROWS_QUANTISED ? 2 : ESZ);
    if constexpr (ROWS == ROWS_CODES) xs[i] = p.x_scale + row * scale_stride(p.K);
  }
#pragma unroll
  for (int q = 0; q < PARTS; ++q) {
    const void *m = stream ? (q ? p.w[1][1] : p.w[1][0]) : (q ? p.w[0][1] : p.w[0][0]);
    w[q] = reinterpret_cast<const char *>(m) + size_t(min(n0 + lr, p.N - 1)) * p.K * ESZ;
    if constexpr (ROWS != ROWS_BF16) {
      const uint8_t *s = stream ? (q ? p.w_scale[1][1] : p.w_scale[1][0]) : (q ? p.w_scale[0][1] : p.w_scale[0][0]);
      ws[q] = s + size_t(n0 / 128) * scale_stride(p.K);
    }
  }
  f32x4 acc[PARTS][MB];
#pragma unroll
  for (int q = 0; q < PARTS; ++q)
#pragma unroll
    for (int i = 0; i < MB; ++i) acc[q][i] = f32x4{0.f, 0.f, 0.f, 0.f};
  const int steps = (p.K + KS - 1) / KS, s0 = steps * wid / kWaves, s1 = steps * (wid + 1) / kWaves;
  const int bytes = p.K * ESZ;  // of a row of w
  using S = Step<ROWS, PARTS, MB>;
  // pieces behind the end of k are read from its last bytes and cleared
  auto load = [&](int s, S &v) __attribute__((always_inline)) {
    const int at = 128 * s + 32 * lg, from = min(at, bytes - 32 < 0 ? 0 : bytes - 32);
    const bool whole = bytes >= 32;  // a row of 16 bytes: K = 8 of bf16 or 16 codes
#pragma unroll
    for (int q = 0; q < PARTS; ++q) {
      if (whole) v.w[q].load(w[q] + from);
      else v.w[q].load16(w[q]);
      if constexpr (ROWS != ROWS_BF16) v.sw[q] = ws[q][s];
    }
#pragma unroll
    for (int i = 0; i < MB; ++i) {
      if constexpr (ROWS == ROWS_QUANTISED) {
        const int f2 = 2 * from;
        if (whole) {
          v.x[i][0].load(x[i] + f2);
          v.x[i][1].load(x[i] + f2 + 32);
        } else {
          v.x[i][0].load(x[i]);
          v.x[i][1].lo = v.x[i][1].hi = i32x4(0);
        }
      } else {
        if (whole) v.x[i][0].load(x[i] + from);
        else v.x[i][0].load16(x[i]);
        if constexpr (ROWS == ROWS_CODES) v.sx[i] = xs[i][s];
      }
    }
  };
  auto mul = [&](int s, S &v) __attribute__((always_inline)) {
    const int at = 128 * s + 32 * lg, valid = bytes - at;  // bytes of w in the lane's piece
    if (128 * s + 128 > bytes) {
      // a piece that begins inside the row but ends behind it was read from earlier on: its bytes move up
      const bool moved = bytes >= 32 && valid > 0 && valid < 32;
#pragma unroll
      for (int q = 0; q < PARTS; ++q) {
        if (moved) v.w[q].lo = v.w[q].hi;
        v.w[q].clip(valid);
      }
#pragma unroll
      for (int i = 0; i < MB; ++i) {
        if constexpr (ROWS == ROWS_QUANTISED) {
          if (moved) v.x[i][0] = v.x[i][1];
          v.x[i][0].clip(2 * valid);
          v.x[i][1].clip(2 * valid - 32);
        } else {
          if (moved) v.x[i][0].lo = v.x[i][0].hi;
          v.x[i][0].clip(valid);
        }
      }
    }
#pragma unroll
    for (int i = 0; i < MB; ++i) {
      if constexpr (ROWS == ROWS_BF16) {
#pragma unroll
        for (int h = 0; h < 2; ++h)
#pragma unroll
          for (int q = 0; q < PARTS; ++q)
            acc[q][i] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(v.w[q].half(h), v.x[i][0].half(h), acc[q][i], 0, 0, 0);
      } else {
        i32x8 xc;
        uint32_t sx;
        if constexpr (ROWS == ROWS_CODES) {
          xc = v.x[i][0].all();
          sx = v.sx[i];
        } else {
          float f[4][8];
          uint32_t top = 0;
#pragma unroll
          for (int h = 0; h < 4; ++h) {
            v.x[i][h >> 1].values(h & 1, f[h]);
#pragma unroll
            for (int e = 0; e < 8; ++e) top = max(top, abs_bits(f[h][e]));
          }
          top = max(top, uint32_t(__shfl_xor(int(top), 16, 64)));
          top = max(top, uint32_t(__shfl_xor(int(top), 32, 64)));
          const bool finite = top < 0x7f800000u;
          const int k = finite ? pow2_exponent(__uint_as_float(top)) : 0;
          const float inv = pow2_inverse(k);
#pragma unroll
          for (int h = 0; h < 4; ++h) {
            xc[2 * h] = int(fp8x4(f[h][0] * inv, f[h][1] * inv, f[h][2] * inv, f[h][3] * inv));
            xc[2 * h + 1] = int(fp8x4(f[h][4] * inv, f[h][5] * inv, f[h][6] * inv, f[h][7] * inv));
          }
          sx = finite ? 127 + k : 255;  // NaN, whatever the codes are
        }
#pragma unroll
        for (int m = 0; m < 4; ++m) {
          const bf16x8 xb = wide_codes(uint32_t(xc[2 * m]), uint32_t(xc[2 * m + 1]), sx << 23);
#pragma unroll
          for (int q = 0; q < PARTS; ++q) {
            const i32x8 wc = v.w[q].all();
            acc[q][i] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(wide_codes(uint32_t(wc[2 * m]), uint32_t(wc[2 * m + 1]), v.sw[q] << 23), xb,
                                                                acc[q][i], 0, 0, 0);
          }
        }
      }
    }
  };
  if (s0 < s1) {
    S a[D], b[D];
    auto chunk = [&](int s, S (&v)[D]) __attribute__((always_inline)) {  // past the wave's steps: its last again
#pragma unroll
      for (int d = 0; d < D; ++d) load(min(s + d, s1 - 1), v[d]);
    };
    auto take = [&](int s, S (&v)[D]) __attribute__((always_inline)) {
#pragma unroll
      for (int d = 0; d < D; ++d)
        if (s + d < s1) mul(s + d, v[d]);
    };
    chunk(s0, a);
#pragma unroll 1
    for (int s = s0; s < s1; s += 2 * D) {
      if (s + D < s1) chunk(s + D, b);
      take(s, a);
      if (s + D >= s1) break;
      if (s + 2 * D < s1) chunk(s + 2 * D, a);
      take(s + D, b);
    }
  }
#pragma unroll
  for (int q = 0; q < PARTS; ++q)
#pragma unroll
    for (int i = 0; i < MB; ++i) sums[wid][q * MB + i][lane] = acc[q][i];
  __syncthreads();
  // wave i finishes rows 16 i + lr, columns 4 lg .. + 3
  if (wid >= MB || 16 * wid + lr >= rows || n0 + 4 * lg >= p.N) return;
  f32x4 v[PARTS];
#pragma unroll
  for (int q = 0; q < PARTS; ++q) {
    v[q] = sums[0][q * MB + wid][lane];
#pragma unroll
    for (int k = 1; k < kWaves; ++k) v[q] += sums[k][q * MB + wid][lane];
  }
  finish_out<GATED>(p, stream, list[16 * wid + lr], n0 + 4 * lg, v[0], v[PARTS - 1]);
}

template <int ROWS, bool GATED>
static hipError_t run(const ProductProblem &p, hipStream_t st) {
  const dim3 grid((p.N + 15) / 16, p.merged ? 1 : 2), block(64 * kWaves);
  if constexpr (ROWS == ROWS_QUANTISED) {
    hipLaunchKernelGGL((k_product_few<ROWS, GATED, 1>), grid, block, 0, st, p);
  } else {
    if (p.rows <= 16) hipLaunchKernelGGL((k_product_few<ROWS, GATED, 1>), grid, block, 0, st, p);
    else if (p.rows <= 32) hipLaunchKernelGGL((k_product_few<ROWS, GATED, 2>), grid, block, 0, st, p);
    else hipLaunchKernelGGL((k_product_few<ROWS, GATED, 4>), grid, block, 0, st, p);
  }
  return hipGetLastError();
}

}  // namespace few

hipError_t launch_product_few(const ProductProblem &p, hipStream_t st) {
  if (!p.w_scale[0][0]) return p.parts == 2 ? few::run<few::ROWS_BF16, true>(p, st) : few::run<few::ROWS_BF16, false>(p, st);
  if (p.x_scale) return p.parts == 2 ? few::run<few::ROWS_CODES, true>(p, st) : few::run<few::ROWS_CODES, false>(p, st);
  return p.parts == 2 ? few::run<few::ROWS_QUANTISED, true>(p, st) : few::run<few::ROWS_QUANTISED, false>(p, st);
}

}  // namespace hilo
