// Shared device helpers for the gfx950 kernels of libhilo.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#define HILO_DEV __device__ __forceinline__

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef __bf16 bf16x4 __attribute__((ext_vector_type(4)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef float f32x16 __attribute__((ext_vector_type(16)));

namespace hilo {

constexpr int kXcds = 8;  // MI355X: 8 accelerator complex dies, each with its own L2

// The dispatcher hands workgroup b to XCD b % 8.  Remap so that each XCD receives a contiguous
// range of logical tiles (neighbouring tiles then share that XCD's L2).
HILO_DEV int xcd_remap(int b, int n) {
  int q = n / kXcds, r = n % kXcds;
  int x = b % kXcds, k = b / kXcds;
  return x * q + (x < r ? x : r) + k;
}

// v, of which nothing derived is known before this point: what rarely executed code forms from the lane number
// is then formed there, not hoisted out of the loop around it and kept in registers through that loop.
HILO_DEV int opaque(int v) {
  asm volatile("" : "+v"(v));
  return v;
}

HILO_DEV float bf2f(uint16_t b) { return __uint_as_float(uint32_t(b) << 16); }

// float -> bf16 bits, round to nearest even (NaN stays NaN).
HILO_DEV uint16_t f2bf(float f) {
  return __builtin_bit_cast(uint16_t, static_cast<__bf16>(f));
}

HILO_DEV uint32_t pack_bf16x2(float lo, float hi) {
  return uint32_t(f2bf(lo)) | (uint32_t(f2bf(hi)) << 16);
}

// The same in one instruction of two conversions (the pair above takes two, a shift and an or).
HILO_DEV uint32_t bf16_pair(float lo, float hi) {
  typedef float f32x2 __attribute__((ext_vector_type(2)));
  typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
  return __builtin_bit_cast(uint32_t, __builtin_convertvector(f32x2{lo, hi}, bf16x2));
}

// 8 bf16 (one 16-byte load) -> 8 floats
HILO_DEV void unpack8(const uint4 &u, float *f) {
  f[0] = __uint_as_float(u.x << 16); f[1] = __uint_as_float(u.x & 0xffff0000u);
  f[2] = __uint_as_float(u.y << 16); f[3] = __uint_as_float(u.y & 0xffff0000u);
  f[4] = __uint_as_float(u.z << 16); f[5] = __uint_as_float(u.z & 0xffff0000u);
  f[6] = __uint_as_float(u.w << 16); f[7] = __uint_as_float(u.w & 0xffff0000u);
}

HILO_DEV long long wave_sum_i64(long long v) {
#pragma unroll
  for (int off = 32; off > 0; off >>= 1) v += __shfl_xor(v, off, 64);
  return v;
}

HILO_DEV long long wave_max_i64(long long v) {
#pragma unroll
  for (int off = 32; off > 0; off >>= 1) {
    long long o = __shfl_xor(v, off, 64);
    v = o > v ? o : v;
  }
  return v;
}

HILO_DEV float wave_sum_f32(float v) {
#pragma unroll
  for (int off = 32; off > 0; off >>= 1) v += __shfl_xor(v, off, 64);
  return v;
}

// FP8 E4M3 codes of four values after scaling: clamp to the format's range (the conversion itself
// would turn an overflow into NaN), then round to nearest even.
HILO_DEV uint32_t fp8x4(float a, float b, float c, float d) {
  const float m = 448.0f;
  a = fminf(fmaxf(a, -m), m); b = fminf(fmaxf(b, -m), m);
  c = fminf(fmaxf(c, -m), m); d = fminf(fmaxf(d, -m), m);
  int w = __builtin_amdgcn_cvt_pk_fp8_f32(a, b, 0, false);
  w = __builtin_amdgcn_cvt_pk_fp8_f32(c, d, w, true);
  return uint32_t(w);
}

// Power-of-two scale of a row for E4M3 codes: the least k with 448 * 2^k >= amax (amax = f * 2^e,
// f in [1, 2): k = e - 8 when f <= 1.75, else e - 7), clamped below at -127, the least E8M0 scale;
// 0 for an all-zero row.  Codes are then x * 2^-k (exact), all within [-448, 448].
HILO_DEV int pow2_exponent(float amax) {
  const uint32_t b = __float_as_uint(amax);
  const int e = int((b >> 23) & 0xff);
  if (amax == 0.f) return 0;
  if (e == 0) return -127;  // subnormal: far below 448 * 2^-127
  const int k = e - 127 - ((b & 0x7fffff) <= 0x600000u ? 8 : 7);
  return k < -127 ? -127 : k;
}
// 2^-k for k in [-127, 127] as a float (always a normal number for the k above)
HILO_DEV float pow2_inverse(int k) { return __uint_as_float(uint32_t(127 - k) << 23); }

// Reductions over a wave in the vector unit: within rows of 16 lanes by DPP (neighbours, pairs, half rows, rows), then
// the four rows' values from lanes 0, 16, 32, 48.  A step takes a few cycles where one through LDS takes some sixty.
template <int CTRL>
HILO_DEV int dpp(int v) { return __builtin_amdgcn_update_dpp(0, v, CTRL, 0xf, 0xf, true); }
constexpr int kDppXor1 = 0xb1, kDppXor2 = 0x4e, kDppHalfMirror = 0x141, kDppMirror = 0x140;
HILO_DEV float lane_f32(float v, int l) { return __int_as_float(__builtin_amdgcn_readlane(__float_as_int(v), l)); }
HILO_DEV float wave_total(float v) {
  v += __int_as_float(dpp<kDppXor1>(__float_as_int(v)));
  v += __int_as_float(dpp<kDppXor2>(__float_as_int(v)));
  v += __int_as_float(dpp<kDppHalfMirror>(__float_as_int(v)));
  v += __int_as_float(dpp<kDppMirror>(__float_as_int(v)));
  return (lane_f32(v, 0) + lane_f32(v, 16)) + (lane_f32(v, 32) + lane_f32(v, 48));
}
HILO_DEV uint32_t wave_max_u32(uint32_t v) {
  v = max(v, uint32_t(dpp<kDppXor1>(int(v))));
  v = max(v, uint32_t(dpp<kDppXor2>(int(v))));
  v = max(v, uint32_t(dpp<kDppHalfMirror>(int(v))));
  v = max(v, uint32_t(dpp<kDppMirror>(int(v))));
  const uint32_t a = __builtin_amdgcn_readlane(int(v), 0), b = __builtin_amdgcn_readlane(int(v), 16);
  const uint32_t c = __builtin_amdgcn_readlane(int(v), 32), d = __builtin_amdgcn_readlane(int(v), 48);
  return max(max(a, b), max(c, d));
}

// int8 codes of a row with a float32 scale.  The row's largest magnitude is taken on the bits of |x|: they order as the
// values do, infinity above every number and NaN above that, so a row that holds either gets a scale that is not
// finite and nothing formed from it passes for a number.  Rows below 2^-120, whose inverse would overflow, count as 0.
HILO_DEV uint32_t abs_bits(float v) { return __float_as_uint(v) & 0x7fffffffu; }
HILO_DEV float i8_inverse(uint32_t top) {
  return top < 0x03800000u || top >= 0x7f800000u ? 0.f : __fmul_rn(__fdiv_rn(1.0f, __uint_as_float(top)), 127.0f);
}
HILO_DEV float i8_scale(uint32_t top) { return top < 0x03800000u ? 0.f : __fdiv_rn(__uint_as_float(top), 127.0f); }
// Codes of four values times the inverse, products at most 127 in magnitude (three roundings above it round to 127): adding
// 1.5 * 2^23 rounds to a whole number, to nearest even, and leaves its low byte in the lowest bits; a NaN's is 0.
HILO_DEV uint32_t i8x4(float a, float b, float c, float d, float inv) {
#pragma clang fp contract(off)  // a product is rounded before it is made whole: that is what the codes are
  constexpr float m = 12582912.0f;
  const float ma = a * inv, mb = b * inv, mc = c * inv, md = d * inv;
  const uint32_t lo = __builtin_amdgcn_perm(__float_as_uint(mb + m), __float_as_uint(ma + m), 0x0c0c0400u);
  const uint32_t hi = __builtin_amdgcn_perm(__float_as_uint(md + m), __float_as_uint(mc + m), 0x04000c0cu);
  return lo | hi;
}

// Sample boundary i of the packed sequence.  The boundaries do not change while a kernel runs, so
// they are read through the constant address space: the compiler then uses scalar loads with their
// own wait, where a vector load inside a pipelined loop is followed by a wait for every global load
// in flight (a drained prefetch per tile or unit).
HILO_DEV int cu_at(const int *cu, int i) { return ((const __attribute__((address_space(4))) int *)cu)[i]; }

// Sample that packed row r belongs to: largest s with cu[s] <= r (cu has B+1 entries).
HILO_DEV int sample_of_row(const int32_t *cu, int B, int r) {
  int lo = 0, hi = B;  // answer in [lo, hi)
  while (hi - lo > 1) {
    int mid = (lo + hi) >> 1;
    if (cu[mid] <= r) lo = mid; else hi = mid;
  }
  return lo;
}

}  // namespace hilo
