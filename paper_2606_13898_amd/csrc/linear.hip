// Products in 8-bit integers with a scale per token and per output channel (hilo_linear_i8), and the quantisation of
// rows (hilo_quantize_rows_i8):
//   acc = sum_k a[m][k] w[n][k] in int32, exact in any order (|acc| < 2^31 for K <= 65536);
//   out = act(acc * (a_scale[m] * w_scale[n]) + bias[n])
// Image rows take the image stream's weights, text rows the text stream's; tiles never straddle a segment.
#include "common.h"
#include "kernels.h"
#include "tiles.h"

namespace hilo {

typedef int i32x4 __attribute__((ext_vector_type(4)));

// ------------------------------------------------------------------------------- quantisation

// One row per group of W waves, NC chunks of 8 values a lane (cols <= 512 W NC), read once; LOOP: any number of
// columns, read twice.
template <bool BF16, int W, int NC, bool LOOP>
__global__ __launch_bounds__(256) void k_quantize_rows_i8(const void *__restrict__ x, int rows, int cols,
                                                          int8_t *__restrict__ codes, float *__restrict__ scale,
                                                          const int *__restrict__ limit) {
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int row = W == 1 ? blockIdx.x * 4 + wave : blockIdx.x;
  if (row >= (limit ? min(rows, cu_at(limit, 0)) : rows)) return;
  const int c0 = 8 * (W == 1 ? threadIdx.x & 63 : threadIdx.x);
  auto load = [&](int c, float (&f)[8]) __attribute__((always_inline)) {
    if constexpr (BF16) {
      unpack8(*reinterpret_cast<const uint4 *>(reinterpret_cast<const uint16_t *>(x) + size_t(row) * cols + c), f);
    } else {
      const float4 *u = reinterpret_cast<const float4 *>(reinterpret_cast<const float *>(x) + size_t(row) * cols + c);
      const float4 a = u[0], b = u[1];
      f[0] = a.x; f[1] = a.y; f[2] = a.z; f[3] = a.w;
      f[4] = b.x; f[5] = b.y; f[6] = b.z; f[7] = b.w;
    }
  };
  auto store = [&](int c, const float (&f)[8], float inv) __attribute__((always_inline)) {
    *reinterpret_cast<uint2 *>(codes + size_t(row) * cols + c) =
        make_uint2(i8x4(f[0] * inv, f[1] * inv, f[2] * inv, f[3] * inv), i8x4(f[4] * inv, f[5] * inv, f[6] * inv, f[7] * inv));
  };
  float v[NC][8];
  uint32_t top = 0;
  auto take = [&](const float (&f)[8]) __attribute__((always_inline)) {
#pragma unroll
    for (int e = 0; e < 8; ++e) top = max(top, abs_bits(f[e]));
  };
  if constexpr (LOOP) {
    for (int c = c0; c < cols; c += 512 * W) {
      load(c, v[0]);
      take(v[0]);
    }
  } else {
#pragma unroll
    for (int k = 0; k < NC; ++k) {
      const int c = c0 + k * 512 * W;
      if (c < cols) {
        load(c, v[k]);
        take(v[k]);
      }
    }
  }
  top = wave_max_u32(top);
  if constexpr (W > 1) {
    __shared__ uint32_t tops[W];
    if ((threadIdx.x & 63) == 0) tops[wave] = top;
    __syncthreads();
#pragma unroll
    for (int w = 0; w < W; ++w) top = max(top, tops[w]);
  }
  const float inv = i8_inverse(top);
  if (c0 == 0) scale[row] = i8_scale(top);
  if constexpr (LOOP) {
    for (int c = c0; c < cols; c += 512 * W) {
      load(c, v[0]);
      store(c, v[0], inv);
    }
  } else {
#pragma unroll
    for (int k = 0; k < NC; ++k) {
      const int c = c0 + k * 512 * W;
      if (c < cols) store(c, v[k], inv);
    }
  }
}

hipError_t launch_quantize_rows_i8(bool bf16, const void *x, int rows, int cols, int8_t *codes, float *scale,
                                   const int *limit, hipStream_t st) {
  if (rows <= 0) return hipSuccess;
#define HILO_Q8(W, NC, LOOP)                                                                                     \
  do {                                                                                                           \
    const dim3 grid(W == 1 ? (unsigned(rows) + 3) / 4 : unsigned(rows));                                         \
    if (bf16) hipLaunchKernelGGL((k_quantize_rows_i8<true, W, NC, LOOP>), grid, dim3(256), 0, st, x, rows, cols, codes, scale, limit); \
    else hipLaunchKernelGGL((k_quantize_rows_i8<false, W, NC, LOOP>), grid, dim3(256), 0, st, x, rows, cols, codes, scale, limit);    \
  } while (0)
  if (cols <= 512) HILO_Q8(1, 1, false);
  else if (cols <= 1024) HILO_Q8(1, 2, false);
  else if (cols <= 2048) HILO_Q8(4, 1, false);
  else if (cols <= 4096) HILO_Q8(4, 2, false);
  else if (cols <= 8192) HILO_Q8(4, 4, false);
  else if (cols <= 16384) HILO_Q8(4, 8, false);
  else HILO_Q8(4, 1, true);
#undef HILO_Q8
  return hipGetLastError();
}

// ------------------------------------------------------------------------------------- products

// Four consecutive columns n .. n + 3 of row m (N % 4 == 0: all inside).
template <bool BF16, bool GELU>
HILO_DEV void i8_out4(const GemmProblem &p, int sigma, size_t m, int n, const i32x4 &acc) {
  const float4 ws = *reinterpret_cast<const float4 *>((sigma ? p.w_scale[1] : p.w_scale[0]) + n);
  const float sa = p.a_scale[m];
  const void *bias = sigma ? p.bias[1] : p.bias[0];
  float b[4] = {0.f, 0.f, 0.f, 0.f};
  if (bias) {
    if constexpr (BF16) {
      const uint2 u = *reinterpret_cast<const uint2 *>(reinterpret_cast<const uint16_t *>(bias) + n);
      b[0] = __uint_as_float(u.x << 16); b[1] = __uint_as_float(u.x & 0xffff0000u);
      b[2] = __uint_as_float(u.y << 16); b[3] = __uint_as_float(u.y & 0xffff0000u);
    } else {
      const float4 u = *reinterpret_cast<const float4 *>(reinterpret_cast<const float *>(bias) + n);
      b[0] = u.x; b[1] = u.y; b[2] = u.z; b[3] = u.w;
    }
  }
  // the exact sum is rounded to 24 bits once here; it and the product of the scales are what float32 costs
  float v[4] = {float(acc[0]) * (sa * ws.x) + b[0], float(acc[1]) * (sa * ws.y) + b[1],
                float(acc[2]) * (sa * ws.z) + b[2], float(acc[3]) * (sa * ws.w) + b[3]};
  if constexpr (GELU) {
#pragma unroll
    for (int e = 0; e < 4; ++e) v[e] = gelu_tanh(v[e]);
  }
  if constexpr (BF16)
    *reinterpret_cast<uint2 *>(reinterpret_cast<uint16_t *>(p.out) + m * p.N + n) =
        make_uint2(pack_bf16x2(v[0], v[1]), pack_bf16x2(v[2], v[3]));
  else
    *reinterpret_cast<float4 *>(reinterpret_cast<float *>(p.out) + m * p.N + n) = make_float4(v[0], v[1], v[2], v[3]);
}

// Tiles of 16 MB rows x 16 NB columns, K split over the NW waves of a workgroup in steps of 64, their sums added
// through LDS.  Fragments come straight from global memory, 16 bytes a lane: lane (lr, lg) holds bytes 16 lg .. of row
// lr's step.
template <bool BF16, bool GELU, int MB, int NB, int NW>
__global__ __launch_bounds__(64 * NW) void k_linear_i8_direct(GemmProblem p) {
  __shared__ i32x4 part[NW][MB * NB][64];
  const int lane = threadIdx.x & 63, wid = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int lr = lane & 15, lg = lane >> 4;
  const int tilesN = (p.N + 16 * NB - 1) / (16 * NB), tiles = row_tiles_total(p, 16 * MB) * tilesN;
  const int steps = (p.K + 63) / 64, s0 = steps * wid / NW, s1 = steps * (wid + 1) / NW;
  for (int t = blockIdx.x; t < tiles; t += gridDim.x) {
    const int n0 = t % tilesN * (16 * NB);
    const TileRows tr = uni(decode_row_tile(p, 16 * MB, t / tilesN));
    const int8_t *A[MB], *W[NB];
#pragma unroll
    for (int i = 0; i < MB; ++i)
      A[i] = reinterpret_cast<const int8_t *>(p.A) + size_t(tr.row0 + min(16 * i + lr, tr.nrows - 1)) * p.K;
#pragma unroll
    for (int j = 0; j < NB; ++j)
      W[j] = reinterpret_cast<const int8_t *>(tr.sigma ? p.W[1] : p.W[0]) + size_t(min(n0 + 16 * j + lr, p.N - 1)) * p.K;
    i32x4 acc[MB][NB];
#pragma unroll
    for (int i = 0; i < MB; ++i)
#pragma unroll
      for (int j = 0; j < NB; ++j) acc[i][j] = i32x4{0, 0, 0, 0};
    for (int s = s0; s < s1; ++s) {
      const int k = 64 * s + 16 * lg, kc = min(k, p.K - 16);  // K % 16 == 0: a chunk is inside or behind K
      i32x4 a[MB], b[NB];
#pragma unroll
      for (int i = 0; i < MB; ++i) {
        a[i] = *reinterpret_cast<const i32x4 *>(A[i] + kc);
        if (k != kc) a[i] = i32x4{0, 0, 0, 0};
      }
#pragma unroll
      for (int j = 0; j < NB; ++j) b[j] = *reinterpret_cast<const i32x4 *>(W[j] + kc);
#pragma unroll
      for (int i = 0; i < MB; ++i)
#pragma unroll
        for (int j = 0; j < NB; ++j) acc[i][j] = __builtin_amdgcn_mfma_i32_16x16x64_i8(b[j], a[i], acc[i][j], 0, 0, 0);
    }
#pragma unroll
    for (int i = 0; i < MB; ++i)
#pragma unroll
      for (int j = 0; j < NB; ++j) part[wid][i * NB + j][lane] = acc[i][j];
    __syncthreads();
    for (int f = wid; f < MB * NB; f += NW) {
      i32x4 v = part[0][f][lane];
#pragma unroll
      for (int w = 1; w < NW; ++w) v += part[w][f][lane];
      const int rl = 16 * (f / NB) + lr, n = n0 + 16 * (f % NB) + 4 * lg;
      if (rl < tr.nrows && n < p.N) i8_out4<BF16, GELU>(p, tr.sigma, size_t(tr.row0 + rl), n, v);
    }
    __syncthreads();  // the next tile's sums go to the same LDS
  }
}

// Buffers of at most this many rows take the direct tiles.
constexpr long long kDirectRows = 64;
size_t linear_i8_part_bytes(long long rows) { return rows <= kDirectRows ? 0 : kSkPartBytes; }

template <bool BF16, bool GELU>
static hipError_t run_linear_i8(const GemmProblem &p, hipStream_t st) {
  const long long few = (long long)p.B * ((p.max_img_rows + 63) / 64 + (p.L + 63) / 64) * ((p.N + 31) / 32);
  if (few <= 0) return hipSuccess;
  hipLaunchKernelGGL((k_linear_i8_direct<BF16, GELU, 4, 2, 4>), dim3(unsigned(few < (1 << 16) ? few : (1 << 16))), dim3(256),
                     0, st, p);
  return hipGetLastError();
}

hipError_t launch_linear_i8(bool bf16, bool gelu, const GemmProblem &p, hipStream_t st) {
  if (p.max_img_rows > kDirectRows) return launch_linear_i8_tiled(bf16, gelu, p, st);
  if (bf16) return gelu ? run_linear_i8<true, true>(p, st) : run_linear_i8<true, false>(p, st);
  return gelu ? run_linear_i8<false, true>(p, st) : run_linear_i8<false, false>(p, st);
}

}  // namespace hilo
