// Products in 8-bit integers with a scale per token and per output channel (hilo_linear_i8), and the quantisation of
// rows (hilo_quantize_rows_i8):
//   acc = sum_k a[m][k] w[n][k] in int32, exact in any order (|acc| < 2^31 for K <= 65536);
//   out = act(acc * (a_scale[m] * w_scale[n]) + bias[n])
// Image rows take the image stream's weights, text rows the text stream's; tiles never straddle a segment.
#include <algorithm>

#include "common.h"
#include "kernels.h"
#include "tiles.h"

namespace hilo {

typedef int i32x4 __attribute__((ext_vector_type(4)));

// 8 values of a float row as they lie in memory: loads stand apart from what is done with them, so that a lane's are all
// in flight at once.
template <bool BF16>
struct Raw8 {
  uint4 u[BF16 ? 1 : 2];
  HILO_DEV void load(const void *x, size_t i) {
    const uint4 *p = reinterpret_cast<const uint4 *>(reinterpret_cast<const char *>(x) + i * (BF16 ? 2 : 4));
    u[0] = p[0];
    if constexpr (!BF16) u[1] = p[1];
  }
  HILO_DEV void zero() {
    u[0] = make_uint4(0u, 0u, 0u, 0u);
    if constexpr (!BF16) u[1] = u[0];
  }
  HILO_DEV void values(float (&f)[8]) const {
    if constexpr (BF16) {
      unpack8(u[0], f);
    } else {
      f[0] = __uint_as_float(u[0].x); f[1] = __uint_as_float(u[0].y); f[2] = __uint_as_float(u[0].z); f[3] = __uint_as_float(u[0].w);
      f[4] = __uint_as_float(u[1].x); f[5] = __uint_as_float(u[1].y); f[6] = __uint_as_float(u[1].z); f[7] = __uint_as_float(u[1].w);
    }
  }
  HILO_DEV uint32_t top(uint32_t t) const {
    float f[8];
    values(f);
#pragma unroll
    for (int e = 0; e < 8; ++e) t = max(t, abs_bits(f[e]));
    return t;
  }
  HILO_DEV uint2 codes(float inv) const {
    float f[8];
    values(f);
    return make_uint2(i8x4(f[0], f[1], f[2], f[3], inv), i8x4(f[4], f[5], f[6], f[7], inv));
  }
};

// ------------------------------------------------------------------------------- quantisation

// One row per group of W waves, NC chunks of 8 values a lane (cols <= 512 W NC), read once; LOOP: any number of
// columns, NC chunks at a time, read twice.  A lane behind the last column reads the last chunk again, which changes
// no maximum.  Bound by memory: 22560 rows of 3072 bf16, 208 MB, in 37 us where the last level's cache holds what was
// written before (5.6 TB/s), 46 where it does not (4.5); 2766 rows in 7 to 8.  One wave a row up to 2048 columns, four
// above (22560 rows of 1536 on one and four 19.7 and 22.5 us, of 2048 25.7 and 26.5, of 3072 38.9 and 37.3).
template <bool BF16, int W, int NC, bool LOOP>
__global__ __launch_bounds__(256) void k_quantize_rows_i8(const void *__restrict__ x, int rows, int cols,
                                                          int8_t *__restrict__ codes, float *__restrict__ scale,
                                                          const int *__restrict__ limit) {
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int row = W == 1 ? blockIdx.x * 4 + wave : blockIdx.x;
  if (row >= (limit ? min(rows, cu_at(limit, 0)) : rows)) return;
  const int c0 = 8 * (W == 1 ? threadIdx.x & 63 : threadIdx.x);
  const size_t at = size_t(row) * cols;
  Raw8<BF16> v[NC];
  uint32_t top = 0;
  auto load = [&](int c) __attribute__((always_inline)) {
#pragma unroll
    for (int k = 0; k < NC; ++k) v[k].load(x, at + min(c + k * 512 * W, cols - 8));
  };
  auto take = [&]() __attribute__((always_inline)) {
#pragma unroll
    for (int k = 0; k < NC; ++k) top = v[k].top(top);
  };
  load(c0);
  take();
  if constexpr (LOOP) {
    for (int c = c0 + NC * 512 * W; c < cols; c += NC * 512 * W) {
      load(c);
      take();
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
  for (int c = c0; c < (LOOP ? cols : c0 + 1); c += NC * 512 * W) {
    if constexpr (LOOP) load(c);
#pragma unroll
    for (int k = 0; k < NC; ++k)
      if (c + k * 512 * W < cols) *reinterpret_cast<uint2 *>(codes + at + c + k * 512 * W) = v[k].codes(inv);
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
  else if (cols <= 2048) HILO_Q8(1, 4, false);
  else if (cols <= 4096) HILO_Q8(4, 2, false);
  else if (cols <= 8192) HILO_Q8(4, 4, false);
  else if (cols <= 16384) HILO_Q8(4, 8, false);
  else HILO_Q8(4, 4, true);
#undef HILO_Q8
  return hipGetLastError();
}

// ------------------------------------------------------------------------------------- products

// Scales and bias of four consecutive columns n .. n + 3 (N % 4 == 0: inside, or n is behind N and nothing is read),
// taken early: they arrive while the sums are formed.
template <bool BF16>
struct I8Cols {
  float4 s;
  float b[4];
  HILO_DEV I8Cols(const GemmProblem &p, int sigma, int n) : s(make_float4(0.f, 0.f, 0.f, 0.f)), b{0.f, 0.f, 0.f, 0.f} {
    if (n >= p.N) return;
    s = *reinterpret_cast<const float4 *>((sigma ? p.w_scale[1] : p.w_scale[0]) + n);
    const void *bias = sigma ? p.bias[1] : p.bias[0];
    if (!bias) return;
    if constexpr (BF16) {
      const uint2 u = *reinterpret_cast<const uint2 *>(reinterpret_cast<const uint16_t *>(bias) + n);
      b[0] = __uint_as_float(u.x << 16); b[1] = __uint_as_float(u.x & 0xffff0000u);
      b[2] = __uint_as_float(u.y << 16); b[3] = __uint_as_float(u.y & 0xffff0000u);
    } else {
      const float4 u = *reinterpret_cast<const float4 *>(reinterpret_cast<const float *>(bias) + n);
      b[0] = u.x; b[1] = u.y; b[2] = u.z; b[3] = u.w;
    }
  }
};

// Those columns of row m from the sums.
template <bool BF16, bool GELU>
HILO_DEV void i8_out4(const GemmProblem &p, size_t m, int n, const i32x4 &acc, float sa, const I8Cols<BF16> &c) {
  // the exact sum is rounded to 24 bits once here; it and the product of the scales are what float32 costs
  float v[4] = {float(acc[0]) * (sa * c.s.x) + c.b[0], float(acc[1]) * (sa * c.s.y) + c.b[1],
                float(acc[2]) * (sa * c.s.z) + c.b[2], float(acc[3]) * (sa * c.s.w) + c.b[3]};
  if constexpr (GELU) gelu_tanh4(v);
  if constexpr (BF16)
    *reinterpret_cast<uint2 *>(reinterpret_cast<uint16_t *>(p.out) + m * p.N + n) = make_uint2(bf16_pair(v[0], v[1]), bf16_pair(v[2], v[3]));
  else
    *reinterpret_cast<float4 *>(reinterpret_cast<float *>(p.out) + m * p.N + n) = make_float4(v[0], v[1], v[2], v[3]);
}

// 16 bytes of a row at k, of which those behind K (a multiple of 16) do not matter.
HILO_DEV i32x4 chunk_at(const int8_t *row, int k, int K) { return *reinterpret_cast<const i32x4 *>(row + min(k, K - 16)); }

// This wave's LDS writes are done and every wave is here; loads from global memory stay in flight.
HILO_DEV void lds_barrier() {
  __builtin_amdgcn_s_waitcnt(0xc07f);  // lgkmcnt(0)
  asm volatile("s_barrier" ::: "memory");
}

// The rows of one stream's tile t of BM rows, gathered over the samples (a sample may have one row), of at most 64 rows
// in all: rows[i] for i < the count, which is 0 where no such tile is.  Ends with every wave past a barrier.
struct FewRows {
  int sigma, n;
};
HILO_DEV FewRows few_rows(const GemmProblem &p, int BM, int t, int *rows) {
  const int lane = threadIdx.x & 63, T = min(cu_at(p.cu, p.B), p.max_img_rows);  // max_img_rows: at most 64
  const bool in = lane < T;
  bool text = false;
  if (p.L > 0 && in) text = lane >= p.cu[sample_of_row(p.cu, p.B, lane) + 1] - p.L;
  const uint64_t m1 = __ballot(in && text), m0 = __ballot(in && !text);
  const int n0 = int(__popcll(m0)), n1 = int(__popcll(m1));  // signed: a tile behind the last has fewer than no rows
  const int tiles0 = (n0 + BM - 1) / BM;
  const int sigma = t >= tiles0 ? 1 : 0, first = (sigma ? t - tiles0 : t) * BM;
  const uint64_t mine = sigma ? m1 : m0;
  const int at = int(__popcll(mine & ((1ull << lane) - 1))) - first, left = (sigma ? n1 : n0) - first;
  if (threadIdx.x < 64 && ((mine >> lane) & 1) && at >= 0 && at < BM) rows[at] = lane;
  __syncthreads();
  return FewRows{uni(sigma), uni(left < 0 ? 0 : left < BM ? left : BM)};
}

// Few rows: tiles of 16 MB rows x `width` columns (at most 16 NB), K split over the four waves of a workgroup in steps of
// 128, their sums added through LDS.  What bounds it is the weights' way from memory: every wave streams its columns'
// bytes, 32 a lane and step (whole lines of 16 rows), up to 2 GS steps ahead of the matrix core, and tiles are narrow so
// that the CUs share them evenly (2 rows of 3072 -> 18432: 57 MB of weights in 12.5 us, 4.5 TB/s).  MR > 0 (MB = 1): x are
// float rows, which every workgroup quantises for itself into LDS, MR at a time -- each wave the part of K that it
// multiplies, while its first weights are on their way; dynamic LDS holds the buffers' rows of codes.
template <bool BF16, bool GELU, int MB, int NB, int MR>
__global__ __launch_bounds__(256) void k_linear_i8_few(GemmProblem p, int width) {
  constexpr int NW = 4, GS = NB == 1 ? 3 : 2;
  constexpr bool FUSED = MR > 0;
  __shared__ i32x4 part[NW][MB * NB][64];
  __shared__ uint32_t tops[16][NW];
  __shared__ int rows[16 * MB];
  extern __shared__ __attribute__((aligned(16))) uint8_t codes[];
  const int lane = threadIdx.x & 63, wid = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int lr = lane & 15, lg = lane >> 4;
  const int n0 = blockIdx.x * width, n1 = min(n0 + width, p.N);
  const int steps = (p.K + 127) / 128, s0 = steps * wid / NW, s1 = steps * (wid + 1) / NW;
  const int kl = 16 * lg;
  const int8_t *W[NB];
  i32x4 w[2][GS][2][NB];
  auto load_w = [&](int s, i32x4 (&d)[GS][2][NB]) __attribute__((always_inline)) {
    if (s >= s1) return;
#pragma unroll
    for (int g = 0; g < GS; ++g)
#pragma unroll
      for (int h = 0; h < 2; ++h)
#pragma unroll
        for (int j = 0; j < NB; ++j) d[g][h][j] = chunk_at(W[j], 128 * min(s + g, steps - 1) + kl + 64 * h, p.K);
  };
  auto first_w = [&](int sigma) __attribute__((always_inline)) {
#pragma unroll
    for (int j = 0; j < NB; ++j)
      W[j] = reinterpret_cast<const int8_t *>(sigma ? p.W[1] : p.W[0]) + size_t(min(n0 + 16 * j + lr, n1 - 1)) * p.K;
    load_w(s0, w[0]);
    load_w(s0 + GS, w[1]);
  };
  if (p.L == 0) first_w(0);  // whose rows these are need not be known first
  const FewRows tr = few_rows(p, 16 * MB, blockIdx.y, rows);
  if (tr.n == 0) return;
  if (p.L != 0) first_w(tr.sigma);
  // wave wid finishes blocks wid, wid + NW, ... of the tile, all of one column block
  static_assert(MB * NB == 1 || NW % NB == 0, "blocks of a wave");
  const I8Cols<BF16> cols(p, tr.sigma, n0 + 16 * (wid % NB) + 4 * lg);
  const int ldc = 128 * steps + 16;  // 16 rows' chunks at one column fall on all banks
  float sa = 0.f;
  if constexpr (FUSED) {
    const int k0 = 128 * s0, k1 = 128 * s1;
    // MR rows, or their last again, and one chunk of 512 values of each at a time
    const int l8 = 8 * lane;
    for (int m0 = 0; m0 < tr.n; m0 += MR) {
      uint32_t top[MR];
      size_t at[MR];
#pragma unroll
      for (int m = 0; m < MR; ++m) {
        top[m] = 0;
        at[m] = size_t(rows[min(m0 + m, tr.n - 1)]) * p.K;
      }
      for (int c = k0; c < min(k1, p.K); c += 512) {
        Raw8<BF16> v[MR];
#pragma unroll
        for (int m = 0; m < MR; ++m) v[m].load(p.A, at[m] + min(c + l8, p.K - 8));
#pragma unroll
        for (int m = 0; m < MR; ++m) top[m] = v[m].top(top[m]);
      }
#pragma unroll
      for (int m = 0; m < MR; ++m) {
        top[m] = wave_max_u32(top[m]);
        if (lane == 0) tops[min(m0 + m, tr.n - 1)][wid] = top[m];
      }
    }
    lds_barrier();
    for (int m0 = 0; m0 < tr.n; m0 += MR) {
      float inv[MR];
      size_t at[MR];
#pragma unroll
      for (int m = 0; m < MR; ++m) {
        const int r = min(m0 + m, tr.n - 1);
        const uint32_t top = max(max(tops[r][0], tops[r][1]), max(tops[r][2], tops[r][3]));
        inv[m] = i8_inverse(top);
        if (r == lr) sa = i8_scale(top);
        at[m] = size_t(rows[r]) * p.K;
      }
      for (int c = k0; c < k1; c += 512) {
        Raw8<BF16> v[MR];
#pragma unroll
        for (int m = 0; m < MR; ++m) v[m].load(p.A, at[m] + min(c + l8, p.K - 8));
        if (c + l8 >= k1) continue;
#pragma unroll
        for (int m = 0; m < MR; ++m) {
          if (c + l8 >= p.K) v[m].zero();
          if (m0 + m < tr.n) *reinterpret_cast<uint2 *>(codes + (m0 + m) * ldc + c + l8) = v[m].codes(inv[m]);
        }
      }
    }
    __builtin_amdgcn_s_waitcnt(0xc07f);  // a wave reads back only what it wrote
    asm volatile("" ::: "memory");
  }
  const int8_t *A[MB];
#pragma unroll
  for (int i = 0; i < MB; ++i)
    A[i] = reinterpret_cast<const int8_t *>(p.A) + size_t(rows[min(16 * i + lr, tr.n - 1)]) * p.K;
  const uint8_t *cr = codes + min(lr, tr.n - 1) * ldc;
  i32x4 acc[MB][NB];
#pragma unroll
  for (int i = 0; i < MB; ++i)
#pragma unroll
    for (int j = 0; j < NB; ++j) acc[i][j] = i32x4{0, 0, 0, 0};
  auto mul = [&](int s, const i32x4 (&d)[GS][2][NB]) __attribute__((always_inline)) {
#pragma unroll
    for (int g = 0; g < GS; ++g)
      if (s + g < s1) {
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          const int k = 128 * (s + g) + kl + 64 * h;
#pragma unroll
          for (int i = 0; i < MB; ++i) {
            i32x4 a;
            if constexpr (FUSED) {
              a = *reinterpret_cast<const i32x4 *>(cr + k);
            } else {
              a = chunk_at(A[i], k, p.K);
              if (k >= p.K) a = i32x4{0, 0, 0, 0};
            }
#pragma unroll
            for (int j = 0; j < NB; ++j)
              acc[i][j] = __builtin_amdgcn_mfma_i32_16x16x64_i8(d[g][h][j], a, acc[i][j], 0, 0, 0);
          }
        }
      }
  };
#pragma unroll 1
  for (int s = s0; s < s1; s += 2 * GS) {
    mul(s, w[0]);
    load_w(s + 2 * GS, w[0]);
    mul(s + GS, w[1]);
    load_w(s + 3 * GS, w[1]);
  }
#pragma unroll
  for (int i = 0; i < MB; ++i)
#pragma unroll
    for (int j = 0; j < NB; ++j) part[wid][i * NB + j][lane] = acc[i][j];
  lds_barrier();
#pragma unroll
  for (int f = wid; f < MB * NB; f += NW) {
    const i32x4 v = (part[0][f][lane] + part[1][f][lane]) + (part[2][f][lane] + part[3][f][lane]);
    const int rl = 16 * (f / NB) + lr, n = n0 + 16 * (f % NB) + 4 * lg;
    if (rl < tr.n && n < n1) i8_out4<BF16, GELU>(p, size_t(rows[rl]), n, v, FUSED ? sa : p.a_scale[rows[rl]], cols);
  }
}

// Small products of float rows: tiles of 32 rows x 64 columns whose rows the workgroup quantises for itself into LDS,
// 8 lanes a row and NC chunks of 8 values a lane (K <= 64 NC), then every wave multiplies them by its 16 columns.  One
// launch, no codes in memory; each row is quantised N / 64 times over, which is why only small problems come here (551
// float32 rows of 256 -> 1024 in 5.6 us, a chain of load, maximum, LDS, product and store).
constexpr int kSmallK = 768;
template <bool BF16, bool GELU, int NC>
__global__ __launch_bounds__(256) void k_linear_i8_small(GemmProblem p) {
  constexpr int MB = 2, LDC = 64 * NC + 16;  // 16 rows' chunks at one column fall on all banks
  __shared__ float scale[16 * MB];
  __shared__ __attribute__((aligned(16))) uint8_t codes[16 * MB * LDC];
  const int lane = threadIdx.x & 63, wid = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int lr = lane & 15, lg = lane >> 4;
  const int tilesN = (p.N + 63) / 64, t = blockIdx.x;
  if (t >= row_tiles_total(p, 16 * MB) * tilesN) return;
  const int n = t % tilesN * 64 + 16 * wid;
  const TileRows tr = uni(decode_row_tile(p, 16 * MB, t / tilesN));
  const int steps = (p.K + 63) / 64;
  // all of the lane's part of its row
  const int r = threadIdx.x >> 3, l = threadIdx.x & 7;
  const size_t row = size_t(tr.row0 + min(r, tr.nrows - 1)) * p.K;
  Raw8<BF16> v[NC];
#pragma unroll
  for (int k = 0; k < NC; ++k) v[k].load(p.A, row + min(64 * k + 8 * l, p.K - 8));
  // and the wave's columns
  const int8_t *W = reinterpret_cast<const int8_t *>(tr.sigma ? p.W[1] : p.W[0]) + size_t(min(n + lr, p.N - 1)) * p.K;
  i32x4 w[NC];
#pragma unroll
  for (int s = 0; s < NC; ++s) w[s] = chunk_at(W, 64 * min(s, steps - 1) + 16 * lg, p.K);
  const I8Cols<BF16> cols(p, tr.sigma, n + 4 * lg);
  uint32_t top = 0;
#pragma unroll
  for (int k = 0; k < NC; ++k) top = v[k].top(top);  // behind K: the row's last values again
#pragma unroll
  for (int off = 4; off > 0; off >>= 1) top = max(top, uint32_t(__shfl_xor(int(top), off, 64)));
  const float inv = i8_inverse(top);
  if (l == 0) scale[r] = i8_scale(top);
#pragma unroll
  for (int k = 0; k < NC; ++k) {
    if (64 * k + 8 * l >= p.K) v[k].zero();
    *reinterpret_cast<uint2 *>(codes + r * LDC + 64 * k + 8 * l) = v[k].codes(inv);
  }
  lds_barrier();
  i32x4 acc[MB];
#pragma unroll
  for (int i = 0; i < MB; ++i) acc[i] = i32x4{0, 0, 0, 0};
#pragma unroll
  for (int s = 0; s < NC; ++s)
    if (s < steps) {
#pragma unroll
      for (int i = 0; i < MB; ++i) {
        const i32x4 a = *reinterpret_cast<const i32x4 *>(codes + (16 * i + lr) * LDC + 64 * s + 16 * lg);
        acc[i] = __builtin_amdgcn_mfma_i32_16x16x64_i8(w[s], a, acc[i], 0, 0, 0);
      }
    }
  if (n + 4 * lg >= p.N) return;
#pragma unroll
  for (int i = 0; i < MB; ++i) {
    const int rl = 16 * i + lr;
    if (rl < tr.nrows) i8_out4<BF16, GELU>(p, size_t(tr.row0 + rl), n + 4 * lg, acc[i], scale[rl], cols);
  }
}

// Buffers of at most this many rows take the narrow tiles (few_rows numbers no more).  Codes in, on one side and on the
// other the projections' tiles: 16 rows of 3072 -> 9216 9.8 and 19.4 us, 64 rows 18.7 and 19.1, of 3072 -> 3072 9.5 and
// 13.2, of 12288 -> 3072 28.7 and 30.9, of 1024 -> 1024 7.7 and 7.8 (both near a launch's own time).
constexpr long long kFewRows = 64;
size_t linear_i8_part_bytes(long long rows, int K) { return rows <= kFewRows || !linear_i8_cuts(K) ? 0 : kSkPartBytes; }

// Whether float rows are quantised by the kernel that multiplies them, or by a launch before it.
// Up to four rows, whose codes fit the LDS: every workgroup reads them all, so more of them cost what the launch does.
// bf16, fused and apart: 1 row of 3072 -> 18432 12.4 and 14.7 us, 4 rows 14.3 and 15.0, of 3072 -> 3072 7.6 and 10.6, of
// 8192 -> 3072 12.1 and 15.5; 5 rows of 3072 -> 9216 14.4 and 12.3, 8 rows -> 18432 18.9 and 15.7.
static bool fused_few(const GemmProblem &p) { return p.max_img_rows <= 4 && p.max_img_rows * (p.K + 144) <= 49152; }
// Short rows: a tile of 32 rows takes the time of its rows' bytes (float32's count three quarters) and 400 more each; apart
// costs the launch, the codes' way through memory and a larger kernel's start.  Fused and apart at the product below, in us:
//   bf16     551 x 256 -> 1024  (8e6)  7.6, 10.6    2000 x 512 -> 1024 (46e6) 10.7, 13.2    8000 x 128 -> 512  (42e6) 10.5, 11.7
//           1000 x 768 -> 2048 (62e6) 14.4, 14.2    1500 x 768 -> 2048 (93e6) 18.0, 14.2   16000 x 128 -> 1024 (168e6) 27.5, 18.8
//   float32 1000 x 768 -> 1536 (65e6) 13.4, 15.4    8000 x 128 -> 1024 (100e6) 18.1, 17.0
//            700 x 768 -> 2048 (61e6) 14.0, 16.0     900 x 768 -> 2048 (78e6)  16.5, 16.0
//           2500 x 512 -> 1024 (77e6) 14.4, 15.5    3000 x 512 -> 1024 (93e6)  16.2, 15.7
// The two meet at 65e6 to 75e6 in bf16 and 75e6 to 90e6 in float32, but for K = 256, where fused stays ahead further than that:
// 5000 x 256 -> 1024 12.6, 15.9 (bf16, 73e6) and 14.9, 17.7 (float32, 93e6).
static bool fused_small(const GemmProblem &p, bool bf16) {
  return p.K <= kSmallK && double(p.max_img_rows) * ((p.N + 63) / 64) * (p.K * (bf16 ? 2 : 3) + 400) <= 65e6;
}
bool linear_i8_fuses(bool bf16, const GemmProblem &p) { return fused_few(p) || fused_small(p, bf16); }

// Columns of a tile, up to 32 in one or two MFMA blocks (lanes behind them read the last column again, which costs no
// memory time): those with which the fullest CU has the least to do, as the workgroups of a CU share its way to memory.
// A workgroup costs its columns, the rows it reads for them and a start; two blocks, which leave fewer steps in flight,
// a little more.  12, 16, 20, 24, 32 columns, K = 3072, in us (18432 / 256 CUs = 72):
//    2 rows -> 18432 15.1, 13.6, 14.1, 12.8, 14.6     4 rows 17.2, 16.4, 15.7, 14.3, 15.6
//   16 rows -> 18432 18.1, 17.1, 16.5, 14.6, 15.8     -> 9216 10.6, 11.3, 9.9, 10.1, 11.3
//   64 rows -> 18432 42.5, 36.9, 34.1, 27.2, 28.2     -> 9216 22.9, 23.3, 18.3, 18.9, 19.6    -> 3072 9.5, 9.6, 11.8, 12.0, 12.4
//    2 rows -> 12288 10.6, 10.3, 11.3, 10.6, 11.0
static int few_width(int rows, int N, int row_tiles) {
  int best = 0;
  long long least = 0;
  for (int w = 8; w <= 32; w += 4) {
    const long long tiles = (long long)((N + w - 1) / w) * row_tiles;
    const long long cost = (tiles + 255) / 256 * (w + (w > 16 ? 4 : 0) + 4 + rows);
    if (best == 0 || cost < least) {
      best = w;
      least = cost;
    }
  }
  return best;
}

template <bool BF16, bool GELU>
static hipError_t run_linear_i8(const GemmProblem &p, hipStream_t st) {
  const int rows = p.max_img_rows;
  if (p.a_scale == nullptr && !fused_few(p)) {
    // row tiles: a part of one in every segment that has rows
    const long long tiles = (rows / 32 + std::min<long long>(2LL * p.B, rows)) * ((p.N + 63) / 64);
    const dim3 grid{unsigned(tiles)};
    if (p.K <= 256) hipLaunchKernelGGL((k_linear_i8_small<BF16, GELU, 4>), grid, dim3(256), 0, st, p);
    else if (p.K <= 512) hipLaunchKernelGGL((k_linear_i8_small<BF16, GELU, 8>), grid, dim3(256), 0, st, p);
    else hipLaunchKernelGGL((k_linear_i8_small<BF16, GELU, 12>), grid, dim3(256), 0, st, p);
    return hipGetLastError();
  }
  const int bm = rows <= 16 ? 16 : 64, row_tiles = (p.L > 0 ? 2 : 1) * ((rows + bm - 1) / bm);  // of either stream
  const int bn = few_width(rows, p.N, row_tiles);
  const dim3 grid(unsigned((p.N + bn - 1) / bn), unsigned(row_tiles));
  const size_t lds = p.a_scale == nullptr ? size_t(rows) * ((p.K + 127) / 128 * 128 + 16) : 0;
#define HILO_FEW(MB, NB, MR) hipLaunchKernelGGL((k_linear_i8_few<BF16, GELU, MB, NB, MR>), grid, dim3(256), lds, st, p, bn)
#define HILO_FEW_ROWS(NB)                        \
  do {                                           \
    if (p.a_scale != nullptr) {                  \
      if (rows <= 16) HILO_FEW(1, NB, 0);        \
      else HILO_FEW(4, NB, 0);                   \
    } else if (rows == 1) HILO_FEW(1, NB, 1);    \
    else if (rows == 2) HILO_FEW(1, NB, 2);      \
    else HILO_FEW(1, NB, 4);                     \
  } while (0)
  if (bn <= 16) HILO_FEW_ROWS(1);
  else HILO_FEW_ROWS(2);
#undef HILO_FEW_ROWS
#undef HILO_FEW
  return hipGetLastError();
}

hipError_t launch_linear_i8(bool bf16, bool gelu, const GemmProblem &p, hipStream_t st) {
  if (p.a_scale != nullptr && p.max_img_rows > kFewRows) return launch_linear_i8_tiled(bf16, gelu, p, st);
  if (bf16) return gelu ? run_linear_i8<true, true>(p, st) : run_linear_i8<true, false>(p, st);
  return gelu ? run_linear_i8<false, true>(p, st) : run_linear_i8<false, false>(p, st);
}

}  // namespace hilo
