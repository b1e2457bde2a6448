// Norms before and after a block of the network, fused with its gate and residual scale (hilo_norm_residual), and
// the backward pass.  Per row, with the modulation of its (sample, stream) and the gains of its stream:
//   u = norm(y) * post;  x' = alpha x + gate u;  h = norm(x') * pre * (1 + scale) + shift
// Everything in float32; x and x' are float32, y and h the block's type, or h int8 codes with a scale per row.
// What bounds both directions is memory: a row is read once, stays in registers through both norms and is written once.
#include "common.h"
#include "kernels.h"

namespace hilo {

namespace {

HILO_DEV float sum4(const float4 &a) { return (a.x + a.y) + (a.z + a.w); }
HILO_DEV float dot4(const float4 &a, const float4 &b) { return (a.x * b.x + a.y * b.y) + (a.z * b.z + a.w * b.w); }
HILO_DEV float4 ld4(const float *p) { return *reinterpret_cast<const float4 *>(p); }

template <bool BF16>
HILO_DEV float4 load4(const void *p, size_t i) {
  if constexpr (BF16) {
    const uint2 u = *reinterpret_cast<const uint2 *>(reinterpret_cast<const uint16_t *>(p) + i);
    return make_float4(__uint_as_float(u.x << 16), __uint_as_float(u.x & 0xffff0000u), __uint_as_float(u.y << 16),
                       __uint_as_float(u.y & 0xffff0000u));
  } else {
    return ld4(reinterpret_cast<const float *>(p) + i);
  }
}

template <bool BF16>
HILO_DEV void store4(void *p, size_t i, const float4 &v) {
  if constexpr (BF16) {
    *reinterpret_cast<uint2 *>(reinterpret_cast<uint16_t *>(p) + i) = make_uint2(pack_bf16x2(v.x, v.y), pack_bf16x2(v.z, v.w));
  } else {
    *reinterpret_cast<float4 *>(reinterpret_cast<float *>(p) + i) = v;
  }
}

// Sums of two values over the W waves of a row's group, on every lane.  red: two sets of W pairs, used in turn, so
// that one barrier per sum is enough (a set is written again only after the barrier of the other).
template <int W>
struct GroupSum {
  float2 *red;
  int turn = 0;
  HILO_DEV float2 operator()(float a, float b) {
    a = wave_sum_f32(a);
    b = wave_sum_f32(b);
    if constexpr (W == 1) return make_float2(a, b);
    float2 *r = red + turn * W;
    turn ^= 1;
    if ((threadIdx.x & 63) == 0) r[threadIdx.x >> 6] = make_float2(a, b);
    __syncthreads();
    float2 s = r[0];
#pragma unroll
    for (int w = 1; w < W; ++w) {
      s.x += r[w].x;
      s.y += r[w].y;
    }
    return s;
  }
};

// Mean and 1 / deviation of a row held as NV float4 a lane (columns past D are zero and not counted).  The deviation
// is taken from the differences to the mean, not from the sum of squares: a row far from zero keeps its digits.
template <int W, int NV>
HILO_DEV float2 row_stats(const float4 (&v)[NV], int c0, int D, bool rms, float eps, GroupSum<W> &sum) {
  float mean = 0.f;
  if (!rms) {
    float s = 0.f;
#pragma unroll
    for (int k = 0; k < NV; ++k) s += sum4(v[k]);
    mean = sum(s, 0.f).x / float(D);
  }
  float q = 0.f;
#pragma unroll
  for (int k = 0; k < NV; ++k) {
    if (c0 + k * 256 * W < D) {
      const float4 d = make_float4(v[k].x - mean, v[k].y - mean, v[k].z - mean, v[k].w - mean);
      q += dot4(d, d);
    }
  }
  return make_float2(mean, 1.0f / sqrtf(sum(q, 0.f).x / float(D) + eps));
}

}  // namespace

// W waves a row, NV float4 a lane: D <= 256 W NV.  A workgroup of 4 waves holds 4 / W rows (8 waves: one).
// OUT: h as 0 dtype, 1 int8 codes and row scales.
template <bool BF16, int OUT, int W, int NV>
__global__ __launch_bounds__(W > 4 ? 64 * W : 256) void k_norm_residual(NormProblem p) {
  __shared__ float2 red[2 * W];
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int row = W == 1 ? blockIdx.x * 4 + wave : blockIdx.x;
  if (row >= min(p.rows, cu_at(p.cu, p.B))) return;
  const int s = sample_of_row(p.cu, p.B, row);
  const int sigma = row >= cu_at(p.cu, s + 1) - p.L ? 1 : 0;
  const size_t m = size_t(2 * s + sigma) * p.mod_stride;
  const int c0 = 4 * (W == 1 ? threadIdx.x & 63 : threadIdx.x);
  const float *post = sigma ? p.post[1] : p.post[0], *pre = sigma ? p.pre[1] : p.pre[0];
  GroupSum<W> sum{red};
  float4 x[NV];
  const float4 zero = make_float4(0.f, 0.f, 0.f, 0.f), one = make_float4(1.f, 1.f, 1.f, 1.f);
#pragma unroll
  for (int k = 0; k < NV; ++k) {
    const int c = c0 + k * 256 * W;
    x[k] = c < p.D ? ld4(p.x + size_t(row) * p.D + c) : zero;
  }
  float4 st = zero;
  if (p.y) {
    float4 y[NV];
#pragma unroll
    for (int k = 0; k < NV; ++k) {
      const int c = c0 + k * 256 * W;
      y[k] = c < p.D ? load4<BF16>(p.y, size_t(row) * p.D + c) : zero;
    }
    const float2 t = row_stats<W, NV>(y, c0, p.D, p.rms, p.eps, sum);
    st.x = t.x;
    st.y = t.y;
#pragma unroll
    for (int k = 0; k < NV; ++k) {
      const int c = c0 + k * 256 * W;
      if (c < p.D) {
        const float4 g = p.gate ? ld4(p.gate + m + c) : one, w = post ? ld4(post + c) : one;
        x[k].x = p.alpha * x[k].x + g.x * ((y[k].x - t.x) * t.y * w.x);
        x[k].y = p.alpha * x[k].y + g.y * ((y[k].y - t.x) * t.y * w.y);
        x[k].z = p.alpha * x[k].z + g.z * ((y[k].z - t.x) * t.y * w.z);
        x[k].w = p.alpha * x[k].w + g.w * ((y[k].w - t.x) * t.y * w.w);
        *reinterpret_cast<float4 *>(p.x_out + size_t(row) * p.D + c) = x[k];
      }
    }
  }
  if (p.h) {
    const float2 t = row_stats<W, NV>(x, c0, p.D, p.rms, p.eps, sum);
    st.z = t.x;
    st.w = t.y;
    uint32_t top = 0;
#pragma unroll
    for (int k = 0; k < NV; ++k) {
      const int c = c0 + k * 256 * W;
      if (c < p.D) {
        const float4 a = p.scale ? ld4(p.scale + m + c) : zero, b = p.shift ? ld4(p.shift + m + c) : zero;
        const float4 w = pre ? ld4(pre + c) : one;
        x[k].x = (x[k].x - t.x) * t.y * w.x * (1.f + a.x) + b.x;
        x[k].y = (x[k].y - t.x) * t.y * w.y * (1.f + a.y) + b.y;
        x[k].z = (x[k].z - t.x) * t.y * w.z * (1.f + a.z) + b.z;
        x[k].w = (x[k].w - t.x) * t.y * w.w * (1.f + a.w) + b.w;
        if constexpr (OUT == 0) store4<BF16>(p.h, size_t(row) * p.D + c, x[k]);
        else top = max(max(max(abs_bits(x[k].x), abs_bits(x[k].y)), max(abs_bits(x[k].z), abs_bits(x[k].w))), top);
      }
    }
    if constexpr (OUT == 1) {
      top = wave_max_u32(top);
      if constexpr (W > 1) {
        __shared__ uint32_t tops[W];
        if ((threadIdx.x & 63) == 0) tops[wave] = top;
        __syncthreads();
#pragma unroll
        for (int w = 0; w < W; ++w) top = max(top, tops[w]);
      }
      const float inv = i8_inverse(top);
      if (c0 == 0) p.h_scale[row] = i8_scale(top);
      int8_t *o = reinterpret_cast<int8_t *>(p.h) + size_t(row) * p.D;
#pragma unroll
      for (int k = 0; k < NV; ++k) {
        const int c = c0 + k * 256 * W;
        if (c < p.D)
          *reinterpret_cast<uint32_t *>(o + c) = i8x4(x[k].x * inv, x[k].y * inv, x[k].z * inv, x[k].w * inv);
      }
    }
  }
  if (p.stats && c0 == 0) *reinterpret_cast<float4 *>(p.stats + 4 * size_t(row)) = st;
}

hipError_t launch_norm_residual(bool bf16, const NormProblem &p, hipStream_t st) {
  if (p.rows <= 0) return hipSuccess;
#define HILO_NR(W, NV)                                                                                            \
  do {                                                                                                            \
    const dim3 grid(W == 1 ? (unsigned(p.rows) + 3) / 4 : unsigned(p.rows)), block(W > 4 ? 64 * W : 256);            \
    if (p.h_scale) {                                                                                                \
      if (bf16) hipLaunchKernelGGL((k_norm_residual<true, 1, W, NV>), grid, block, 0, st, p);                       \
      else hipLaunchKernelGGL((k_norm_residual<false, 1, W, NV>), grid, block, 0, st, p);                           \
    } else {                                                                                                        \
      if (bf16) hipLaunchKernelGGL((k_norm_residual<true, 0, W, NV>), grid, block, 0, st, p);                       \
      else hipLaunchKernelGGL((k_norm_residual<false, 0, W, NV>), grid, block, 0, st, p);                           \
    }                                                                                                               \
  } while (0)
  if (p.D <= 256) HILO_NR(1, 1);
  else if (p.D <= 512) HILO_NR(1, 2);
  else if (p.D <= 1024) HILO_NR(1, 4);
  else if (p.D <= 2048) HILO_NR(4, 2);
  else if (p.D <= 3072) HILO_NR(4, 3);
  else if (p.D <= 4096) HILO_NR(4, 4);
  else HILO_NR(4, 8);
#undef HILO_NR
  return hipGetLastError();
}

// ------------------------------------------------------------------------------------- backward
//
// With xh = norm(x'), yh = norm(y) (stats kept by the forward pass):
//   n = dh (1 + scale) pre;  g = dx' + r_x (n - mean(n) - xh mean(n xh));  dx = alpha g
//   e = g gate post;  dy = r_y (e - mean(e) - yh mean(e yh))        (RMS: without the means of n and e)
// and, summed over the rows of a (sample, stream):  A = sum g yh, B = sum dh xh, C = sum dh, from which
//   dgate = post A;  dscale = pre B;  dshift = C;  dpost = sum over samples of gate A;  dpre = of (1 + scale) B.
// A worker (W waves) takes a consecutive share of all rows and keeps A, B and C of the segment it is in in registers;
// where the segment ends, and at its last row, it leaves them in a slot of its own.  Shares are never empty (no more
// workers than rows), so (worker + segment) numbers the slots without gaps or collisions, and the sums are taken in
// worker order by k_norm_sums: the same result every time, and no atomics.

struct NormSlots {
  int R, P;  // rows, workers that have rows
};
HILO_DEV NormSlots norm_slots(const int *cu, int B, int rows, int P) {
  const int R = min(rows, cu_at(cu, B));
  return NormSlots{R, min(P, R)};
}
HILO_DEV int norm_row0(const NormSlots &q, int w) { return int((long long)q.R * w / q.P); }
HILO_DEV int norm_owner(const NormSlots &q, int row) { return int(((long long)(row + 1) * q.P - 1) / q.R); }

template <bool BF16, int W, int NV>
__global__ __launch_bounds__(W > 4 ? 64 * W : 256) void k_norm_residual_back(NormBackProblem p) {
  __shared__ float2 red[2 * W];
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int w = W == 1 ? blockIdx.x * 4 + wave : blockIdx.x;
  const NormSlots q = norm_slots(p.cu, p.B, p.rows, p.P);
  if (w >= q.P) return;
  const int c0 = 4 * (W == 1 ? threadIdx.x & 63 : threadIdx.x);
  const float4 zero = make_float4(0.f, 0.f, 0.f, 0.f), one = make_float4(1.f, 1.f, 1.f, 1.f);
  const float inv_d = 1.0f / float(p.D), center = p.rms ? 0.f : 1.f;
  GroupSum<W> sum{red};
  const int last = norm_row0(q, w + 1);
  int row = norm_row0(q, w);
  while (row < last) {
    const int s = sample_of_row(p.cu, p.B, row);
    const int ts = cu_at(p.cu, s + 1) - p.L;
    const int sigma = row >= ts ? 1 : 0, end = min(last, sigma ? ts + p.L : ts);
    const size_t m = size_t(2 * s + sigma) * p.mod_stride;
    const float *post = sigma ? p.post[1] : p.post[0], *pre = sigma ? p.pre[1] : p.pre[0];
    float4 fx[NV], fy[NV];  // (1 + scale) pre and gate post
    float4 A[NV], Bs[NV], C[NV];
#pragma unroll
    for (int k = 0; k < NV; ++k) {
      const int c = c0 + k * 256 * W;
      A[k] = Bs[k] = C[k] = zero;
      fx[k] = fy[k] = one;
      if (c < p.D) {
        if (p.scale) {
          const float4 a = ld4(p.scale + m + c);
          fx[k] = make_float4(1.f + a.x, 1.f + a.y, 1.f + a.z, 1.f + a.w);
        }
        if (pre) {
          const float4 a = ld4(pre + c);
          fx[k] = make_float4(fx[k].x * a.x, fx[k].y * a.y, fx[k].z * a.z, fx[k].w * a.w);
        }
        if (p.gate) fy[k] = ld4(p.gate + m + c);
        if (post) {
          const float4 a = ld4(post + c);
          fy[k] = make_float4(fy[k].x * a.x, fy[k].y * a.y, fy[k].z * a.z, fy[k].w * a.w);
        }
      }
    }
    for (; row < end; ++row) {
      const float4 st = ld4(p.stats + 4 * size_t(row));
      float4 g[NV];
#pragma unroll
      for (int k = 0; k < NV; ++k) {
        const int c = c0 + k * 256 * W;
        g[k] = p.dx_out && c < p.D ? ld4(p.dx_out + size_t(row) * p.D + c) : zero;
      }
      if (p.dh) {
        float4 xh[NV], n[NV];
        float a = 0.f, b = 0.f;
#pragma unroll
        for (int k = 0; k < NV; ++k) {
          const int c = c0 + k * 256 * W;
          xh[k] = n[k] = zero;
          if (c < p.D) {
            const float4 x = ld4(p.x_out + size_t(row) * p.D + c), d = load4<BF16>(p.dh, size_t(row) * p.D + c);
            xh[k] = make_float4((x.x - st.z) * st.w, (x.y - st.z) * st.w, (x.z - st.z) * st.w, (x.w - st.z) * st.w);
            C[k] = make_float4(C[k].x + d.x, C[k].y + d.y, C[k].z + d.z, C[k].w + d.w);
            Bs[k] = make_float4(Bs[k].x + d.x * xh[k].x, Bs[k].y + d.y * xh[k].y, Bs[k].z + d.z * xh[k].z,
                                Bs[k].w + d.w * xh[k].w);
            n[k] = make_float4(d.x * fx[k].x, d.y * fx[k].y, d.z * fx[k].z, d.w * fx[k].w);
          }
          a += sum4(n[k]);
          b += dot4(n[k], xh[k]);
        }
        const float2 t = sum(a, b);
        const float mn = center * t.x * inv_d, mx = t.y * inv_d;
#pragma unroll
        for (int k = 0; k < NV; ++k) {
          g[k].x += st.w * (n[k].x - mn - xh[k].x * mx);
          g[k].y += st.w * (n[k].y - mn - xh[k].y * mx);
          g[k].z += st.w * (n[k].z - mn - xh[k].z * mx);
          g[k].w += st.w * (n[k].w - mn - xh[k].w * mx);
        }
      }
      if (p.y) {
        float4 yh[NV], e[NV];
        float a = 0.f, b = 0.f;
#pragma unroll
        for (int k = 0; k < NV; ++k) {
          const int c = c0 + k * 256 * W;
          yh[k] = e[k] = zero;
          if (c < p.D) {
            const float4 y = load4<BF16>(p.y, size_t(row) * p.D + c);
            yh[k] = make_float4((y.x - st.x) * st.y, (y.y - st.x) * st.y, (y.z - st.x) * st.y, (y.w - st.x) * st.y);
            A[k] = make_float4(A[k].x + g[k].x * yh[k].x, A[k].y + g[k].y * yh[k].y, A[k].z + g[k].z * yh[k].z,
                               A[k].w + g[k].w * yh[k].w);
            e[k] = make_float4(g[k].x * fy[k].x, g[k].y * fy[k].y, g[k].z * fy[k].z, g[k].w * fy[k].w);
          }
          a += sum4(e[k]);
          b += dot4(e[k], yh[k]);
        }
        const float2 t = sum(a, b);
        const float mn = center * t.x * inv_d, mx = t.y * inv_d;
#pragma unroll
        for (int k = 0; k < NV; ++k) {
          const int c = c0 + k * 256 * W;
          if (c < p.D)
            store4<BF16>(p.dy, size_t(row) * p.D + c,
                         make_float4(st.y * (e[k].x - mn - yh[k].x * mx), st.y * (e[k].y - mn - yh[k].y * mx),
                                     st.y * (e[k].z - mn - yh[k].z * mx), st.y * (e[k].w - mn - yh[k].w * mx)));
        }
      }
#pragma unroll
      for (int k = 0; k < NV; ++k) {
        const int c = c0 + k * 256 * W;
        if (c < p.D)
          *reinterpret_cast<float4 *>(p.dx + size_t(row) * p.D + c) =
              make_float4(p.alpha * g[k].x, p.alpha * g[k].y, p.alpha * g[k].z, p.alpha * g[k].w);
      }
    }
    if (p.part) {
      float *slot = p.part + size_t(w + 2 * s + sigma) * 3 * p.D;
#pragma unroll
      for (int k = 0; k < NV; ++k) {
        const int c = c0 + k * 256 * W;
        if (c < p.D) {
          *reinterpret_cast<float4 *>(slot + c) = A[k];
          *reinterpret_cast<float4 *>(slot + p.D + c) = Bs[k];
          *reinterpret_cast<float4 *>(slot + 2 * p.D + c) = C[k];
        }
      }
    }
  }
}

// Sums the slots of one segment: blockIdx.x segment, blockIdx.y 64 columns, blockIdx.z which of A, B, C.  16 lanes of
// four columns by 16 groups of slots, joined in group order.  A and B go on to the gains (sums: [2 B][2][D]).
__global__ __launch_bounds__(256) void k_norm_sums(NormBackProblem p, float *sums) {
  __shared__ float4 red[16][16];
  const int seg = blockIdx.x, s = seg >> 1, sigma = seg & 1, which = blockIdx.z;
  const NormSlots q = norm_slots(p.cu, p.B, p.rows, p.P);
  const int lo = cu_at(p.cu, s), hi = cu_at(p.cu, s + 1), ts = hi - p.L;
  const int a = min(sigma ? ts : lo, q.R), b = min(sigma ? hi : ts, q.R);
  const int lane = threadIdx.x & 15, grp = threadIdx.x >> 4, c = blockIdx.y * 64 + 4 * lane;
  float4 v = make_float4(0.f, 0.f, 0.f, 0.f);
  if (a < b && c < p.D) {
    const int w1 = norm_owner(q, b - 1);
    for (int w = norm_owner(q, a) + grp; w <= w1; w += 16) {
      const float4 t = ld4(p.part + (size_t(w + seg) * 3 + which) * p.D + c);
      v = make_float4(v.x + t.x, v.y + t.y, v.z + t.z, v.w + t.w);
    }
  }
  red[grp][lane] = v;
  __syncthreads();
  if (grp != 0 || c >= p.D) return;
#pragma unroll
  for (int g = 1; g < 16; ++g) {
    const float4 t = red[g][lane];
    v = make_float4(v.x + t.x, v.y + t.y, v.z + t.z, v.w + t.w);
  }
  if (which < 2) *reinterpret_cast<float4 *>(sums + (size_t(seg) * 2 + which) * p.D + c) = v;
  const float *gain = which == 0 ? (sigma ? p.post[1] : p.post[0]) : which == 1 ? (sigma ? p.pre[1] : p.pre[0]) : nullptr;
  float *out = which == 0 ? p.dgate : which == 1 ? p.dscale : p.dshift;
  if (!out) return;
  if (gain) {
    const float4 t = ld4(gain + c);
    v = make_float4(v.x * t.x, v.y * t.y, v.z * t.z, v.w * t.w);
  }
  *reinterpret_cast<float4 *>(out + size_t(seg) * p.dmod_stride + c) = v;
}

// The gains' gradients: blockIdx.y 0 post, 1 pre; over the samples of a stream, or of both where they share one gain.
__global__ __launch_bounds__(256) void k_norm_gains(NormBackProblem p, const float *sums) {
  const int c = blockIdx.x * 256 + threadIdx.x, which = blockIdx.y;
  if (c >= p.D) return;
  float *out[2] = {which ? p.dpre[0] : p.dpost[0], which ? p.dpre[1] : p.dpost[1]};
  float v[2] = {0.f, 0.f};
  for (int seg = 0; seg < 2 * p.B; ++seg) {
    const float *mod = which ? p.scale : p.gate;
    const float f = mod ? mod[size_t(seg) * p.mod_stride + c] + float(which) : 1.f;
    v[seg & 1] += f * sums[(size_t(seg) * 2 + which) * p.D + c];
  }
  if (out[0] && out[0] == out[1]) {
    out[0][c] = v[0] + v[1];
    return;
  }
  if (out[0]) out[0][c] = v[0];
  if (out[1]) out[1][c] = v[1];
}

static int norm_back_waves(int D) { return D <= 1024 ? 1 : D <= 4096 ? 4 : 8; }

// Workers: about 8 rows each, so that their slots (12 bytes a column) are a small part of what they read, and no more
// than fill the card.
static int norm_back_workers(int rows, int D) {
  const int most = norm_back_waves(D) == 1 ? 4096 : 1024, want = (rows + 7) / 8;
  return want < 1 ? 1 : want < most ? want : most;
}

size_t norm_back_bytes(int rows, int B, int D) {
  return ((size_t(norm_back_workers(rows, D)) + 2 * size_t(B)) * 3 + 4 * size_t(B)) * size_t(D) * sizeof(float);
}

hipError_t launch_norm_residual_back(bool bf16, NormBackProblem p, hipStream_t st) {
  p.P = norm_back_workers(p.rows, p.D);
  float *sums = p.part ? p.part + (size_t(p.P) + 2 * size_t(p.B)) * 3 * p.D : nullptr;
  if (p.rows > 0) {
#define HILO_NB(W, NV)                                                                                     \
  do {                                                                                                     \
    const dim3 grid(W == 1 ? unsigned(p.P + 3) / 4 : unsigned(p.P)), block(W > 4 ? 64 * W : 256);           \
    if (bf16) hipLaunchKernelGGL((k_norm_residual_back<true, W, NV>), grid, block, 0, st, p);              \
    else hipLaunchKernelGGL((k_norm_residual_back<false, W, NV>), grid, block, 0, st, p);                  \
  } while (0)
    if (p.D <= 256) HILO_NB(1, 1);
    else if (p.D <= 512) HILO_NB(1, 2);
    else if (p.D <= 1024) HILO_NB(1, 4);
    else if (p.D <= 2048) HILO_NB(4, 2);
    else if (p.D <= 3072) HILO_NB(4, 3);
    else if (p.D <= 4096) HILO_NB(4, 4);
    else HILO_NB(8, 4);
#undef HILO_NB
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
  }
  if (!p.part) return hipSuccess;
  hipLaunchKernelGGL(k_norm_sums, dim3(2 * p.B, (p.D + 63) / 64, 3), dim3(256), 0, st, p, sums);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess || !(p.dpost[0] || p.dpost[1] || p.dpre[0] || p.dpre[1])) return e;
  hipLaunchKernelGGL(k_norm_gains, dim3((p.D + 255) / 256, 2), dim3(256), 0, st, p, sums);
  return hipGetLastError();
}

}  // namespace hilo
