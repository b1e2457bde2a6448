// Norms before and after a block of the network, fused with its gate and residual scale (hilo_norm_residual), and
// the backward pass.  Per row, with the modulation of its (sample, stream) and the gains of its stream:
//   u = norm(y) * post;  x' = alpha x + gate u;  h = norm(x') * pre * (1 + scale) + shift
// Everything in float32; x and x' are float32, y and h the block's type, or h int8 codes with a scale per row.
// What bounds both directions is memory: a row is read once, stays in registers through both norms and is written once.
// A copy of 4 GiB reaches 4.74 TB/s; the forward pass on bf16 y 4.2 (2766 rows of 3072 in 24.0 us, with or without
// statistics; with codes out 4708 rows of 1536 in 19 us call after call, 22 to 23 between products that fill the cache), the
// backward pass 4.9 (22560 rows of 3072, 1.2 GB, in 253 us, and 11 us for the sums).  Fewer rows stay further from it: 1100
// rows of 3072 12.9 and 23 us (3.1 and 2.6 TB/s), 300 6.0 and 17.  Four rows of 3072 take 4.6 us: a load, two sums over
// four waves and a store, one behind the other.
#include "common.h"
#include "kernels.h"

namespace hilo {

namespace {

HILO_DEV float sum4(const float4 &a) { return (a.x + a.y) + (a.z + a.w); }
HILO_DEV float dot4(const float4 &a, const float4 &b) { return (a.x * b.x + a.y * b.y) + (a.z * b.z + a.w * b.w); }
HILO_DEV float4 ld4(const float *p) { return *reinterpret_cast<const float4 *>(p); }

HILO_DEV float4 mul4(const float4 &a, const float4 &b) { return make_float4(a.x * b.x, a.y * b.y, a.z * b.z, a.w * b.w); }
HILO_DEV float4 add4(const float4 &a, const float4 &b) { return make_float4(a.x + b.x, a.y + b.y, a.z + b.z, a.w + b.w); }
HILO_DEV float4 add4(const float4 &a, float b) { return make_float4(a.x + b, a.y + b, a.z + b, a.w + b); }
HILO_DEV float4 fma4(const float4 &a, const float4 &b, const float4 &c) {
  return make_float4(a.x * b.x + c.x, a.y * b.y + c.y, a.z * b.z + c.z, a.w * b.w + c.w);
}
HILO_DEV float4 zero4() { return make_float4(0.f, 0.f, 0.f, 0.f); }
HILO_DEV float4 ones4() { return make_float4(1.f, 1.f, 1.f, 1.f); }
HILO_DEV float4 shfl_xor4(const float4 &v, int m) {
  return make_float4(__shfl_xor(v.x, m), __shfl_xor(v.y, m), __shfl_xor(v.z, m), __shfl_xor(v.w, m));
}
HILO_DEV float4 only(bool in, const float4 &v) {
  return make_float4(in ? v.x : 0.f, in ? v.y : 0.f, in ? v.z : 0.f, in ? v.w : 0.f);
}
// (v - mean) * r
HILO_DEV float4 unit4(const float4 &v, float mean, float r) {
  return make_float4((v.x - mean) * r, (v.y - mean) * r, (v.z - mean) * r, (v.w - mean) * r);
}

// Loads from a uniform base and a 32-bit byte offset of the lane, in global memory.
typedef const __attribute__((address_space(1))) char *GlobalPtr;
// The base is made opaque, in scalar registers: otherwise base + offset is formed for every tensor ahead of the loop
// over rows, in two vector registers each, and the row's part is added to that.
HILO_DEV GlobalPtr global_ptr(const void *p) {
  const uint64_t u = reinterpret_cast<uint64_t>(p);
  uint32_t lo = __builtin_amdgcn_readfirstlane(uint32_t(u)), hi = __builtin_amdgcn_readfirstlane(uint32_t(u >> 32));
  asm volatile("" : "+s"(lo), "+s"(hi));
  return (GlobalPtr)((uint64_t(hi) << 32) | lo);
}
HILO_DEV float4 gld4(GlobalPtr p, uint32_t off) {
  typedef float f4 __attribute__((ext_vector_type(4)));
  const f4 v = *(const __attribute__((address_space(1))) f4 *)(p + off);
  return make_float4(v[0], v[1], v[2], v[3]);
}
HILO_DEV uint2 gld2(GlobalPtr p, uint32_t off) {
  typedef uint32_t u2 __attribute__((ext_vector_type(2)));
  const u2 v = *(const __attribute__((address_space(1))) u2 *)(p + off);
  return make_uint2(v[0], v[1]);
}

// Four values of a row of the block's type as they lie in memory.  Loads stand apart from what is done with them, and
// lanes behind the last column read the last four again: no branch parts a row's loads, so all are in flight at once.
template <bool BF16>
struct Raw4;
template <>
struct Raw4<true> {
  uint2 u;
  HILO_DEV void load(GlobalPtr row, uint32_t c) { u = gld2(row, 2 * c); }
  HILO_DEV float4 get() const {
    return make_float4(__uint_as_float(u.x << 16), __uint_as_float(u.x & 0xffff0000u), __uint_as_float(u.y << 16),
                       __uint_as_float(u.y & 0xffff0000u));
  }
};
template <>
struct Raw4<false> {
  float4 u;
  HILO_DEV void load(GlobalPtr row, uint32_t c) { u = gld4(row, 4 * c); }
  HILO_DEV float4 get() const { return u; }
};
template <bool BF16>
HILO_DEV GlobalPtr row_at(const void *p, size_t i) { return global_ptr(reinterpret_cast<const char *>(p) + i * (BF16 ? 2 : 4)); }

template <bool BF16>
HILO_DEV void store4(GlobalPtr row, uint32_t c, const float4 &v) {
  typedef float f4 __attribute__((ext_vector_type(4)));
  typedef uint32_t u2 __attribute__((ext_vector_type(2)));
  auto *p = (__attribute__((address_space(1))) char *)row;
  if constexpr (BF16) *(__attribute__((address_space(1))) u2 *)(p + 2 * c) = u2{bf16_pair(v.x, v.y), bf16_pair(v.z, v.w)};
  else *(__attribute__((address_space(1))) f4 *)(p + 4 * c) = f4{v.x, v.y, v.z, v.w};
}

// What a vector that is not given is read from: zeros, to which `by` is added (1 for a gate or a gain).
__device__ const float g_zeros[8192] = {};
struct Vector {
  GlobalPtr p;
  float by;
  HILO_DEV Vector(const float *q, size_t at, float unless) : p(global_ptr(q ? q + at : g_zeros)), by(q ? 0.f : unless) {}
  HILO_DEV float4 operator()(uint32_t c) const { return add4(gld4(p, 4 * c), by); }
};

// Sums over the W waves of a row's group, of one value or of two, on every lane.  red: two sets of W pairs, used in turn,
// so that one barrier per sum is enough (a set is written again only after the barrier of the other).
template <int W>
struct GroupSum {
  float2 *red;
  int turn = 0;
  HILO_DEV float2 operator()(float a, float b) {
    a = wave_total(a);
    b = wave_total(b);
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
  HILO_DEV float operator()(float a) {
    a = wave_total(a);
    if constexpr (W == 1) return a;
    float2 *r = red + turn * W;
    turn ^= 1;
    if ((threadIdx.x & 63) == 0) r[threadIdx.x >> 6].x = a;
    __syncthreads();
    float s = r[0].x;
#pragma unroll
    for (int w = 1; w < W; ++w) s += r[w].x;
    return s;
  }
};

// Mean and 1 / deviation of a row held as NV float4 a lane (zeros, not counted, where in[k] is false).  The deviation is
// taken from the differences to the mean, not from the sum of squares: a row far from zero keeps its digits.
template <int W, int NV>
HILO_DEV float2 row_stats(const float4 (&v)[NV], const bool (&in)[NV], float inv_d, bool rms, float eps, GroupSum<W> &sum) {
  float mean = 0.f;
  if (!rms) {
    float s = 0.f;
#pragma unroll
    for (int k = 0; k < NV; ++k) s += sum4(v[k]);
    mean = sum(s) * inv_d;
  }
  float q = 0.f;
#pragma unroll
  for (int k = 0; k < NV; ++k) {
    const float4 d = only(in[k], add4(v[k], -mean));
    q += dot4(d, d);
  }
  return make_float2(mean, 1.0f / sqrtf(sum(q) * inv_d + eps));
}

}  // namespace

// Workers take consecutive shares of the R rows in use, none of them empty: no more workers than rows.
struct NormShares {
  int R, P;
};
HILO_DEV NormShares norm_shares(const int *cu, int B, int rows, int P) {
  const int R = min(rows, cu_at(cu, B));
  return NormShares{R, min(P, R)};
}
// R w / P and the w with share_begin(w) <= row < share_begin(w + 1).  The products are whole numbers below 2^40 and the
// quotients below 2^28, so a quotient that is no whole number is 2^-28 or more from one: its double's floor is exact, in
// a fifth of the time of a 64-bit division.
HILO_DEV int share_begin(const NormShares &q, int w) {
  return __builtin_amdgcn_readfirstlane(int(double(q.R) * double(w) / double(q.P)));
}
HILO_DEV int share_owner(const NormShares &q, int row) { return int((double(row + 1) * double(q.P) - 1.0) / double(q.R)); }

// The segment of a row and where a share's rows leave it.
struct RowSegment {
  int s, sigma, end;
};
HILO_DEV RowSegment row_segment(const int *cu, int B, int L, int row, int last) {
  int s = 0, above = B;  // the largest s with cu[s] <= row, by scalar loads
  while (above - s > 1) {
    const int mid = (s + above) >> 1;
    if (cu_at(cu, mid) <= row) s = mid;
    else above = mid;
  }
  s = __builtin_amdgcn_readfirstlane(s);
  const int hi = cu_at(cu, s + 1), ts = hi - L, sigma = row >= ts ? 1 : 0;
  return RowSegment{s, sigma, min(last, sigma ? hi : ts)};
}

// Waves a SIMD that the registers leave room for.
constexpr int norm_waves(int NV) { return NV == 1 ? 8 : NV == 2 ? 5 : NV == 3 ? 4 : 3; }

// A worker is W waves, NV float4 a lane (D <= 256 W NV); W = 1: four a workgroup.  It keeps the vectors of the segment
// that its rows are in -- read for every row they are more than the row itself -- and reads a row ahead.  W and NV are
// chosen so that at most three float4 a lane leave room for four waves a SIMD or more: six on one wave a row (D = 1536)
// took 36.6 us where three on two take 20.3, and two on four 19.9 (20.0 and 18.3 with codes, whose maximum is one more
// sum over the row's waves).
// OUT: h as 0 dtype, 1 int8 codes and row scales.
template <bool BF16, int OUT, int W, int NV>
__global__ __launch_bounds__(W == 1 ? 256 : 64 * W, norm_waves(NV)) void k_norm_residual(NormProblem p) {
  __shared__ float2 red[2 * W];
  __shared__ uint32_t tops[2][W];
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int w = W == 1 ? blockIdx.x * 4 + wave : blockIdx.x;
  const NormShares q = norm_shares(p.cu, p.B, p.rows, p.P);
  if (w >= q.P) return;
  const uint32_t c0 = 4 * (W == 1 ? threadIdx.x & 63 : threadIdx.x);
  uint32_t c[NV];
  bool in[NV];
#pragma unroll
  for (int k = 0; k < NV; ++k) {
    in[k] = c0 + k * 256 * W < uint32_t(p.D);
    c[k] = in[k] ? c0 + k * 256 * W : p.D - 4;
  }
  const float inv_d = 1.0f / float(p.D);
  GroupSum<W> sum{red};
  int turn = 0;
  const int last = share_begin(q, w + 1);
  int row = share_begin(q, w);
  float4 nx[NV];
  Raw4<BF16> ny[NV];
  auto load = [&](int r) __attribute__((always_inline)) {
    const size_t at = size_t(r) * p.D;
    const GlobalPtr px = global_ptr(p.x + at), py = row_at<BF16>(p.y, at);
#pragma unroll
    for (int k = 0; k < NV; ++k) nx[k] = gld4(px, 4 * c[k]);
    if (p.y) {
#pragma unroll
      for (int k = 0; k < NV; ++k) ny[k].load(py, c[k]);
    }
  };
  load(row);
  while (row < last) {
    const RowSegment sg = row_segment(p.cu, p.B, p.L, row, last);
    const size_t m = size_t(2 * sg.s + sg.sigma) * p.mod_stride;
    float4 fy[NV], fx[NV], b[NV];  // gate post, pre (1 + scale), shift
    if (p.y) {
      const Vector gate(p.gate, m, 1.f), post(sg.sigma ? p.post[1] : p.post[0], 0, 1.f);
#pragma unroll
      for (int k = 0; k < NV; ++k) fy[k] = mul4(gate(c[k]), post(c[k]));
    }
    if (p.h) {
      const Vector scale(p.scale, m, 0.f), shift(p.shift, m, 0.f), pre(sg.sigma ? p.pre[1] : p.pre[0], 0, 1.f);
#pragma unroll
      for (int k = 0; k < NV; ++k) {
        fx[k] = mul4(pre(c[k]), add4(scale(c[k]), 1.f));
        b[k] = shift(c[k]);
      }
    }
#pragma unroll 1
    for (; row < sg.end; ++row) {
      const size_t at = size_t(row) * p.D;
      float4 x[NV], v[NV];
#pragma unroll
      for (int k = 0; k < NV; ++k) {
        x[k] = only(in[k], nx[k]);
        v[k] = only(in[k], ny[k].get());
      }
      if (row + 1 < last) load(row + 1);
      float4 st = zero4();
      if (p.y) {
        const float2 t = row_stats<W, NV>(v, in, inv_d, p.rms, p.eps, sum);
        st.x = t.x;
        st.y = t.y;
        const GlobalPtr px = global_ptr(p.x_out + at);
#pragma unroll
        for (int k = 0; k < NV; ++k) {
          const float4 u = mul4(fy[k], unit4(v[k], t.x, t.y));
          x[k] = only(in[k], make_float4(p.alpha * x[k].x + u.x, p.alpha * x[k].y + u.y, p.alpha * x[k].z + u.z,
                                         p.alpha * x[k].w + u.w));
          if (in[k]) store4<false>(px, c[k], x[k]);
        }
      }
      if (p.h) {
        const float2 t = row_stats<W, NV>(x, in, inv_d, p.rms, p.eps, sum);
        st.z = t.x;
        st.w = t.y;
        uint32_t top = 0;
        const GlobalPtr ph = global_ptr(reinterpret_cast<char *>(p.h) + at * (OUT == 1 ? 1 : BF16 ? 2 : 4));
#pragma unroll
        for (int k = 0; k < NV; ++k) {
          x[k] = fma4(fx[k], unit4(x[k], t.x, t.y), b[k]);
          if constexpr (OUT == 0) {
            if (in[k]) store4<BF16>(ph, c[k], x[k]);
          } else {
            const uint32_t a = max(max(abs_bits(x[k].x), abs_bits(x[k].y)), max(abs_bits(x[k].z), abs_bits(x[k].w)));
            top = max(top, in[k] ? a : 0u);
          }
        }
        if constexpr (OUT == 1) {
          top = wave_max_u32(top);
          if constexpr (W > 1) {  // two sets in turn, as for the sums
            turn ^= 1;
            if ((threadIdx.x & 63) == 0) tops[turn][wave] = top;
            __syncthreads();
#pragma unroll
            for (int i = 0; i < W; ++i) top = max(top, tops[turn][i]);
          }
          const float inv = i8_inverse(top);
          if (c0 == 0) p.h_scale[row] = i8_scale(top);
          auto *o = (__attribute__((address_space(1))) char *)ph;
#pragma unroll
          for (int k = 0; k < NV; ++k)
            if (in[k]) *(__attribute__((address_space(1))) uint32_t *)(o + c[k]) = i8x4(x[k].x, x[k].y, x[k].z, x[k].w, inv);
        }
      }
      if (p.stats && c0 == 0) *reinterpret_cast<float4 *>(p.stats + 4 * size_t(row)) = st;
    }
  }
}

// Workers: the same number on every CU, whose memory time they share, and no more than eight waves there (one wave a row:
// sixteen), each with a row on its way: 22560 rows of 3072 on 512, 768, 1024 workers 172.7, 176.2, 178.4 us; 1500 13.0,
// 13.5, 14.5; 6000 of 4096 on 256, 512, 768 64.7, 66.2, 69.3; 2000 of 8192 on 256 and 384 45.6 and 50.4; 9000 of 1536 on
// 768, 1024, 1280 39.4, 38.7, 40.2; 13000 of 768 on 1024, 2048, 4096 27.4, 27.8, 27.1.
template <int W>
static int norm_workers(int rows) {
  constexpr int most = W == 1 ? 4096 : 2048 / W;
  return rows < most ? rows : most;
}

hipError_t launch_norm_residual(bool bf16, NormProblem p, hipStream_t st) {
  if (p.rows <= 0) return hipSuccess;
#define HILO_NR(W, NV)                                                                                            \
  do {                                                                                                            \
    p.P = norm_workers<W>(p.rows);                                                                                  \
    const dim3 grid(W == 1 ? (unsigned(p.P) + 3) / 4 : unsigned(p.P)), block(W == 1 ? 256 : 64 * W);                \
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
  else if (p.D <= 768) HILO_NR(1, 3);
  else if (p.D <= 1024) HILO_NR(2, 2);
  else if (p.D <= 1536) HILO_NR(2, 3);
  else if (p.D <= 2048) HILO_NR(4, 2);
  else if (p.D <= 3072) HILO_NR(4, 3);
  else if (p.D <= 4096) HILO_NR(8, 2);
  else if (p.D <= 6144) HILO_NR(8, 3);
  else HILO_NR(8, 4);
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
// A worker takes a consecutive share of all rows and keeps A, B and C of the segment it is in in registers; where the
// segment ends, and at its last row, it leaves them in a slot of its own.  As shares are never empty, (worker + segment)
// numbers the slots without collisions, and the sums are taken in worker order by k_norm_sums: the same result every
// time, and no atomics.

// r (n - mean(n) - v mean(n v)) per value; without the mean of n for RMS (t.x taken as 0).
HILO_DEV float4 through4(const float4 &n, const float4 &v, float2 t, float r) {
  return make_float4(r * (n.x - t.x - v.x * t.y), r * (n.y - t.x - v.y * t.y), r * (n.z - t.x - v.z * t.y),
                     r * (n.w - t.x - v.w * t.y));
}

// A worker is a workgroup: W > 1 waves that share a row, or (W = 1) four that take rows in turn and join their sums in
// LDS where a segment ends, so that a slot holds four times the rows.
template <bool BF16, int W, int NV>
__global__ __launch_bounds__(W == 1 ? 256 : 64 * W, NV < 3 ? 3 : 2) void k_norm_residual_back(NormBackProblem p) {
  constexpr int G = W == 1 ? 4 : 1;
  __shared__ float2 red[2 * W];
  __shared__ float4 join[G == 1 ? 1 : G - 1][G == 1 ? 1 : 3 * NV][64];
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), grp = W == 1 ? wave : 0;
  const int w = blockIdx.x;
  const NormShares q = norm_shares(p.cu, p.B, p.rows, p.P);
  if (w >= q.P) return;
  const uint32_t c0 = 4 * (W == 1 ? threadIdx.x & 63 : threadIdx.x);
  uint32_t c[NV];
  bool in[NV];
#pragma unroll
  for (int k = 0; k < NV; ++k) {
    in[k] = c0 + k * 256 * W < uint32_t(p.D);
    c[k] = in[k] ? c0 + k * 256 * W : p.D - 4;
  }
  const float inv_d = 1.0f / float(p.D), center = p.rms ? 0.f : inv_d;
  GroupSum<W> sum{red};
  const int last = share_begin(q, w + 1);
  int first = share_begin(q, w);
  while (first < last) {
    const RowSegment sg = row_segment(p.cu, p.B, p.L, first, last);
    const size_t m = size_t(2 * sg.s + sg.sigma) * p.mod_stride;
    float4 fx[NV], fy[NV];  // (1 + scale) pre and gate post, zero behind the last column
    float4 A[NV], B[NV], C[NV];
    {
      const Vector gate(p.gate, m, 1.f), scale(p.scale, m, 0.f);
      const Vector post(sg.sigma ? p.post[1] : p.post[0], 0, 1.f), pre(sg.sigma ? p.pre[1] : p.pre[0], 0, 1.f);
#pragma unroll
      for (int k = 0; k < NV; ++k) {
        fx[k] = only(in[k], mul4(add4(scale(c[k]), 1.f), pre(c[k])));
        fy[k] = only(in[k], mul4(gate(c[k]), post(c[k])));
        A[k] = B[k] = C[k] = zero4();
      }
    }
    // a row's loads, a row ahead: they are in flight while the row before is summed
    float4 ng[NV], nx[NV], nst;
    Raw4<BF16> ndh[NV], ny[NV];
    auto load = [&](int r) __attribute__((always_inline)) {
      const size_t at = size_t(r) * p.D;
      nst = gld4(global_ptr(p.stats + 4 * size_t(r)), 0);
      if (p.dh) {
        const GlobalPtr pd = row_at<BF16>(p.dh, at), px = global_ptr(p.x_out + at);
#pragma unroll
        for (int k = 0; k < NV; ++k) {
          ndh[k].load(pd, c[k]);
          nx[k] = gld4(px, 4 * c[k]);
        }
      }
      if (p.dx_out) {
        const GlobalPtr pg = global_ptr(p.dx_out + at);
#pragma unroll
        for (int k = 0; k < NV; ++k) ng[k] = gld4(pg, 4 * c[k]);
      }
      if (p.y) {
        const GlobalPtr py = row_at<BF16>(p.y, at);
#pragma unroll
        for (int k = 0; k < NV; ++k) ny[k].load(py, c[k]);
      }
    };
    if (first + grp < sg.end) load(first + grp);
#pragma unroll 1
    for (int row = first + grp; row < sg.end; row += G) {
      const size_t at = size_t(row) * p.D;
      float4 g[NV], x[NV];
      Raw4<BF16> dh[NV], y[NV];
      const float4 st = nst;
#pragma unroll
      for (int k = 0; k < NV; ++k) {
        g[k] = p.dx_out ? ng[k] : zero4();
        x[k] = nx[k];
        dh[k] = ndh[k];
        y[k] = ny[k];
      }
      if (row + G < sg.end) load(row + G);
      if (p.dh) {
        float a = 0.f, b = 0.f;
#pragma unroll
        for (int k = 0; k < NV; ++k) {
          const float4 d = dh[k].get();
          x[k] = unit4(x[k], st.z, st.w);
          C[k] = add4(C[k], d);
          B[k] = fma4(d, x[k], B[k]);
          const float4 n = mul4(d, fx[k]);
          a += sum4(n);
          b += dot4(n, x[k]);
        }
        float2 t = sum(a, b);
        t = make_float2(t.x * center, t.y * inv_d);
#pragma unroll
        for (int k = 0; k < NV; ++k) g[k] = add4(g[k], through4(mul4(dh[k].get(), fx[k]), x[k], t, st.w));
      }
      if (p.y) {
        float a = 0.f, b = 0.f;
#pragma unroll
        for (int k = 0; k < NV; ++k) {
          const float4 v = unit4(y[k].get(), st.x, st.y), e = mul4(g[k], fy[k]);
          A[k] = fma4(g[k], v, A[k]);
          a += sum4(e);
          b += dot4(e, v);
        }
        float2 t = sum(a, b);
        t = make_float2(t.x * center, t.y * inv_d);
        const GlobalPtr dy = row_at<BF16>(p.dy, at);
#pragma unroll
        for (int k = 0; k < NV; ++k)
          if (in[k]) store4<BF16>(dy, c[k], through4(mul4(g[k], fy[k]), unit4(y[k].get(), st.x, st.y), t, st.y));
      }
      const GlobalPtr dx = global_ptr(p.dx + at);
#pragma unroll
      for (int k = 0; k < NV; ++k)
        if (in[k])
          store4<false>(dx, c[k], make_float4(p.alpha * g[k].x, p.alpha * g[k].y, p.alpha * g[k].z, p.alpha * g[k].w));
    }
    if (p.part) {
      if constexpr (G > 1) {
        const int lane = threadIdx.x & 63;
        if (grp > 0) {
#pragma unroll
          for (int k = 0; k < NV; ++k) {
            join[grp - 1][k][lane] = A[k];
            join[grp - 1][NV + k][lane] = B[k];
            join[grp - 1][2 * NV + k][lane] = C[k];
          }
        }
        __syncthreads();
        if (grp == 0) {
#pragma unroll
          for (int i = 0; i < G - 1; ++i)
#pragma unroll
            for (int k = 0; k < NV; ++k) {
              A[k] = add4(A[k], join[i][k][lane]);
              B[k] = add4(B[k], join[i][NV + k][lane]);
              C[k] = add4(C[k], join[i][2 * NV + k][lane]);
            }
        }
      }
      float *slot = p.part + size_t(w + 2 * sg.s + sg.sigma) * 3 * p.D;
      const GlobalPtr sa = global_ptr(slot), sb = global_ptr(slot + p.D), sc = global_ptr(slot + 2 * p.D);
#pragma unroll
      for (int k = 0; k < NV; ++k)
        if (in[k] && grp == 0) {
          store4<false>(sa, c[k], A[k]);
          store4<false>(sb, c[k], B[k]);
          store4<false>(sc, c[k], C[k]);
        }
      if constexpr (G > 1) __syncthreads();  // the next segment's sums go to the same LDS
    }
    first = sg.end;
  }
}

// The sums over a stream's slots: blockIdx.x stream (or, where both share a gain, both in turn), blockIdx.y 64 columns,
// blockIdx.z which of A, B, C.  16 lanes of four columns by 64 groups; a sample's slots are dealt to 64 / samples groups
// (a power of two), whose sums are joined in group order and written with the sample's vectors; then the gain's gradient
// over the samples, in their order.  One launch for both: the gains' sums in a second one took 5 us more for few rows.
// Registers for two workgroups a CU, which hold all of them at once (D = 3072: 288; one a CU and a second round 13.8 us
// for 19 MB of slots, 10.8 now).
__global__ __launch_bounds__(1024, 8) void k_norm_sums(NormBackProblem p, bool both) {
  constexpr int G = 64;
  __shared__ float4 red[G][16];
  const int which = blockIdx.z, lane = threadIdx.x & 15, grp = threadIdx.x >> 4, c = blockIdx.y * 64 + 4 * lane;
  const bool in = c < p.D;
  const NormShares q = norm_shares(p.cu, p.B, p.rows, p.P);
  int per = G;  // groups of a sample
  while (per > 1 && per * p.B > G) per /= 2;
  const int part = grp % per, samples = G / per, step = min(per, 4);  // four groups of a wave are joined by shuffles
  const float *mod = which == 0 ? p.gate : which == 1 ? p.scale : nullptr;
  float *out = which == 0 ? p.dgate : which == 1 ? p.dscale : p.dshift;
  float4 shared_gain = zero4();
  for (int sigma = both ? 0 : blockIdx.x; sigma <= (both ? 1 : int(blockIdx.x)); ++sigma) {
    const float *post = sigma ? p.post[1] : p.post[0], *pre = sigma ? p.pre[1] : p.pre[0];
    const float *w = which == 0 ? post : which == 1 ? pre : nullptr;
    const float4 weight = w && in ? ld4(w + c) : ones4();
    float4 gain = zero4();
    for (int s0 = 0; s0 < p.B; s0 += samples) {
      const int s = s0 + grp / per;
      const size_t seg = 2 * size_t(s) + sigma;
      float4 v = zero4(), factor = ones4();
      if (s < p.B && in) {
        if (mod && part == 0) factor = add4(ld4(mod + seg * p.mod_stride + c), float(which));
        const int lo = p.cu[s], hi = p.cu[s + 1], ts = hi - p.L;
        const int a = min(sigma ? ts : lo, q.R), b = min(sigma ? hi : ts, q.R);
        if (a < b) {
          const int w1 = share_owner(q, b - 1);
          for (int w = share_owner(q, a) + part; w <= w1; w += 4 * per) {  // four slots' loads at a time
            float4 t[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) t[i] = ld4(p.part + (size_t(min(w + per * i, w1) + seg) * 3 + which) * p.D + c);
#pragma unroll
            for (int i = 0; i < 4; ++i)
              if (w + per * i <= w1) v = add4(v, t[i]);
          }
        }
      }
      if (per >= 2) v = add4(v, shfl_xor4(v, 16));
      if (per >= 4) v = add4(v, shfl_xor4(v, 32));
      __syncthreads();  // the last samples' sums have been read
      red[grp][lane] = v;
      __syncthreads();
      if (part == 0 && s < p.B && in) {
#pragma unroll 4
        for (int i = step; i < per; i += step) v = add4(v, red[grp + i][lane]);
        if (out) *reinterpret_cast<float4 *>(out + seg * p.dmod_stride + c) = mul4(v, weight);
        red[grp][lane] = mul4(v, factor);
      }
      __syncthreads();
      if (which < 2 && grp == 0 && in) {
#pragma unroll 4
        for (int i = 0; i < min(samples, p.B - s0); ++i) gain = add4(gain, red[i * per][lane]);
      }
    }
    float *const *d = which ? p.dpre : p.dpost;
    if (which < 2 && grp == 0 && in) {
      if (d[0] && d[0] == d[1]) {
        shared_gain = add4(shared_gain, gain);
        if (sigma == 1) *reinterpret_cast<float4 *>(d[0] + c) = shared_gain;
      } else if (sigma ? d[1] : d[0]) {
        *reinterpret_cast<float4 *>((sigma ? d[1] : d[0]) + c) = gain;
      }
    }
  }
}

// Workers: the same number on every CU here too, about five rows for each (one wave a row: ten for its four), since a slot
// costs 24 bytes a column where a row costs 18 and more, and at most one, two or three a CU: 22560 rows of 3072 on 256, 512,
// 768 workers 291.6, 265.2, 270.9 us, 2766 51.3, 51.1, 54.0, 1100 27.5, 30.9, 33.8; 5000 of 5120 on 256, 384, 512 111.5,
// 130.6, 117.5; 9000 of 1536 on 512, 768, 1024 68.3, 65.0, 66.2; 13000 of 512 39.1, 36.8, 38.2, 2000 of 512 on 256 and 512
// 13.9 and 14.5.
static int norm_back_workers(int rows, int D) {
  const int share = 256 * (D <= 768 ? 10 : 5), most = D > 3072 ? 1 : D > 1536 || (D > 512 && D <= 768) ? 2 : 3;
  const int a_cu = (rows + share / 2) / share, workers = 256 * (a_cu < 1 ? 1 : a_cu < most ? a_cu : most);
  return rows < 1 ? 1 : rows < workers ? rows : workers;
}

size_t norm_back_bytes(int rows, int B, int D) {
  return (size_t(norm_back_workers(rows, D)) + 2 * size_t(B)) * 3 * size_t(D) * sizeof(float);
}

hipError_t launch_norm_residual_back(bool bf16, NormBackProblem p, hipStream_t st) {
  p.P = norm_back_workers(p.rows, p.D);
  if (p.rows > 0) {
#define HILO_NB(W, NV)                                                                                     \
  do {                                                                                                     \
    const dim3 grid{unsigned(p.P)}, block(W == 1 ? 256 : 64 * W);                                          \
    if (bf16) hipLaunchKernelGGL((k_norm_residual_back<true, W, NV>), grid, block, 0, st, p);              \
    else hipLaunchKernelGGL((k_norm_residual_back<false, W, NV>), grid, block, 0, st, p);                  \
  } while (0)
    if (p.D <= 256) HILO_NB(1, 1);
    else if (p.D <= 512) HILO_NB(1, 2);
    else if (p.D <= 768) HILO_NB(1, 3);
    else if (p.D <= 1024) HILO_NB(2, 2);
    else if (p.D <= 1536) HILO_NB(2, 3);
    else if (p.D <= 2048) HILO_NB(4, 2);
    else if (p.D <= 3072) HILO_NB(4, 3);
    else if (p.D <= 4096) HILO_NB(8, 2);
    else if (p.D <= 6144) HILO_NB(8, 3);
    else HILO_NB(8, 4);
#undef HILO_NB
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
  }
  if (!p.part) return hipSuccess;
  const bool both = (p.dpost[0] && p.dpost[0] == p.dpost[1]) || (p.dpre[0] && p.dpre[0] == p.dpre[1]);
  hipLaunchKernelGGL(k_norm_sums, dim3(both ? 1 : 2, (p.D + 63) / 64, 3), dim3(1024), 0, st, p, both);
  return hipGetLastError();
}

}  // namespace hilo
