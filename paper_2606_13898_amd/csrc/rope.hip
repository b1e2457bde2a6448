// Rotary positions with several axes on packed rows (hilo_rope), and the positions of a compressed sequence's
// tokens (hilo_token_positions).
//
// Pair j of a head turns by t = position(axis of j) * frequency(j):  (a, b) -> (a cos t - b sin t, b cos t + a sin t).
// All heads of a row turn alike, so a workgroup forms the cosines and sines of its rows once, in 64 bits, keeps them
// as floats in LDS and streams the heads past them.  What bounds it is memory: every value is read and written once.
// 2766 rows of 48 bf16 heads of 128 out of a packed projection, 68 MB, in 11.8 us (5.7 TB/s: a part comes from the last
// level's cache; a copy of 4 GiB reaches 4.7); 22560 rows of 16 float32 heads of 64, 185 MB, in 35.0 us (5.3 TB/s).  One
// row takes 2.8 us, most of it the launch and the one chain of doubles to a cosine.
#include "common.h"
#include "kernels.h"

namespace hilo {

namespace {

// cos and sin of 2 pi t.  The turn is reduced in double (a position of millions of turns keeps its fraction: k_rope forms
// the frequencies in double too, as powers of 2 whose logarithms the host takes), to at most an eighth from the nearest
// quarter; there the Taylor series of both, to the 13th and 12th power, are off by less than 2^-40.  Rounded to float once.
HILO_DEV float2 turn(double t) {
  const double q = rint(4.0 * t);
  const double x = (t - 0.25 * q) * 6.283185307179586476925;
  const double y = x * x;
  const double s = x * (1.0 + y * (-1.0 / 6 + y * (1.0 / 120 + y * (-1.0 / 5040 + y * (1.0 / 362880 + y * (-1.0 / 39916800 + y * (1.0 / 6227020800.0)))))));
  const double c = 1.0 + y * (-0.5 + y * (1.0 / 24 + y * (-1.0 / 720 + y * (1.0 / 40320 + y * (-1.0 / 3628800 + y * (1.0 / 479001600.0))))));
  const int k = int(q - 4.0 * floor(0.25 * q));  // quarter 0 .. 3 (a NaN position: 0, with a NaN series)
  const double cc = (k & 1) ? s : c, ss = (k & 1) ? c : s;
  return make_float2(float(k == 1 || k == 2 ? -cc : cc), float(k >= 2 ? -ss : ss));
}

// 2^x, |x| kept to 1000: the whole part in the exponent, e^y of the rest, at most half an octave, by its Taylor series to
// the 14th power (off by less than 2^-56).
HILO_DEV double pow2(double x) {
  x = fmin(fmax(x, -1000.0), 1000.0);
  const double k = rint(x), y = (x - k) * 0.69314718055994530942;
  double s = 1.0;
#pragma unroll
  for (int i = 14; i > 0; --i) s = 1.0 + (y * s) * (1.0 / double(i));
  return s * __longlong_as_double((long long)(int(k) + 1023) << 52);
}

template <int BYTES>
struct Raw;
template <> struct Raw<2> { using T = uint16_t; };
template <> struct Raw<4> { using T = uint32_t; };
template <> struct Raw<8> { using T = uint2; };
template <> struct Raw<16> { using T = uint4; };

// V consecutive values of a row.
template <bool BF16, int V>
struct Vec {
  using E = std::conditional_t<BF16, uint16_t, float>;
  union {
    typename Raw<V * sizeof(E)>::T raw;
    E e[V];
  };
  HILO_DEV float get(int i) const {
    if constexpr (BF16) return bf2f(e[i]);
    else return e[i];
  }
  HILO_DEV void set(int i, float v) {
    if constexpr (BF16) e[i] = f2bf(v);
    else e[i] = v;
  }
};

}  // namespace

// A unit is V pairs of one head (two vectors of V values: at columns j and j + n, or 2 j and 2 j + V), or, where
// rows are copied, V columns behind the rotated ones.  A workgroup takes p.block_rows rows.
template <bool BF16, int V, bool ADJ>
__global__ __launch_bounds__(256) void k_rope(RopeProblem p) {
  using E = std::conditional_t<BF16, uint16_t, float>;
  using VV = Vec<BF16, V>;
  // rows may start at any value: the launcher takes a V whose bytes divide every address, and a VV asks for no more
  static_assert(sizeof(VV) == V * sizeof(E) && alignof(VV) == V * sizeof(E), "a vector is its values and no more");
  __shared__ float2 cs[kRopeTable];
  const int rows = p.rows_end ? min((long long)p.rows, (long long)cu_at(p.rows_end, 0)) : p.rows;
  const int row0 = blockIdx.x * p.block_rows, nr = min(p.block_rows, rows - row0);
  if (nr <= 0) return;
  for (int i = threadIdx.x; i < nr * p.n; i += 256) {
    const int r = i / p.n, j = i - r * p.n;
    const int a = (j >= p.first[1]) + (j >= p.first[2]) + (j >= p.first[3]);
    const int first = a == 0 ? 0 : a == 1 ? p.first[1] : a == 2 ? p.first[2] : p.first[3];
    const double step = a == 0 ? p.step[0] : a == 1 ? p.step[1] : a == 2 ? p.step[2] : p.step[3];
    const double freq = pow2(-step * double(p.one_spectrum ? j : j - first)) * 0.15915494309189533577;  // in turns
    float2 v = turn(double(p.pos[size_t(row0 + r) * p.axes + a]) * freq);
    if (p.backward) v.y = -v.y;
    cs[i] = v;
  }
  __syncthreads();
  const int per_head = p.units_head, units = nr * p.heads * per_head;
  const int turned = p.n / V;
  for (int i = threadIdx.x; i < units; i += 256) {
    const int q = i / per_head, u = i - q * per_head, r = q / p.heads, h = q - r * p.heads;
    const size_t row = size_t(row0 + r);
    const E *x = reinterpret_cast<const E *>(p.x) + row * p.ldx + size_t(h) * p.hd;
    E *o = reinterpret_cast<E *>(p.out) + row * p.ldo + size_t(h) * p.hd;
    if (u >= turned) {
      const int c = 2 * p.n + (u - turned) * V;
      reinterpret_cast<VV *>(o + c)->raw = reinterpret_cast<const VV *>(x + c)->raw;
      continue;
    }
    const float2 *t = cs + r * p.n + u * V;
    const int c0 = ADJ ? 2 * u * V : u * V, c1 = ADJ ? c0 + V : c0 + p.n;
    VV a, b, y, z;
    a.raw = reinterpret_cast<const VV *>(x + c0)->raw;
    b.raw = reinterpret_cast<const VV *>(x + c1)->raw;
#pragma unroll
    for (int e = 0; e < V; ++e) {
      const float2 w = t[e];
      // value k of the 2 V in column order is element k % V of a or b
      const int ka = ADJ ? 2 * e : e, kb = ADJ ? 2 * e + 1 : V + e;
      const float av = ka < V ? a.get(ka % V) : b.get(ka % V), bv = kb < V ? a.get(kb % V) : b.get(kb % V);
      const float u0 = av * w.x - bv * w.y, u1 = bv * w.x + av * w.y;
      if (ka < V) y.set(ka % V, u0);
      else z.set(ka % V, u0);
      if (kb < V) y.set(kb % V, u1);
      else z.set(kb % V, u1);
    }
    reinterpret_cast<VV *>(o + c0)->raw = y.raw;
    reinterpret_cast<VV *>(o + c1)->raw = z.raw;
  }
}

hipError_t launch_rope(bool bf16, RopeProblem p, hipStream_t st) {
  if (p.rows <= 0) return hipSuccess;
  const bool copy = p.x != p.out || p.ldx != p.ldo;
  const int e = bf16 ? 2 : 4, rest = p.hd - 2 * p.n;
  // the widest vectors that the columns and both addresses allow
  int V = bf16 ? 8 : 4;
  auto fits = [&](int v) {
    const uintptr_t a = uintptr_t(p.x) | uintptr_t(p.out) | uintptr_t(p.ldx * e) | uintptr_t(p.ldo * e);
    return p.n % v == 0 && rest % v == 0 && p.hd % v == 0 && a % uintptr_t(v * e) == 0;
  };
  while (V > 1 && !fits(V)) V /= 2;
  p.units_head = p.n / V + (copy ? rest / V : 0);
  // rows of a workgroup: a unit a thread and no more than one row over, and a table that fits.  Forming the table (about 70
  // operations in doubles a row and pair, for all heads) hides behind other workgroups' loads, better the more there are:
  // with 1, 2, 4, 9 units a thread 7680 rows of 48 heads of 128 38.1, 39.1, 40.6, 41.5 us, 1100 6.8, 6.7, 7.4, 9.6,
  // 22560 float32 rows of 16 heads of 64 35.0, 36.0, 36.6, 40.7
  const int row_units = p.heads * p.units_head;
  const int br = (256 + row_units - 1) / row_units;
  p.block_rows = br < kRopeTable / p.n ? br : kRopeTable / p.n;
  const dim3 grid{unsigned((p.rows + p.block_rows - 1) / p.block_rows)};
#define HILO_ROPE(B, VV)                                                              \
  do {                                                                                \
    if (p.adjacent) hipLaunchKernelGGL((k_rope<B, VV, true>), grid, dim3(256), 0, st, p); \
    else hipLaunchKernelGGL((k_rope<B, VV, false>), grid, dim3(256), 0, st, p);       \
  } while (0)
  if (bf16) {
    if (V == 8) HILO_ROPE(true, 8);
    else if (V == 4) HILO_ROPE(true, 4);
    else if (V == 2) HILO_ROPE(true, 2);
    else HILO_ROPE(true, 1);
  } else {
    if (V == 4) HILO_ROPE(false, 4);
    else if (V == 2) HILO_ROPE(false, 2);
    else HILO_ROPE(false, 1);
  }
#undef HILO_ROPE
  return hipGetLastError();
}

// One thread per row slot (the slots of the compress pass: every grid's fine patches and pooled blocks, then text).  A
// launch's own time: 2763 tokens of one image in 2.2 us, 40112 of 16 images in 2.3 (captured, call after call).
__global__ __launch_bounds__(256) void k_token_positions(const int *__restrict__ fine_idx, const int *__restrict__ pool_idx,
                                                         const int *__restrict__ counts, const int *__restrict__ cu,
                                                         const int *__restrict__ seg, const float *__restrict__ text_pos,
                                                         float *__restrict__ pos, int G, int I, int N, int W, int L,
                                                         long long nslots) {
  const int R = N + N / 4;
  const long long slot = (long long)blockIdx.x * 256 + threadIdx.x, img = (long long)G * R;
  if (slot >= nslots) return;
  float t, h, w;
  size_t dst;
  if (slot < img) {
    const int g = int(slot / R), k = int(slot - (long long)g * R);
    const int nf = counts[2 * g], np = counts[2 * g + 1];
    if (k >= nf + np) return;
    dst = size_t(seg[g]) + k;
    t = float(g % I);
    if (k < nf) {
      const int p = fine_idx[size_t(g) * N + k];
      h = float(p / W);
      w = float(p % W);
    } else {
      const int b = pool_idx[size_t(g) * (N / 4) + (k - nf)];
      h = float(b / (W / 2) * 2) + 0.5f;
      w = float(b % (W / 2) * 2) + 0.5f;
    }
  } else {
    const long long i = slot - img;
    const int s = int(i / L), j = int(i - (long long)s * L);
    dst = size_t(cu[s + 1]) - L + j;
    t = text_pos ? text_pos[3 * j] : 0.f;
    h = text_pos ? text_pos[3 * j + 1] : 0.f;
    w = text_pos ? text_pos[3 * j + 2] : 0.f;
  }
  pos[3 * dst] = t;
  pos[3 * dst + 1] = h;
  pos[3 * dst + 2] = w;
}

hipError_t launch_token_positions(const int *fine_idx, const int *pool_idx, const int *counts, const int *cu,
                                  const int *seg, const float *text_pos, float *pos, int B, int I, int H, int W, int L,
                                  hipStream_t st) {
  const int N = H * W;
  const long long nslots = (long long)B * I * (N + N / 4) + (long long)B * L;
  hipLaunchKernelGGL(k_token_positions, dim3(unsigned((nslots + 255) / 256)), dim3(256), 0, st, fine_idx, pool_idx, counts,
                     cu, seg, text_pos, pos, B * I, I, N, W, L, nslots);
  return hipGetLastError();
}

}  // namespace hilo
