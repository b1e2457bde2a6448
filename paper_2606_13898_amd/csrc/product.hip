// Products of a feed-forward with their gradients (hilo_linear, hilo_linear_backward, hilo_linear_fp8):
//   PRODUCT_OUT  u = x w^T + b, or with a gate act(x wg^T + bg) u
//   PRODUCT_DX   dx = sum over parts of d_part w_part
//   PRODUCT_DW   dw_part = d_part^T x over the rows of a stream
// Here in float32 on the matrix cores, of float32 operands or of codes; bf16 and FP8 have kernels of their own
// (product_bf16.hip, product_fp8.hip, product_few.hip).  And what stands beside the products: the way back through the
// gate, sums over rows, quantisation.
#include <algorithm>

#include "product.h"

namespace hilo {

enum ProductType { TYPE_F32, TYPE_BF16, TYPE_FP8 };

// 8 consecutive values of an operand
template <int TYPE>
struct Chunk {
  uint4 u[TYPE == TYPE_F32 ? 2 : 1];
  float scale;
  HILO_DEV void zero() {
    u[0] = make_uint4(0u, 0u, 0u, 0u);
    if constexpr (TYPE == TYPE_F32) u[1] = u[0];
    scale = 0.f;
  }
  HILO_DEV void load(const void *x, size_t i) {
    if constexpr (TYPE == TYPE_FP8) {
      const uint2 v = *reinterpret_cast<const uint2 *>(reinterpret_cast<const uint8_t *>(x) + i);
      u[0].x = v.x;
      u[0].y = v.y;
    } else {
      const uint4 *p = reinterpret_cast<const uint4 *>(reinterpret_cast<const char *>(x) + i * (TYPE == TYPE_BF16 ? 2 : 4));
      u[0] = p[0];
      if constexpr (TYPE == TYPE_F32) u[1] = p[1];
    }
  }
  HILO_DEV void values(float (&f)[8]) const {
    if constexpr (TYPE == TYPE_BF16) {
      unpack8(u[0], f);
    } else if constexpr (TYPE == TYPE_FP8) {
      const uint32_t w[2] = {u[0].x, u[0].y};
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        const auto a = __builtin_amdgcn_cvt_pk_f32_fp8(w[h], false), b = __builtin_amdgcn_cvt_pk_f32_fp8(w[h], true);
        f[4 * h] = a[0] * scale; f[4 * h + 1] = a[1] * scale;
        f[4 * h + 2] = b[0] * scale; f[4 * h + 3] = b[1] * scale;
      }
    } else {
      f[0] = __uint_as_float(u[0].x); f[1] = __uint_as_float(u[0].y); f[2] = __uint_as_float(u[0].z); f[3] = __uint_as_float(u[0].w);
      f[4] = __uint_as_float(u[1].x); f[5] = __uint_as_float(u[1].y); f[6] = __uint_as_float(u[1].z); f[7] = __uint_as_float(u[1].w);
    }
  }
};

template <bool BF16>
HILO_DEV void store8(void *o, size_t i, const float (&f)[8]) {
  if constexpr (BF16) {
    *reinterpret_cast<uint4 *>(reinterpret_cast<uint16_t *>(o) + i) =
        make_uint4(bf16_pair(f[0], f[1]), bf16_pair(f[2], f[3]), bf16_pair(f[4], f[5]), bf16_pair(f[6], f[7]));
  } else {
    float4 *q = reinterpret_cast<float4 *>(reinterpret_cast<float *>(o) + i);
    q[0] = make_float4(f[0], f[1], f[2], f[3]);
    q[1] = make_float4(f[4], f[5], f[6], f[7]);
  }
}

// The value of an E8M0 byte; 255 stands for NaN.
HILO_DEV float e8m0(uint8_t b) {
  return b == 255 ? __uint_as_float(0x7fc00000u) : b == 0 ? __uint_as_float(0x00400000u) : __uint_as_float(uint32_t(b) << 23);
}

// Tiles of 64 x 64 outputs (with a gate, of 32 columns of either part) on two groups of 4 waves of 32 x 32: a group takes every
// other step of 32 values of k, through two LDS buffers of its own, with kAhead steps more on their way to registers, and
// the groups' sums meet in LDS.  Both operands lie in LDS as [row][k], whichever index is last in memory; rows are kPad
// values long, so that 16 lanes' 16-byte reads fall on all banks once.  A lane of group lg takes k = 16 s + 4 lg .. + 3.
//
// Bound by the float32 MFMA: 2048 x 4096 -> 4096 in 558 us, 123 TFLOP/s (the library's product reaches 131), its dx alone 587, its
// dw 646, whose operands both are transposed on their way to LDS.  Small ones by a launch, two loads on their way and the
// tiles' number: 551 x 256 -> 1024 with a gate, 288 tiles for 256 CUs, 15.2 us, of which 6.6 do not grow with K.  Both
// products of its gradients in a launch, and what is left in another: 33.9 us; in launches of their own 48.4.  Transposing
// with four lanes' stores on a bank: 39.3.
constexpr int kStep = 32, kPad = 36, kAhead = 2;

// 8 values of a step of an operand, as a thread loads them and lays them into LDS as [row][k].
template <int TYPE>
struct Piece {
  typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
  typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
  u32x4 u[TYPE == TYPE_F32 ? 2 : 1];  // codes: the first two
  uint32_t scale;
  static HILO_DEV int half(int wid) { return (TYPE == TYPE_F32 ? wid >> 1 : wid) & 1; }
  // With k first 16 lanes have 16 columns of 8 k, so that the 8-byte stores to 16 rows of LDS fall on 32 banks, not on 8.
  static HILO_DEV int k_first(int tid) { return 8 * (tid >> 6) + 2 * (tid >> 2 & 3); }
  static HILO_DEV int col_first(int tid) { return 16 * (tid >> 4 & 3) + 4 * (tid & 3); }
  // From the tile's first value x[at] on, `pitch` values from row to row of memory, of which there are `rows` of `cols`.
  // K_LAST: a row has consecutive k.  float32: 4 values of two rows 32 apart, codes: 8 of one; PAIRED: rows of 16 columns
  // of one part and of the other.  Otherwise a row of memory has one k: 4 values of each of two consecutive k.
  template <bool K_LAST, bool PAIRED = false>
  HILO_DEV void load(const void *x, size_t at, int pitch, int rows, int cols, int tid) {
    constexpr int E = TYPE == TYPE_F32 ? 4 : 1;
    const auto rsrc = __builtin_amdgcn_make_buffer_rsrc(const_cast<char *>(reinterpret_cast<const char *>(x)) + at * E, 0,
                                                        int(kBehind - 1), 0x00020000);
    if constexpr (TYPE == TYPE_F32) {
#pragma unroll
      for (int j = 0; j < 2; ++j) {
        int q = K_LAST ? (tid >> 3) + 32 * j : k_first(tid) + j;
        if (PAIRED) q = (tid >> 3 & 15) + 16 * j;
        const int c = K_LAST ? 4 * (tid & 7) : col_first(tid);
        u[j] = __builtin_amdgcn_raw_buffer_load_b128(rsrc, q < rows && c < cols ? (q * pitch + c) * E : kBehind, 0, 0);
      }
    } else {
      static_assert(K_LAST || TYPE == TYPE_F32, "codes are loaded for the first product alone");
      int q = tid >> 2;
      if (PAIRED) q = 16 * (q >> 5) + (q & 15);
      const int c = 8 * (tid & 3);
      const u32x2 v = __builtin_amdgcn_raw_buffer_load_b64(rsrc, q < rows && c < cols ? q * pitch + c : kBehind, 0, 0);
      u[0] = u32x4{v[0], v[1], 0u, 0u};
    }
  }
  HILO_DEV void load_scale(const uint8_t *x, int pitch, int rows, int cols, int tid) {
    const auto rsrc = __builtin_amdgcn_make_buffer_rsrc(const_cast<uint8_t *>(x), 0, int(kBehind - 1), 0x00020000);
    const int q = tid >> 2;
    scale = __builtin_amdgcn_raw_buffer_load_b8(rsrc, q < rows && cols > 0 ? q * pitch : kBehind, 0, 0);
  }
  template <bool K_LAST>
  HILO_DEV void store(float (&lds)[64][kPad], int tid) const {
    if constexpr (TYPE == TYPE_FP8) {
      const float s = e8m0(uint8_t(scale));
      f32x4 f[2];
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        const auto v = __builtin_amdgcn_cvt_pk_f32_fp8(u[0][h], false), w = __builtin_amdgcn_cvt_pk_f32_fp8(u[0][h], true);
        f[h] = f32x4{v[0] * s, v[1] * s, w[0] * s, w[1] * s};
      }
      f32x4 *to = reinterpret_cast<f32x4 *>(&lds[tid >> 2][8 * (tid & 3)]);
      to[0] = f[0];
      to[1] = f[1];
    } else if constexpr (K_LAST) {
#pragma unroll
      for (int j = 0; j < 2; ++j) *reinterpret_cast<u32x4 *>(&lds[(tid >> 3) + 32 * j][4 * (tid & 7)]) = u[j];
    } else {
#pragma unroll
      for (int e = 0; e < 4; ++e) *reinterpret_cast<u32x2 *>(&lds[col_first(tid) + e][k_first(tid)]) = u32x2{u[0][e], u[1][e]};
    }
  }
};

typedef float ProductLds[2][2][2][64][kPad];  // [group][buffer][operand][row][k]

// The items of workgroup `block` of `blocks`.
template <int TYPE, int KIND, bool GATED>
HILO_DEV void product_items(const ProductProblem &p, int block, int blocks, ProductLds &buffers) {
  constexpr bool AK = KIND != PRODUCT_DW, BK = KIND == PRODUCT_OUT;  // operand's last index is k
  constexpr int BN = GATED && KIND == PRODUCT_OUT ? 32 : 64;         // columns of a tile
  const int tid = threadIdx.x & 255, lane = tid & 63, wid = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int group = __builtin_amdgcn_readfirstlane(threadIdx.x >> 8);
  float (&lds)[2][2][64][kPad] = buffers[group];
  const int lr = lane & 15, lg = lane >> 4, wm = wid >> 1, wn = wid & 1;
  const int cols = KIND == PRODUCT_OUT ? p.N : p.K, tn_count = (cols + BN - 1) / BN;
  const int tm_count = KIND == PRODUCT_DW ? (p.N + 63) / 64 : row_tiles_bound(p, 64);
  const int tr_count = KIND == PRODUCT_DW ? tm_count * p.outs : tm_count;
  // steps of the whole sum; of a segment's rows in DW
  const int parts = KIND == PRODUCT_DX ? p.parts : 1, per = (KIND == PRODUCT_OUT ? p.K : p.N) + kStep - 1, each = per / kStep;
  // a workgroup keeps its columns and its split, and goes from row tile to row tile
  const uint32_t wide = uint32_t(tn_count) * p.splits;
  const int across = int(uint32_t(block) % wide), tn = int(uint32_t(across) / uint32_t(p.splits)), split = across - tn * p.splits, n0 = tn * BN;
  for (int tr = int(uint32_t(block) / wide); tr < tr_count; tr += int(uint32_t(blocks) / wide)) {
    int o = 0, stream = 0, part = 0, row0 = 0, rows = 64;
    if constexpr (KIND == PRODUCT_DW) {
      int t = tr;
      for (; t >= tm_count; t -= tm_count) ++o;
      row0 = t * 64;
      stream = p.out_stream[o];
      part = p.out_part[o];
      rows = min(64, p.N - row0);
    } else {
      const RowTile rt = find_row_tile(p, 64, tr);
      if (rt.n == 0) continue;  // behind the last
      row0 = uni(rt.row0);
      rows = uni(rt.n);
      stream = uni(rt.stream);
    }
    // ---- where the sum runs: pieces of k, walked from step s0 to s1
    int total = 0;
    if constexpr (KIND == PRODUCT_DW) {
      for (int i = stream; i < segments(p); i += 2) total += (max(segment(p, i).n, 0) + kStep - 1) / kStep;
    } else {
      total = parts * each;
    }
    const int least = int(uint32_t(total) / uint32_t(p.splits)), over = total - least * p.splits;
    const int s0 = least * split + min(split, over), s1 = s0 + least + (split < over ? 1 : 0);
    int seg = stream, seg_lo = 0, seg_n = 0, seg_s = 0;  // DW: the segment of the step, its first step
    if constexpr (KIND == PRODUCT_DW) {
      if (s0 < s1) {
        Segment g = segment(p, seg);
        while ((g.n + kStep - 1) / kStep <= s0 - seg_s) {
          seg_s += (max(g.n, 0) + kStep - 1) / kStep;
          seg += 2;
          g = segment(p, seg);
        }
        seg_lo = g.lo;
        seg_n = g.n;
      }
    }
    // A step's operands, of a step behind the last zeros.  No load stands behind a branch, so that a wait knows how many it
    // leaves on their way.
    auto load = [&](int s, Piece<TYPE> &a, Piece<TYPE> &b) __attribute__((always_inline)) {
      const bool more = s < s1;
      int k0 = 0, kn = 0;  // first k of the step in its piece, and how many there are from there
      if constexpr (KIND == PRODUCT_DW) {
        if (more) {
          while (s - seg_s >= (seg_n + kStep - 1) / kStep) {
            seg_s += (max(seg_n, 0) + kStep - 1) / kStep;
            seg += 2;
            const Segment g = segment(p, seg);
            seg_lo = g.lo;
            seg_n = g.n;
          }
          k0 = (s - seg_s) * kStep;
          kn = seg_n - k0;
        }
        const size_t row = size_t(seg_lo) + k0;
        a.template load<false>(p.d, (row * p.parts + part) * p.N + row0, p.parts * p.N, kn, p.N - row0, tid);
        b.template load<false>(p.x, row * p.K + n0, p.K, kn, p.K - n0, tid);
      } else {
        const int dpart = KIND == PRODUCT_DX && more && s >= each ? 1 : 0;
        if (more) {
          k0 = (s - dpart * each) * kStep;
          kn = per - kStep + 1 - k0;
        }
        if constexpr (KIND == PRODUCT_DX) {
          a.template load<true>(p.d, (size_t(row0) * p.parts + dpart) * p.N + k0, p.parts * p.N, rows, kn, tid);
          const void *w = stream ? (dpart ? p.w[1][1] : p.w[1][0]) : (dpart ? p.w[0][1] : p.w[0][0]);
          b.template load<false>(w, size_t(k0) * p.K + n0, p.K, kn, p.K - n0, tid);
        } else {
          a.template load<true>(p.x, size_t(row0) * p.K + k0, p.K, rows, kn, tid);
          // with a gate rows of 16 columns of one part and of the other, in turn; a wave's are of one part
          const int wp = GATED ? Piece<TYPE>::half(wid) : 0;
          const void *w = stream ? (wp ? p.w[1][1] : p.w[1][0]) : (wp ? p.w[0][1] : p.w[0][0]);
          b.template load<true, GATED>(w, size_t(n0) * p.K + k0, p.K, p.N - n0, kn, tid);
          if constexpr (TYPE == TYPE_FP8) {
            const uint8_t *ws = stream ? (wp ? p.w_scale[1][1] : p.w_scale[1][0]) : (wp ? p.w_scale[0][1] : p.w_scale[0][0]);
            a.load_scale(p.x_scale + size_t(row0) * scale_stride(p.K) + k0 / 128, scale_stride(p.K), rows, kn, tid);
            b.load_scale(ws + size_t(n0 / 128) * scale_stride(p.K) + k0 / 128, 0, 64, kn, tid);  // one of all the tile's columns
          }
        }
      }
    };
    auto store = [&](int buf, const Piece<TYPE> &a, const Piece<TYPE> &b) __attribute__((always_inline)) {
      a.template store<AK>(lds[buf][0], tid);
      b.template store<BK>(lds[buf][1], tid);
    };
    f32x4 acc[2][2];
#pragma unroll
    for (int i = 0; i < 2; ++i)
#pragma unroll
      for (int j = 0; j < 2; ++j) acc[i][j] = f32x4{0.f, 0.f, 0.f, 0.f};
    if (s0 < s1) {
      Piece<TYPE> a[kAhead], b[kAhead];
#pragma unroll
      for (int k = 0; k < kAhead; ++k) load(s0 + group + 2 * k, a[k], b[k]);
      // step s of the group out of buffer buf
      auto step = [&](int s, int buf, Piece<TYPE> &ca, Piece<TYPE> &cb) __attribute__((always_inline)) {
        store(buf, ca, cb);
        load(s + 2 * kAhead, ca, cb);
        __syncthreads();
#pragma unroll
        for (int h = 0; h < kStep / 16; ++h) {
          f32x4 av[2], bv[2];
#pragma unroll
          for (int i = 0; i < 2; ++i) {
            av[i] = *reinterpret_cast<const f32x4 *>(&lds[buf][0][32 * wm + 16 * i + lr][16 * h + 4 * lg]);
            bv[i] = *reinterpret_cast<const f32x4 *>(&lds[buf][1][32 * wn + 16 * i + lr][16 * h + 4 * lg]);
          }
#pragma unroll
          for (int e = 0; e < 4; ++e)
#pragma unroll
            for (int i = 0; i < 2; ++i)
#pragma unroll
              for (int j = 0; j < 2; ++j) acc[i][j] = __builtin_amdgcn_mfma_f32_16x16x4f32(bv[j][e], av[i][e], acc[i][j], 0, 0, 0);
        }
      };
      static_assert(kAhead == 2, "a buffer for every other step");
#pragma unroll 1
      for (int s = s0;; s += 2) {  // both groups the same number of steps
        step(s + group, 0, a[0], b[0]);
        s += 2;
        if (s >= s1) break;
        step(s + group, 1, a[1], b[1]);
        if (s + 2 >= s1) break;
      }
    }
    // ---- group g finishes row block g of every wave's two
    __syncthreads();
    f32x4 *meet = reinterpret_cast<f32x4 *>(buffers) + (group * 4 + wid) * 128 + lane;
#pragma unroll
    for (int j = 0; j < 2; ++j) meet[64 * j] = group ? acc[0][j] : acc[1][j];
    __syncthreads();
    f32x4 sum[2];
#pragma unroll
    for (int j = 0; j < 2; ++j) {
      const f32x4 other = (reinterpret_cast<f32x4 *>(buffers) + ((1 - group) * 4 + wid) * 128 + lane)[64 * j];
      sum[j] = group ? other + acc[1][j] : acc[0][j] + other;  // group 0's first, in either group
    }
    __syncthreads();  // the next item's first steps go to the same LDS
    // lane (lr, lg): row lr of the block, columns 16 j + 4 lg .. + 3 of the wave's 32
    const int r = 32 * wm + 16 * group + lr;
    if (r < rows) {
      const size_t row = size_t(row0) + r;
      if constexpr (KIND == PRODUCT_OUT && GATED) {
        const int n = n0 + 16 * wn + 4 * lg;
        if (n >= p.N) continue;  // nothing behind it in this item
        if (p.splits > 1) {
          float *q = p.part + (size_t(split) * p.rows + row) * 2 * p.N + n;
          *reinterpret_cast<f32x4 *>(q) = sum[0];
          *reinterpret_cast<f32x4 *>(q + p.N) = sum[1];
        } else {
          finish_out<true>(p, stream, row, n, sum[0], sum[1]);
        }
      } else {
#pragma unroll
        for (int j = 0; j < 2; ++j) {
          const int n = n0 + 32 * wn + 16 * j + 4 * lg;
          if (n >= cols) continue;
          if (p.splits > 1) {
            const size_t all = KIND == PRODUCT_DW ? size_t(p.outs) * p.N : size_t(p.rows);
            const size_t at = KIND == PRODUCT_DW ? size_t(o) * p.N + row : row;
            *reinterpret_cast<f32x4 *>(p.part + (split * all + at) * cols + n) = sum[j];
          } else if constexpr (KIND == PRODUCT_OUT) {
            finish_out<false>(p, stream, row, n, sum[j], sum[j]);
          } else if constexpr (KIND == PRODUCT_DX) {
            store4(p.dx, row * p.K + n, sum[j], p.bf16);
          } else {
            store4(p.dw[o], row * p.K + n, sum[j], p.bf16);
          }
        }
      }
    }
  }
}

template <int TYPE, int KIND, bool GATED>
__global__ __launch_bounds__(512) void k_product(ProductProblem p) {
  __shared__ __attribute__((aligned(16))) ProductLds buffers;
  product_items<TYPE, KIND, GATED>(p, blockIdx.x, gridDim.x, buffers);
}

// Both products of a float32 backward pass in one launch: the first blocks_x workgroups have dx, the others dw.
__global__ __launch_bounds__(512) void k_product_back(ProductProblem x, ProductProblem w, int blocks_x) {
  __shared__ __attribute__((aligned(16))) ProductLds buffers;
  if (int(blockIdx.x) < blocks_x) product_items<TYPE_F32, PRODUCT_DX, false>(x, blockIdx.x, blocks_x, buffers);
  else product_items<TYPE_F32, PRODUCT_DW, false>(w, blockIdx.x - blocks_x, gridDim.x - blocks_x, buffers);
}

// Sums of the splits, in order, and the last step, by workgroup `block` of `blocks`.  A thread has four columns of a row.
template <int KIND, bool GATED>
HILO_DEV void join_items(const ProductProblem &p, int block, int blocks) {
  const int cols = KIND == PRODUCT_OUT ? p.N : p.K, quads = cols / 4;
  const long long all = KIND == PRODUCT_DW ? (long long)p.outs * p.N : p.rows;
  const long long rows = KIND == PRODUCT_DW ? all : cu_at(p.cu, p.B);
  constexpr int W = KIND == PRODUCT_OUT && GATED ? 2 : 1;
  for (long long t = block * 256ll + threadIdx.x; t < rows * quads; t += blocks * 256ll) {
    const long long row = t / quads;
    const int n = int(t - row * quads) * 4;
    f32x4 v[W];
#pragma unroll
    for (int w = 0; w < W; ++w) v[w] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll 4
    for (int s = 0; s < p.splits; ++s)
#pragma unroll
      for (int w = 0; w < W; ++w)
        v[w] += *reinterpret_cast<const f32x4 *>(p.part + (s * all + row) * (W * cols) + w * cols + n);
    if constexpr (KIND == PRODUCT_OUT) {
      int stream = 0;
      if (!p.merged) {
        const int s = sample_of_row(p.cu, p.B, int(row));
        stream = row >= p.cu[s + 1] - p.L;
      }
      finish_out<GATED>(p, stream, size_t(row), n, v[0], v[W - 1]);
    } else if constexpr (KIND == PRODUCT_DX) {
      store4(p.dx, row * p.K + n, v[0], p.bf16);
    } else {
      const int o = int(row / p.N);
      store4(p.dw[o], (row - (long long)o * p.N) * p.K + n, v[0], p.bf16);
    }
  }
}

template <int KIND, bool GATED>
__global__ __launch_bounds__(256) void k_product_join(ProductProblem p) {
  join_items<KIND, GATED>(p, blockIdx.x, gridDim.x);
}

// Splits of the sum, no shorter than 4 steps each, where tiles are fewer than two for each of the 256 CUs; one in a backward
// pass, whose two products run together.  They do not depend on what else a call forms, so that an output alone has
// the same bits: the weights' gradients are cut as if the call formed all of them, one for each part, or by stream for each
// part of either.  (512 x 256 -> 1024: 11.2 us on 128 tiles in 4 splits, their sums included)
constexpr long long kSplitTiles = 512;
static long long most_splits(int kind, long long rows, int K, int N, int parts) {
  const long long steps = kind == PRODUCT_OUT ? K / kStep : kind == PRODUCT_DX ? (long long)parts * N / kStep : rows / kStep;
  return std::max(1ll, steps / 4);
}
static int splits_of(int kind, long long rows, int K, int N, int parts, int B, bool merged) {
  const long long tm = kind == PRODUCT_DW ? (long long)parts * (merged ? 1 : 2) * ((N + 63) / 64) : (rows + 63) / 64 + (merged ? 0 : 2 * B - 1);  // row_tiles_bound
  const int bn = kind == PRODUCT_OUT && parts == 2 ? 32 : 64, cols = kind == PRODUCT_OUT ? N : K;
  const long long tiles = std::max(1ll, tm * ((cols + bn - 1) / bn));
  return int(std::min(std::max(1ll, (kind == PRODUCT_OUT ? kSplitTiles : kSplitTiles / 2) / tiles), most_splits(kind, rows, K, N, parts)));
}

// Bounds the partial sums of any call, and grows with the sizes: a tile's are 64 x 64.  Weights' gradients without text may
// be twice as many as they are cut for (stream 1's are zeros), of at most half as many tiles as other sums.
size_t product_part_bytes(bool bf16, int kind, long long rows, int K, int N, int parts) {
  if (bf16) return kind == PRODUCT_OUT && rows <= kProductFewRows ? 0 : product_tiles_part_bytes();
  const long long most = most_splits(kind, rows, K, N, parts);
  if (most == 1) return 0;
  const long long each = kind == PRODUCT_OUT ? rows * parts * N : kind == PRODUCT_DX ? rows * K : 4ll * N * K;
  return size_t(std::min((most * each + 63) / 64, kSplitTiles * 64)) * 64 * sizeof(float);
}

// Sets the splits; workgroups of the product and of the sums of its splits.
static int product_blocks(int kind, ProductProblem &p) {
  p.splits = splits_of(kind, p.rows, p.K, p.N, p.parts, p.B, p.merged);
  const long long tm = kind == PRODUCT_DW ? (long long)p.outs * ((p.N + 63) / 64) : row_tiles_bound(p, 64);
  const int cols = kind == PRODUCT_OUT ? p.N : p.K, bn = kind == PRODUCT_OUT && p.parts == 2 ? 32 : 64;
  const int wide = (cols + bn - 1) / bn * p.splits;  // of one row tile
  return int(std::min(tm, std::max(1ll, (1ll << 20) / wide))) * wide;
}
static int join_blocks(int kind, const ProductProblem &p) {
  if (p.splits == 1) return 0;
  const long long quads = (kind == PRODUCT_DW ? (long long)p.outs * p.N : p.rows) * ((kind == PRODUCT_OUT ? p.N : p.K) / 4);
  return int(std::min((quads + 255) / 256, 4096ll));
}

template <int TYPE, int KIND, bool GATED>
static hipError_t run(ProductProblem &p, hipStream_t st) {
  const int blocks = product_blocks(KIND, p);
  if (blocks <= 0) return hipSuccess;
  hipLaunchKernelGGL((k_product<TYPE, KIND, GATED>), dim3(blocks), dim3(512), 0, st, p);
  const hipError_t e = hipGetLastError();
  const int joins = join_blocks(KIND, p);
  if (e != hipSuccess || joins == 0) return e;
  hipLaunchKernelGGL((k_product_join<KIND, GATED>), dim3(joins), dim3(256), 0, st, p);
  return hipGetLastError();
}

template <int TYPE>
static hipError_t run_kind(int kind, ProductProblem &p, hipStream_t st) {
  const bool gated = p.parts == 2;
  if (kind == PRODUCT_OUT) return gated ? run<TYPE, PRODUCT_OUT, true>(p, st) : run<TYPE, PRODUCT_OUT, false>(p, st);
  if (kind == PRODUCT_DX) return run<TYPE, PRODUCT_DX, false>(p, st);
  return p.outs > 0 ? run<TYPE, PRODUCT_DW, false>(p, st) : hipSuccess;
}

hipError_t launch_product(int kind, ProductProblem p, hipStream_t st) {
  if (kind == PRODUCT_DW && p.outs == 0) return hipSuccess;
  if (!p.bf16) return run_kind<TYPE_F32>(kind, p, st);
  return kind == PRODUCT_OUT && p.rows <= kProductFewRows ? launch_product_few(p, st) : launch_product_tiles(kind, p, st);
}

// How an FP8 product is formed: of few rows; on FP8 tiles where bf16 leaves; from widened rows where codes or float32 leave; and
// where that makes few tiles, float32 ones cut along k.  Those run at 0.1 PFLOP/s whatever their number, a widened tile's
// window of 64 takes 0.7 us alone, as 17 tiles' take there.  Measured, widened and cut (us, float32 out): 16 tiles
// 400 x 1024 -> 1024 24.5 and 23.4, 32 tiles 1000 x 256 -> 1024 16.7 and 19.6, 2 tiles 209 x 6272 -> 144 83 and 25.  Codes take a
// launch more there, 5 us: what 120 such windows of tiles fewer than 17 save (a feed of 209 rows, 6272 wide: 95 and 46).
enum Fp8Way { FP8_FEW, FP8_TILES, FP8_WIDE, FP8_SPLIT };
constexpr int kSplitTilesMost = 17;
static Fp8Way fp8_way(bool bf16, bool coded, long long rows, int K, int N, int parts) {
  if (rows <= kProductFewRows) return FP8_FEW;
  if (!coded && bf16) return FP8_TILES;
  const int cols = parts == 2 ? 128 : 256;
  const long long tiles = (rows + 127) / 128 * ((N + cols - 1) / cols);
  return (kSplitTilesMost - tiles) * K > (coded ? 120 * 64 : 0) ? FP8_SPLIT : FP8_WIDE;
}
// Partial sums, and float32 rows that codes are formed from (of FP8_SPLIT, behind them)
size_t product_fp8_part_bytes(long long rows, int K, int N, int parts) {
  if (rows <= kProductFewRows) return size_t(rows) * N * sizeof(float);
  const size_t coded = std::min<size_t>(size_t(rows) * N, kSplitTilesMost * 128 * 128) * sizeof(float);
  return std::max(product_tiles_part_bytes(), product_part_bytes(false, PRODUCT_OUT, rows, K, N, parts) + coded);
}
Fp8Rows product_fp8_rows(const ProductProblem &p) {
  const Fp8Way way = fp8_way(p.bf16, p.out_scale != nullptr, p.rows, p.K, p.N, p.parts);
  if (way == FP8_WIDE) return FP8_ROWS_WIDE;
  return way == FP8_FEW && p.bf16 && p.rows <= 16 ? FP8_ROWS_ANY : FP8_ROWS_CODES;
}
hipError_t launch_product_fp8(ProductProblem p, hipStream_t st) {
  const Fp8Way way = fp8_way(p.bf16, p.out_scale != nullptr, p.rows, p.K, p.N, p.parts);
  if (way == FP8_TILES) return launch_product_fp8_tiles(p, st);
  if (way == FP8_WIDE) return launch_product_fp8_wide(p, st);
  // codes: a scale's 128 columns are several workgroups', so they are formed from float32 rows in a launch of their own
  void *codes = p.out;
  p.out_f32 = !p.bf16 || p.out_scale;
  if (p.out_scale) p.out = p.part + (way == FP8_FEW ? 0 : product_part_bytes(false, PRODUCT_OUT, p.rows, p.K, p.N, p.parts) / sizeof(float));
  const hipError_t e = way == FP8_FEW ? launch_product_few(p, st)
                       : p.parts == 2 ? run<TYPE_FP8, PRODUCT_OUT, true>(p, st)
                                      : run<TYPE_FP8, PRODUCT_OUT, false>(p, st);
  if (e != hipSuccess || !p.out_scale) return e;
  return launch_quantize_blocks(false, p.out, p.rows, p.N, 1, p.cu + p.B, reinterpret_cast<uint8_t *>(codes), p.out_scale, st);
}

// ------------------------------------------------------------------------ through the gate, and sums over rows
//
//   du = dout act(g), dg = dout u act'(g); db_part = sum over a stream's rows of d_part
// du and dg are formed and summed in float32, and rounded to the dtype as operands of the products: in bf16 that rounding, 2^-9
// of each value at its mean, is most of a gradient's error (2.3e-3 beside 1.7e-3 of exact ones rounded at the end).
//
// Bound by memory: with a gate five values a column are read or written.  A workgroup has block_rows rows of a segment and
// 512 columns: a wave every fourth row, a lane 8 columns, four rows on their way.  What a column's rows sum to goes to part[row block][parts][N], and k_gate_back_sum adds those of a stream's
// blocks in their order.  22560 x 8192 bf16: 373 us for 1.85 GB, 5.0 TB/s (a copy reaches 5.2), and 13 for the sums.
constexpr int kBackCols = 512;
// Rows of a block: the fewest of 4, 16, 64, 256 that leave at most 2048 workgroups (256 CUs have 8 each), or 256.  1005 x 8208
// bf16 in blocks of 16: 17.9 us and 4.4 for the sums, of 4 20.2 and 5.6; 551 x 1024 float32 of 4 6.2 and 4.1, of 16 8.2 and 3.2.
constexpr long long kBackItems = 2048;
static int back_rows(long long rows, int N) {
  int b = 4;
  while (b < 256 && (rows + b - 1) / b * ((N + kBackCols - 1) / kBackCols) > kBackItems) b *= 4;
  return b;
}

template <bool BF16, bool GATED>
__global__ __launch_bounds__(256) void k_gate_back(GateBackProblem p) {
  constexpr int PARTS = GATED ? 2 : 1, TYPE = BF16 ? TYPE_BF16 : TYPE_F32, AHEAD = 4;
  __shared__ float sums[3][PARTS][8][64];
  const int lane = threadIdx.x & 63, wid = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int tn_count = (p.N + kBackCols - 1) / kBackCols;
  const long long tiles = (long long)row_tiles_bound(p, p.block_rows) * tn_count;
  for (long long t = blockIdx.x; t < tiles; t += gridDim.x) {
    const int tr = int(t / tn_count), n = int(t - (long long)tr * tn_count) * kBackCols + 8 * lane;
    const RowTile rt = find_row_tile(p, p.block_rows, tr);
    if (rt.n == 0) continue;  // behind the last
    float db[PARTS][8];
#pragma unroll
    for (int q = 0; q < PARTS; ++q)
#pragma unroll
      for (int e = 0; e < 8; ++e) db[q][e] = 0.f;
    if (n < p.N) {
#pragma unroll 1
      for (int r0 = wid; r0 < rt.n; r0 += 4 * AHEAD) {
        Chunk<TYPE> d[AHEAD], g[AHEAD], u[AHEAD];
#pragma unroll
        for (int a = 0; a < AHEAD; ++a) {
          const size_t row = size_t(rt.row0) + min(r0 + 4 * a, rt.n - 1);  // behind the last row: it again, left out below
          d[a].load(p.dout, row * p.N + n);
          if constexpr (GATED) {
            g[a].load(p.pre, row * 2 * p.N + n);
            u[a].load(p.pre, row * 2 * p.N + p.N + n);
          }
        }
#pragma unroll
        for (int a = 0; a < AHEAD; ++a) {
          if (r0 + 4 * a >= rt.n) break;
          float dv[8];
          d[a].values(dv);
          if constexpr (GATED) {
            float gv[8], uv[8];
            g[a].values(gv);
            u[a].values(uv);
#pragma unroll
            for (int e = 0; e < 8; ++e) {
              float act, slope;
              gate_slope<!BF16>(gv[e], p.silu, act, slope);
              gv[e] = dv[e] * uv[e] * slope;
              uv[e] = dv[e] * act;
              db[0][e] += gv[e];
              db[1][e] += uv[e];
            }
            const size_t at = (size_t(rt.row0) + r0 + 4 * a) * 2 * p.N + n;
            store8<BF16>(p.dpre, at, gv);
            store8<BF16>(p.dpre, at + p.N, uv);
          } else {
#pragma unroll
            for (int e = 0; e < 8; ++e) db[0][e] += dv[e];
          }
        }
      }
    }
    if (p.part) {
      if (wid > 0) {
#pragma unroll
        for (int q = 0; q < PARTS; ++q)
#pragma unroll
          for (int e = 0; e < 8; ++e) sums[wid - 1][q][e][lane] = db[q][e];
      }
      __syncthreads();
      if (wid == 0 && n < p.N) {
#pragma unroll
        for (int q = 0; q < PARTS; ++q) {
#pragma unroll
          for (int e = 0; e < 8; ++e) db[q][e] = ((db[q][e] + sums[0][q][e][lane]) + sums[1][q][e][lane]) + sums[2][q][e][lane];
          store8<false>(p.part, (size_t(tr) * PARTS + q) * p.N + n, db[q]);
        }
      }
      __syncthreads();
    }
  }
}

// A workgroup of W waves has 64 columns (block) of one sum.  Its row blocks go to kBackSums partial sums in turn, whatever W is, so
// that a call's other gradients do not change a bias's bits; a wave has every W-th partial sum, eight row blocks of each on
// their way.
constexpr int kBackSums = 8;
template <bool BF16, int W>
HILO_DEV void sum_columns(const GateBackProblem &p, int block, int which) {
  constexpr int V = kBackSums / W;
  __shared__ float sums[kBackSums][64];
  const int lane = threadIdx.x & 63, wid = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int stream = which / p.parts, part = which % p.parts;
  void *db = stream ? p.db[1][part] : p.db[0][part];
  const bool both = p.db[0][part] == p.db[1][part];
  if (!db || (both && stream)) return;
  const int n = block * 64 + lane;
  float v[V];
#pragma unroll
  for (int j = 0; j < V; ++j) v[j] = 0.f;
  int t0 = 0;  // blocks before the segment
  for (int i = 0; i < segments(p); ++i) {
    const Segment s = segment(p, i);
    const int tiles = (s.n + p.block_rows - 1) / p.block_rows;
    if (both || s.stream == stream) {
      const float *from = p.part + (size_t(t0) * p.parts + part) * p.N + min(n, p.N - 1);
#pragma unroll 1
      for (int t = wid; t < tiles; t += 8 * kBackSums) {
        float w[V][8];
#pragma unroll
        for (int j = 0; j < V; ++j)
#pragma unroll
          for (int k = 0; k < 8; ++k) w[j][k] = from[size_t(min(t + W * j + kBackSums * k, tiles - 1)) * p.parts * p.N];
#pragma unroll
        for (int j = 0; j < V; ++j)
#pragma unroll
          for (int k = 0; k < 8; ++k) v[j] += t + W * j + kBackSums * k < tiles ? w[j][k] : 0.f;
      }
    }
    t0 += tiles;
  }
#pragma unroll
  for (int j = 0; j < V; ++j) sums[wid + W * j][lane] = v[j];
  __syncthreads();
  if (wid == 0 && n < p.N) {
    float s = sums[0][lane];
#pragma unroll
    for (int k = 1; k < kBackSums; ++k) s += sums[k][lane];
    if (BF16) reinterpret_cast<uint16_t *>(db)[n] = f2bf(s);
    else reinterpret_cast<float *>(db)[n] = s;
  }
}

template <bool BF16>
__global__ __launch_bounds__(512) void k_gate_back_sum(GateBackProblem p) {
  sum_columns<BF16, 8>(p, blockIdx.x, blockIdx.y);
}

// What is left of a float32 backward pass, in one launch: sums of the splits of dx and of dw, and over the rows.
__global__ __launch_bounds__(256) void k_join_back(ProductProblem x, ProductProblem w, GateBackProblem g, int blocks_x, int blocks_w) {
  int block = blockIdx.x;
  if (block < blocks_x) return join_items<PRODUCT_DX, false>(x, block, blocks_x);
  block -= blocks_x;
  if (block < blocks_w) return join_items<PRODUCT_DW, false>(w, block, blocks_w);
  block -= blocks_w;
  const int cols = (g.N + 63) / 64;
  sum_columns<false, 4>(g, block % cols, block / cols);
}

// Bounds the blocks, and grows with the rows.
size_t gate_back_bytes(long long rows, int N, int parts, int B) {
  const long long most = kBackItems / ((N + kBackCols - 1) / kBackCols), blocks = std::max(std::min((rows + 3) / 4, most), (rows + 255) / 256);
  return (size_t(blocks) + 2 * size_t(B)) * parts * N * sizeof(float);
}

template <bool BF16, bool GATED>
static hipError_t run_gate_back(const GateBackProblem &p, hipStream_t st) {
  if (p.rows > 0 && (GATED || p.part)) {
    const long long tiles = (long long)row_tiles_bound(p, p.block_rows) * ((p.N + kBackCols - 1) / kBackCols);
    hipLaunchKernelGGL((k_gate_back<BF16, GATED>), dim3(unsigned(std::min(tiles, 1ll << 20))), dim3(256), 0, st, p);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
  }
  if (!p.part || p.sums_later) return hipSuccess;
  hipLaunchKernelGGL((k_gate_back_sum<BF16>), dim3((p.N + 63) / 64, 2 * p.parts), dim3(512), 0, st, p);
  return hipGetLastError();
}

hipError_t launch_gate_back(bool bf16, GateBackProblem p, hipStream_t st) {
  p.block_rows = back_rows(p.rows, p.N);
  if (p.parts == 2) return bf16 ? run_gate_back<true, true>(p, st) : run_gate_back<false, true>(p, st);
  return bf16 ? run_gate_back<true, false>(p, st) : run_gate_back<false, false>(p, st);
}

hipError_t launch_product_back(ProductProblem x, ProductProblem w, GateBackProblem g, hipStream_t st) {
  g.block_rows = back_rows(g.rows, g.N);
  const int bx = product_blocks(PRODUCT_DX, x), bw = product_blocks(PRODUCT_DW, w);
  hipLaunchKernelGGL(k_product_back, dim3(bx + bw), dim3(512), 0, st, x, w, bx);
  const hipError_t e = hipGetLastError();
  const int jx = join_blocks(PRODUCT_DX, x), jw = join_blocks(PRODUCT_DW, w), sums = g.part ? (g.N + 63) / 64 * 2 * g.parts : 0;
  if (e != hipSuccess || jx + jw + sums == 0) return e;
  hipLaunchKernelGGL(k_join_back, dim3(jx + jw + sums), dim3(256), 0, st, x, w, g, jx, jw);
  return hipGetLastError();
}

// ----------------------------------------------------------------------------------- quantisation of blocks

// The codes of 8 values times 2^-k, and the bits that say whether they are finite: the largest |x|'s, as they order.
HILO_DEV uint2 block_codes(const float (&f)[8], uint32_t top) {
  if (top >= 0x7f800000u) return make_uint2(0x7f7f7f7fu, 0x7f7f7f7fu);
  const float inv = pow2_inverse(pow2_exponent(__uint_as_float(top)));
  return make_uint2(fp8x4(f[0] * inv, f[1] * inv, f[2] * inv, f[3] * inv), fp8x4(f[4] * inv, f[5] * inv, f[6] * inv, f[7] * inv));
}
HILO_DEV uint8_t block_scale(uint32_t top) {
  return top >= 0x7f800000u ? 255 : uint8_t(127 + pow2_exponent(__uint_as_float(top)));
}

// The largest magnitude's bits over 16 lanes' 8 values each
HILO_DEV uint32_t top16(const float (&f)[8]) {
  uint32_t top = 0;
#pragma unroll
  for (int e = 0; e < 8; ++e) top = max(top, abs_bits(f[e]));
  top = max(top, uint32_t(dpp<kDppXor1>(int(top))));
  top = max(top, uint32_t(dpp<kDppXor2>(int(top))));
  top = max(top, uint32_t(dpp<kDppHalfMirror>(int(top))));
  return max(top, uint32_t(dpp<kDppMirror>(int(top))));
}

// x is rounded to codes here, the one loss of an FP8 product: x 2^-k with the block's largest in (224, 448], exact but for the
// rounding to 4 bits.  Bound by memory.
// Rows: 16 lanes have the 128 columns of a scale, 8 a lane; a wave 512 columns of a row at a time.  2766 x 3072 bf16: 8.0 us,
// 25.5 MB at 3.2 TB/s, ramp and tail; 22560 x 3072 40.9, 5.1 TB/s.
template <bool BF16>
__global__ __launch_bounds__(256) void k_quantize_blocks(const void *__restrict__ x, int rows, int cols, const int *__restrict__ limit,
                                                         uint8_t *__restrict__ codes, uint8_t *__restrict__ scale) {
  const int lane = threadIdx.x & 63, wid = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int end = limit ? min(rows, cu_at(limit, 0)) : rows, groups = scale_stride(cols) / 4;
  const long long units = (long long)end * groups;
  for (long long t = blockIdx.x * 4ll + wid; t < units; t += gridDim.x * 4ll) {
    const int row = int(t / groups), c = int(t - (long long)row * groups) * 512 + 8 * lane;
    Chunk<BF16 ? TYPE_BF16 : TYPE_F32> v;
    v.zero();
    if (c < cols) v.load(x, size_t(row) * cols + c);
    float f[8];
    v.values(f);
    const uint32_t top = top16(f);
    if (c < cols) *reinterpret_cast<uint2 *>(codes + size_t(row) * cols + c) = block_codes(f, top);
    if ((lane & 15) == 0) scale[size_t(row) * scale_stride(cols) + c / 128] = c < cols ? block_scale(top) : 0;
  }
}

// Rows as the values that codes and scales stand for, in bf16, which holds them exactly: of x, or of codes of it (TYPE_FP8).
template <int TYPE>
__global__ __launch_bounds__(256) void k_widen_rows(const void *__restrict__ x, const uint8_t *__restrict__ scale, int rows, int cols,
                                                    const int *__restrict__ limit, uint16_t *__restrict__ out) {
  const int lane = threadIdx.x & 63, wid = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int end = min(rows, cu_at(limit, 0)), groups = (cols + 511) / 512;
  const long long units = (long long)end * groups;
  for (long long t = blockIdx.x * 4ll + wid; t < units; t += gridDim.x * 4ll) {
    const int row = int(t / groups), c = int(t - (long long)row * groups) * 512 + 8 * lane;
    Chunk<TYPE> v;
    v.zero();
    if (c < cols) v.load(x, size_t(row) * cols + c);
    uint2 codes;
    uint32_t s;
    if constexpr (TYPE == TYPE_FP8) {
      codes = make_uint2(v.u[0].x, v.u[0].y);
      s = c < cols ? scale[size_t(row) * scale_stride(cols) + c / 128] : 0;
    } else {
      float f[8];
      v.values(f);
      const uint32_t top = top16(f);
      codes = block_codes(f, top);
      s = block_scale(top);
    }
    if (c < cols) *reinterpret_cast<bf16x8 *>(out + size_t(row) * cols + c) = wide_codes(codes.x, codes.y, s << 23);
  }
}

hipError_t launch_widen_rows(bool bf16, const void *x, const uint8_t *scale, int rows, int cols, const int *limit, void *out, hipStream_t st) {
  const long long units = (long long)rows * ((cols + 511) / 512);
  const dim3 grid(unsigned(std::min((units + 3) / 4, 1ll << 20)));
  uint16_t *o = reinterpret_cast<uint16_t *>(out);
  if (scale) hipLaunchKernelGGL((k_widen_rows<TYPE_FP8>), grid, dim3(256), 0, st, x, scale, rows, cols, limit, o);
  else if (bf16) hipLaunchKernelGGL((k_widen_rows<TYPE_BF16>), grid, dim3(256), 0, st, x, scale, rows, cols, limit, o);
  else hipLaunchKernelGGL((k_widen_rows<TYPE_F32>), grid, dim3(256), 0, st, x, scale, rows, cols, limit, o);
  return hipGetLastError();
}

// Blocks of 128 x 128: a workgroup each, a thread 8 rows of 8 columns, held while the largest is found.  Bound by memory: 8192 x
// 3072 bf16 17.0 us, 75.5 MB at 4.5 TB/s, float32 24.8 at 5.1; 1024 x 1024, 64 workgroups, 5.6.
template <bool BF16>
__global__ __launch_bounds__(256) void k_quantize_tiles(const void *__restrict__ x, int rows, int cols, const int *__restrict__ limit,
                                                        uint8_t *__restrict__ codes, uint8_t *__restrict__ scale) {
  __shared__ uint32_t tops[4];
  const int end = limit ? min(rows, cu_at(limit, 0)) : rows;
  const int c = blockIdx.x * 128 + 8 * (threadIdx.x & 15);
  for (int r0 = blockIdx.y * 128; r0 < end; r0 += gridDim.y * 128) {
    Chunk<BF16 ? TYPE_BF16 : TYPE_F32> v[8];
    uint32_t top = 0;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const int r = r0 + 16 * i + (threadIdx.x >> 4);
      v[i].zero();
      if (r < end && c < cols) v[i].load(x, size_t(r) * cols + c);
    }
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      float f[8];
      v[i].values(f);
#pragma unroll
      for (int e = 0; e < 8; ++e) top = max(top, abs_bits(f[e]));
    }
    top = wave_max_u32(top);
    if ((threadIdx.x & 63) == 0) tops[threadIdx.x >> 6] = top;
    __syncthreads();
    top = max(max(tops[0], tops[1]), max(tops[2], tops[3]));
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const int r = r0 + 16 * i + (threadIdx.x >> 4);
      float f[8];
      v[i].values(f);
      if (r < end && c < cols) *reinterpret_cast<uint2 *>(codes + size_t(r) * cols + c) = block_codes(f, top);
    }
    // the last blocks' threads fill the group of four up with zeros
    if (threadIdx.x == 0) scale[size_t(r0 / 128) * scale_stride(cols) + blockIdx.x] = blockIdx.x * 128 < cols ? block_scale(top) : 0;
    __syncthreads();
  }
}

hipError_t launch_quantize_blocks(bool bf16, const void *x, int rows, int cols, int block_rows, const int *limit, uint8_t *codes,
                                  uint8_t *scale, hipStream_t st) {
  if (rows <= 0) return hipSuccess;
  if (block_rows == 1) {
    const long long units = (long long)rows * (scale_stride(cols) / 4);
    const dim3 grid(unsigned(std::min((units + 3) / 4, 1ll << 20)));
    if (bf16) hipLaunchKernelGGL((k_quantize_blocks<true>), grid, dim3(256), 0, st, x, rows, cols, limit, codes, scale);
    else hipLaunchKernelGGL((k_quantize_blocks<false>), grid, dim3(256), 0, st, x, rows, cols, limit, codes, scale);
  } else {
    const dim3 grid(scale_stride(cols), unsigned(std::min((rows + 127) / 128, 4096)));
    if (bf16) hipLaunchKernelGGL((k_quantize_tiles<true>), grid, dim3(256), 0, st, x, rows, cols, limit, codes, scale);
    else hipLaunchKernelGGL((k_quantize_tiles<false>), grid, dim3(256), 0, st, x, rows, cols, limit, codes, scale);
  }
  return hipGetLastError();
}

}  // namespace hilo
