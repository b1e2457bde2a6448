// The bf16 products of a feed-forward and their gradients on large tiles (product.hip has their mathematics).
//
// One persistent workgroup of 8 waves a CU (WM x WN, a wave's tile in 16 x 16 MFMA blocks).  K goes through
// LDS in windows of 64 values, filled by direct loads to LDS some windows ahead, also of the tiles to come; while the MFMAs of one half of
// a window run, the fragments of the next half are read.  One barrier a window.
//
// An operand lies in memory with k last (x and w of the forward product, the gradients dpre of dx), or with k first (w of
// dx, both of dw), and goes to LDS as it lies there:
//   k last   a window is 128-byte rows, a fragment read 16 bytes a lane; 16-byte chunk c of row r at c ^ (r / 2) % 8
//   k first  a window is 64 rows of the tile's columns; a fragment is two transposing reads, in which 16 lanes take four
//            rows of 16 columns and each gets a column's four values; 32-byte chunk c of row k at c ^ f(k), f(k) = k % 4 + 4
//            (k / 8 % 2), so that the rows that 32 lanes read at once lie in eight groups of banks
// What lies behind the last row, column or k is never read: the loads' buffer ends there, and they leave zeros.
//
// Bound by the matrix cores at the power limit, and by what feeds them: a window of 256 x 256 takes 1.46 to 1.67 us on all CUs
// (1.25 to 1.35 PFLOP/s; the library's large product reaches 1.30), 1.07 on few.  The rest: a tile's epilogue, 7 us, which
// does not run beside the next tile's products (128 of a lane's 256 registers are accumulators, so there are no second ones),
// and turns that are not full.  2766 x 3072 -> 8192 with a gate 270 to 276 us, 1.02 PFLOP/s; 4708 x 4096 -> 1536 64;
// 22560 x 3072 -> 8192, gradients of both parts, 4.1 ms, 1.11.  The next tile's first windows are loaded before a tile's stores and
// not waited for behind them.
#include <algorithm>

#include "product_tiles.h"

namespace hilo {
namespace pt {

template <int BM_, int BN_, int KIND_, bool GATED_>
struct Geo {
  static constexpr int WM = BM_ > BN_ ? 4 : 2, WN = 8 / WM;  // waves
  static constexpr int BM = BM_, BN = BN_, KIND = KIND_;
  static constexpr bool GATED = GATED_ && KIND == PRODUCT_OUT;  // two products a tile, half its columns each
  static constexpr bool AK = KIND != PRODUCT_DW, BK = KIND == PRODUCT_OUT;  // k last
  static constexpr int MB = BM / WM / 16, NB = BN / WN / 16;
  static constexpr int LA = BM / 64, LB = BN / 64;  // load instructions of a wave for a window
  static constexpr int WB = (BM + BN) * 128;
  static constexpr int SLOTS = 3 * WB + 2048 <= 160 * 1024 ? 3 : 2;
  static constexpr int LDS = SLOTS * WB + 2048;  // and 256 bytes a wave for biases
  static constexpr int COLS = GATED ? BN / 2 : BN;  // columns of the output
};

// Windows of a tile's sum; of a stream's segments in DW.
template <int KIND>
HILO_DEV int windows(const ProductProblem &p, int stream) {
  if constexpr (KIND == PRODUCT_OUT) return (p.K + 63) / 64;
  if constexpr (KIND == PRODUCT_DX) return p.parts * ((p.N + 63) / 64);
  int n = 0;
  for (int i = stream; i < segments(p); i += 2) n += (segment(p, i).n + 63) / 64;
  return n;
}

template <int OFF>
HILO_DEV void read_tr(u32x2 &d, uint32_t addr) {
  asm volatile("ds_read_b64_tr_b16 %0, %1 offset:%2" : "=v"(d) : "v"(addr), "n"(OFF) : "memory");
}

// A fragment: 8 values of k of a row, in one read or two.
template <bool LAST>
struct Frag;
template <>
struct Frag<true> {
  u32x4 v;
  HILO_DEV bf16x8 get() const { return __builtin_bit_cast(bf16x8, v); }
  HILO_DEV void pin() { asm volatile("" : "+v"(v)); }
};
template <>
struct Frag<false> {
  u32x2 lo, hi;
  HILO_DEV bf16x8 get() const { return __builtin_bit_cast(bf16x8, __builtin_shufflevector(lo, hi, 0, 1, 2, 3)); }
  HILO_DEV void pin() { asm volatile("" : "+v"(lo), "+v"(hi)); }
};

// Two blocks of 16 columns of a row, four a lane: lanes of groups 0 and 2 get 8 of the first's, of 1 and 3 of the second's,
// so that a store writes 64 consecutive bytes of 16 rows.  tile: its first row, row: values to the lane's, c: the first
// block's column.
HILO_DEV void store_blocks(uint16_t *tile, uint32_t row, int c, int end, int lg, f32x4 a, f32x4 b, bool in) {
  uint32_t x0 = bf16_pair(a[0], a[1]), x1 = bf16_pair(a[2], a[3]), y0 = bf16_pair(b[0], b[1]), y1 = bf16_pair(b[2], b[3]);
  swap16(x0, y0);
  swap16(x1, y1);
  c += 16 * (lg & 1) + 8 * (lg >> 1);
  if (in && c < end) *reinterpret_cast<uint4 *>(tile + (row + c)) = make_uint4(x0, x1, y0, y1);
}
HILO_DEV void store_block(uint16_t *tile, uint32_t row, int c, int end, int lg, f32x4 a, bool in) {
  c += 4 * lg;
  if (in && c < end) *reinterpret_cast<uint2 *>(tile + (row + c)) = make_uint2(bf16_pair(a[0], a[1]), bf16_pair(a[2], a[3]));
}

// Biases of a wave's columns, four a lane of every block.
template <typename G>
struct Bias {
  uint2 v[G::NB];
  HILO_DEV static int part(int j) { return G::GATED ? j / (G::NB / 2) : 0; }
  HILO_DEV static const void *of_part(const ProductProblem &p, const Place &z, int q) {
    return z.stream ? (q ? p.bias[1][1] : p.bias[1][0]) : (q ? p.bias[0][1] : p.bias[0][0]);
  }
  HILO_DEV void load(const ProductProblem &p, const Place &z, int wn, int lg) {
#pragma unroll
    for (int j = 0; j < G::NB; ++j) {
      const void *b = of_part(p, z, part(j));
      const int n = min(z.n0 + wn * (G::COLS / G::WN) + 16 * (G::GATED ? j % (G::NB / 2) : j) + 4 * lg, p.N - 4);
      v[j] = b ? *reinterpret_cast<const uint2 *>(reinterpret_cast<const uint16_t *>(b) + n) : make_uint2(0u, 0u);
    }
  }
  // of what bias_to_lds left
  HILO_DEV void take(const ProductProblem &p, const Place &z, uint32_t area, int lg) {
    u32x2 r[G::NB];
    auto rd = [&](auto jj) __attribute__((always_inline)) {
      constexpr int j = decltype(jj)::value;
      if constexpr (j < G::NB) read8<32 * j>(r[j], area + 8 * lg);
    };
    rd(Int<0>{}); rd(Int<1>{}); rd(Int<2>{}); rd(Int<3>{});
    __builtin_amdgcn_s_waitcnt(0xc07f);
#pragma unroll
    for (int j = 0; j < G::NB; ++j) {
      asm volatile("" : "+v"(r[j]));
      v[j] = of_part(p, z, part(j)) ? make_uint2(r[j][0], r[j][1]) : make_uint2(0u, 0u);
    }
  }
  HILO_DEV f32x4 of(int j) const {
    return f32x4{__uint_as_float(v[j].x << 16), __uint_as_float(v[j].x & 0xffff0000u), __uint_as_float(v[j].y << 16),
                 __uint_as_float(v[j].y & 0xffff0000u)};
  }
};

// The last step of a row block: row 16 i + lr of the wave's rows, columns 16 j + 4 lg .. + 3 of block j.
template <typename G>
HILO_DEV void finish_row(const ProductProblem &p, const Place &z, const Bias<G> &bias, int wid, int i, int lane, f32x4 (&acc)[G::NB]) {
  const int lr = lane & 15, lg = lane >> 4, wn = wid % G::WN;
  const int rl = (wid / G::WN) * (G::BM / G::WM) + 16 * i + lr;
  const bool in = rl < z.rows;
  const int n = z.n0 + wn * (G::COLS / G::WN), end = G::KIND == PRODUCT_OUT ? p.N : p.K;
  // blocks J0 .. J0 + COUNT - 1
  auto put = [&](void *out, size_t ld, size_t from, auto first, auto count) __attribute__((always_inline)) {
    uint16_t *tile = reinterpret_cast<uint16_t *>(out) + size_t(z.row0) * ld + from;
    const uint32_t r = uint32_t(rl) * uint32_t(ld);
    constexpr int J0 = decltype(first)::value, COUNT = decltype(count)::value;
#pragma unroll
    for (int j = 0; j + 1 < COUNT; j += 2) store_blocks(tile, r, n + 16 * j, end, lg, acc[J0 + j], acc[J0 + j + 1], in);
    if constexpr (COUNT % 2 == 1) store_block(tile, r, n + 16 * (COUNT - 1), end, lg, acc[J0 + COUNT - 1], in);
  };
  if constexpr (G::KIND == PRODUCT_OUT) {
#pragma unroll
    for (int j = 0; j < G::NB; ++j) acc[j] += bias.of(j);
    if constexpr (G::GATED) {
      constexpr int H = G::NB / 2;
      if (p.pre) {
        put(p.pre, 2 * size_t(p.N), 0, Int<0>{}, Int<H>{});
        put(p.pre, 2 * size_t(p.N), p.N, Int<H>{}, Int<H>{});
      }
#pragma unroll
      for (int j = 0; j < H; ++j)
#pragma unroll
        for (int e = 0; e < 4; ++e) acc[j][e] = gate_act<false>(acc[j][e], p.silu) * acc[H + j][e];
      put(p.out, p.N, 0, Int<0>{}, Int<H>{});
    } else {
      put(p.out, p.N, 0, Int<0>{}, Int<G::NB>{});
    }
  } else if constexpr (G::KIND == PRODUCT_DX) {
    put(p.dx, p.K, 0, Int<0>{}, Int<G::NB>{});
  } else {
    put(p.dw[z.o], p.K, 0, Int<0>{}, Int<G::NB>{});
  }
}

// Partial sums in register order.
template <typename G>
HILO_DEV size_t part_at(int slot, int wid, int i, int j, int lane) {
  return size_t(slot) * G::BM * G::BN + ((size_t(wid) * G::MB * G::NB + i * G::NB + j) * 64 + lane) * 4;
}

template <typename G>
HILO_DEV void run(const ProductProblem &p, const Plan &q, int pid, uint8_t *lds) {
  constexpr int BM = G::BM, BN = G::BN, KIND = G::KIND, MB = G::MB, NB = G::NB, LA = G::LA, LB = G::LB, WB = G::WB, S = G::SLOTS;
  constexpr bool AK = G::AK, BK = G::BK;
  const int lane = threadIdx.x & 63;
  const int wid = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int lr = lane & 15, lg = lane >> 4, wm = wid / G::WN, wn = wid % G::WN;
  // bytes between rows of the operands as they lie in memory
  const uint32_t lda = 2u * (KIND == PRODUCT_OUT ? p.K : p.parts * p.N), ldb = 2u * p.K;

  // ---- loads: wave wid fills 1 / 8 of either operand's window, LA and LB instructions; offsets into the window's rows
  uint32_t oa[LA], ob[LB];
  auto offsets = [&](auto last, auto blk, uint32_t ld, int row_base, uint32_t (&o)[decltype(blk)::value / 64]) {
    constexpr int BLK = decltype(blk)::value;
#pragma unroll
    for (int i = 0; i < BLK / 64; ++i) {
      if constexpr (decltype(last)::value != 0) {
        const int r = 8 * i + (lane >> 3);  // of the wave's rows; wid * BLK / 8 is a multiple of 16
        const int c = (lane & 7) ^ ((r >> 1) & 7);
        o[i] = uint32_t(row_base + r) * ld + 16u * c;
      } else {
        const int at = wid * (BLK * 16) + i * 1024 + lane * 16, k = at / (BLK * 2), c = at % (BLK * 2) / 16;
        const int f = (k & 3) | ((k >> 3) & 1) << 2;
        o[i] = uint32_t(k) * ld + 16u * (c ^ (2 * f));
      }
    }
  };
  // with a gate, the columns of W of a wave of the product are half the gate's, half the other's; a wave loads rows of one part
  constexpr int WC = BN / G::WN;
  const int wgrp = wid * (BN / 8) / WC, win = wid * (BN / 8) % WC, wpart = G::GATED ? win / (WC / 2) : 0;
  offsets(Int<AK>{}, Int<BM>{}, lda, wid * (BM / 8), oa);
  offsets(Int<BK>{}, Int<BN>{}, ldb, G::GATED ? wgrp * (WC / 2) + win % (WC / 2) : wid * (BN / 8), ob);

  int lu = pid, lslot = 0;
  int lw = 0, lwe = 0;              // windows of the item yet to load
  int lk = 0, lkn = 0, lpiece = 0;  // k within the piece, the piece's length, which piece
  const char *la = nullptr, *lb = nullptr;
  uint32_t ra = 0, rb = 0;          // bytes: rows of the tile (k last), or columns of a row (k first)
  Place lz{0, 0, 0, 0, 0, 0};
  bool more = true;
  auto ld_piece = [&]() __attribute__((always_inline)) {  // bases of piece lpiece
    if constexpr (KIND == PRODUCT_OUT) {
      const int part = wpart;
      const void *w = lz.stream ? (part ? p.w[1][1] : p.w[1][0]) : (part ? p.w[0][1] : p.w[0][0]);
      la = reinterpret_cast<const char *>(p.x) + size_t(lz.row0) * lda;
      lb = reinterpret_cast<const char *>(w) + size_t(lz.n0) * ldb;
      lkn = p.K;
      ra = uint32_t(lz.rows - 1) * lda + 2u * p.K;
      rb = uint32_t(min(G::COLS, p.N - lz.n0) - 1) * ldb + 2u * p.K;
    } else if constexpr (KIND == PRODUCT_DX) {
      const void *w = lz.stream ? (lpiece ? p.w[1][1] : p.w[1][0]) : (lpiece ? p.w[0][1] : p.w[0][0]);
      la = reinterpret_cast<const char *>(p.d) + size_t(lz.row0) * lda + size_t(lpiece) * p.N * 2;
      lb = reinterpret_cast<const char *>(w) + size_t(lz.n0) * 2;
      lkn = p.N;
      ra = uint32_t(lz.rows - 1) * lda + 2u * p.N;
      rb = 2u * (p.K - lz.n0);
    } else {
      const Segment s = segment(p, lpiece);
      la = reinterpret_cast<const char *>(p.d) + size_t(s.lo) * lda + (size_t(lz.part) * p.N + lz.row0) * 2;
      lb = reinterpret_cast<const char *>(p.x) + size_t(s.lo) * ldb + size_t(lz.n0) * 2;
      lkn = s.n;
      ra = 2u * (p.N - lz.row0);
      rb = 2u * (p.K - lz.n0);
    }
  };
  auto ld_item = [&]() __attribute__((always_inline)) {  // the next item that has windows
    while (true) {
      const Item it = item_at(q, lu);
      if (!it.valid) {
        more = false;
        return;
      }
      lu += P;
      lz = place_of<G>(p, q, it.t);
      const int n = windows<KIND>(p, lz.stream);
      lw = int((long long)n * it.pc / it.n);
      lwe = int((long long)n * (it.pc + 1) / it.n);
      if (lw == lwe) continue;
      int w = lw;  // windows before it within its piece
      if constexpr (KIND == PRODUCT_OUT) {
        lpiece = 0;
      } else if constexpr (KIND == PRODUCT_DX) {
        const int per = (p.N + 63) / 64;
        lpiece = w / per;
        w -= lpiece * per;
      } else {
        lpiece = lz.stream;
        int n1 = (segment(p, lpiece).n + 63) / 64;
        while (w >= n1) {
          w -= n1;
          lpiece += 2;
          n1 = (segment(p, lpiece).n + 63) / 64;
        }
      }
      ld_piece();
      lk = 64 * w;
      return;
    }
  };
  // the next window: to the next piece or item where this one ends
  auto ld_step = [&]() __attribute__((always_inline)) {
    if (!more) return;
    if (lw == lwe) {
      ld_item();
    } else if (KIND != PRODUCT_OUT && lk >= lkn) {
      if constexpr (KIND == PRODUCT_DX) {
        ++lpiece;
        ld_piece();
      } else {
        do {
          lpiece += 2;
          ld_piece();
        } while (lkn <= 0);
      }
      lk = 0;
    }
  };
  auto ld_operand = [&](auto last, auto blk, const char *base, uint32_t reach, uint32_t ld, const uint32_t (&o)[decltype(blk)::value / 64],
                        uint8_t *d) __attribute__((always_inline)) {
    constexpr int BLK = decltype(blk)::value;
    const int kv = min(64, lkn - lk);
    uint32_t bytes;
    if constexpr (decltype(last)::value != 0) {
      bytes = reach - 2u * uint32_t(lk);
      base += size_t(lk) * 2;
    } else {
      bytes = uint32_t(kv - 1) * ld + reach;
      base += size_t(lk) * ld;
    }
    if (!more) bytes = 0;
    // chunks of k behind the end: offsets behind the buffer's.  The chunk of instruction i is that of 0, or its bit 2 the other
    // way round
    const int lane = opaque(threadIdx.x & 63), c = (lane & 7) ^ ((lane >> 4) & 3);
    const bool in[2] = {8 * c < kv, 8 * (c ^ 4) < kv};
#pragma unroll
    for (int i = 0; i < BLK / 64; ++i)
      buffer_to_lds(base, bytes, decltype(last)::value == 0 || in[i & 1] ? o[i] : kBehind, d + i * 1024);
  };
  auto ld_a = [&]() __attribute__((always_inline)) {
    ld_operand(Int<AK>{}, Int<BM>{}, la, ra, lda, oa, lds + lslot * WB + wid * (BM * 16));
  };
  auto ld_b = [&]() __attribute__((always_inline)) {
    ld_operand(Int<BK>{}, Int<BN>{}, lb, rb, ldb, ob, lds + lslot * WB + BM * 128 + wid * (BN * 16));
    lk += 64;
    ++lw;
    lslot = lslot == S - 1 ? 0 : lslot + 1;
  };

  // ---- fragments
  const uint32_t lds0 = (uint32_t)(uintptr_t)lds;
  const int f = (lr >> 2) | (lg & 1) << 2;
  uint32_t fa[2], fb[2];  // k last: of either half; k first: [0]
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    const uint32_t chunk = uint32_t((4 * h + lg) ^ ((lr >> 1) & 7)) * 16;
    fa[h] = lds0 + (AK ? (wm * (BM / G::WM) + lr) * 128 + chunk : (8 * lg + (lr >> 2)) * (BM * 2) + 8 * (lr & 3) + (f << 5));
    fb[h] = lds0 + BM * 128 + (BK ? (wn * (BN / G::WN) + lr) * 128 + chunk : (8 * lg + (lr >> 2)) * (BN * 2) + 8 * (lr & 3) + (f << 5));
  }
  f32x4 acc[MB][NB];
  Frag<AK> a[2][MB];
  Frag<BK> b[2][NB];
  uint32_t so = 0;  // byte offset of the window being read
  // read x of set h: W's fragments first
  auto rd = [&](auto hh, auto xx) __attribute__((always_inline)) {
    constexpr int h = decltype(hh)::value, x = decltype(xx)::value;
    if constexpr (x < NB) {
      if constexpr (BK) {
        read16<x * 2048>(b[h][x].v, fb[h] + so);
      } else {
        const uint32_t at = (fb[0] + so) ^ uint32_t((wn * NB + x) << 5);
        read_tr<h * 32 * BN * 2>(b[h][x].lo, at);
        read_tr<(h * 32 + 4) * BN * 2>(b[h][x].hi, at);
      }
    } else if constexpr (x < NB + MB) {
      constexpr int i = x - NB;
      if constexpr (AK) {
        read16<i * 2048>(a[h][i].v, fa[h] + so);
      } else {
        const uint32_t at = (fa[0] + so) ^ uint32_t((wm * MB + i) << 5);
        read_tr<h * 32 * BM * 2>(a[h][i].lo, at);
        read_tr<(h * 32 + 4) * BM * 2>(a[h][i].hi, at);
      }
    }
  };
  auto rd_wait = [&](auto hh) __attribute__((always_inline)) {
    constexpr int h = decltype(hh)::value;
    __builtin_amdgcn_s_waitcnt(0xc07f);  // lgkmcnt(0), in the form the compiler's own wait tracking sees
#pragma unroll
    for (int i = 0; i < MB; ++i) a[h][i].pin();
#pragma unroll
    for (int j = 0; j < NB; ++j) b[h][j].pin();
    __builtin_amdgcn_sched_barrier(0);
  };
  auto rd_all = [&](auto hh) __attribute__((always_inline)) {
    auto r4 = [&](auto x) __attribute__((always_inline)) {
      constexpr int x0 = decltype(x)::value;
      rd(hh, Int<x0>{}); rd(hh, Int<x0 + 1>{}); rd(hh, Int<x0 + 2>{}); rd(hh, Int<x0 + 3>{});
    };
    static_assert(MB + NB <= 12, "reads of a set");
    r4(Int<0>{}); r4(Int<4>{}); r4(Int<8>{});
    rd_wait(hh);
  };
  // the MFMAs of set h, row by row; after each row but the last a share of the reads of the other set; with ld the loads of a window
  auto half = [&](auto hh, auto ldd) __attribute__((always_inline)) {
    constexpr int h = decltype(hh)::value;
    constexpr int RPB = (NB + MB + MB - 2) / (MB - 1);
    auto row = [&](auto ii) __attribute__((always_inline)) {
      constexpr int i = decltype(ii)::value;
      if constexpr (i < MB) {
#pragma unroll
        for (int j = 0; j < NB; ++j) acc[i][j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(b[h][j].get(), a[h][i].get(), acc[i][j], 0, 0, 0);
        __builtin_amdgcn_sched_barrier(0);
        if constexpr (i < MB - 1) {
          static_assert(RPB <= 3, "reads per row");
          rd(Int<1 - h>{}, Int<i * RPB>{});
          if constexpr (RPB > 1) rd(Int<1 - h>{}, Int<i * RPB + 1>{});
          if constexpr (RPB > 2) rd(Int<1 - h>{}, Int<i * RPB + 2>{});
        }
        if constexpr (decltype(ldd)::value != 0) {
          if constexpr (i == 0) ld_a();
          if constexpr (i == MB / 2) ld_b();
        }
        __builtin_amdgcn_sched_barrier(0);
      }
    };
    row(Int<0>{}); row(Int<1>{}); row(Int<2>{}); row(Int<3>{});
    row(Int<4>{}); row(Int<5>{}); row(Int<6>{}); row(Int<7>{});
  };
  // this wave has read the window, and all but the last issued windows have landed; on to the next.  Not waited for in the
  // first S - 1 windows of a tile: theirs have landed before the stores of the tile before, which wait_vm would wait for as well
  int landed = S - 1;
  auto next_window = [&]() __attribute__((always_inline)) {
    // (MFMAs before a branch would be moved behind it, past the reads that they are to run beside)
#pragma unroll
    for (int i = 0; i < MB; ++i)
#pragma unroll
      for (int j = 0; j < NB; ++j) asm volatile("" : "+v"(acc[i][j]));
    if (landed > 0) --landed;
    else wait_vm<(S - 2) * (LA + LB)>();
    asm volatile("s_barrier" ::: "memory");
    __builtin_amdgcn_sched_barrier(0);
    so = so == (S - 1) * WB ? 0 : so + WB;
  };

#pragma unroll 1
  for (int w = 0; w < S; ++w) {
    ld_step();
    ld_a();
    ld_b();
  }
  wait_vm<0>();
  asm volatile("s_barrier" ::: "memory");
  for (int u = pid;; u += P) {
    const Item it = item_at(q, u);
    if (!it.valid) break;
    const Place z = place_of<G>(p, q, it.t);
    const int n = windows<KIND>(p, z.stream);
    const int w0 = int((long long)n * it.pc / it.n), w1 = int((long long)n * (it.pc + 1) / it.n);
    uint8_t *area = lds + S * WB + wid * 256;
    if constexpr (KIND == PRODUCT_OUT) {
      if (it.n == 1) bias_to_lds<BN / G::WN, G::GATED ? 2 : 1>(p, z, z.n0 + wn * (G::COLS / G::WN), area, true);
    }
#pragma unroll
    for (int i = 0; i < MB; ++i)
#pragma unroll
      for (int j = 0; j < NB; ++j) acc[i][j] = f32x4{0.f, 0.f, 0.f, 0.f};
    rd_all(Int<0>{});
#pragma unroll 1
    for (int w = w0; w < w1; ++w) {
      ld_step();
      half(Int<0>{}, Int<0>{});
      rd_wait(Int<1>{});
      next_window();
      half(Int<1>{}, Int<1>{});
      rd_wait(Int<0>{});
    }
    wait_vm<0>();  // the next tile's first windows, and the biases
    landed = S - 1;
    const int lane = opaque(threadIdx.x & 63);
    if (it.n > 1) {
#pragma unroll
      for (int i = 0; i < MB; ++i)
#pragma unroll
        for (int j = 0; j < NB; ++j) *reinterpret_cast<f32x4 *>(p.part + part_at<G>(it.slot, wid, i, j, lane)) = acc[i][j];
    } else {
      Bias<G> bias;
      if constexpr (KIND == PRODUCT_OUT) {
        bias.take(p, z, lds0 + S * WB + wid * 256, lane >> 4);
      }
#pragma unroll
      for (int i = 0; i < MB; ++i) {
        finish_row<G>(p, z, bias, wid, i, lane, acc[i]);
        asm volatile("" ::: "memory");
      }
    }
  }
  wait_vm<0>();
}

// A wave of the fixup adds one row block of one wave's part of a cut tile, pieces in order.
template <typename G>
HILO_DEV void fix(const ProductProblem &p, const Plan &q) {
  if (q.s == 1) return;
  const int lane = threadIdx.x & 63;
  const int items = q.tail * 8 * G::MB;
  for (int x = blockIdx.x * 8 + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6); x < items; x += gridDim.x * 8) {
    const int v = x / (8 * G::MB), rem = x - v * 8 * G::MB, wid = rem / G::MB, i = rem - wid * G::MB;
    const Place z = place_of<G>(p, q, q.full + v);
    Bias<G> bias;
    if constexpr (G::KIND == PRODUCT_OUT) bias.load(p, z, wid % G::WN, lane >> 4);
    f32x4 acc[G::NB];
#pragma unroll
    for (int j = 0; j < G::NB; ++j) acc[j] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll 4
    for (int pc = 0; pc < q.s; ++pc)
#pragma unroll
      for (int j = 0; j < G::NB; ++j)
        acc[j] += *reinterpret_cast<const f32x4 *>(p.part + part_at<G>(pc * q.tail + v, wid, i, j, lane));
    finish_row<G>(p, z, bias, wid, i, lane, acc);
  }
}

// 256 x 256, 256 x 128, 128 x 128: the larger one loads less for a product, the smaller one leaves fewer CUs idle.  Each is best
// somewhere (us): 18900 x 296 -> 3392 68, 79, 93; 4700 x 4096 -> 1536 78, 62, 73; 1000 x 4096 -> 4096 56, 47, 40.
constexpr Cost kCost[3][3] = {{{146, 700, 700, 50, 7}, {84, 500, 650, 35, 3}, {50, 400, 600, 22, 1}},   // by kind of product
                              {{160, 700, 700, 50, 7}, {100, 500, 650, 35, 3}, {65, 400, 600, 22, 1}},
                              {{155, 700, 700, 50, 7}, {90, 500, 650, 35, 3}, {55, 400, 600, 22, 1}}};
template <int I, int KIND, bool GATED>
using Tile = Geo<I < 2 ? 256 : 128, I < 1 ? 256 : 128, KIND, GATED>;

// Row tiles of outputs (DW) or as the caller counts them, for each tile the plan and its cost: which is quickest.
template <int KIND, bool GATED, typename F>
HILO_BOTH int choose(const ProductProblem &p, int nk, F &&row_tiles, Plan &q) {
  q = make_plan<Tile<0, KIND, GATED>>(p, row_tiles(256), nk, kCost[KIND][0]);
  const Plan a = make_plan<Tile<1, KIND, GATED>>(p, q.R, nk, kCost[KIND][1]);
  const Plan b = make_plan<Tile<2, KIND, GATED>>(p, row_tiles(128), nk, kCost[KIND][2]);
  int best = 0;
  long long cost = plan_cost(q.T, nk, kCost[KIND][0], p.splits);
  const long long ca = plan_cost(a.T, nk, kCost[KIND][1], p.splits), cb = plan_cost(b.T, nk, kCost[KIND][2], p.splits);
  if (ca < cost) {
    best = 1;
    cost = ca;
    q = a;
  }
  if (cb < cost) {
    best = 2;
    q = b;
  }
  return best;
}
// On the device, which knows the rows; the main kernel and the fixup find the same.
template <int KIND, bool GATED>
HILO_DEV int choose(const ProductProblem &p, Plan &q) {
  int nk = windows<KIND>(p, 0);
  if constexpr (KIND == PRODUCT_DW) {
    if (!p.merged) nk = max(nk, windows<KIND>(p, 1));
    return choose<KIND, GATED>(p, nk, [&](int bm) { return p.outs * ((p.N + bm - 1) / bm); }, q);
  }
  return choose<KIND, GATED>(p, nk, [&](int bm) { return count_row_tiles(p, bm); }, q);
}

template <int KIND, bool GATED>
__global__ __launch_bounds__(512, 2) void k_product_tiles(ProductProblem p) {
  constexpr auto bytes = [](auto g) { return decltype(g)::LDS; };
  constexpr int L0 = bytes(Tile<0, KIND, GATED>{}), L1 = bytes(Tile<1, KIND, GATED>{}), L2 = bytes(Tile<2, KIND, GATED>{});
  __shared__ __attribute__((aligned(1024))) uint8_t lds[std::max(L0, std::max(L1, L2))];
  const int pid = xcd_remap(blockIdx.x, P);
  Plan q;
  switch (choose<KIND, GATED>(p, q)) {
    case 0: run<Tile<0, KIND, GATED>>(p, q, pid, lds); break;
    case 1: run<Tile<1, KIND, GATED>>(p, q, pid, lds); break;
    default: run<Tile<2, KIND, GATED>>(p, q, pid, lds);
  }
}

// dx and the weights' gradients in a launch, whole 256 x 256 tiles of the one and then of the others: a workgroup's first of
// the latter follows the last of the former, and the two have one last turn between them.  2766 x 8192 -> 3072: 264 us, in
// launches of their own 303.
__global__ __launch_bounds__(512, 2) void k_product_back_tiles(ProductProblem x, ProductProblem w) {
  using GX = Tile<0, PRODUCT_DX, false>;
  using GW = Tile<0, PRODUCT_DW, false>;
  __shared__ __attribute__((aligned(1024))) uint8_t lds[std::max(GX::LDS, GW::LDS)];
  const int pid = xcd_remap(blockIdx.x, P);
  const Plan qx = make_plan<GX>(x, count_row_tiles(x, 256), 1, kCost[PRODUCT_DX][0]);
  run<GX>(x, qx, pid, lds);
  asm volatile("s_barrier" ::: "memory");
  const Plan qw = make_plan<GW>(w, w.outs * ((w.N + 255) / 256), 1, kCost[PRODUCT_DW][0]);
  run<GW>(w, qw, (pid + P - qx.tail) % P, lds);
}

template <int KIND, bool GATED>
__global__ __launch_bounds__(512) void k_product_fix(ProductProblem p) {
  Plan q;
  switch (choose<KIND, GATED>(p, q)) {
    case 0: fix<Tile<0, KIND, GATED>>(p, q); break;
    case 1: fix<Tile<1, KIND, GATED>>(p, q); break;
    default: fix<Tile<2, KIND, GATED>>(p, q);
  }
}

}  // namespace pt

size_t product_tiles_part_bytes() { return size_t(pt::P) * 256 * 256 * sizeof(float); }

// The plan, and its cost, where all the rows of the buffers are in use.
template <int KIND, bool GATED>
static long long plan_rows(ProductProblem p, pt::Plan &q) {
  const int nk = KIND == PRODUCT_OUT ? (p.K + 63) / 64 : KIND == PRODUCT_DX ? p.parts * ((p.N + 63) / 64) : (p.rows + 63) / 64;
  p.splits = pt::kSearch;
  const int best = pt::choose<KIND, GATED>(
      p, nk, [&](int bm) { return KIND == PRODUCT_DW ? p.outs * ((p.N + bm - 1) / bm) : (p.rows + bm - 1) / bm; }, q);
  return pt::plan_cost(q.T, nk, pt::kCost[KIND][best], pt::kSearch);
}

template <int KIND, bool GATED>
static hipError_t run_tiles(ProductProblem p, hipStream_t st) {
  pt::Plan q;
  plan_rows<KIND, GATED>(p, q);
  p.splits = q.s > 1 ? q.s : 0;
  hipLaunchKernelGGL((pt::k_product_tiles<KIND, GATED>), dim3(pt::P), dim3(512), 0, st, p);
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess || !p.splits) return e;
  hipLaunchKernelGGL((pt::k_product_fix<KIND, GATED>), dim3(pt::P), dim3(512), 0, st, p);
  return hipGetLastError();
}

// The longest of the workgroups' shares of whole 256 x 256 tiles, in order: of dx, where `both`, and of the weights' gradients.
static long long shares(const ProductProblem &x, const ProductProblem &w, bool both) {
  long long each[pt::P] = {};
  int at = 0;
  auto add = [&](int kind, int tiles, int nk) {
    const long long cost = pt::kCost[kind][0].windows(nk) + pt::kCost[kind][0].tile;
    for (int k = 0; k < pt::P; ++k) each[(at + k) % pt::P] += (tiles / pt::P + (k < tiles % pt::P)) * cost;
    at += tiles % pt::P;
  };
  const int cols = (x.K + 255) / 256;
  if (both) add(PRODUCT_DX, (x.rows + 255) / 256 * cols, x.parts * ((x.N + 63) / 64));
  for (int o = 0; o < w.outs; ++o) {
    const long long text = std::min<long long>(x.rows, (long long)x.B * x.L);
    const long long rows = w.merged ? x.rows : w.out_stream[o] ? text : x.rows - text;
    add(PRODUCT_DW, (w.N + 255) / 256 * cols, int((rows + 63) / 64));
  }
  return *std::max_element(each, each + pt::P);
}

// Whether both products in one launch are quicker than each with a plan of its own.
static bool one_launch(const ProductProblem &x, const ProductProblem &w) {
  pt::Plan q;
  const long long dx = plan_rows<PRODUCT_DX, false>(x, q), dw = plan_rows<PRODUCT_DW, false>(w, q);
  return shares(x, w, true) < dx + (w.merged ? dw : std::min(dw, shares(x, w, false)));
}

hipError_t launch_product_back_tiles(ProductProblem x, ProductProblem w, hipStream_t st) {
  if (!one_launch(x, w)) {
    const hipError_t e = run_tiles<PRODUCT_DX, false>(x, st);
    return e != hipSuccess ? e : run_tiles<PRODUCT_DW, false>(w, st);
  }
  x.splits = w.splits = 0;
  hipLaunchKernelGGL(pt::k_product_back_tiles, dim3(pt::P), dim3(512), 0, st, x, w);
  return hipGetLastError();
}

hipError_t launch_product_tiles(int kind, const ProductProblem &p, hipStream_t st) {
  if (kind == PRODUCT_OUT) return p.parts == 2 ? run_tiles<PRODUCT_OUT, true>(p, st) : run_tiles<PRODUCT_OUT, false>(p, st);
  if (kind == PRODUCT_DX) return run_tiles<PRODUCT_DX, false>(p, st);
  return run_tiles<PRODUCT_DW, false>(p, st);
}

}  // namespace hilo
