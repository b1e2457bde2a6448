// Products on E4M3 codes with a power-of-two scale for each block of 128 (hilo_linear_fp8) on large tiles.
//
// The loop is product_bf16.hip's with k last in both operands: a window is 128 codes of 128-byte rows, just the block that
// has one scale, and v_mfma_scale_f32_32x32x64_f8f6f4 takes both operands' scales, so that they cost no arithmetic.  Four
// windows' scales of a row of x are a dword, which goes to LDS beside each window; those of w are the same for a wave's
// columns (128 x 128 blocks).
//
// The instruction aligns the products of eight consecutive k to the one with the largest exponents and cuts what lies more than 13
// bits below (each group's sum is then added in float32's precision): enough for outputs of bf16, not for float32's or for
// codes, which go another way (run_wide).
//
// Bound by the matrix cores and the loads that feed them: 22560 x 3072 -> 8192 with a gate from codes 976 us (2.3 PFLOP/s; the
// library's large product reaches 2.57); 2766 x 3072 -> 9216 96, two turns for 1.55 turns' tiles.
//
// A wave's 128 x 64 are 32 x 32 blocks: lane l holds row l % 32 and, W's rows being read in the order perm, columns
// 16 (l / 32) .. + 15 of a block in register order.  With a gate the two blocks of columns are the gate's and the other's.
#include <algorithm>

#include "product_tiles.h"

namespace hilo {

typedef int i32x8 __attribute__((ext_vector_type(8)));

namespace pt {

template <int BM_, int BN_, bool GATED_>
struct Geo8 {
  static constexpr int BM = BM_, BN = BN_, KIND = PRODUCT_OUT;
  static constexpr bool GATED = GATED_;
  static constexpr int MB = BM / 64, NB = BN / 128;  // blocks of 32 x 32 of a wave
  static constexpr int LA = BM / 64, LB = BN / 64;
  static constexpr int WB = (BM + BN) * 128;
  static constexpr int RING = 4, RB = BM * 4;        // windows' scales of x, bytes of one
  static constexpr int SLOTS = 3 * WB + RING * RB + 2048 <= 160 * 1024 ? 3 : 2;
  static constexpr int AREAS = SLOTS * WB + RING * RB, LDS = AREAS + 2048;  // 256 bytes a wave for biases
  static constexpr int COLS = GATED ? BN / 2 : BN;
  static_assert(RING > SLOTS, "a window's scales last until it is multiplied");
  static_assert(!GATED || NB == 2, "a block of either part");
};

// 16-byte chunk c of row r lies at c ^ swz(r); perm: the row of W that lane r of a block reads.
HILO_DEV int swz(int r) { return ((r >> 1) & 3) ^ ((((r >> 3) ^ (r >> 4)) & 1) << 2); }
HILO_DEV int perm(int r) { return ((r & 4) ? 16 : 0) + 4 * (r >> 3) + (r & 3); }

template <int OFF>
HILO_DEV void read4(uint32_t &d, uint32_t addr) {
  asm volatile("ds_read_b32 %0, %1 offset:%2" : "=v"(d) : "v"(addr), "n"(OFF) : "memory");
}
// Four scales of w: uniform, by a scalar load.
HILO_DEV uint32_t scales_at(const uint8_t *s, int group) {
  return reinterpret_cast<const __attribute__((address_space(4))) uint32_t *>(reinterpret_cast<uint64_t>(s))[group];
}
HILO_DEV i32x8 cat8(u32x4 lo, u32x4 hi) {
  return __builtin_bit_cast(i32x8, __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7));
}

HILO_DEV void store16(uint16_t *o, const float (&v)[16]) {
#pragma unroll
  for (int h = 0; h < 2; ++h)
    reinterpret_cast<uint4 *>(o)[h] = make_uint4(bf16_pair(v[8 * h], v[8 * h + 1]), bf16_pair(v[8 * h + 2], v[8 * h + 3]),
                                                 bf16_pair(v[8 * h + 4], v[8 * h + 5]), bf16_pair(v[8 * h + 6], v[8 * h + 7]));
}

// Column of a wave's block j of its part, for lane half g.
template <typename G>
HILO_DEV int col8(const Place &z, int wn, int j, int g) {
  return z.n0 + wn * (G::COLS / 4) + (G::GATED ? 0 : 32 * j) + 16 * g;
}
// Biases of a lane's 16 columns of every block, bf16.
template <typename G>
struct Bias8 {
  u32x4 v[G::NB][2];
  HILO_DEV static const void *of_block(const ProductProblem &p, const Place &z, int j) {
    const int q = G::GATED ? j : 0;
    return z.stream ? (q ? p.bias[1][1] : p.bias[1][0]) : (q ? p.bias[0][1] : p.bias[0][0]);
  }
  HILO_DEV void load(const ProductProblem &p, const Place &z, int wn, int g) {
#pragma unroll
    for (int j = 0; j < G::NB; ++j) {
      const uint16_t *b = reinterpret_cast<const uint16_t *>(of_block(p, z, j));
      const int n = min(col8<G>(z, wn, j, g), p.N - 16);
#pragma unroll
      for (int h = 0; h < 2; ++h) v[j][h] = b ? *reinterpret_cast<const u32x4 *>(b + n + 8 * h) : u32x4(0u);
    }
  }
  // of what bias_to_lds left
  HILO_DEV void take(const ProductProblem &p, const Place &z, uint32_t area, int g) {
    auto rd = [&](auto jj) __attribute__((always_inline)) {
      constexpr int j = decltype(jj)::value;
      if constexpr (j < G::NB) {
        read16<64 * j>(v[j][0], area + 32 * g);
        read16<64 * j + 16>(v[j][1], area + 32 * g);
      }
    };
    rd(Int<0>{}); rd(Int<1>{});
    __builtin_amdgcn_s_waitcnt(0xc07f);
#pragma unroll
    for (int j = 0; j < G::NB; ++j)
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        asm volatile("" : "+v"(v[j][h]));
        if (!of_block(p, z, j)) v[j][h] = u32x4(0u);
      }
  }
  HILO_DEV float of(int j, int e) const {
    const uint32_t w = v[j][e >> 3][(e >> 1) & 3];
    return __uint_as_float(e & 1 ? w & 0xffff0000u : w << 16);
  }
};

// The last step of a row block but for codes: rows 32 i + l % 32 of the wave's.
template <typename G>
HILO_DEV void finish8(const ProductProblem &p, const Place &z, const Bias8<G> &bias, int wid, int i, int lane, f32x16 (&acc)[G::NB]) {
  const int rl = (wid >> 2) * (G::BM / 2) + 32 * i + (lane & 31), wn = wid & 3, g = lane >> 5;
  uint16_t *tile = reinterpret_cast<uint16_t *>(p.out) + size_t(z.row0) * p.N;
  const uint32_t row = uint32_t(rl) * uint32_t(p.N);
  if constexpr (G::GATED) {
#pragma unroll
    for (int e = 0; e < 16; ++e) acc[0][e] = gate_act<false>(acc[0][e] + bias.of(0, e), p.silu) * (acc[1][e] + bias.of(1, e));
  }
#pragma unroll
  for (int j = 0; j < (G::GATED ? 1 : G::NB); ++j) {
    const int n = col8<G>(z, wn, j, g);
    float v[16];
#pragma unroll
    for (int e = 0; e < 16; ++e) v[e] = G::GATED ? acc[j][e] : acc[j][e] + bias.of(j, e);
    if (rl < z.rows && n < p.N) store16(tile + (row + uint32_t(n)), v);
  }
}

// A block of a partial tile, by quads: 64 lanes' 16 bytes side by side.
template <typename G>
HILO_DEV float *part_at8(float *part, int slot, int wid, int i, int j, int lane) {
  return part + size_t(slot) * G::BM * G::BN + (size_t(wid) * G::MB * G::NB + i * G::NB + j) * 1024 + lane * 4;
}
HILO_DEV void store_part8(float *to, const f32x16 &v) {
#pragma unroll
  for (int e = 0; e < 4; ++e)
    *reinterpret_cast<f32x4 *>(to + 256 * e) = f32x4{v[4 * e], v[4 * e + 1], v[4 * e + 2], v[4 * e + 3]};
}
HILO_DEV void add_part8(f32x16 &v, const f32x4 (&w)[4]) {
#pragma unroll
  for (int e = 0; e < 16; ++e) v[e] += w[e >> 2][e & 3];
}

// A workgroup's loads, product_bf16.hip's with k last, and a window's scales: windows of its items one after another.
template <typename G>
struct Loads8 {
  static constexpr int BM = G::BM, BN = G::BN, LA = G::LA, LB = G::LB, WB = G::WB, S = G::SLOTS;
  const ProductProblem &p;
  const Plan &q;
  uint8_t *lds;
  int wid;
  uint32_t ld, lds_scale;
  int nk;
  uint32_t oa, ob;  // of instruction 0
  int lu, slot = 0, ring = 0, w = 0, we = 0, rows = 0;
  const char *la = nullptr, *lb = nullptr, *lsc = nullptr;
  uint32_t ra = 0, rb = 0;
  bool more = true;

  HILO_DEV Loads8(const ProductProblem &p_, const Plan &q_, int pid, uint8_t *lds_, int wid_)
      : p(p_), q(q_), lds(lds_), wid(wid_), ld(p_.K), lds_scale(scale_stride(p_.K)), nk((p_.K + 127) / 128), lu(pid) {
    const int lane = threadIdx.x & 63, r = lane >> 3;
    const int wrow = G::GATED ? (wid >> 1) * (BN / 8) : wid * (BN / 8);  // first row of W, of its part, that the wave loads
    oa = uint32_t(wid * (BM / 8) + r) * ld + 16u * ((lane & 7) ^ swz(wid * (BM / 8) + r));
    ob = uint32_t(wrow + r) * ld + 16u * ((lane & 7) ^ swz(wid * (BN / 8) + r));
  }
  // to the next item where this one ends
  HILO_DEV void step() {
    if (!more || w < we) return;
    const Item it = item_at(q, lu);
    if (!it.valid) {
      more = false;
      return;
    }
    lu += P;
    const Place z = place_of<G>(p, q, it.t);
    w = int((long long)nk * it.pc / it.n);
    we = int((long long)nk * (it.pc + 1) / it.n);
    const int part = G::GATED ? wid & 1 : 0;
    const void *m = z.stream ? (part ? p.w[1][1] : p.w[1][0]) : (part ? p.w[0][1] : p.w[0][0]);
    la = reinterpret_cast<const char *>(p.x) + size_t(z.row0) * ld;
    lb = reinterpret_cast<const char *>(m) + size_t(z.n0) * ld;
    lsc = reinterpret_cast<const char *>(p.x_scale) + size_t(z.row0) * lds_scale;
    rows = z.rows;
    ra = uint32_t(z.rows) * ld;
    rb = uint32_t(min(G::COLS, p.N - z.n0)) * ld;
  }
  template <int L>
  HILO_DEV void window(const char *base, uint32_t reach, uint32_t o, int lds_base, uint8_t *d) {
    // the chunk of instruction i (8 rows) is that of instruction 0, or its bit 2 the other way round; chunks of k behind the end: offsets behind the buffer's
    const int kv = p.K - 128 * w, lane = opaque(threadIdx.x & 63), c = (lane & 7) ^ swz(lds_base + (lane >> 3));
    const uint32_t o0 = 16 * c < kv ? o : kBehind, o1 = 16 * (c ^ 4) < kv ? o + (c & 4 ? -64 : 64) : kBehind;
    const uint32_t bytes = more ? reach - 128u * uint32_t(w) : 0u;
    base += size_t(w) * 128;
#pragma unroll
    for (int i = 0; i < L; ++i) buffer_to_lds(base, bytes, ((i ^ (i >> 1)) & 1 ? o1 : o0) + uint32_t(8 * i) * ld, d + i * 1024);
  }
  HILO_DEV void a() {
    constexpr int N = BM / 64;
    const int r = 64 * (wid % N) + opaque(threadIdx.x & 63);
    __builtin_amdgcn_raw_ptr_buffer_load_lds(
        __builtin_amdgcn_make_buffer_rsrc(const_cast<char *>(lsc), 0, more ? int(uint32_t(rows) * lds_scale) : 0, 0x00020000),
        (__attribute__((address_space(3))) void *)(lds + S * WB + ring * G::RB + 256 * (wid % N)), 4,
        int(uint32_t(r) * lds_scale + 4u * (uint32_t(w) >> 2)), 0, 0, 0);
    ring = (ring + 1) & (G::RING - 1);
    window<LA>(la, ra, oa, wid * (BM / 8), lds + slot * WB + wid * (BM * 16));
  }
  HILO_DEV void b() {
    window<LB>(lb, rb, ob, wid * (BN / 8), lds + slot * WB + BM * 128 + wid * (BN * 16));
    ++w;
    slot = slot == S - 1 ? 0 : slot + 1;
  }
  // the first S windows
  HILO_DEV void start() {
#pragma unroll 1
    for (int i = 0; i < S; ++i) {
      step();
      a();
      b();
    }
    wait_vm<0>();
    asm volatile("s_barrier" ::: "memory");
  }
  // this wave has read a window, and all but the last issued windows have landed; first: as product_bf16.hip's next_window
  template <bool FIRST>
  HILO_DEV void next() {
    if constexpr (!FIRST) wait_vm<(S - 2) * (LA + LB + 1)>();
    asm volatile("s_barrier" ::: "memory");
    __builtin_amdgcn_sched_barrier(0);
  }
};

template <typename G>
HILO_DEV void run8(const ProductProblem &p, const Plan &q, int pid, uint8_t *lds) {
  constexpr int BM = G::BM, BN = G::BN, MB = G::MB, NB = G::NB, WB = G::WB, S = G::SLOTS;
  const int lane = threadIdx.x & 63;
  const int wid = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int wm = wid >> 2, wn = wid & 3;
  Loads8<G> loads(p, q, pid, lds, wid);
  const int nk = loads.nk;

  // ---- fragments: of half h, chunks 4 h + g and 4 h + 2 + g of a row (g = lane / 32)
  const uint32_t lds0 = (uint32_t)(uintptr_t)lds;
  const int r32 = lane & 31, g32 = lane >> 5;
  const int w32 = perm(r32);
  const uint32_t fa = lds0 + (wm * (BM / 2) + r32) * 128 + (g32 ^ swz(r32)) * 16;
  const uint32_t fb = lds0 + BM * 128 + (wn * (BN / 4) + w32) * 128 + (g32 ^ swz(w32)) * 16;
  f32x16 acc[MB][NB];
  u32x4 a[2][MB][2], b[2][NB][2];
  uint32_t sa[MB], sb[NB], sn[MB];  // scales of this window in the lowest byte; the next window's rows', as they lie in LDS
  uint32_t so = 0;
  int ring = 0;
  auto rd = [&](auto hh, auto xx) __attribute__((always_inline)) {
    constexpr int h = decltype(hh)::value, x = decltype(xx)::value / 2, c = decltype(xx)::value % 2;
    if constexpr (x < NB) read16<x * 4096>(b[h][x][c], (fb + so) ^ uint32_t(32 * (2 * h + c)));
    else if constexpr (x < NB + MB) read16<(x - NB) * 4096>(a[h][x - NB][c], (fa + so) ^ uint32_t(32 * (2 * h + c)));
  };
  auto rd_wait = [&](auto hh) __attribute__((always_inline)) {
    constexpr int h = decltype(hh)::value;
    __builtin_amdgcn_s_waitcnt(0xc07f);
#pragma unroll
    for (int c = 0; c < 2; ++c) {
#pragma unroll
      for (int i = 0; i < MB; ++i) asm volatile("" : "+v"(a[h][i][c]));
#pragma unroll
      for (int j = 0; j < NB; ++j) asm volatile("" : "+v"(b[h][j][c]));
    }
    __builtin_amdgcn_sched_barrier(0);
  };
  auto rd_all = [&](auto hh) __attribute__((always_inline)) {
    auto r4 = [&](auto x) __attribute__((always_inline)) {
      constexpr int x0 = decltype(x)::value;
      rd(hh, Int<x0>{}); rd(hh, Int<x0 + 1>{}); rd(hh, Int<x0 + 2>{}); rd(hh, Int<x0 + 3>{});
    };
    static_assert(2 * (MB + NB) <= 12, "reads of a set");
    r4(Int<0>{}); r4(Int<4>{}); r4(Int<8>{});
    rd_wait(hh);
  };
  const uint8_t *ws[2] = {nullptr, nullptr};
  const uint32_t fs = lds0 + S * WB + 4 * (wm * (BM / 2) + r32);
  auto rd_scales = [&]() __attribute__((always_inline)) {
    auto row = [&](auto ii) __attribute__((always_inline)) {
      constexpr int i = decltype(ii)::value;
      if constexpr (i < MB) read4<128 * i>(sn[i], fs + ring * G::RB);
    };
    row(Int<0>{}); row(Int<1>{}); row(Int<2>{}); row(Int<3>{});
  };
  auto take_scales = [&](int w) __attribute__((always_inline)) {  // behind a wait
    const int shift = 8 * (w & 3);
#pragma unroll
    for (int i = 0; i < MB; ++i) {
      asm volatile("" : "+v"(sn[i]));
      sa[i] = sn[i] >> shift;
    }
#pragma unroll
    for (int j = 0; j < NB; ++j) sb[j] = scales_at(ws[G::GATED ? j : 0], w >> 2) >> shift;
  };
  // the MFMAs of set h in MB NB groups of one
  auto half = [&](auto hh, auto ldd) __attribute__((always_inline)) {
    constexpr int h = decltype(hh)::value, GR = MB * NB;
    constexpr int RPB = (2 * (MB + NB) + GR - 2) / (GR - 1);
    auto group = [&](auto ii) __attribute__((always_inline)) {
      constexpr int i = decltype(ii)::value;
      if constexpr (i < GR) {
        constexpr int bi = i / NB, bj = i % NB;
        acc[bi][bj] = __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(cat8(b[h][bj][0], b[h][bj][1]), cat8(a[h][bi][0], a[h][bi][1]),
                                                                      acc[bi][bj], 0, 0, 0, int(sb[bj]), 0, int(sa[bi]));
        __builtin_amdgcn_sched_barrier(0);
        if constexpr (i < GR - 1 || GR == 1) {
          static_assert(RPB <= 6, "reads per group");
          rd(Int<1 - h>{}, Int<i * RPB>{});
          if constexpr (RPB > 1) rd(Int<1 - h>{}, Int<i * RPB + 1>{});
          if constexpr (RPB > 2) rd(Int<1 - h>{}, Int<i * RPB + 2>{});
          if constexpr (RPB > 3) rd(Int<1 - h>{}, Int<i * RPB + 3>{});
          if constexpr (RPB > 4) rd(Int<1 - h>{}, Int<i * RPB + 4>{});
          if constexpr (RPB > 5) rd(Int<1 - h>{}, Int<i * RPB + 5>{});
        }
        if constexpr (decltype(ldd)::value != 0) {
          if constexpr (i == 0) loads.a();
          if constexpr (i == GR / 2) loads.b();
        }
        __builtin_amdgcn_sched_barrier(0);
      }
    };
    group(Int<0>{}); group(Int<1>{}); group(Int<2>{}); group(Int<3>{});
    group(Int<4>{}); group(Int<5>{}); group(Int<6>{}); group(Int<7>{});
  };

  loads.start();
  for (int u = pid;; u += P) {
    const Item it = item_at(q, u);
    if (!it.valid) break;
    const Place z = place_of<G>(p, q, it.t);
    const int w0 = int((long long)nk * it.pc / it.n), w1 = int((long long)nk * (it.pc + 1) / it.n);
#pragma unroll
    for (int j = 0; j < 2; ++j) {
      const uint8_t *s = z.stream ? (j ? p.w_scale[1][1] : p.w_scale[1][0]) : (j ? p.w_scale[0][1] : p.w_scale[0][0]);
      ws[j] = s + size_t((G::GATED ? z.n0 : min(z.n0 + wn * (BN / 4), p.N - 1)) / 128) * loads.lds_scale;
    }
    if (it.n == 1) bias_to_lds<BN / 4, G::GATED ? 2 : 1>(p, z, z.n0 + wn * (G::COLS / 4), lds + G::AREAS + wid * 256, true);
#pragma unroll
    for (int i = 0; i < MB; ++i)
#pragma unroll
      for (int j = 0; j < NB; ++j) acc[i][j] = f32x16(0.f);
    rd_scales();
    rd_all(Int<0>{});
    take_scales(w0);
    auto window = [&](auto first, int w) __attribute__((always_inline)) {
      loads.step();  // its branch lies here because MFMAs before a branch are moved behind it
      half(Int<0>{}, Int<0>{});
      rd_wait(Int<1>{});
      loads.template next<decltype(first)::value != 0>();
      so = so == (S - 1) * WB ? 0 : so + WB;
      ring = (ring + 1) & (G::RING - 1);
      rd_scales();
      half(Int<1>{}, Int<1>{});
      rd_wait(Int<0>{});
      take_scales(min(w + 1, nk - 1));
    };
    int w = w0;
#pragma unroll
    for (int k = 0; k < S - 1; ++k)
      if (w < w1) {
        window(Int<1>{}, w);
        ++w;
      }
#pragma unroll 1
    for (; w < w1; ++w) window(Int<0>{}, w);
    wait_vm<0>();  // the next tile's first windows, and the biases
    const int lane = opaque(threadIdx.x & 63);
    if (it.n > 1) {
#pragma unroll
      for (int i = 0; i < MB; ++i)
#pragma unroll
        for (int j = 0; j < NB; ++j) store_part8(part_at8<G>(p.part, it.slot, wid, i, j, lane), acc[i][j]);
      continue;
    }
    Bias8<G> bias;
    bias.take(p, z, lds0 + G::AREAS + wid * 256, lane >> 5);
#pragma unroll
    for (int i = 0; i < MB; ++i) {
      finish8<G>(p, z, bias, wid, i, lane, acc[i]);
      asm volatile("" ::: "memory");
    }
  }
  wait_vm<0>();
}

// Where the instruction's 13 bits are too few -- codes out, since h next to the border between two codes gets the other one
// some ten times as often as with float32 sums, and float32 out -- the products are of bf16, which holds a code times its
// scale exactly, at half the rate.  x comes as such bf16 rows (k_widen_rows); W's codes are widened behind LDS, 16 of a row by
// a lane, which takes about as long as the MFMAs they feed (16 cycles for two values).  Tiles of 128 x 256, windows of 64 values;
// W is loaded for two windows at once, whole lines.  An MFMA of half h of a window multiplies values 16 g + 8 h .. + 7 of
// lane group g.  4096 cubed 132 us, 1.04 PFLOP/s; a window takes 0.7 us alone, 0.9 on all CUs, of which its MFMAs and
// conversions are 0.58.  4708 x 1536 -> 4096 with a gate into codes 129 us, 7 of them k_widen_rows: 4.6 turns of tiles in 5, each
// 24 windows and 8 us of activations, maxima, codes.  Of a float32 call the activations are as exact as finish_out's, so that
// its codes are of the values that it leaves without out_scale: 10 us more there.
template <bool GATED_, bool EXACT_>
struct GeoW {
  static constexpr int BM = 128, BN = 256, KIND = PRODUCT_OUT;
  static constexpr bool GATED = GATED_;
  static constexpr bool EXACT = EXACT_;  // the gate of float32 calls
  static constexpr int MB = 4, NB = 4;  // blocks of 16 x 16 of a wave, 2 x 4 waves
  static constexpr int COLS = GATED ? BN / 2 : BN;
  static constexpr int XB = BM * 128, XSLOTS = 4, WB = BN * 128;  // a window of x, two of W in two slots
  static constexpr int W0 = XSLOTS * XB, TOPS = W0 + 2 * WB;      // codes out: a row's largest values by wave
  static constexpr int AREAS = TOPS + BM * 16, LDS = AREAS + 2048;  // 256 bytes a wave for biases
  static_assert(LDS <= 160 * 1024, "LDS");
};

// Four of a wave's biases from value i on, of either type.
HILO_DEV f32x4 take_bias4(uint32_t area, int i, bool some, bool bf16) {
  u32x4 r;
  u32x2 h;
  if (bf16) {
    asm volatile("ds_read_b64 %0, %1\n\ts_waitcnt lgkmcnt(0)" : "=v"(h) : "v"(area + 2 * i) : "memory");
    r = u32x4{h[0] << 16, h[0] & 0xffff0000u, h[1] << 16, h[1] & 0xffff0000u};
  } else {
    asm volatile("ds_read_b128 %0, %1\n\ts_waitcnt lgkmcnt(0)" : "=v"(r) : "v"(area + 4 * i) : "memory");
  }
  return some ? __builtin_bit_cast(f32x4, r) : f32x4(0.f);
}

template <typename G>
HILO_DEV void run_wide(const ProductProblem &p, const Plan &q, int pid, uint8_t *lds) {
  constexpr int BM = G::BM, BN = G::BN, MB = G::MB, NB = G::NB;
  const int lane = threadIdx.x & 63;
  const int wid = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int lr = lane & 15, lg = lane >> 4, wm = wid >> 2, wn = wid & 3;
  const uint32_t lda = 2u * p.K, ldb = p.K;
  const int nv = (p.K + 127) / 128, stride = scale_stride(p.K);  // pairs of windows

  // ---- loads of a pair of windows: 16 rows of x a wave, two instructions for each window, and 32 of W, four; with a gate a
  // wave's rows of W are of one part.  The chunk of instruction i (8 rows) is that of instruction 0, or its bit 2 the
  // other way round
  const uint32_t oa = uint32_t(wid * 16 + (lane >> 3)) * lda + 16u * ((lane & 7) ^ (lane >> 4));
  const uint32_t ob = uint32_t((G::GATED ? wid >> 1 : wid) * 32 + (lane >> 3)) * ldb + 16u * ((lane & 7) ^ (lane >> 4));
  int lu = pid, lv = nv, lx = 0, lslot = 0;
  const char *la = nullptr, *lb = nullptr;
  uint32_t ra = 0, rb = 0;
  bool more = true;
  auto ld_step = [&]() __attribute__((always_inline)) {  // before a pair of windows
    if (!more || lv < nv) return;
    const Item it = item_at(q, lu);
    if (!it.valid) {
      more = false;
      return;
    }
    lu += P;
    const Place z = place_of<G>(p, q, it.t);
    lv = 0;
    const int part = G::GATED ? wid & 1 : 0;
    const void *w = z.stream ? (part ? p.w[1][1] : p.w[1][0]) : (part ? p.w[0][1] : p.w[0][0]);
    la = reinterpret_cast<const char *>(p.x) + size_t(z.row0) * lda;
    lb = reinterpret_cast<const char *>(w) + size_t(z.n0) * ldb;
    ra = uint32_t(z.rows) * lda;
    rb = uint32_t(min(G::COLS, p.N - z.n0)) * ldb;
  };
  // chunks behind the end of k: offsets behind the buffer's
  auto ld_x = [&](int h) __attribute__((always_inline)) {  // window h of the pair
    const int k = 128 * lv + 64 * h, kv = p.K - k, lane = opaque(threadIdx.x & 63), c = (lane & 7) ^ (lane >> 4);
    const uint32_t bytes = more && kv > 0 ? ra - 2u * uint32_t(k) : 0u, o1 = oa + 8 * lda + (c & 4 ? -64 : 64);
    uint8_t *at = lds + lx * G::XB + wid * 2048;
    buffer_to_lds(la + size_t(k) * 2, bytes, 8 * c < kv ? oa : kBehind, at);
    buffer_to_lds(la + size_t(k) * 2, bytes, 8 * (c ^ 4) < kv ? o1 : kBehind, at + 1024);
    lx = (lx + 1) & (G::XSLOTS - 1);
  };
  auto ld_w = [&]() __attribute__((always_inline)) {
    const int kv = p.K - 128 * lv, lane = opaque(threadIdx.x & 63), c = (lane & 7) ^ (lane >> 4);
    const uint32_t bytes = more ? rb - 128u * uint32_t(lv) : 0u;
    const uint32_t o0 = 16 * c < kv ? ob : kBehind, o1 = 16 * (c ^ 4) < kv ? ob + (c & 4 ? -64 : 64) : kBehind;
    uint8_t *at = lds + G::W0 + lslot * G::WB + wid * 4096;
#pragma unroll
    for (int i = 0; i < 4; ++i) buffer_to_lds(lb + size_t(lv) * 128, bytes, (i & 1 ? o1 : o0) + uint32_t(8 * i) * ldb, at + i * 1024);
    lslot ^= 1;
  };

  // ---- fragments
  const uint32_t lds0 = (uint32_t)(uintptr_t)lds;
  uint32_t fa[2];
#pragma unroll
  for (int h = 0; h < 2; ++h) fa[h] = lds0 + (wm * (BM / 2) + lr) * 128 + ((2 * lg + h) ^ ((lr >> 1) & 7)) * 16;
  uint32_t fb[2];  // of either window of a pair
#pragma unroll
  for (int h = 0; h < 2; ++h) fb[h] = lds0 + G::W0 + (wn * (BN / 4) + lr) * 128 + ((4 * h + lg) ^ ((lr >> 1) & 7)) * 16;
  f32x4 acc[MB][NB];
  // of two windows: x by halves; W's codes, read a window before they are widened, and that one before they are multiplied
  u32x4 a[2][2][MB], b[2][NB];
  bf16x8 wb[2][2][NB];
  uint32_t sx = G::XB, sw = G::WB;  // byte offsets of the next window of x, and of the next pair of W
  const uint8_t *ws[2] = {nullptr, nullptr};
  uint32_t s0, s1;  // of the window that is widened
  auto scales = [&](int v) __attribute__((always_inline)) {  // of pair v: a float32 number's exponent
    const int shift = 8 * (v & 3);
    s0 = (scales_at(ws[0], v >> 2) >> shift & 255u) << 23;
    s1 = (scales_at(ws[G::GATED ? 1 : 0], v >> 2) >> shift & 255u) << 23;
  };
  auto rd_a = [&](auto set, auto gg) __attribute__((always_inline)) {
    constexpr int s = decltype(set)::value, h = decltype(gg)::value / 4, i = decltype(gg)::value % 4;
    read16<i * 2048>(a[s][h][i], fa[h] + sx);
  };
  auto rd_b = [&](auto set, auto jj) __attribute__((always_inline)) {  // window `set` of the pair
    constexpr int s = decltype(set)::value, j = decltype(jj)::value;
    read16<j * 2048>(b[s][j], fb[s] + sw);
  };
  auto wait = [&](auto set) __attribute__((always_inline)) {  // for a of a set, b of the other
    constexpr int s = decltype(set)::value;
    __builtin_amdgcn_sched_barrier(0);
    __builtin_amdgcn_s_waitcnt(0xc07f);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      asm volatile("" : "+v"(a[s][0][i]));
      asm volatile("" : "+v"(a[s][1][i]));
      asm volatile("" : "+v"(b[1 - s][i]));
    }
    __builtin_amdgcn_sched_barrier(0);
  };
  // Window w = 2 v + s, while W's codes of w + 1 are widened, x of w + 1 and W of w + 2 are read.  One barrier, at which every
  // wave has read x of w and W of w + 1, so that x of w + 4 goes to the slot of w, and for even w W's pair v + 2 to that of
  // v.  What is read behind it has landed: of the loads issued since, 2 + 2 of x (even w), or 2 of x, 4 of W and 2 of x
  auto window = [&](auto set, auto first, int v) __attribute__((always_inline)) {  // window s of pair v
    constexpr int s = decltype(set)::value;
    if constexpr (s == 0) ld_step();
    // in a tile's first pair it has landed before the stores of the tile before, which would be waited for as well
    if constexpr (decltype(first)::value == 0) wait_vm<s == 0 ? 4 : 8>();
    asm volatile("s_barrier" ::: "memory");
    __builtin_amdgcn_sched_barrier(0);
    auto group = [&](auto gg) __attribute__((always_inline)) {
      constexpr int g = decltype(gg)::value, h = g / 4, i = g % 4;
#pragma unroll
      for (int j = 0; j < NB; ++j)
        acc[i][j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(wb[s][h][j], __builtin_bit_cast(bf16x8, a[s][h][i]), acc[i][j], 0, 0, 0);
      wb[1 - s][h][i] = wide_codes(b[1 - s][i][2 * h], b[1 - s][i][2 * h + 1], i < NB / 2 ? s0 : s1);
      if constexpr (g < 4) {
        rd_b(Int<s>{}, Int<g>{});
        rd_a(Int<1 - s>{}, Int<2 * g>{});
        rd_a(Int<1 - s>{}, Int<2 * g + 1>{});
      }
      if constexpr (g == 4 && s == 0) ld_w();
      if constexpr (g == 5) ld_x(s);
      if constexpr (g == 5 && s == 1) ++lv;
      __builtin_amdgcn_sched_barrier(0);
    };
    group(Int<0>{}); group(Int<1>{}); group(Int<2>{}); group(Int<3>{});
    group(Int<4>{}); group(Int<5>{}); group(Int<6>{}); group(Int<7>{});
    if constexpr (s == 0) scales(min(v + 1, nv - 1));
    wait(Int<1 - s>{});
    sx = sx == 3 * G::XB ? 0 : sx + G::XB;
    if constexpr (s == 1) sw ^= G::WB;
  };
#pragma unroll 1
  for (int v = 0; v < 2; ++v) {
    ld_step();
    ld_w();
    ld_x(0);
    ld_x(1);
    ++lv;
  }
  wait_vm<0>();
  asm volatile("s_barrier" ::: "memory");
  for (int u = pid;; u += P) {
    const Item it = item_at(q, u);
    if (!it.valid) break;
    const Place z = place_of<G>(p, q, it.t);
#pragma unroll
    for (int j = 0; j < 2; ++j) {
      const uint8_t *s = z.stream ? (j ? p.w_scale[1][1] : p.w_scale[1][0]) : (j ? p.w_scale[0][1] : p.w_scale[0][0]);
      ws[j] = s + size_t((G::GATED ? z.n0 : min(z.n0 + wn * (BN / 4), p.N - 1)) / 128) * stride;
    }
    if (G::GATED && p.out_scale) bias_to_lds<BN / 4, 2>(p, z, z.n0 + wn * (G::COLS / 4), lds + G::AREAS + wid * 256, p.bf16);
#pragma unroll
    for (int i = 0; i < MB; ++i)
#pragma unroll
      for (int j = 0; j < NB; ++j) acc[i][j] = f32x4{0.f, 0.f, 0.f, 0.f};
    // x of the first window, and W of the first two: all have landed.  (The last window of the item before read them too, but
    // widened W with its own scales)
    sx = sx == 0 ? 3 * G::XB : sx - G::XB;
    sw ^= G::WB;
    rd_b(Int<0>{}, Int<0>{}); rd_b(Int<0>{}, Int<1>{}); rd_b(Int<0>{}, Int<2>{}); rd_b(Int<0>{}, Int<3>{});
    rd_b(Int<1>{}, Int<0>{}); rd_b(Int<1>{}, Int<1>{}); rd_b(Int<1>{}, Int<2>{}); rd_b(Int<1>{}, Int<3>{});
    rd_a(Int<0>{}, Int<0>{}); rd_a(Int<0>{}, Int<1>{}); rd_a(Int<0>{}, Int<2>{}); rd_a(Int<0>{}, Int<3>{});
    rd_a(Int<0>{}, Int<4>{}); rd_a(Int<0>{}, Int<5>{}); rd_a(Int<0>{}, Int<6>{}); rd_a(Int<0>{}, Int<7>{});
    sx = sx == 3 * G::XB ? 0 : sx + G::XB;
    sw ^= G::WB;
    scales(0);
    wait(Int<0>{});
#pragma unroll
    for (int j = 0; j < NB; ++j) {
      asm volatile("" : "+v"(b[0][j]));
#pragma unroll
      for (int h = 0; h < 2; ++h) wb[0][h][j] = wide_codes(b[0][j][2 * h], b[0][j][2 * h + 1], j < NB / 2 ? s0 : s1);
    }
    window(Int<0>{}, Int<1>{}, 0);
    window(Int<1>{}, Int<1>{}, 0);
#pragma unroll 1
    for (int v = 1; v < nv; ++v) {
      window(Int<0>{}, Int<0>{}, v);
      window(Int<1>{}, Int<0>{}, v);
    }
    wait_vm<0>();  // the next tile's first windows, and the biases
    const int lane = opaque(threadIdx.x & 63), lr = lane & 15, lg = lane >> 4;
    // lane (lr, lg): rows 16 i + lr, columns 16 j + 4 lg .. + 3 of block j; with a gate blocks 0 and 1 are the gate's
    const int n = z.n0 + wn * (G::COLS / 4) + 4 * lg;
    if (!p.out_scale) {
#pragma unroll
      for (int i = 0; i < MB; ++i) {
        const int rl = wm * (BM / 2) + 16 * i + lr;
        const size_t row = size_t(z.row0) + rl;
#pragma unroll
        for (int j = 0; j < (G::GATED ? 2 : NB); ++j)
          if (rl < z.rows && n + 16 * j < p.N) finish_out<G::GATED>(p, z.stream, row, n + 16 * j, acc[i][j], acc[i][G::GATED ? 2 + j : j]);
        asm volatile("" ::: "memory");
      }
      continue;
    }
    if constexpr (G::GATED) {
      // the tile's 128 columns have one scale a row, from the largest of four waves' 32 columns
      const uint32_t tops = lds0 + G::TOPS;
      f32x4 bias[NB];
#pragma unroll
      for (int j = 0; j < NB; ++j) {
        const void *v = z.stream ? (j / 2 ? p.bias[1][1] : p.bias[1][0]) : (j / 2 ? p.bias[0][1] : p.bias[0][0]);
        bias[j] = take_bias4(lds0 + G::AREAS + wid * 256, 32 * (j / 2) + 16 * (j & 1) + 4 * lg, v != nullptr, p.bf16);
      }
#pragma unroll
      for (int i = 0; i < MB; ++i) {
        uint32_t top = 0;
#pragma unroll
        for (int j = 0; j < 2; ++j)
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            const float h = gate_act<G::EXACT>(acc[i][j][e] + bias[j][e], p.silu) * (acc[i][2 + j][e] + bias[2 + j][e]);
            acc[i][j][e] = h;
            top = n + 16 * j < p.N ? max(top, abs_bits(h)) : top;
          }
        uint32_t other = top;
        swap16(top, other);
        top = max(top, other);
        other = top;
        swap32(top, other);
        top = max(top, other);
        if (lg == 0) asm volatile("ds_write_b32 %0, %1" ::"v"(tops + 16 * (wm * (BM / 2) + 16 * i + lr) + 4 * wn), "v"(top) : "memory");
      }
      asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory");
#pragma unroll
      for (int i = 0; i < MB; ++i) {
        const int rl = wm * (BM / 2) + 16 * i + lr;
        u32x4 t;
        asm volatile("ds_read_b128 %0, %1\n\ts_waitcnt lgkmcnt(0)" : "=v"(t) : "v"(tops + 16 * rl) : "memory");
        const uint32_t top = max(max(t[0], t[1]), max(t[2], t[3]));
        const bool finite = top < 0x7f800000u;
        const int k = finite ? pow2_exponent(__uint_as_float(top)) : 0;
        const float inv = pow2_inverse(k);
        uint32_t c[2];
#pragma unroll
        for (int j = 0; j < 2; ++j) {
          c[j] = fp8x4(acc[i][j][0] * inv, acc[i][j][1] * inv, acc[i][j][2] * inv, acc[i][j][3] * inv);
          c[j] = finite ? c[j] : 0x7f7f7f7fu;
        }
        swap16(c[0], c[1]);  // 8 columns of a block a lane
        const int col = z.n0 + wn * 32 + 16 * (lg & 1) + 8 * (lg >> 1);
        if (rl < z.rows) {
          const size_t row = size_t(z.row0) + rl;
          if (col < p.N) *reinterpret_cast<uint2 *>(reinterpret_cast<uint8_t *>(p.out) + row * p.N + col) = make_uint2(c[0], c[1]);
          if (wn == 0 && lg == 0) {
            uint8_t *s = p.out_scale + row * scale_stride(p.N);
            const int at = z.n0 / 128, end = z.n0 + 128 >= p.N ? scale_stride(p.N) : at + 1;
            s[at] = finite ? uint8_t(127 + k) : 255;
            for (int x = at + 1; x < end; ++x) s[x] = 0;
          }
        }
      }
    }
  }
  wait_vm<0>();
}

template <typename G>
HILO_DEV void fix8(const ProductProblem &p, const Plan &q) {
  if (q.s == 1) return;
  const int lane = threadIdx.x & 63;
  const int items = q.tail * 8 * G::MB;
  for (int x = blockIdx.x * 8 + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6); x < items; x += gridDim.x * 8) {
    const int v = x / (8 * G::MB), rem = x - v * 8 * G::MB, wid = rem / G::MB, i = rem - wid * G::MB;
    const Place z = place_of<G>(p, q, q.full + v);
    Bias8<G> bias;
    bias.load(p, z, wid & 3, lane >> 5);
    f32x16 acc[G::NB];
#pragma unroll
    for (int j = 0; j < G::NB; ++j) acc[j] = f32x16(0.f);
#pragma unroll 1
    for (int pc = 0; pc < q.s; pc += 2) {  // two pieces' loads at once
      f32x4 w[2][G::NB][4];
#pragma unroll
      for (int k = 0; k < 2; ++k)
#pragma unroll
        for (int j = 0; j < G::NB; ++j) {
          const float *from = part_at8<G>(p.part, min(pc + k, q.s - 1) * q.tail + v, wid, i, j, lane);
#pragma unroll
          for (int e = 0; e < 4; ++e) w[k][j][e] = *reinterpret_cast<const f32x4 *>(from + 256 * e);
        }
      __builtin_amdgcn_sched_barrier(0);
#pragma unroll
      for (int j = 0; j < G::NB; ++j) {
        add_part8(acc[j], w[0][j]);
        if (pc + 1 < q.s) add_part8(acc[j], w[1][j]);
      }
    }
    finish8<G>(p, z, bias, wid, i, lane, acc);
  }
}

// 256 x 256, 128 x 256 (us): 2766 x 3072 -> 9216 96 and 108; 1000 x 4096 -> 4096 48 and 40.
constexpr Cost kCost8[2] = {{150, 600, 600, 80, 7}, {80, 400, 600, 40, 2}};

// 256 x 256 tiles or 128 x 256.
template <bool GATED, typename F>
HILO_BOTH bool choose8(const ProductProblem &p, F &&row_tiles, Plan &q) {
  const int nk = (p.K + 127) / 128;
  const Plan a = make_plan<Geo8<256, 256, GATED>>(p, row_tiles(256), nk, kCost8[0]);
  const Plan b = make_plan<Geo8<128, 256, GATED>>(p, row_tiles(128), nk, kCost8[1]);
  const bool large = plan_cost(a.T, nk, kCost8[0], p.splits) <= plan_cost(b.T, nk, kCost8[1], p.splits);
  q = large ? a : b;
  return large;
}
template <bool GATED>
HILO_DEV bool choose8(const ProductProblem &p, Plan &q) {
  return choose8<GATED>(p, [&](int bm) { return count_row_tiles(p, bm); }, q);
}

template <bool GATED>
__global__ __launch_bounds__(512, 2) void k_product_fp8(ProductProblem p) {
  using G0 = Geo8<256, 256, GATED>;
  using G1 = Geo8<128, 256, GATED>;
  __shared__ __attribute__((aligned(1024))) uint8_t lds[G0::LDS > G1::LDS ? G0::LDS : G1::LDS];
  const int pid = xcd_remap(blockIdx.x, P);
  Plan q;
  if (choose8<GATED>(p, q)) run8<G0>(p, q, pid, lds);
  else run8<G1>(p, q, pid, lds);
}

template <bool GATED>
__global__ __launch_bounds__(512) void k_product_fp8_fix(ProductProblem p) {
  Plan q;
  if (choose8<GATED>(p, q)) fix8<Geo8<256, 256, GATED>>(p, q);
  else fix8<Geo8<128, 256, GATED>>(p, q);
}

template <bool GATED, bool EXACT>
__global__ __launch_bounds__(512, 2) void k_product_fp8_wide(ProductProblem p) {
  using G = GeoW<GATED, EXACT>;
  __shared__ __attribute__((aligned(1024))) uint8_t lds[G::LDS];
  const Plan q = make_plan<G>(p, count_row_tiles(p, G::BM), 1, kCost8[1]);
  run_wide<G>(p, q, xcd_remap(blockIdx.x, P), lds);
}

}  // namespace pt

template <bool GATED>
static hipError_t run_tiles8(ProductProblem p, hipStream_t st) {
  pt::Plan q;
  p.splits = pt::kSearch;
  pt::choose8<GATED>(p, [&](int bm) { return (p.rows + bm - 1) / bm; }, q);
  p.splits = q.s > 1 ? q.s : 0;
  hipLaunchKernelGGL((pt::k_product_fp8<GATED>), dim3(pt::P), dim3(512), 0, st, p);
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess || !p.splits) return e;
  hipLaunchKernelGGL((pt::k_product_fp8_fix<GATED>), dim3(pt::P), dim3(512), 0, st, p);
  return hipGetLastError();
}

hipError_t launch_product_fp8_wide(ProductProblem p, hipStream_t st) {
  p.splits = 0;  // whole tiles
  if (p.parts == 1) hipLaunchKernelGGL((pt::k_product_fp8_wide<false, false>), dim3(pt::P), dim3(512), 0, st, p);
  else if (p.bf16) hipLaunchKernelGGL((pt::k_product_fp8_wide<true, false>), dim3(pt::P), dim3(512), 0, st, p);
  else hipLaunchKernelGGL((pt::k_product_fp8_wide<true, true>), dim3(pt::P), dim3(512), 0, st, p);
  return hipGetLastError();
}

hipError_t launch_product_fp8_tiles(const ProductProblem &p, hipStream_t st) {
  return p.parts == 2 ? run_tiles8<true>(p, st) : run_tiles8<false>(p, st);
}

}  // namespace hilo
