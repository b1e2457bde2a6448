// The schedule of the products on large tiles, bf16 and FP8: whole tiles in turns of a tile a workgroup, the last turn cut along
// k; where a tile lies; loads to LDS.
#pragma once

#include "product.h"

namespace hilo {

typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));

namespace pt {

constexpr int P = kGemmWorkgroups;

// Tiles in groups of 8 row tiles by all column tiles, row tile fastest: the 32 workgroups of an XCD then share 8 + 4 slices
// of the operands.
HILO_DEV void tile_at(int R, int TN, int t, int &r, int &c) {
  const int grp = t / (8 * TN), in = t - grp * 8 * TN, gm = min(8, R - grp * 8);
  c = in / gm;
  r = grp * 8 + in - c * gm;
}

// Tiles run whole, P at a time; what is left over for a last turn is cut along k into s pieces each, no more than there are
// workgroups for, where that is quicker than a whole turn.  Pieces leave float32 tiles that the fixup adds up in their order,
// a launch of its own.  Only the device knows the rows: the host launches the fixup, and says how many pieces there are at
// most (splits), as all the rows of the buffers would have it.
struct Plan {
  int R, TN, T, full, tail, s;
};
struct Item {
  int t, pc, n, slot;  // tile, piece of n, slot of its partial sums (n > 1)
  bool valid;
};
HILO_DEV Item item_at(const Plan &q, int u) {
  if (u < q.full) return Item{u, 0, 1, 0, true};
  const int v = u - q.full;
  if (v >= q.tail * q.s) return Item{0, 0, 1, 0, false};
  const int pc = v / q.tail;
  return Item{q.full + v - pc * q.tail, pc, q.s, v, true};
}

// In units of 10 ns: a window and a tile's rest; beside their windows pieces of the last turn cost a launch, and each level
// of pieces and each piece its share (a partial tile written and read).  Fitted to calls that were made with each tile
// and each number of pieces; what they choose is within a tenth of the best on most of them.  Measured (us, one tile size):
//   bf16 128 x 128, 100 x 4096 -> 256    1 piece 33.9, 2 25.0, 4 18.3, 8 15.9, 16 16.9, 32 18.2
//   bf16 256 x 256, 2000 x 4096 -> 1536  1 87, 2 68, 4 49, 5 49;  of 256 x 128 60 whole, of 128 x 128 39 whole: taken
//   FP8 128 x 256, 500 x 8192 -> 1024    1 59, 2 45, 4 35, 8 32.5, 16 35
struct Cost {
  int window, tile, fix, level, piece;
  __host__ __device__ __forceinline__ int pieces(int s, int tail) const { return fix + s * (level + tail * piece); }
  // of nk windows; beyond 2^20 of them, 2^20's
  __host__ __device__ __forceinline__ int windows(int nk) const { return (nk < 1 << 20 ? nk : 1 << 20) * window; }
};
#define HILO_BOTH __host__ __device__ __forceinline__
// Pieces of a tile of the last turn: none (splits 0), at most splits, or on the host (kSearch) as many as are quickest.
constexpr int kSearch = -1;
HILO_BOTH int plan_tail(int tail, int nk, Cost c, int splits) {
  if (tail == 0 || splits == 0) return 1;
  const int most = P / tail < nk / 4 ? P / tail : nk / 4, all = c.windows(nk);
  int s = most < splits ? most : splits;
  if (splits == kSearch)
    for (s = 1; s < most && all > s * (s + 1) * (c.level + tail * c.piece);) ++s;  // one more saves more than it costs
  return s > 1 && all - int(unsigned(all) / unsigned(s)) > c.pieces(s, tail) ? s : 1;
}
HILO_BOTH long long plan_cost(int T, int nk, Cost c, int splits) {
  const int tail = T % P, s = plan_tail(tail, nk, c, splits), all = c.windows(nk);
  return (long long)(T / P) * (all + c.tile) + (tail ? int(unsigned(all) / unsigned(s)) + c.tile + (s > 1 ? c.pieces(s, tail) : 0) : 0);
}
template <typename G>
HILO_BOTH Plan make_plan(const ProductProblem &p, int R, int nk, Cost c) {
  Plan q;
  q.R = R;
  q.TN = ((G::KIND == PRODUCT_OUT ? p.N : p.K) + G::COLS - 1) / G::COLS;
  q.T = q.R * q.TN;
  q.tail = q.T % P;
  q.full = q.T - q.tail;
  q.s = plan_tail(q.tail, nk, c, p.splits);
  return q;
}

// Where a tile lies: rows row0 .. + rows of the output (DW: of output o), columns from n0, stream, and for the backward
// products the part.
struct Place {
  int row0, rows, n0, stream, part, o;
};
template <typename G>
HILO_DEV Place place_of(const ProductProblem &p, const Plan &q, int t) {
  int r, c;
  Place z;
  if constexpr (G::KIND == PRODUCT_DW) {
    const int per = q.R / p.outs * q.TN;  // R: the row tiles of all outputs
    z.o = t / per;
    tile_at(q.R / p.outs, q.TN, t - z.o * per, r, c);
    z.stream = p.out_stream[z.o];
    z.part = p.out_part[z.o];
    z.row0 = r * G::BM;
    z.rows = min(G::BM, p.N - z.row0);
  } else {
    tile_at(q.R, q.TN, t, r, c);
    z.o = z.part = 0;
    const RowTile rt = find_row_tile(p, G::BM, r);
    z.row0 = rt.row0;
    z.rows = rt.n;
    z.stream = rt.stream;
  }
  z.n0 = c * G::COLS;
  return Place{uni(z.row0), uni(z.rows), uni(z.n0), uni(z.stream), uni(z.part), uni(z.o)};
}

// One 16-byte load per lane straight to LDS, zeros where the offset lies behind the buffer's end: lane l's bytes land at
// 16 l of the wave's 1 KiB.
HILO_DEV void buffer_to_lds(const char *base, uint32_t bytes, uint32_t offset, void *lds_wave_base) {
  __builtin_amdgcn_raw_ptr_buffer_load_lds(
      __builtin_amdgcn_make_buffer_rsrc(const_cast<char *>(base), 0, int(bytes), 0x00020000),
      (__attribute__((address_space(3))) void *)lds_wave_base, 16, int(offset), 0, 0, 0);
}

template <int N>
HILO_DEV void wait_vm() { asm volatile("s_waitcnt vmcnt(%0)" ::"n"(N) : "memory"); }
template <int V>
struct Int {
  static constexpr int value = V;
};
template <int OFF>
HILO_DEV void read16(u32x4 &d, uint32_t addr) {
  asm volatile("ds_read_b128 %0, %1 offset:%2" : "=v"(d) : "v"(addr), "n"(OFF) : "memory");
}

// Exchanges rows of 16 lanes: x gets y's row 0 in its row 1, its row 2 in its row 3; y x's rows 1 and 3 in its rows 0 and 2.
HILO_DEV void swap16(uint32_t &x, uint32_t &y) {
  const auto r = __builtin_amdgcn_permlane16_swap(x, y, false, false);
  x = r[0];
  y = r[1];
}

// The same of halves of 32 lanes.
HILO_DEV void swap32(uint32_t &x, uint32_t &y) {
  const auto r = __builtin_amdgcn_permlane32_swap(x, y, false, false);
  x = r[0];
  y = r[1];
}

// Biases of a wave's WC columns (PARTS: half of either part) for the end of its tile: by a direct load to LDS when the tile begins, as
// they lie in memory, so that nothing is waited for then.  n: the wave's first column of its part; area: 256 bytes.
template <int WC, int PARTS>
HILO_DEV void bias_to_lds(const ProductProblem &p, const Place &z, int n, void *area, bool bf16) {
  const char *b[2];
#pragma unroll
  for (int q = 0; q < 2; ++q) b[q] = reinterpret_cast<const char *>(z.stream ? (q ? p.bias[1][1] : p.bias[1][0]) : (q ? p.bias[0][1] : p.bias[0][0]));
  if (!b[0] && (PARTS == 1 || !b[1])) return;
  const int each = bf16 ? 2 : 1, at = opaque(threadIdx.x & 63) * each % WC;  // values of a lane's 4 bytes
  const int part = at / (WC / PARTS), col = at % (WC / PARTS);
  const char *base = PARTS == 1 || (part == 0 ? b[0] != nullptr : b[1] == nullptr) ? b[0] : b[1];  // a part without: the other's
  __builtin_amdgcn_global_load_lds(base + size_t(min(n + col, p.N - each)) * (4 / each), (__attribute__((address_space(3))) void *)area, 4, 0, 0);
}
template <int OFF>
HILO_DEV void read8(u32x2 &d, uint32_t addr) {
  asm volatile("ds_read_b64 %0, %1 offset:%2" : "=v"(d) : "v"(addr), "n"(OFF) : "memory");
}

}  // namespace pt
}  // namespace hilo
