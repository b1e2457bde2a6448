// The library's own plans of the products on large tiles, from the kernels' sources: host code alone, for a test that compares
// them with product_schedule.py's.  A line of stdin is a call: kind (0 to 3 as there, 4: dx and the weights' gradients), rows of
// the buffers, in, out, parts, streams, then what the device counts: windows of the sum, row tiles of 256 rows and of 128; for
// kind 4 samples, text rows and 0.  Printed: index of the tile size, tiles, pieces; of kind 4 whether it is one launch.
#include <cstdio>

#include "product_bf16.hip"
#include "product_fp8.hip"

using namespace hilo;

template <int KIND, bool GATED>
static void plan(ProductProblem p, int nk, int r256, int r128) {
  pt::Plan q;
  plan_rows<KIND, GATED>(p, q);
  p.splits = q.s > 1 ? q.s : 0;
  const int i = pt::choose<KIND, GATED>(
      p, nk, [&](int bm) { return KIND == PRODUCT_DW ? p.outs * ((p.N + bm - 1) / bm) : bm == 256 ? r256 : r128; }, q);
  std::printf("%d %d %d\n", i, q.T, q.s);
}

template <bool GATED>
static void plan8(ProductProblem p, int r256, int r128) {
  pt::Plan q;
  p.splits = pt::kSearch;
  pt::choose8<GATED>(p, [&](int bm) { return (p.rows + bm - 1) / bm; }, q);
  p.splits = q.s > 1 ? q.s : 0;
  const bool large = pt::choose8<GATED>(p, [&](int bm) { return bm == 256 ? r256 : r128; }, q);
  std::printf("%d %d %d\n", large ? 0 : 1, q.T, q.s);
}

int main() {
  int kind, streams, a, b, c;
  ProductProblem p{};
  while (std::scanf("%d %d %d %d %d %d %d %d %d", &kind, &p.rows, &p.K, &p.N, &p.parts, &streams, &a, &b, &c) == 9) {
    p.merged = streams == 1;
    p.outs = 0;
    for (int k = 0; k < streams; ++k)
      for (int q = 0; q < p.parts; ++q) {
        p.out_stream[p.outs] = k;
        p.out_part[p.outs++] = q;
      }
    if (kind == 0) p.parts == 2 ? plan<PRODUCT_OUT, true>(p, a, b, c) : plan<PRODUCT_OUT, false>(p, a, b, c);
    if (kind == 1) plan<PRODUCT_DX, false>(p, a, b, c);
    if (kind == 2) plan<PRODUCT_DW, false>(p, a, b, c);
    if (kind == 3) p.parts == 2 ? plan8<true>(p, b, c) : plan8<false>(p, b, c);
    if (kind == 4) {
      p.B = a;
      p.L = b;
      std::printf("%d\n", one_launch(p, p));
    }
  }
}
