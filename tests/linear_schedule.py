"""The plans of the int8 products on the host (gemm.hip: choose_tile_i8 and the plans it shares with the projections), and
the shapes with which the GPU tests reach each kind."""
import schedule_model as M

# (sample lengths, text rows, K, N) and (tile, tiles, pieces per tile, data-parallel units, stream-K units, workgroups
# sharing those).  K is no multiple of 128 in most: the last step is part of one
SHAPES = [
    # 192 x 192: whole tiles in one wave; one tile in 128 pieces of a step; pieces with a stream-K tail; one piece, a tail
    (([300], 100, 528, 520), (192, 9, 1, 9, 0, 256)),
    (([128], 0, 16384, 100), (192, 1, 128, 0, 128, 128)),
    (([200, 90], 40, 8336, 1000), (192, 24, 11, 256, 8, 8)),
    (([5000], 0, 2064, 13312), (192, 1890, 1, 1792, 98, 139)),
    # 256 x 256: one wave of whole tiles; four; pieces
    (([4096], 0, 1040, 4096), (256, 256, 1, 256, 0, 256)),
    (([15000], 0, 2048, 3900), (256, 944, 1, 944, 0, 256)),
    (([2040], 0, 16400, 2040), (256, 64, 4, 256, 0, 0)),
]


def describe(lens, text, K, N):
    segs, nk = [(n - text, text) for n in lens], -(-K // 128)
    c192, c256 = (M.cost(False, M.row_tiles(segs, t) * -(-N // t), nk, *M.TILE_COSTS[t]) for t in (192, 256))
    tile = 256 if c256 < c192 else 192
    T = M.row_tiles(segs, tile) * -(-N // tile)
    s, U, dp, _, _, Pk = M.plan(T, M.WORKGROUPS, nk)
    return tile, T, s, dp, U - dp, Pk
