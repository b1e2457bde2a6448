"""The plans of the int8 products on the host (gemm.hip: choose_tile_i8 and the plans it shares with the projections), and
the shapes with which the GPU tests reach each kind."""
import schedule_model as M

WORKGROUPS = 256
# estimates of choose_tile_i8 in units of 10 ns: a K step, a tile's rest without and with GELU, K pieces in all, per tile
# (128 x 128 tiles are not cut)
COSTS = {192: (91, 560, 730, 2700, 20), 256: (148, 600, 870, 4500, 35), 128: (46, 390, 430, None, None)}
START = 250  # the first windows

# (sample lengths, text rows, K, N) and (tile, tiles, pieces per tile, data-parallel units, stream-K units, workgroups
# sharing those), or ("small", tiles, turns).  K is no multiple of 128 in most: the last step is part of one
SHAPES = [
    # 64 x 32: one turn; two (many samples of a row)
    (([300], 100, 1040, 520), ("small", 102, 1)),
    (([1] * 520, 0, 80, 32), ("small", 520, 2)),
    # 128 x 128: whole tiles in one wave, few and 7/8 of one with a K that would else be cut, and in two
    (([700], 0, 4112, 4092), (128, 192, 1, 192, 0, 256)),
    (([900], 100, 2064, 2040), (128, 128, 1, 128, 0, 256)),
    (([2048], 0, 65536, 2044), (128, 256, 1, 256, 0, 256)),
    (([1] * 300, 0, 80, 64), (128, 300, 1, 300, 0, 256)),
    # 192 x 192: whole tiles in one wave, and in two; one tile in 256 pieces; pieces with a stream-K tail, whole and cut
    (([2500], 30, 528, 2048), (192, 154, 1, 154, 0, 256)),
    (([2766], 512, 1552, 6144), (192, 480, 1, 480, 0, 256)),
    (([190], 0, 65536, 100), (192, 1, 256, 256, 0, 0)),
    (([500], 40, 8336, 2040), (192, 44, 6, 256, 8, 8)),
    (([700], 40, 16400, 2000), (192, 55, 5, 256, 19, 42)),
    # 256 x 256: one wave of whole tiles; five; pieces
    (([4096], 0, 1040, 4096), (256, 256, 1, 256, 0, 256)),
    (([5000], 0, 2064, 13312), (256, 1040, 1, 1040, 0, 256)),
    (([1536], 0, 65536, 2044), (256, 48, 6, 256, 32, 230)),
]


def choose(segs, nk, N, gelu=False):
    P, found = WORKGROUPS, []
    for tile, (step, rest, rest_gelu, piece, piece_t) in COSTS.items():
        T = M.row_tiles(segs, tile) * -(-N // tile)
        if T >= P or M.whole_tiles(T, P, nk):
            found.append((-(-T // P) * (nk * step + (rest_gelu if gelu else rest)) + START, tile))
        elif piece is not None:
            found.append((T * nk // P * step + piece + piece_t * T, tile))
    tiles = M.row_tiles(segs, 64) * -(-N // 32)
    one, two, turn = M.SMALL_COSTS
    found.append((-(-tiles // (2 * P)) * (-(-nk // 4) * (one if tiles <= P else two) + turn), "small"))
    return min(found, key=lambda f: f[0])[1]


def plan(T, P, nk):
    return (1, T, T, nk, 0, P) if T >= P else M.plan(T, P, nk)


def describe(lens, text, K, N, gelu=False):
    segs, nk = [(n - text, text) for n in lens], -(-K // 128)
    tile = choose(segs, nk, N, gelu)
    if tile == "small":
        tiles = M.row_tiles(segs, 64) * -(-N // 32)
        return tile, tiles, -(-tiles // (2 * WORKGROUPS))
    T = M.row_tiles(segs, tile) * -(-N // tile)
    s, U, dp, _, _, Pk = plan(T, WORKGROUPS, nk)
    return tile, T, s, dp, U - dp, Pk
