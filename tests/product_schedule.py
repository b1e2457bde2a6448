"""The plans of the feed-forward products on large tiles (product_tiles.h, product_bf16.hip, product_fp8.hip) on the host, and
calls with which the GPU tests reach each kind."""

WORKGROUPS = 256
OUT, DX, DW, FP8 = range(4)
TILES = {OUT: ((256, 256), (256, 128), (128, 128)), FP8: ((256, 256), (128, 256))}
TILES[DX] = TILES[DW] = TILES[OUT]
# window, tile, and of pieces: launch, level, piece; in units of 10 ns
COSTS = {OUT: ((146, 700, 700, 50, 7), (84, 500, 650, 35, 3), (50, 400, 600, 22, 1)),
         DX: ((160, 700, 700, 50, 7), (100, 500, 650, 35, 3), (65, 400, 600, 22, 1)),
         DW: ((155, 700, 700, 50, 7), (90, 500, 650, 35, 3), (55, 400, 600, 22, 1)),
         FP8: ((150, 600, 600, 80, 7), (80, 400, 600, 40, 2))}
SEARCH = -1

# kind, image rows of each sample, text rows, in, out, streams, parts, and with 3 rows more in the buffers: tile, tiles, pieces.
# Each tile whole and cut, in one turn and in more
SHAPES = [
    (OUT, [65], 0, 8, 8, 1, 1, ((128, 128), 1, 1)),
    (OUT, [84], 0, 1192, 8, 1, 1, ((128, 128), 1, 4)),
    (OUT, [527, 57], 105, 40, 11064, 2, 1, ((128, 128), 696, 1)),
    (OUT, [46, 54], 29, 4872, 10864, 2, 1, ((128, 128), 340, 3)),
    (OUT, [50], 143, 8, 11856, 2, 1, ((256, 128), 186, 1)),
    (OUT, [580, 7802], 0, 4400, 152, 1, 1, ((256, 128), 66, 3)),
    (OUT, [1756, 15118], 0, 8, 776, 1, 1, ((256, 128), 462, 1)),
    (OUT, [8262], 0, 1952, 992, 1, 1, ((256, 128), 264, 7)),
    (OUT, [33, 206], 18, 8, 9368, 2, 1, ((256, 256), 148, 1)),
    (OUT, [204], 27, 9304, 5896, 2, 1, ((256, 256), 48, 5)),
    (OUT, [410, 50], 52, 8, 15704, 2, 1, ((256, 256), 310, 1)),
    (OUT, [11824, 1208], 144, 1144, 1272, 2, 1, ((256, 256), 270, 4)),
    (OUT, [65], 0, 8, 8, 1, 2, ((128, 128), 1, 1)),
    (OUT, [78], 0, 1264, 8, 1, 2, ((128, 128), 1, 5)),
    (OUT, [144, 43], 92, 8, 8392, 2, 2, ((128, 128), 660, 1)),
    (OUT, [56], 76, 4128, 8744, 2, 2, ((128, 128), 274, 9)),
    (OUT, [15401, 1442], 0, 8, 72, 1, 2, ((256, 128), 132, 1)),
    (OUT, [131], 0, 6808, 2784, 1, 2, ((256, 128), 44, 5)),
    (OUT, [563, 108], 118, 8, 5384, 2, 2, ((256, 128), 510, 1)),
    (OUT, [446], 0, 1808, 8536, 1, 2, ((256, 128), 268, 6)),
    (OUT, [111], 22, 8, 9192, 2, 2, ((256, 256), 144, 1)),
    (OUT, [38, 52], 174, 9608, 1376, 2, 2, ((256, 256), 44, 5)),
    (OUT, [119, 35], 88, 8, 13552, 2, 2, ((256, 256), 424, 1)),
    (OUT, [952], 0, 1000, 8424, 1, 2, ((256, 256), 264, 4)),
    (DX, [66], 0, 8, 8, 1, 1, ((128, 128), 1, 1)),
    (DX, [75], 5, 8, 976, 2, 1, ((128, 128), 2, 4)),
    (DX, [383, 63], 98, 13712, 8, 2, 1, ((128, 128), 648, 1)),
    (DX, [11106], 0, 296, 2736, 1, 1, ((128, 128), 261, 10)),
    (DX, [136, 101], 12, 7904, 8, 2, 1, ((256, 128), 248, 1)),
    (DX, [5612], 0, 144, 4312, 1, 1, ((256, 128), 44, 5)),
    (DX, [16108, 650], 101, 808, 8, 2, 1, ((256, 128), 476, 1)),
    (DX, [11422], 0, 656, 2440, 1, 1, ((256, 128), 270, 7)),
    (DX, [290, 178], 9, 8304, 8, 2, 1, ((256, 256), 165, 1)),
    (DX, [138], 30, 5712, 8464, 2, 1, ((256, 256), 46, 5)),
    (DX, [307, 294], 140, 12024, 8, 2, 1, ((256, 256), 282, 1)),
    (DX, [5885, 10788], 188, 1008, 880, 2, 1, ((256, 256), 272, 3)),
    (DX, [65], 0, 8, 8, 1, 2, ((128, 128), 1, 1)),
    (DX, [40], 30, 8, 504, 2, 2, ((128, 128), 2, 4)),
    (DX, [70, 87], 6, 12040, 72, 2, 2, ((128, 128), 380, 1)),
    (DX, [39, 36], 50, 8232, 1632, 2, 2, ((128, 128), 260, 3)),
    (DX, [155], 18, 12952, 8, 2, 2, ((256, 128), 204, 1)),
    (DX, [157], 0, 5792, 2080, 1, 2, ((256, 128), 46, 5)),
    (DX, [37, 611], 35, 10768, 8, 2, 2, ((256, 128), 510, 1)),
    (DX, [12924, 133], 0, 536, 992, 1, 2, ((256, 128), 260, 8)),
    (DX, [166, 106], 10, 10168, 8, 2, 2, ((256, 256), 160, 1)),
    (DX, [79], 131, 5456, 3992, 2, 2, ((256, 256), 44, 5)),
    (DX, [327, 308], 16, 14008, 8, 2, 2, ((256, 256), 330, 1)),
    (DX, [4198, 471], 0, 3512, 328, 1, 2, ((256, 256), 266, 3)),
    (DW, [67], 0, 8, 8, 1, 1, ((128, 128), 1, 1)),
    (DW, [57, 980], 0, 8, 8, 1, 1, ((128, 128), 1, 4)),
    (DW, [70, 40], 15, 8400, 312, 2, 1, ((128, 128), 396, 1)),
    (DW, [1448, 1421], 32, 160, 8864, 2, 1, ((128, 128), 280, 7)),
    (DW, [45], 31, 8880, 160, 2, 1, ((256, 128), 140, 1)),
    (DW, [5896], 155, 8, 5456, 2, 1, ((256, 128), 44, 5)),
    (DW, [35], 63, 1120, 6800, 2, 1, ((256, 128), 486, 1)),
    (DW, [664, 1223], 100, 280, 10952, 2, 1, ((256, 128), 258, 7)),
    (DW, [47], 45, 10672, 288, 2, 1, ((256, 256), 168, 1)),
    (DW, [4618, 7019], 13, 2864, 280, 2, 1, ((256, 256), 48, 5)),
    (DW, [43], 29, 2424, 3352, 2, 1, ((256, 256), 280, 1)),
    (DW, [832], 90, 736, 10936, 2, 1, ((256, 256), 258, 3)),
    (DW, [65], 0, 8, 8, 1, 2, ((128, 128), 2, 1)),
    (DW, [1028], 0, 8, 8, 1, 2, ((128, 128), 2, 4)),
    (DW, [44, 66], 31, 8920, 8, 2, 2, ((128, 128), 280, 1)),
    (DW, [1139], 95, 8240, 8, 2, 2, ((128, 128), 260, 4)),
    (DW, [73], 8, 8, 10040, 2, 2, ((256, 128), 160, 1)),
    (DW, [3694, 53], 163, 8, 4192, 2, 2, ((256, 128), 68, 3)),
    (DW, [70], 6, 616, 5944, 2, 2, ((256, 128), 480, 1)),
    (DW, [2090, 181], 51, 8592, 136, 2, 2, ((256, 128), 272, 6)),
    (DW, [38], 30, 12912, 8, 2, 2, ((256, 256), 204, 1)),
    (DW, [10854], 54, 1480, 288, 2, 2, ((256, 256), 48, 5)),
    (DW, [39], 36, 9000, 288, 2, 2, ((256, 256), 288, 1)),
    (DW, [842, 80], 27, 3272, 1200, 2, 2, ((256, 256), 260, 4)),
    (FP8, [66], 0, 16, 16, 1, 1, ((128, 256), 1, 1)),
    (FP8, [70], 0, 1680, 16, 1, 1, ((128, 256), 1, 3)),
    (FP8, [770], 37, 16, 13936, 2, 1, ((128, 256), 440, 1)),
    (FP8, [1961], 0, 2864, 4176, 1, 1, ((128, 256), 272, 5)),
    (FP8, [205, 91], 11, 16, 16160, 2, 1, ((256, 256), 256, 1)),
    (FP8, [67, 1038], 146, 16, 14240, 2, 1, ((256, 256), 448, 1)),
    (FP8, [69], 0, 16, 16, 1, 2, ((128, 256), 1, 1)),
    (FP8, [68], 0, 1936, 16, 1, 2, ((128, 256), 1, 4)),
    (FP8, [38, 44], 15, 32, 13984, 2, 2, ((128, 256), 440, 1)),
    (FP8, [256], 12, 2576, 11344, 2, 2, ((128, 256), 267, 5)),
    (FP8, [99, 135], 16, 16, 6944, 2, 2, ((256, 256), 220, 1)),
    (FP8, [686], 25, 16, 15248, 2, 2, ((256, 256), 480, 1)),
    (FP8, [8383], 0, 11760, 352, 1, 1, ((256, 256), 66, 3)),
    (FP8, [148], 0, 12064, 8528, 1, 2, ((256, 256), 67, 3)),
]
# calls whose gradients are formed in one launch: image rows, text rows, in, out, streams, parts
TOGETHER = [
    ([579], 0, 7136, 536, 1, 1),
    ([361, 1719], 0, 7712, 880, 1, 1),
    ([155, 132], 106, 272, 296, 2, 1),
    ([1055, 665], 243, 7704, 312, 2, 1),
    ([2450], 0, 7112, 472, 1, 2),
    ([471, 190], 256, 272, 272, 2, 2),
    ([259, 2337], 287, 5128, 272, 2, 2),
]


def tail_pieces(tail, nk, cost, splits):
    if tail == 0 or splits == 0:
        return 1
    window, _, fix, level, piece = cost
    most, every = min(WORKGROUPS // tail, nk // 4), nk * window
    s = min(most, splits)
    if splits == SEARCH:
        s = 1
        while s < most and every > s * (s + 1) * (level + tail * piece):
            s += 1
    return s if s > 1 and every - every // s > fix + s * (level + tail * piece) else 1


def plan_cost(T, nk, cost, splits):
    tail, every = T % WORKGROUPS, nk * cost[0]
    s = tail_pieces(tail, nk, cost, splits)
    last = every // s + cost[1] + (cost[2] + s * (cost[3] + tail * cost[4]) if s > 1 else 0)
    return T // WORKGROUPS * (every + cost[1]) + (last if tail else 0)


def choose(kind, row_tiles, cols, nk, splits):
    """Index of the tile size, tiles, pieces of those of the last turn."""
    best = None
    for i, ((bm, bn), cost) in enumerate(zip(TILES[kind], COSTS[kind])):
        T = row_tiles(bm) * -(-cols // bn)
        c = plan_cost(T, nk, cost, splits)
        if best is None or c < best[0]:
            best = c, i, T, tail_pieces(T % WORKGROUPS, nk, cost, splits)
    return best[1:]


def segments(lens, text, merged):
    """Rows of each segment and its stream, of samples with lens image rows and text rows each."""
    if merged:
        return [(sum(lens) + text * len(lens), 0)]
    return [s for n in lens for s in ((n, 0), (text, 1))]


def describe(kind, lens, text, K, N, streams=1, parts=1, behind=0):
    """(tile, tiles, pieces): the main kernel's plan in a call whose buffers hold `behind` rows more."""
    rows, segs = sum(lens) + text * len(lens) + behind, segments(lens, text, streams == 1)
    if kind == DW:
        outs = parts * streams
        nk = max(sum(-(-n // 64) for n, s in segs if s == k) for k in range(streams))
        host = choose(kind, lambda bm: outs * -(-N // bm), K, -(-rows // 64), SEARCH)
        i, T, s = choose(kind, lambda bm: outs * -(-N // bm), K, nk, host[2] if host[2] > 1 else 0)
    else:
        nk = {OUT: -(-K // 64), DX: parts * -(-N // 64), FP8: -(-K // 128)}[kind]
        cols = K if kind == DX else N * parts if parts == 1 else None
        if cols is None:  # half a tile's columns are the gate's
            halves = [(bm, bn // 2) for bm, bn in TILES[kind]]
            return _gated(kind, halves, rows, segs, N, nk)
        host = choose(kind, lambda bm: -(-rows // bm), cols, nk, SEARCH)
        i, T, s = choose(kind, lambda bm: sum(-(-n // bm) for n, _ in segs), cols, nk, host[2] if host[2] > 1 else 0)
    return TILES[kind][i], T, s


def _gated(kind, halves, rows, segs, N, nk):
    def pick(tiles_of, splits):
        found = []
        for i, ((bm, bn), cost) in enumerate(zip(halves, COSTS[kind])):
            T = tiles_of(bm) * -(-N // bn)
            found.append((plan_cost(T, nk, cost, splits), i, T, tail_pieces(T % WORKGROUPS, nk, cost, splits)))
        return min(found)[1:]
    host = pick(lambda bm: -(-rows // bm), SEARCH)
    i, T, s = pick(lambda bm: sum(-(-n // bm) for n, _ in segs), host[2] if host[2] > 1 else 0)
    return TILES[kind][i], T, s


def together(lens, text, K, N, streams, parts, behind=0):
    """Whether dx and the weights' gradients of a call are formed in one launch."""
    rows = sum(lens) + text * len(lens) + behind

    def cost(kind, row_tiles, cols, nk):
        return min(plan_cost(row_tiles(bm) * -(-cols // bn), nk, c, SEARCH) for (bm, bn), c in zip(TILES[kind], COSTS[kind]))

    def shares(both):
        each, at = [0] * WORKGROUPS, 0
        runs = [(DX, -(-rows // 256) * -(-K // 256), parts * -(-N // 64))] if both else []
        words = min(rows, text * len(lens))
        for k in range(streams):
            for _ in range(parts):
                mine = rows if streams == 1 else words if k else rows - words
                runs.append((DW, -(-N // 256) * -(-K // 256), -(-mine // 64)))
        for kind, tiles, nk in runs:
            c = COSTS[kind][0]
            for j in range(WORKGROUPS):
                each[(at + j) % WORKGROUPS] += (tiles // WORKGROUPS + (j < tiles % WORKGROUPS)) * (nk * c[0] + c[1])
            at += tiles % WORKGROUPS
        return max(each)

    dx = cost(DX, lambda bm: -(-rows // bm), K, parts * -(-N // 64))
    dw = cost(DW, lambda bm: parts * streams * -(-N // bm), K, -(-rows // 64))
    return shares(True) < dx + (dw if streams == 1 else min(dw, shares(False)))
