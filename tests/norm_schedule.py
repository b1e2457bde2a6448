"""How the sandwich norms' kernels share rows, on the host (norm.hip: the launchers' tables of forms, norm_workers,
norm_back_workers, norm_shares, k_norm_sums), and the shapes with which the GPU tests reach every form with workers that
take several rows and cross from one segment into the next."""
# widths up to D run on W waves a row with NV float4 a lane, in both directions
FORMS = [(256, 1, 1), (512, 1, 2), (768, 1, 3), (1024, 2, 2), (1536, 2, 3), (2048, 4, 2), (3072, 4, 3), (4096, 8, 2),
         (6144, 8, 3), (8192, 8, 4)]
SUM_GROUPS = 64  # of k_norm_sums


def form(D):
    return next((W, NV) for top, W, NV in FORMS if D <= top)


def workers(rows, D):
    W = form(D)[0]
    return min(rows, 4096 if W == 1 else 2048 // W)


def back_workers(rows, D):
    share = 256 * (10 if D <= 768 else 5)
    most = 1 if D > 3072 else 2 if D > 1536 or 512 < D <= 768 else 3
    return max(1, min(rows, 256 * min(max((rows + share // 2) // share, 1), most)))


def shares(used, P):
    """(first row, end) of every worker's rows."""
    P = min(P, used)
    return [(used * w // P, used * (w + 1) // P) for w in range(P)]


def segments(lens, text):
    """(first row, end) of the segments that have rows."""
    found, at = [], 0
    for n in lens:
        found += [(at, at + n - text), (at + n - text, at + n)]
        at += n
    return [(a, b) for a, b in found if a < b]


def describe(lens, text, P):
    """(rows of the largest share, shares that hold rows of more than one segment, segments in one share at most)."""
    segs, most, crossing, met = segments(lens, text), 0, 0, 0
    for a, b in shares(sum(lens), P):
        n = sum(lo < b and hi > a for lo, hi in segs)
        most, crossing, met = max(most, b - a), crossing + (n > 1), max(met, n)
    return most, crossing, met


def longest_sum(lens, text, D, P):
    """Additions in turn of a segment's sum: a worker's (or each of its four waves') rows and their joint, a group's slots,
    the groups' joint."""
    B, G = len(lens), SUM_GROUPS
    per = G
    while per > 1 and per * B > G:
        per //= 2
    most, slots, all_shares = 0, 0, shares(sum(lens), P)
    for lo, hi in segments(lens, text):
        mine = [min(b, hi) - max(a, lo) for a, b in all_shares if a < hi and b > lo]
        most, slots = max(most, max(mine)), max(slots, len(mine))
    rows = -(-most // 4) + 3 if form(D)[0] == 1 else most
    return rows + -(-slots // per) + min(per, 4) // 2 + max(per // 4 - 1, 0)


def lens(rows):
    """Samples of `rows` rows in all, 4 of each text: one of text alone, one of a single image row."""
    return [rows * 2 // 5, 4, 5, rows - rows * 2 // 5 - 9]


TEXT = 4
# (D, rows): the first and the last width of every form, on more rows than it has workers, so that a share has three rows or
# more (backward, one wave a row: nine, three for one of its four waves)
FORWARD_ROWS = {1: 9000, 2: 2400, 4: 1200, 8: 600}
BACKWARD_ROWS = {1: 2300, 2: 1000, 4: 600, 8: 520}
WIDTHS = [D for low, (top, _, _) in zip([0] + [f[0] for f in FORMS], FORMS) for D in (low + 4, top)]
FORWARD = [(D, FORWARD_ROWS[form(D)[0]]) for D in WIDTHS]
# ... and the first with three and with two workers a CU
BACKWARD = [(D, BACKWARD_ROWS[form(D)[0]]) for D in WIDTHS] + [(1028, 4000), (2052, 2100)]
