"""hilo_rope, hilo_token_positions, hilo_norm_residual and its backward pass, hilo_quantize_rows_i8 and hilo_linear_i8
against their float64 oracle, at the sizes, strides and layouts where they can go wrong.

E is half a step of float32 (2^-24).  A result stored in bf16 adds half a step of its own, HALF["bf16"] relative."""
import numpy as np
import pytest
import torch

import linear_schedule
import norm_schedule
from oracle import hilo_operators as Q
from paper_2606_13898_amd import hilo

pytestmark = pytest.mark.gpu

E = 2.0 ** -24
DT = {"f32": torch.float32, "bf16": torch.bfloat16}
HALF = {"f32": E, "bf16": 2.0 ** -8}


def _cu(lens):
    return np.concatenate([[0], np.cumsum(lens)]).astype(np.int32)


def _dev(a, dtype=torch.float32):
    return torch.from_numpy(np.ascontiguousarray(a)).to(dtype).cuda()


def _np(t):
    return t.detach().cpu().double().numpy()


def _rand(rng, dtype, *shape, std=1.0, mean=0.0):
    """A device tensor and its values in float64."""
    t = _dev(rng.standard_normal(shape) * std + mean, torch.float32).to(DT[dtype])
    return t, _np(t)


def _within(got, want, bound, what):
    over = np.abs(got - want) - bound
    assert np.isfinite(got).all(), f"{what}: not finite"
    at = np.unravel_index(over.argmax(), over.shape)
    assert over.max() <= 0, f"{what}: {got[at]} for {want[at]}, bound {np.broadcast_to(bound, over.shape)[at]} at {at}"


# ------------------------------------------------------------------------------------------ rotary

def _rope_bound(x, pos, heads, pairs, base, adjacent, one_spectrum, want, dtype):
    """Cosine, sine, both products and their sum each off by half a step of at most |u| + |v|: 4 E (|u| + |v|) with the
    sum's rounding counted against the larger |u| + |v|.  The frequency's 64-bit series: below 2^-46 of the angle."""
    rows, n = x.shape[0], sum(pairs)
    a = np.abs(x).reshape(rows, heads, -1)
    far = np.abs(Q.rope_angles(pos, pairs, base, one_spectrum))[:, None] * 2.0 ** -46
    bound = np.zeros_like(a)
    for j in range(n):
        p, q = (2 * j, 2 * j + 1) if adjacent else (j, j + n)
        bound[:, :, p] = bound[:, :, q] = (4 * E + far[:, :, j]) * (a[:, :, p] + a[:, :, q])
    return bound.reshape(rows, -1) + (HALF[dtype] * np.abs(want) if dtype == "bf16" else 0)


# every vector width (by pairs, rest, head size and alignment), one to four axes, an axis without pairs, rotated
# parts, far positions, rows over several workgroups and a table of one row
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("rows,heads,hd,pairs,pad,far", [
    (1, 2, 128, (64,), 0, 40000), (5, 3, 64, (8, 12, 12), 8, 0), (77, 1, 80, (10, 10, 10), 0, 3), (33, 6, 96, (20,), 5, 7),
    (130, 2, 256, (64, 0, 32, 32), 1, 1000000), (3, 5, 2, (1,), 0, 9), (700, 48, 64, (16, 16), 64, 0), (9, 4, 10, (2, 1), 3, 0)])
@pytest.mark.parametrize("adjacent,one_spectrum,backward", [(False, False, False), (True, True, True)])
def test_rope(dtype, rows, heads, hd, pairs, pad, far, adjacent, one_spectrum, backward):
    print(f"[rope] {dtype} rows={rows} heads={heads} hd={hd} pairs={pairs} pad={pad} adj={adjacent}", flush=True)
    rng = np.random.default_rng(rows + hd)
    width = heads * hd
    xt, xv = _rand(rng, dtype, rows, width + pad)
    pos = (rng.integers(0, 200, (rows, len(pairs))) * 0.5).astype(np.float32)
    pos[:, 0] += far
    pos[0, -1] = -3.5
    base = [10000.0, 500.0, 100.0, 7.0][:len(pairs)]
    want = Q.rope(xv[:, :width], pos, heads, pairs, base, adjacent, one_spectrum, backward)
    bound = _rope_bound(xv[:, :width], pos, heads, pairs, base, adjacent, one_spectrum, want, dtype)
    flags = (hilo.ROPE_ADJACENT if adjacent else 0) | (hilo.ROPE_ONE_SPECTRUM if one_spectrum else 0)
    r = hilo.rotary(heads, hd, pairs, base, flags)
    out = torch.full((rows, width + 3), 5.0, dtype=DT[dtype], device="cuda")
    before = xt.clone()
    hilo.hilo_rope(r, xt[:, :width], _dev(pos), out[:, 1:1 + width], backward=backward)
    torch.cuda.synchronize()
    got = _np(out)
    _within(got[:, 1:1 + width], want, bound, "rope")
    assert (got[:, 0] == 5).all() and (got[:, 1 + width:] == 5).all() and torch.equal(xt, before)
    # in place, between columns that stay
    hilo.hilo_rope(r, xt[:, :width], _dev(pos), xt[:, :width], backward=backward)
    torch.cuda.synchronize()
    _within(_np(xt[:, :width]), want, bound, "rope in place")
    assert torch.equal(xt[:, width:], before[:, width:])


def test_rope_turns_back():
    """The gradient's turn undoes the turn: two turns are off by twice one turn's bound."""
    rng = np.random.default_rng(4)
    r = hilo.rotary(7, 64, (8, 12, 12))
    x, xv = _rand(rng, "f32", 50, 7 * 64)
    pos = _dev(rng.uniform(0, 3000, (50, 3)))
    y = torch.empty_like(x)
    hilo.hilo_rope(r, x, pos, y)
    hilo.hilo_rope(r, y, pos, y, backward=True)
    torch.cuda.synchronize()
    _within(_np(y), xv, 16 * E * (np.abs(xv).max() * 2), "there and back")


def test_rope_rows_end():
    """Rows at or behind the last boundary stay as they are."""
    rng = np.random.default_rng(5)
    r = hilo.rotary(2, 64, (32,))
    x, xv = _rand(rng, "bf16", 40, 128)
    pos = _dev(rng.integers(0, 9, (40, 1)))
    for end in (0, 1, 17, 40):
        y = torch.full_like(x, 3.0)
        hilo.hilo_rope(r, x, pos, y, cu=_dev(np.array([0, end // 2, end]), torch.int32))
        torch.cuda.synchronize()
        want = Q.rope(xv, _np(pos), 2, (32,))
        assert (y[end:] == 3).all()
        _within(_np(y)[:end], want[:end], (2.0 ** -8 + 8 * E) * 8, "rows") if end else None


@pytest.mark.parametrize("tokens", [hilo.PARTITION, hilo.OVERLAP, hilo.DROP])
def test_token_positions(tokens):
    rng = np.random.default_rng(6)
    batch, images, H, W, L = 2, 2, 6, 10, 3
    shp = hilo.hilo_shape(batch, images, H, W, L, 64, 1, 64, 64, hilo.F32)
    G, N = batch * images, H * W
    x = _dev(rng.standard_normal((G, N, 64)))
    i32 = dict(dtype=torch.int32, device="cuda")
    energy = torch.empty(G, N, dtype=torch.int64, device="cuda")
    idx, fine, pool = torch.empty(G, N, **i32), torch.empty(G, N, **i32), torch.empty(G, N // 4, **i32)
    counts, cu, seg = torch.empty(G, 2, **i32), torch.empty(batch + 1, **i32), torch.empty(G, **i32)
    hilo.hilo_score(shp, x, energy)
    hilo.hilo_select_tokens(shp, energy, None, 0, hilo.TOPK, None, [0, 15, 4, 9], tokens, idx, fine, pool, counts, cu, seg)
    T = hilo.hilo_max_tokens(shp)
    text = rng.uniform(0, 9, (L, 3)).astype(np.float32)
    for tp in (None, text):
        pos = torch.full((T, 3), -7.0, device="cuda")
        hilo.hilo_token_positions(shp, fine, pool, counts, cu, seg, None if tp is None else _dev(tp), pos)
        torch.cuda.synchronize()
        want = Q.token_positions(batch, images, W, L, fine.cpu().numpy(), pool.cpu().numpy(), counts.cpu().numpy(), tp)
        n = int(cu[-1])
        assert len(want) == n
        np.testing.assert_array_equal(_np(pos)[:n], want)
        assert (pos[n:] == -7).all()


# ------------------------------------------------------------------------------------------- norms

def _norm_bound(v, dv, rms, eps):
    """How far a normalised row may be: v off by dv, the mean by the sum's at most 48 additions a lane and joint, the
    deviation by half of the square sum's, then three roundings of the value."""
    n, m, r = (np.abs(a) for a in Q.norm(v, rms, eps))
    r = r[:, None]
    dm = 0 if rms else 48 * E * np.abs(v).mean(1)[:, None] + dv.max(1)[:, None]
    d = r * (dv + dm + E * np.abs(v - (0 if rms else v.mean(1)[:, None])))
    return d + n * (32 * E + np.sqrt((d * d).mean(1))[:, None])


def _norm_case(seed, dtype, lens, text, D, gains, mod, outlier=0.0):
    rng = np.random.default_rng(seed)
    T, B = int(sum(lens)), len(lens)
    c = dict(cu=_cu(lens), T=T, D=D)
    c["y"], c["yv"] = _rand(rng, dtype, max(T, 1) + 2, D, std=0.7, mean=0.2)
    c["x"], c["xv"] = _rand(rng, "f32", max(T, 1) + 2, D, mean=outlier)
    vec = dict(gate=None, shift=None, scale=None, post_gain=None, pre_gain=None)
    c["dev"], c["ref"] = dict(vec), dict(vec)
    if mod:
        m, mv = _rand(rng, "f32", B, 2, 6, D, std=0.3)
        for i, k in enumerate(("gate", "shift", "scale")):
            c["dev"][k], c["ref"][k] = m[:, :, 2 + i], mv[:, :, 2 + i]
    if gains:
        for k in ("post_gain", "pre_gain"):
            c["dev"][k], c["ref"][k] = _rand(rng, "f32", 2, D, std=0.2, mean=1.0)
    return rng, c


NORM_SHAPES = [([1], 0, 4), ([3, 0, 5], 0, 64), ([6, 4, 9], 4, 100), ([2, 2], 2, 256), ([7], 3, 260), ([5], 0, 512),
               ([4], 1, 1024), ([3, 3], 1, 1028), ([2], 0, 2048), ([9, 1], 1, 2052), ([3], 1, 3072), ([2], 0, 4096),
               ([3], 1, 4100), ([2], 1, 8192)]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("lens,text,D", NORM_SHAPES)
@pytest.mark.parametrize("rms,gains,mod", [(False, False, True), (True, True, True), (False, True, False)])
def test_norm_residual(dtype, lens, text, D, rms, gains, mod):
    print(f"[norm] {dtype} lens={lens} text={text} D={D} rms={rms} gains={gains} mod={mod}", flush=True)
    rng, c = _norm_case(D + sum(lens), dtype, lens, text, D, gains, mod)
    T, alpha, eps = c["T"], 0.75, 1e-6
    kind = hilo.NORM_RMS if rms else hilo.NORM_LAYER
    n = hilo.norms(kind, eps, alpha, **c["dev"])
    x_out, h = torch.full_like(c["x"], 9.0), torch.full_like(c["y"], 9.0)
    stats = torch.full((c["x"].shape[0], 4), 9.0, device="cuda")
    cu = _dev(c["cu"], torch.int32)
    hilo.hilo_norm_residual(n, c["y"], c["x"], x_out, h, cu, text, stats=stats)
    torch.cuda.synchronize()
    want_x, want_h, want_s = Q.norm_residual(c["yv"][:T], c["xv"][:T], c["cu"], text, rms, eps, alpha, **c["ref"])
    gt, po, pr, sc = (np.ones((T, D)) for _ in range(4))
    sh = np.zeros((T, D))
    for a, b, s, k in Q.segments(c["cu"], text):
        if mod:
            gt[a:b], sc[a:b], sh[a:b] = c["ref"]["gate"][s, k], 1 + c["ref"]["scale"][s, k], c["ref"]["shift"][s, k]
        if gains:
            po[a:b], pr[a:b] = c["ref"]["post_gain"][k], c["ref"]["pre_gain"][k]
    yv = c["yv"][:T]
    u = np.abs(Q.norm(yv, rms, eps)[0])
    bx = np.abs(gt * po) * (_norm_bound(yv, np.zeros_like(yv), rms, eps) + 3 * E * u) + 2 * E * (np.abs(alpha * c["xv"][:T]) + np.abs(want_x))
    _within(_np(x_out)[:T], want_x, bx, "x_out")
    v = np.abs(Q.norm(want_x, rms, eps)[0])
    bh = np.abs(pr * sc) * (_norm_bound(want_x, bx, rms, eps) + 4 * E * v) + 2 * E * np.abs(sh) + E * np.abs(want_h)
    bh = bh + (HALF[dtype] * np.abs(want_h) if dtype == "bf16" else 0)
    _within(_np(h)[:T], want_h, bh, "h")
    assert (x_out[T:] == 9).all() and (h[T:] == 9).all() and (stats[T:] == 9).all()
    np.testing.assert_allclose(_np(stats)[:T], want_s, rtol=64 * E, atol=64 * E * (1 + np.abs(want_x).max()))
    # in place, without statistics; only the norm after; only the norm before
    x2, h2 = c["x"].clone(), torch.empty_like(h)
    hilo.hilo_norm_residual(n, c["y"], x2, x2, h2, cu, text)
    x3, h3 = torch.empty_like(x2), torch.empty_like(h)
    hilo.hilo_norm_residual(n, c["y"], c["x"], x3, None, cu, text)
    hilo.hilo_norm_residual(n, None, x_out, None, h3, cu, text)
    torch.cuda.synchronize()
    assert torch.equal(x2[:T], x_out[:T]) and torch.equal(h2[:T], h[:T])
    assert torch.equal(x3[:T], x_out[:T]) and torch.equal(h3[:T], h[:T]) and torch.equal(x2[T:], c["x"][T:])


def test_norm_far_from_zero():
    """A residual stream whose mean is a thousand deviations away keeps the digits that float32 has."""
    rng, c = _norm_case(3, "f32", [5], 0, 1024, False, False, outlier=1000.0)
    h = torch.empty_like(c["x"])
    hilo.hilo_norm_residual(hilo.norms(), None, c["x"], None, h, _dev(c["cu"], torch.int32))
    torch.cuda.synchronize()
    want = Q.norm(c["xv"][:5], False, 1e-6)[0]
    _within(_np(h)[:5], want, _norm_bound(c["xv"][:5], np.zeros((5, 1024)), False, 1e-6) + E * np.abs(want), "h")


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("lens,text,D", [([3, 0, 5], 0, 64), ([6, 4], 2, 256), ([3], 1, 1040), ([2], 1, 3072), ([2], 0, 8192)])
def test_norm_residual_codes(dtype, lens, text, D):
    """h as codes is the quantisation of the float32 h: the float32 block's h, within its own roundings of a half."""
    print(f"[norm codes] {dtype} lens={lens} D={D}", flush=True)
    rng, c = _norm_case(D, dtype, lens, text, D, True, True)
    T, n, cu = c["T"], hilo.norms(hilo.NORM_LAYER, 1e-6, 1.0, **c["dev"]), _dev(c["cu"], torch.int32)
    x_out, x2, h = torch.empty_like(c["x"]), torch.empty_like(c["x"]), torch.empty_like(c["x"])
    codes = torch.full(c["x"].shape, 99, dtype=torch.int8, device="cuda")
    scale = torch.full((c["x"].shape[0],), 9.0, device="cuda")
    hilo.hilo_norm_residual(n, c["y"], c["x"], x_out, codes, cu, text, h_scale=scale)
    hilo.hilo_norm_residual(n, c["y"].float(), c["x"], x2, h, cu, text)  # the same values, float32 h
    torch.cuda.synchronize()
    assert torch.equal(x2[:T], x_out[:T]) and (codes[T:] == 99).all() and (scale[T:] == 9).all()
    want, ws = Q.quantize_rows_i8(h[:T].cpu().numpy())
    np.testing.assert_array_equal(codes[:T].cpu().numpy(), want)
    np.testing.assert_array_equal(scale[:T].cpu().numpy(), ws)


def _back_bounds(c, ref, dx_out, dh, rms, eps, alpha, text, want):
    """Worst cases of the sums: a row's means take at most 48 additions a lane and joint, a segment's sums at most 80 in
    turn (a worker's rows, its group's workers, the groups) here; every factor is off by a few E."""
    T, D = c["T"], c["D"]
    cu = c["cu"]
    bx, by = np.zeros((T, D)), np.zeros((T, D))
    sums = {k: np.zeros_like(v) for k, v in want.items()}
    zero = np.zeros((T, D))

    def through(n, bn, v, bv, r, m):
        # r (n - mean n - v mean(n v)), n off by bn, v off by bv
        nv = (np.abs(n) * np.abs(v)).mean(1)[:, None]
        bnv = (bn * np.abs(v) + np.abs(n) * bv).mean(1)[:, None] + 64 * E * nv
        mn = 0 if rms else np.abs(n).mean(1)[:, None]
        bmn = 0 if rms else bn.mean(1)[:, None] + 64 * E * mn
        b = bn + bmn + np.abs(v) * bnv + bv * nv + 6 * E * (np.abs(n) + mn + np.abs(v) * nv)
        return r * b + 4 * E * r * (np.abs(n) + mn + np.abs(v) * nv)

    for a, b, s, k in Q.segments(cu, text):
        if a == b:
            continue
        xv, yv = c["xv"][a:b], c["yv"][a:b]
        one = 1.0 + (0 if ref["scale"] is None else ref["scale"][s, k])
        pre = 1.0 if ref["pre_gain"] is None else ref["pre_gain"][k]
        gt = np.ones(D) if ref["gate"] is None else ref["gate"][s, k]
        post = np.ones(D) if ref["post_gain"] is None else ref["post_gain"][k]
        g = zero[a:b] if dx_out is None else dx_out[a:b].copy()
        bg = 2 * E * np.abs(g)
        if dh is not None:
            v, m, r = Q.norm(xv, rms, eps)
            bv = E * (2 * np.abs(m * r)[:, None] + 4 * np.abs(v)) + E * np.abs(xv) * r[:, None]
            d = dh[a:b]
            nn = d * one * pre
            bg = bg + through(nn, 4 * E * np.abs(nn), v, bv, r[:, None], m)
            t = nn - v * (nn * v).mean(1)[:, None] - (0 if rms else nn.mean(1)[:, None])
            g = g + r[:, None] * t
            sums["shift"][s, k] = 80 * E * np.abs(d).sum(0)
            sB = (np.abs(d) * bv).sum(0) + 84 * E * np.abs(d * v).sum(0)
            sums["scale"][s, k] = np.abs(pre) * sB
            sums["pre_gain"][k] += np.abs(one) * sB + 16 * E * np.abs(one * (d * v).sum(0))
        bx[a:b] = abs(alpha) * (bg + 2 * E * np.abs(g))
        u, m, r = Q.norm(yv, rms, eps)
        bu = E * (2 * np.abs(m * r)[:, None] + 4 * np.abs(u)) + E * np.abs(yv) * r[:, None]
        f = gt * post
        by[a:b] = through(g * f, np.abs(f) * bg + 4 * E * np.abs(g * f), u, bu, r[:, None], m)
        sA = (bg * np.abs(u) + np.abs(g) * bu).sum(0) + 84 * E * np.abs(g * u).sum(0)
        sums["gate"][s, k] = np.abs(post) * sA
        sums["post_gain"][k] += np.abs(gt) * sA + 16 * E * np.abs(gt * (g * u).sum(0))
    return bx, by, sums


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("lens,text,D", NORM_SHAPES + [([40, 0, 133], 0, 128), ([90, 70], 33, 512), ([150], 20, 1536), ([70], 6, 4608)])
@pytest.mark.parametrize("rms,gains,mod", [(False, True, True), (True, False, True)])
def test_norm_residual_backward(dtype, lens, text, D, rms, gains, mod):
    print(f"[norm back] {dtype} lens={lens} text={text} D={D} rms={rms} gains={gains}", flush=True)
    rng, c = _norm_case(D + sum(lens), dtype, lens, text, D, gains, mod)
    T, B, alpha, eps = c["T"], len(lens), 0.75, 1e-6
    kind, cu = hilo.NORM_RMS if rms else hilo.NORM_LAYER, _dev(c["cu"], torch.int32)
    n = hilo.norms(kind, eps, alpha, **c["dev"])
    rows = c["x"].shape[0]
    stats = torch.zeros(rows, 4, device="cuda")
    st = Q.norm_residual(c["yv"][:T], np.zeros((T, D)), c["cu"], text, rms, eps)[2]
    st[:, 2:] = np.stack(Q.norm(c["xv"][:T], rms, eps)[1:], 1)
    stats[:T] = _dev(st)
    dxo, dxov = _rand(rng, "f32", rows, D, std=0.5)
    dh, dhv = _rand(rng, dtype, rows, D)
    dx, dy = torch.full_like(dxo, 9.0), torch.full_like(dh, 9.0)
    dmod = torch.full((B, 2, 4, D), 9.0, device="cuda")
    dg = torch.full((2, 2, D), 9.0, device="cuda")
    ws = torch.full((hilo.hilo_norm_residual_workspace_bytes(rows, B, D) // 4,), float("nan"), device="cuda")
    grads = hilo.norm_grads(gate=dmod[:, :, 0], shift=dmod[:, :, 1], scale=dmod[:, :, 3], post_gain=dg[0], pre_gain=dg[1])
    hilo.hilo_norm_residual_backward(n, dxo, dh, c["y"], c["x"], stats, dx, dy, grads, cu, text, ws)
    torch.cuda.synchronize()
    r = {k: c["ref"][k] for k in ("gate", "scale", "post_gain", "pre_gain")}
    wx, wy, ws_ = Q.norm_residual_backward(dxov[:T], dhv[:T], c["yv"][:T], c["xv"][:T], c["cu"], text, rms, eps, alpha, **r)
    bx, by, bs = _back_bounds(c, r, dxov[:T], dhv[:T], rms, eps, alpha, text, ws_)
    _within(_np(dx)[:T], wx, bx, "dx")
    _within(_np(dy)[:T], wy, by + (HALF[dtype] * np.abs(wy) if dtype == "bf16" else 0), "dy")
    for k, got in (("gate", dmod[:, :, 0]), ("shift", dmod[:, :, 1]), ("scale", dmod[:, :, 3]), ("post_gain", dg[0]), ("pre_gain", dg[1])):
        _within(_np(got), ws_[k], bs[k] + 1e-30, "d" + k)
    assert (dx[T:] == 9).all() and (dy[T:] == 9).all() and (dmod[:, :, 2] == 9).all()
    # the same bits again, in place; a gain that both streams share gets the sum of both
    first = (dx.clone(), dy.clone(), dmod.clone(), dg.clone())
    dxo2, dh2 = dxo.clone(), dh.clone()
    hilo.hilo_norm_residual_backward(n, dxo2, dh2, c["y"], c["x"], stats, dxo2, dh2, grads, cu, text, ws)
    shared = torch.zeros(2, D, device="cuda")
    hilo.hilo_norm_residual_backward(n, dxo, dh, c["y"], c["x"], stats, dx, dy, hilo.norm_grads(
        post_gain=(shared[0], shared[0]), pre_gain=(shared[1], None)), cu, text, ws)
    torch.cuda.synchronize()
    assert torch.equal(dxo2[:T], first[0][:T]) and torch.equal(dh2[:T], first[1][:T])
    assert torch.equal(dmod, first[2]) and torch.equal(dg, first[3])
    assert torch.equal(shared[0], first[3][0, 0] + first[3][0, 1]) and torch.equal(shared[1], first[3][1, 0])


# samples over the groups that sum their slots: 8, 2 and 1 group a sample, more samples than groups, many slots a sample
@pytest.mark.parametrize("B,most,text,D", [(5, 30, 2, 64), (20, 5, 1, 132), (40, 3, 0, 64), (70, 4, 1, 72), (2, 2000, 77, 64)])
def test_norm_backward_many_samples(B, most, text, D):
    lens = [int(n) + text for n in np.random.default_rng(B).integers(0, most + 1, B)]
    test_norm_residual_backward("f32", lens, text, D, False, True, True)


def test_norm_backward_parts():
    """Without a gradient from elsewhere, without h, without y: the formula with that part left out."""
    rng, c = _norm_case(8, "f32", [5, 3], 2, 128, True, True)
    T, cu = c["T"], _dev(c["cu"], torch.int32)
    n = hilo.norms(hilo.NORM_LAYER, 1e-6, 0.5, **c["dev"])
    r = {k: c["ref"][k] for k in ("gate", "scale", "post_gain", "pre_gain")}
    stats = torch.zeros(T + 2, 4, device="cuda")
    st = np.concatenate([np.stack(Q.norm(v[:T], False, 1e-6)[1:], 1) for v in (c["yv"], c["xv"])], 1)
    stats[:T] = _dev(st)
    dxo, dxov = _rand(rng, "f32", T + 2, 128)
    dh, dhv = _rand(rng, "f32", T + 2, 128)
    for a, b, y in ((None, dh, c["y"]), (dxo, None, c["y"]), (dxo, dh, None), (None, dh, None)):
        dx, dy = torch.empty_like(dxo), torch.empty_like(dh)
        hilo.hilo_norm_residual_backward(n, a, b, y, c["x"], stats, dx, None if y is None else dy, None, cu, 2)
        torch.cuda.synchronize()
        wx, wy, _ = Q.norm_residual_backward(None if a is None else dxov[:T], None if b is None else dhv[:T],
                                             None if y is None else c["yv"][:T], c["xv"][:T], c["cu"], 2, False, 1e-6, 0.5, **r)
        np.testing.assert_allclose(_np(dx)[:T], wx, rtol=0, atol=128 * E * 16)
        if y is not None:
            np.testing.assert_allclose(_np(dy)[:T], wy, rtol=0, atol=128 * E * 16)


def test_norm_backward_against_differences():
    """The gradient's product with a direction is the slope of sum(x_out cx + h ch) along it, by central differences of the
    forward pass.  Outputs up to 8 are off by 64 E each at random signs: 8 * 64 E sqrt(2 T D) over 2 step; the third
    derivative's part, step^2, is below that."""
    rng, c = _norm_case(9, "f32", [6, 5], 2, 64, True, True)
    T, D, cu, step = c["T"], 64, _dev(c["cu"], torch.int32), 2.0 ** -6
    y, x = c["y"][:T].clone(), c["x"][:T].clone()
    n = hilo.norms(hilo.NORM_LAYER, 1e-6, 0.9, **c["dev"])
    cx, ch = _rand(rng, "f32", T, D, std=0.1)[0], _rand(rng, "f32", T, D, std=0.1)[0]

    def forward(y, x, stats=None):
        xo, h = torch.empty_like(x), torch.empty_like(x)
        hilo.hilo_norm_residual(n, y, x, xo, h, cu, 2, stats=stats)
        return xo, h, float((xo.double() * cx.double()).sum() + (h.double() * ch.double()).sum())

    stats, dx, dy = torch.empty(T, 4, device="cuda"), torch.empty_like(x), torch.empty_like(x)
    xo, _, _ = forward(y, x, stats)
    hilo.hilo_norm_residual_backward(n, cx, ch, y, xo, stats, dx, dy, None, cu, 2)
    for _ in range(4):
        vy, vx = _rand(rng, "f32", T, D)[0], _rand(rng, "f32", T, D)[0]
        vy, vx = (v / v.norm() for v in (vy, vx))
        slope = (forward(y + step * vy, x + step * vx)[2] - forward(y - step * vy, x - step * vx)[2]) / (2 * step)
        told = float((dy.double() * vy.double()).sum() + (dx.double() * vx.double()).sum())
        assert abs(slope - told) <= 0.1 * 8 * 64 * E * np.sqrt(2 * T * D) / (2 * step) + step ** 2, (slope, told)


# --------------------------------------------------------------------------------------------- int8

@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("rows,cols", [(1, 16), (5, 512), (7, 528), (3, 1024), (4, 1040), (2, 3072), (3, 4112), (2, 16384), (2, 16400)])
def test_quantize_rows_i8(dtype, rows, cols):
    print(f"[quantize i8] {dtype} {rows} x {cols}", flush=True)
    rng = np.random.default_rng(cols)
    x, _ = _rand(rng, dtype, rows + 3, cols)
    x[0] *= 1e-3
    x[-1] = 0
    x[rows // 2, cols - 1] = 300.0
    for cu, n in ((None, rows + 3), (_dev(np.array([0, rows]), torch.int32), rows)):
        codes = torch.full(x.shape, 99, dtype=torch.int8, device="cuda")
        scale = torch.full((rows + 3,), 9.0, device="cuda")
        hilo.hilo_quantize_rows_i8(x, codes, scale, cu)
        torch.cuda.synchronize()
        want, ws = Q.quantize_rows_i8(x.float().cpu().numpy())
        np.testing.assert_array_equal(codes[:n].cpu().numpy(), want[:n])
        np.testing.assert_array_equal(scale[:n].cpu().numpy(), ws[:n])
        assert (codes[n:] == 99).all() and (scale[n:] == 9).all()


def test_quantize_rows_i8_extremes():
    """Rows of tiny, largest and not finite values: codes that stay in range, a scale that says what the row was."""
    x = torch.zeros(7, 64, device="cuda")
    x[0, 3], x[1, 3], x[2, 3], x[3, 3] = 2.0 ** -126, 2.0 ** -119, 3.4028234663852886e38, float("inf")
    x[4, 3], x[5, 3], x[5, 4], x[6] = float("nan"), float("inf"), float("nan"), -1e-30
    codes, scale = torch.empty(7, 64, dtype=torch.int8, device="cuda"), torch.empty(7, device="cuda")
    hilo.hilo_quantize_rows_i8(x, codes, scale)
    torch.cuda.synchronize()
    assert scale[0] == 0 and (codes[0] == 0).all()
    assert [int(codes[i, 3]) for i in (1, 2)] == [127, 127] and (codes[6] == -127).all()
    assert torch.isfinite(scale[[1, 2, 6]]).all() and (scale[[1, 2, 6]] > 0).all()
    assert torch.isinf(scale[3]) and torch.isnan(scale[4]) and torch.isnan(scale[5])


def _linear_bound(want, size, gelu, dtype):
    """The sum's rounding, the two scales' product, theirs and the bias' sum: 4 half steps of what is added up.  GELU: its
    slope is below 1.13, its own arithmetic below 64 E of 1 + |u|."""
    b = 4 * E * size
    if gelu:
        b = 1.13 * b + 64 * E * (1 + size)
    return b + HALF[dtype] * np.abs(want)


# rows, columns and K on either side of every tile and step; streams with and without text, empty samples, no bias
LINEAR = [([1], 0, 16, 4), ([1], 0, 3072, 96), ([2, 1], 0, 64, 20), ([17], 0, 80, 36), ([40, 0, 33], 0, 128, 100),
          ([31, 60], 9, 272, 64), ([70], 5, 1040, 132), ([5, 3], 3, 48, 260), ([129, 66], 65, 256, 192),
          ([300], 100, 512, 520), ([64], 64, 192, 32), ([3, 2], 1, 5008, 40), ([1, 0, 1], 0, 9200, 52), ([4], 4, 1552, 28),
          ([13], 5, 2304, 48), ([30, 25], 0, 12304, 36), ([40, 9], 3, 2064, 8212), ([500, 333], 77, 768, 196), ([61], 61, 784, 68)]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("lens,text,K,N", LINEAR)
@pytest.mark.parametrize("gelu,bias", [(False, True), (True, False)])
def test_linear_i8(dtype, lens, text, K, N, gelu, bias):
    print(f"[linear i8] {dtype} lens={lens} text={text} K={K} N={N} gelu={gelu} bias={bias}", flush=True)
    run_linear(dtype, lens, text, K, N, gelu, bias, K + N)


def run_linear(dtype, lens, text, K, N, gelu, bias, seed, rows=None, spare=3):
    """hilo_linear_i8 on float rows and on their codes, `rows` of them (all) compared; `spare` rows behind the last."""
    g = torch.Generator().manual_seed(seed)
    cu, T = _cu(lens), int(sum(lens))
    x = torch.randn(T + spare, K, generator=g).to(DT[dtype])
    ws, ref = [], []
    for _ in range(2):
        w = {"w": torch.randint(-127, 128, (N, K), dtype=torch.int8, generator=g), "s": (torch.rand(N, generator=g) + 0.5) * 1e-3,
             "b": torch.randn(N, generator=g).to(DT[dtype]) if bias else None}
        ws.append({k: None if v is None else v.cuda() for k, v in w.items()})
        ref.append({k: None if v is None else v.numpy() if k == "w" else v.double().numpy() for k, v in w.items()})
    plan = hilo.linear_weights_i8(ws)
    out = torch.full((T + spare, N), 9.0, dtype=DT[dtype], device="cuda")
    act = hilo.ACT_GELU if gelu else hilo.ACT_NONE
    wsp = torch.full((hilo.hilo_linear_i8_workspace_bytes(T + spare, K),), 255, dtype=torch.uint8, device="cuda")
    cud, xd = _dev(cu, torch.int32), x.cuda()
    hilo.hilo_linear_i8(plan, xd, out, cud, text, act=act, workspace=wsp)
    torch.cuda.synchronize()
    pick = np.arange(T) if rows is None else rows
    codes, scale = Q.quantize_rows_i8(x[torch.from_numpy(pick)].float().numpy())
    want, size = np.zeros((len(pick), N)), np.zeros((len(pick), N))
    for a, b, _, k in Q.segments(cu, text):
        at = np.flatnonzero((pick >= a) & (pick < b))
        if len(at):
            want[at], size[at] = Q.linear_i8(codes[at], scale[at], [ref[k]], np.array([0, len(at)]), 0, gelu)
    _within(_np(out[torch.from_numpy(pick).cuda()]), want, _linear_bound(want, size, gelu, dtype), "linear")
    assert (out[T:] == 9).all()
    # codes in: the same bits
    cd, sd = torch.empty(T + spare, K, dtype=torch.int8, device="cuda"), torch.empty(T + spare, device="cuda")
    hilo.hilo_quantize_rows_i8(xd, cd, sd)
    out2 = torch.full_like(out, 9.0)
    hilo.hilo_linear_i8(plan, cd, out2, cud, text, x_scale=sd, act=act, workspace=wsp)
    torch.cuda.synchronize()
    assert torch.equal(out, out2)


# buffers of exactly these rows: the forms for one, two and up to four rows, up to 16, up to 64, and the first behind each
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("lens,text,K,N", [([1], 0, 1552, 100), ([1, 1], 0, 3072, 96), ([1, 1, 1], 1, 784, 64), ([3], 1, 12240, 36),
                                           ([2, 1, 1], 0, 4096, 52), ([5], 2, 1024, 68), ([9, 7], 0, 2064, 36), ([17], 3, 896, 132),
                                           ([40, 24], 7, 1168, 8260), ([65], 1, 1040, 72)])
def test_linear_i8_few_rows(dtype, lens, text, K, N):
    print(f"[linear i8 few] {dtype} lens={lens} text={text} K={K} N={N}", flush=True)
    run_linear(dtype, lens, text, K, N, False, True, K, spare=0)


# every width of the few rows' tiles (8 to 32 columns by fours, the last tile part of one), one and two streams
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("lens,text", [([2], 0), ([1, 3], 1), ([9, 5], 2), ([33, 20], 6)])
@pytest.mark.parametrize("N", [1028, 2052, 4100, 5132, 6148, 7172, 12300])
def test_linear_i8_few_rows_widths(dtype, lens, text, N):
    print(f"[linear i8 few width] {dtype} lens={lens} text={text} N={N}", flush=True)
    run_linear(dtype, lens, text, 144, N, True, True, N, spare=0)


# every kind of plan of the large tiles (linear_schedule.py says which each shape reaches), both types of output
@pytest.mark.parametrize("shape", [s for s, _ in linear_schedule.SHAPES], ids=lambda s: f"{sum(s[0])}x{s[2]}x{s[3]}")
@pytest.mark.parametrize("dtype,gelu,bias", [("bf16", True, True), ("f32", False, True), ("bf16", False, False)])
def test_linear_i8_plans(shape, dtype, gelu, bias):
    lens, text, K, N = shape
    print(f"[linear i8 plan] {dtype} lens={lens} text={text} K={K} N={N}", flush=True)
    T = sum(lens)
    rows = None if T * N * K < 3e9 else np.sort(np.random.default_rng(1).choice(T, 100, replace=False))
    run_linear(dtype, lens, text, K, N, gelu, bias, 7, rows)


@pytest.mark.parametrize("spare", [0, 40000])
def test_linear_i8_most_samples(spare):
    """4096 samples, most of two rows: in one launch, and from codes on the larger tiles' kernel."""
    lens = [2, 1, 3, 2] * 1024
    run_linear("bf16", lens, 1, 80, 96, False, True, 3, spare=spare)


def test_linear_i8_largest_sum():
    """Every product the largest: sums at the edge of what K allows stay exact."""
    K = 65536
    for rows in (2, 300):
        x = torch.full((rows, K), 127, dtype=torch.int8, device="cuda")
        w = torch.full((4, K), 127, dtype=torch.int8, device="cuda")
        w[1] = -127
        plan = hilo.linear_weights_i8([{"w": w, "s": torch.ones(4, device="cuda")}])
        out = torch.empty(rows, 4, device="cuda")
        ws = torch.empty(hilo.hilo_linear_i8_workspace_bytes(rows, K), dtype=torch.uint8, device="cuda")
        hilo.hilo_linear_i8(plan, x, out, _dev(np.array([0, rows]), torch.int32), x_scale=torch.ones(rows, device="cuda"), workspace=ws)
        torch.cuda.synchronize()
        top = float(np.float32(127 * 127 * K))
        assert _np(out).tolist() == [[top, -top, top, top]] * rows


def test_linear_i8_not_finite_row():
    """A row that holds an infinity or a NaN comes out not finite; the others are what they are without it."""
    rng = np.random.default_rng(2)
    x, _ = _rand(rng, "bf16", 6, 64)
    w = hilo.quantize_i8_weights(_rand(rng, "bf16", 8, 64)[0])
    plan, cu = hilo.linear_weights_i8([w]), _dev(np.array([0, 6]), torch.int32)
    ws = torch.empty(hilo.hilo_linear_i8_workspace_bytes(6, 64), dtype=torch.uint8, device="cuda")
    out, bad = (torch.empty(6, 8, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    hilo.hilo_linear_i8(plan, x, out, cu, workspace=ws)
    y = x.clone()
    y[2, 5], y[4, 63] = float("inf"), float("nan")
    hilo.hilo_linear_i8(plan, y, bad, cu, workspace=ws)
    torch.cuda.synchronize()
    assert not torch.isfinite(bad[[2, 4]].float()).any()
    assert torch.equal(bad[[0, 1, 3, 5]], out[[0, 1, 3, 5]])


# small tiles, 128 x 128, 192 x 192 and 256 x 256 ones (linear_schedule.py), whole tiles inside; buffers of few rows
@pytest.mark.parametrize("lens,text,K,N,spare", [([300], 100, 1040, 520, 3), ([900], 100, 2064, 2040, 3), ([2500], 30, 528, 2048, 3),
                                                 ([4096], 0, 1040, 4096, 3), ([30], 4, 272, 136, 0)])
def test_linear_i8_output_at_8_bytes(lens, text, K, N, spare):
    """bf16 rows that start 8 bytes behind a multiple of 16: the bits of rows that do not, and nothing beside them."""
    print(f"[linear i8 out] lens={lens} K={K} N={N}", flush=True)
    T, cu = sum(lens) + spare, _dev(_cu(lens), torch.int32)
    g = torch.Generator(device="cuda").manual_seed(N)
    w = [hilo.quantize_i8_weights(torch.randn(N, K, device="cuda", generator=g), torch.randn(N, device="cuda", generator=g).bfloat16())
         for _ in range(2)]
    plan, x = hilo.linear_weights_i8(w), torch.randn(T, K, device="cuda", generator=g).bfloat16()
    ws = torch.empty(hilo.hilo_linear_i8_workspace_bytes(T, K), dtype=torch.uint8, device="cuda")
    out = torch.full((T, N), 9.0, dtype=torch.bfloat16, device="cuda")
    buf = torch.full((T * N + 8,), 9.0, dtype=torch.bfloat16, device="cuda")
    off = buf[4:4 + T * N].view(T, N)
    assert out.data_ptr() % 16 == 0 and off.data_ptr() % 16 == 8
    for act in (hilo.ACT_NONE, hilo.ACT_GELU):
        hilo.hilo_linear_i8(plan, x, out, cu, text, act=act, workspace=ws)
        hilo.hilo_linear_i8(plan, x, off, cu, text, act=act, workspace=ws)
        torch.cuda.synchronize()
        assert torch.equal(off, out) and (off[sum(lens):] == 9).all() and (buf[:4] == 9).all() and (buf[-4:] == 9).all()
        assert out[:sum(lens)].float().std() > 0.1


# ------------------------------------------------------------------- norms whose workers take several rows
#
# The same checks on more rows than there are workers, every form at both ends of its widths (norm_schedule.py): rows read
# ahead, vectors kept over a segment's rows and read again where a share crosses into the next one, sums over a row's waves
# in turn, slots of several segments.  A row's own sums are no longer than above, so its tolerances hold; a segment's are
# within the 80 additions that the backward pass' count (the longest of these shapes' is checked on the host).

def _types(i):
    return [("bf16", False), ("f32", True), ("f32", False), ("bf16", True)][i % 4]


@pytest.mark.parametrize("i,D,rows", [(i, *s) for i, s in enumerate(norm_schedule.FORWARD)])
def test_norm_residual_many_rows(i, D, rows):
    dtype, rms = _types(i)
    test_norm_residual(dtype, norm_schedule.lens(rows), norm_schedule.TEXT, D, rms, True, True)


@pytest.mark.parametrize("i,D,rows", [(i, *s) for i, s in enumerate(norm_schedule.FORWARD)])
def test_norm_residual_codes_many_rows(i, D, rows):
    test_norm_residual_codes(_types(i + 2)[0], norm_schedule.lens(rows), norm_schedule.TEXT, D)


@pytest.mark.parametrize("i,D,rows", [(i, *s) for i, s in enumerate(norm_schedule.BACKWARD)])
def test_norm_residual_backward_many_rows(i, D, rows):
    dtype, rms = _types(i + 1)
    test_norm_residual_backward(dtype, norm_schedule.lens(rows), norm_schedule.TEXT, D, rms, True, True)


# ------------------------------------------------------------ int8 products: forms that the cases above leave out

@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("text,K", [(0, 144), (1, 144), (0, 3088)])
@pytest.mark.parametrize("N", [4100, 5132, 6148, 7172])
def test_linear_i8_one_row_wide(dtype, text, K, N):
    """One float row on tiles of two column blocks (20, 24, 28 and 32 columns, and where a stream has none 12 and 16)."""
    print(f"[linear i8 one row] {dtype} text={text} K={K} N={N}", flush=True)
    run_linear(dtype, [1], text, K, N, text == 0, True, N, spare=0)


@pytest.mark.parametrize("shape", [s for s, _ in linear_schedule.SHAPES], ids=lambda s: f"{sum(s[0])}x{s[2]}x{s[3]}")
@pytest.mark.parametrize("gelu,bias", [(True, True), (False, False)])
def test_linear_i8_plans_f32(shape, gelu, bias):
    """float32 rows out of the large tiles with GELU, and without a bias; test_operators.py holds which plans GELU reaches."""
    lens, text, K, N = shape
    print(f"[linear i8 plan f32] lens={lens} text={text} K={K} N={N} gelu={gelu}", flush=True)
    T = sum(lens)
    rows = None if T * N * K < 3e9 else np.sort(np.random.default_rng(1).choice(T, 100, replace=False))
    run_linear("f32", lens, text, K, N, gelu, bias, 8, rows)
