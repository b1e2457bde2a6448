"""The products of a feed-forward against their definitions in float64: forward, gradients, FP8 blocks.

Tolerances.  A float32 sum of K products x w is off by at most (K + 2) 2^-24 sum |x w| in any order, or (K + 2) 2^-23
where additions cut instead of rounding (the bf16 and FP8 matrix instructions); what the FP8 one cuts beside is
oracle.hilo_products.cut's, for outputs of bf16 and codes (float32 outputs are formed without it).  What the activation
adds, and how errors of g and u reach the output, is oracle.hilo_products'; the last rounding is half a step: 2^-8 (bf16)
or 2^-24 of the value, of codes 2^-4 and half the least step, 2^-10 of the scale."""
import product_schedule
import pytest
import torch

from oracle import hilo_products as P
from paper_2606_13898_amd import hilo

pytestmark = pytest.mark.gpu

F64 = torch.float64
HALF = {torch.float32: 2.0 ** -24, torch.bfloat16: 2.0 ** -8}
ACTS = {None: hilo.ACT_NONE, "silu": hilo.ACT_SILU, "gelu": hilo.ACT_GELU}
BEHIND = 3  # rows behind the last sample: NaN in, left alone out


def pack(images, text):
    cu = [0]
    for n in images:
        cu.append(cu[-1] + n + text)
    return cu


def weights(g, streams, n, k, dt, gate, bias):
    ws = []
    for _ in range(streams):
        d = {}
        for part in ("", "_gate") if gate else ("",):
            d["w" + part] = (torch.randn(n, k, generator=g) * k ** -0.5).to(dt)
            d["b" + part] = (torch.randn(n, generator=g) * 0.3).to(dt) if bias else None
        ws.append(d)
    return ws


def cuda(ds):
    return [{k: None if v is None else v.cuda() for k, v in d.items()} for d in ds]


def rows_like(t, behind):
    """t on the device with `behind` more rows of NaN (of 0x7f codes)."""
    pad = torch.full((BEHIND, *t.shape[1:]), float("nan") if t.dtype.is_floating_point else behind, dtype=t.dtype)
    return torch.cat([t, pad]).cuda()


def near(got, want, bound, what):
    got = got.to(want.device).to(F64)
    off = (got - want).abs()
    bad = ~(off <= bound + 1e-30)
    assert not bad.any(), (what, int(bad.sum()), float((off / (bound + 1e-30)).nan_to_num(1e9).max()),
                           float(got[bad][0]), float(want[bad][0]))


# image rows of each sample, text rows, in, out, streams of weights
SHAPES = [
    ([1], 0, 8, 8, 1),
    ([1], 0, 1024, 520, 1),
    ([7], 0, 264, 136, 1),
    ([33, 0, 5], 3, 64, 72, 2),
    ([0], 9, 40, 1000, 2),
    ([13, 4], 3, 328, 248, 2),
    ([64, 64], 64, 128, 256, 2),
    ([129], 0, 8, 640, 1),
    ([129, 5], 0, 72, 136, 2),
    ([100, 31, 260], 17, 200, 344, 2),
    ([100, 31, 260], 17, 200, 344, 1),
    ([300], 213, 520, 264, 2),
    ([1, 1, 1, 1], 0, 2056, 648, 1),
    ([600], 0, 1032, 1288, 1),
    ([513, 2, 700], 40, 328, 776, 2),
]
KINDS = [(torch.bfloat16, "silu", True), (torch.bfloat16, "gelu", False), (torch.bfloat16, None, True),
         (torch.float32, "silu", False), (torch.float32, "gelu", True), (torch.float32, None, False)]


def case_id(v):
    return str(v).replace("torch.", "").replace(" ", "")


@pytest.mark.parametrize("shape", SHAPES, ids=case_id)
@pytest.mark.parametrize("kind", KINDS, ids=case_id)
def test_forward(shape, kind):
    (images, text, k, n, streams), (dt, act, bias) = shape, kind
    g = torch.Generator().manual_seed(len(images) * 1000 + k + n)
    cu = pack(images, text)
    x = torch.randn(cu[-1], k, generator=g).to(dt)
    ws = weights(g, streams, n, k, dt, act, bias)
    T = cu[-1] + BEHIND
    out = torch.full((T, n), 7.0, dtype=dt, device="cuda")
    pre = torch.full((T, 2, n), 7.0, dtype=dt, device="cuda") if act else None
    need = hilo.hilo_linear_workspace_bytes(dt, T, k, n, len(images), gated=act is not None)
    ws_dev = torch.empty(need, dtype=torch.uint8, device="cuda").fill_(0xff)
    plan = hilo.linear_weights(cuda(ws))
    cud = torch.tensor(cu, dtype=torch.int32, device="cuda")
    hilo.hilo_linear(plan, rows_like(x, 0), out, cud, text, act=ACTS[act], pre=pre, workspace=ws_dev)
    torch.cuda.synchronize()
    assert (out[cu[-1]:] == 7.0).all()
    xd, ulp = x.to(F64), 2.0 ** -23 if dt is torch.bfloat16 else 2.0 ** -24
    u, su = P.affine(xd, ws, "", cu, text)
    eu = (k + 2) * ulp * su
    if act is None:
        near(out[:cu[-1]], u, eu + HALF[dt] * (u.abs() + eu), "out")
        return
    v, sv = P.affine(xd, ws, "_gate", cu, text)
    ev = (k + 2) * ulp * sv
    want, off = P.gated(act, v, u, ev, eu, dt is torch.bfloat16)
    near(out[:cu[-1]], want, off + HALF[dt] * (want.abs() + off), "out")
    assert (pre[cu[-1]:] == 7.0).all()
    near(pre[:cu[-1], 0], v, ev + HALF[dt] * (v.abs() + ev), "g")
    near(pre[:cu[-1], 1], u, eu + HALF[dt] * (u.abs() + eu), "u")
    # without pre: the same bits
    again = torch.zeros_like(out)
    hilo.hilo_linear(plan, rows_like(x, 0), again, cud, text, act=ACTS[act], workspace=ws_dev)
    assert torch.equal(again[:cu[-1]], out[:cu[-1]])


@pytest.mark.parametrize("shape", SHAPES, ids=case_id)
@pytest.mark.parametrize("kind", KINDS, ids=case_id)
def test_backward(shape, kind):
    (images, text, k, n, streams), (dt, act, bias) = shape, kind
    g = torch.Generator().manual_seed(len(images) * 1000 + k + n + 1)
    cu = pack(images, text)
    x = torch.randn(cu[-1], k, generator=g).to(dt)
    dout = torch.randn(cu[-1], n, generator=g).to(dt)
    pre = torch.randn(cu[-1], 2, n, generator=g).to(dt) if act else None
    ws = weights(g, streams, n, k, dt, act, True)
    T = cu[-1] + BEHIND
    dx = torch.full((T, k), 7.0, dtype=dt, device="cuda")
    got = [{name: torch.full_like(v, 7.0, device="cuda") for name, v in d.items()} for d in ws]
    need = hilo.hilo_linear_backward_workspace_bytes(dt, T, k, n, len(images), gated=act is not None)
    ws_dev = torch.empty(need, dtype=torch.uint8, device="cuda").fill_(0xff)
    cud = torch.tensor(cu, dtype=torch.int32, device="cuda")
    args = (hilo.linear_weights(cuda(ws)), rows_like(x, 0), None if pre is None else rows_like(pre, 0), rows_like(dout, 0))
    hilo.hilo_linear_backward(*args, dx, hilo.linear_grads(got), cud, text, act=ACTS[act], workspace=ws_dev)
    torch.cuda.synchronize()
    assert (dx[cu[-1]:] == 7.0).all()
    (wx, bx), want = P.backward(x.to(F64), ws, None if pre is None else pre.to(F64), dout.to(F64), act, cu, text, HALF[dt],
                                streams == 1)
    near(dx[:cu[-1]], wx, bx, "dx")
    for kk, d in enumerate(got):
        for name, t in d.items():
            near(t, *want[kk][name], f"{name} of {kk}")
    # each output alone: the same bits
    alone = torch.zeros_like(dx)
    hilo.hilo_linear_backward(*args, alone, None, cud, text, act=ACTS[act], workspace=ws_dev)
    assert torch.equal(alone[:cu[-1]], dx[:cu[-1]])
    for kk, d in enumerate(got):
        for name, t in d.items():
            one = [{name: torch.zeros_like(t)} if j == kk else {} for j in range(streams)]
            hilo.hilo_linear_backward(*args, None, hilo.linear_grads(one), cud, text, act=ACTS[act], workspace=ws_dev)
            if streams == 2 or len(want) == 1:
                near(one[kk][name], *want[kk][name], f"{name} of {kk} alone")


@pytest.mark.parametrize("dt", [torch.bfloat16, torch.float32], ids=case_id)
@pytest.mark.parametrize("shared", [("w",), ("w_gate", "b"), ("b", "b_gate"), ("w", "b", "b_gate")], ids=str)
def test_backward_partly_shared(dt, shared):
    """Two streams' gradients of which some are one tensor: that one has the sum over both, the others their stream's."""
    g = torch.Generator().manual_seed(len(shared))
    cu, text, k, n = pack([70, 9, 130], 33), 33, 72, 136
    x, dout, pre = (torch.randn(cu[-1], *s, generator=g).to(dt) for s in ((k,), (n,), (2, n)))
    ws = weights(g, 2, n, k, dt, "silu", True)
    got = [{name: torch.full_like(v, 7.0, device="cuda") for name, v in d.items()} for d in ws]
    got[1].update({name: got[0][name] for name in shared})
    dx, cud = torch.zeros(cu[-1], k, dtype=dt, device="cuda"), torch.tensor(cu, dtype=torch.int32, device="cuda")
    ws_dev = torch.empty(hilo.hilo_linear_backward_workspace_bytes(dt, cu[-1], k, n, 3, gated=True), dtype=torch.uint8, device="cuda")
    hilo.hilo_linear_backward(hilo.linear_weights(cuda(ws)), x.cuda(), pre.cuda(), dout.cuda(), dx, hilo.linear_grads(got), cud, text,
                              act=ACTS["silu"], workspace=ws_dev)
    (wx, bx), want = P.backward(x.to(F64), ws, pre.to(F64), dout.to(F64), "silu", cu, text, HALF[dt], False)
    near(dx, wx, bx, "dx")
    for kk in range(2):
        for name, t in got[kk].items():
            if name in shared:
                near(t, *(want[0][name][j] + want[1][name][j] for j in range(2)), name)
            else:
                near(t, *want[kk][name], f"{name} of {kk}")


@pytest.mark.parametrize("dt", [torch.bfloat16, torch.float32], ids=case_id)
@pytest.mark.parametrize("rows, cols", [(1, 16), (5, 128), (130, 144), (77, 1040), (300, 512), (3, 4112)])
@pytest.mark.parametrize("block_rows", [1, 128])
def test_quantize(dt, rows, cols, block_rows):
    g = torch.Generator().manual_seed(rows + cols)
    x = torch.randn(rows, cols, generator=g) * torch.exp2(torch.randint(-30, 30, (rows, 1), generator=g).float())
    x[0, :16] = 0
    if rows > 2:
        x[1] = 0
        x[2] *= 2.0 ** -118  # to float32's least numbers
    x[-1, -1] = 448 * 2.0 ** 9  # the largest value that a scale reaches
    x = x.to(dt)
    codes = torch.full((rows + 2, cols), 9, dtype=torch.uint8, device="cuda")
    scales = torch.full((-(-(rows + 2) // block_rows), hilo.scale_stride(cols)), 9, dtype=torch.uint8, device="cuda")
    cu = torch.tensor([0, rows], dtype=torch.int32, device="cuda")
    hilo.hilo_quantize_blocks(torch.cat([x, torch.full((2, cols), float("inf"), dtype=dt)]).cuda(), codes, scales, block_rows, cu)
    want, k = P.quantize(x.to(F64), block_rows)
    n = -(-rows // block_rows)
    assert torch.equal(scales[:n, :k.shape[1]].cpu().to(F64), k + 127)
    assert (scales[:n, k.shape[1]:] == 0).all() and (codes[rows:] == 9).all() and (scales[n:] == 9).all()
    assert torch.equal(P.decode(codes[:rows].cpu(), scales[:n].cpu(), block_rows), want)


def test_quantize_not_finite():
    for bad in (float("inf"), float("nan"), -float("inf")):
        for block_rows in (1, 128):
            x = torch.ones(2, 256)
            x[1, 130] = bad
            codes, scales = torch.zeros(2, 256, dtype=torch.uint8, device="cuda"), torch.zeros(2 // block_rows or 1, 4, dtype=torch.uint8, device="cuda")
            hilo.hilo_quantize_blocks(x.cuda(), codes, scales, block_rows)
            v = P.decode(codes.cpu(), scales.cpu(), block_rows)
            assert v[1, 128:].isnan().all() and (v[:, :128] == 1).all() and v[0, 128:].isnan().all() == (block_rows == 128)


FP8_SHAPES = [
    ([1], 0, 16, 16, 1),
    ([1], 0, 2064, 528, 1),
    ([7], 0, 272, 144, 1),
    ([33, 0, 5], 3, 64, 80, 2),
    ([0], 9, 48, 1008, 2),
    ([13, 4], 3, 336, 240, 2),
    ([64, 64], 64, 128, 256, 2),
    ([100, 31, 260], 17, 208, 352, 2),
    ([100, 31, 260], 17, 528, 352, 1),
    ([4, 1], 0, 1168, 640, 1),
    ([600], 0, 1040, 1296, 1),
    ([513, 2, 700], 40, 336, 784, 2),
    ([150, 3], 9, 2064, 272, 2),
]


def fp8_weights(g, streams, n, k, dt, act, bias):
    ws = weights(g, streams, n, k, torch.float32, act, bias)
    for d in ws:
        for part in ("", "_gate") if act else ("",):
            if d["b" + part] is not None:
                d["b" + part] = d["b" + part].to(dt)
    plans = [hilo.quantize_block_weights(**{name: None if v is None else v.cuda() for name, v in d.items()}) for d in ws]
    exponents = [{} for _ in ws]
    for d, e in zip(ws, exponents):
        for part in ("", "_gate") if act else ("",):
            d["w" + part], e["w" + part] = P.quantize(d["w" + part].to(F64), 128)
    return ws, exponents, hilo.linear_weights_fp8(plans)


@pytest.mark.parametrize("shape", FP8_SHAPES, ids=case_id)
@pytest.mark.parametrize("kind", KINDS, ids=case_id)
@pytest.mark.parametrize("coded", [False, True])
def test_fp8(shape, kind, coded):
    (images, text, k, n, streams), (dt, act, bias) = shape, kind
    g = torch.Generator().manual_seed(len(images) * 1000 + k + n + 2)
    cu = pack(images, text)
    x = torch.randn(cu[-1], k, generator=g) * torch.exp2(torch.randint(-3, 4, (1, k), generator=g).float())
    x = x.to(dt)
    ws, kws, plan = fp8_weights(g, streams, n, k, dt, act, bias)
    T = cu[-1] + BEHIND
    need = hilo.hilo_linear_fp8_workspace_bytes(T, k, n, gated=act is not None)
    ws_dev = torch.empty(need, dtype=torch.uint8, device="cuda").fill_(0xff)
    cud = torch.tensor(cu, dtype=torch.int32, device="cuda")
    out = torch.full((T, n), 7.0, dtype=dt, device="cuda")
    xin, a = rows_like(x, 0), {}
    if coded:
        codes = torch.full((T, k), 0x7f, dtype=torch.uint8, device="cuda")
        a["x_scale"] = torch.full((T, hilo.scale_stride(k)), 255, dtype=torch.uint8, device="cuda")
        hilo.hilo_quantize_blocks(xin, codes, a["x_scale"], cu=cud)
        xin = codes
    hilo.hilo_linear_fp8(plan, xin, out, cud, text, act=ACTS[act], workspace=ws_dev, **a)
    torch.cuda.synchronize()
    assert (out[cu[-1]:] == 7.0).all()
    (xq, kx), step = P.quantize(x.to(F64), 1), 2.0 ** -23
    u, su = P.affine(xq, ws, "", cu, text)
    eu = (k + 2) * step * su
    cu_, full = P.cut(xq, kx, ws, kws, "", cu, text), dt is torch.float32
    eu = eu if full else eu + cu_
    if act is None:
        near(out[:cu[-1]], u, eu + HALF[dt] * (u.abs() + eu), "out")
        return
    v, sv = P.affine(xq, ws, "_gate", cu, text)
    ev, cv = (k + 2) * step * sv, P.cut(xq, kx, ws, kws, "_gate", cu, text)
    want, off = P.gated(act, v, u, ev if full else ev + cv, eu, True)
    near(out[:cu[-1]], want, off + HALF[dt] * (want.abs() + off), "out")
    # codes out: of the float32 values, whose block may just have another scale
    want, off = P.gated(act, v, u, ev + cv, eu + cu_ if full else eu, True)
    h = torch.full((T, n), 9, dtype=torch.uint8, device="cuda")
    hs = torch.full((T, hilo.scale_stride(n)), 9, dtype=torch.uint8, device="cuda")
    hilo.hilo_linear_fp8(plan, xin, h, cud, text, act=ACTS[act], workspace=ws_dev, out_scale=hs, **a)
    assert (h[cu[-1]:] == 9).all() and (hs[cu[-1]:] == 9).all()
    blocks = -(-n // 128)
    kk = hs[:cu[-1], :blocks].cpu().to(F64) - 127
    lo = torch.stack([(b[0].abs() - b[1]).clamp(min=0).amax(1) for b in zip(want.split(128, 1), off.split(128, 1))], 1)
    hi = torch.stack([(b[0].abs() + b[1]).amax(1) for b in zip(want.split(128, 1), off.split(128, 1))], 1)
    assert ((kk >= P.block_exponent(lo)) & (kk <= P.block_exponent(hi))).all()
    scale = torch.exp2(kk).repeat_interleave(128, 1)[:, :n]
    near(P.decode(h[:cu[-1]].cpu(), hs[:cu[-1]].cpu(), 1), want, off + 2.0 ** -4 * (want.abs() + off) + 2.0 ** -10 * scale, "codes")


# ------------------------------------------------------------------------- each plan of the large tiles, against float64 here

def on_device(shape, seed):
    """Rows, what they are to be multiplied with and their boundaries, on the device; NaN behind the last row."""
    images, text, k, n, streams, parts = shape
    cu, g = pack(images, text), torch.Generator(device="cuda").manual_seed(seed)
    randn = lambda *s: torch.randn(*s, device="cuda", generator=g)  # noqa: E731
    ws = [{f"{v}{part}": randn(*s).mul_(c).to(torch.bfloat16) for part in ("", "_gate")[:parts] for v, s, c in (("w", (n, k), k ** -0.5), ("b", (n,), 0.3))}
          for _ in range(streams)]
    return cu, torch.tensor(cu, dtype=torch.int32, device="cuda"), randn, ws


def padded(t):
    return torch.cat([t, torch.full((BEHIND, *t.shape[1:]), float("nan"), dtype=t.dtype, device="cuda")])


def scratch(nbytes):
    return torch.empty(max(nbytes, 1), dtype=torch.uint8, device="cuda").fill_(0xff)


def backward_bits(shape, seed, form_dx, form_dw):
    """A bf16 backward pass of a shape against float64; biases' sums as well."""
    images, text, k, n, streams, parts = shape
    cu, cud, randn, ws = on_device(shape, seed)
    act, dt = "silu" if parts == 2 else None, torch.bfloat16
    x, dout = randn(cu[-1], k).to(dt), randn(cu[-1], n).to(dt)
    pre = randn(cu[-1], 2, n).to(dt) if act else None
    dx = torch.full((cu[-1] + BEHIND, k), 7.0, dtype=dt, device="cuda") if form_dx else None
    got = [{name: torch.full_like(v, 7.0) for name, v in d.items()} for d in ws] if form_dw else None
    need = hilo.hilo_linear_backward_workspace_bytes(dt, cu[-1] + BEHIND, k, n, len(images), gated=parts == 2)
    hilo.hilo_linear_backward(hilo.linear_weights(ws), padded(x), None if pre is None else padded(pre), padded(dout), dx,
                              hilo.linear_grads(got) if got else None, cud, text, act=ACTS[act], workspace=scratch(need))
    with torch.device("cuda"):
        (wx, bx), want = P.backward(x.to(F64), ws, None if pre is None else pre.to(F64), dout.to(F64), act, cu, text, HALF[dt], streams == 1)
    if form_dx:
        assert (dx[cu[-1]:] == 7.0).all()
        near(dx[:cu[-1]], wx, bx, "dx")
    for kk, d in enumerate(got or []):
        for name, t in d.items():
            near(t, *want[kk][name], f"{name} of {kk}")


@pytest.mark.parametrize("kind, images, text, k, n, streams, parts, plan", product_schedule.SHAPES, ids=str)
def test_plan(kind, images, text, k, n, streams, parts, plan):
    shape, dt = (images, text, k, n, streams, parts), torch.bfloat16
    if kind in (product_schedule.DX, product_schedule.DW):
        return backward_bits(shape, k + n, kind == product_schedule.DX, kind == product_schedule.DW)
    act = "silu" if parts == 2 else None
    cu, cud, randn, ws = on_device(shape, k + n)
    x, out = randn(cu[-1], k).to(dt), torch.full((cu[-1] + BEHIND, n), 7.0, dtype=dt, device="cuda")
    if kind == product_schedule.OUT:
        need = hilo.hilo_linear_workspace_bytes(dt, cu[-1] + BEHIND, k, n, len(images), gated=parts == 2)
        hilo.hilo_linear(hilo.linear_weights(ws), padded(x), out, cud, text, act=ACTS[act], workspace=scratch(need))
        xv, values = x.to(F64), ws
    else:
        codes, scales = torch.empty_like(x, dtype=torch.uint8), torch.empty(cu[-1], hilo.scale_stride(k), dtype=torch.uint8, device="cuda")
        hilo.hilo_quantize_blocks(x, codes, scales)
        plans = [hilo.quantize_block_weights(d["w"], d["b"], d.get("w_gate"), d.get("b_gate")) for d in ws]
        need = hilo.hilo_linear_fp8_workspace_bytes(cu[-1] + BEHIND, k, n, gated=parts == 2)
        hilo.hilo_linear_fp8(hilo.linear_weights_fp8(plans), padded(x), out, cud, text, act=ACTS[act], workspace=scratch(need))
        xv = P.decode(codes, scales, 1)
        kx = scales[:, :-(-k // 128)].to(F64) - 127
        values = [{**d, **{"w" + p: P.decode(q["w" + p], q["s" + p], 128) for p in ("", "_gate")[:parts]}} for d, q in zip(ws, plans)]
        kws = [{"w" + p: q["s" + p][:, :-(-k // 128)].to(F64) - 127 for p in ("", "_gate")[:parts]} for q in plans]
    assert (out[cu[-1]:] == 7.0).all()
    v, e = {}, {}
    with torch.device("cuda"):
        for p in ("", "_gate")[:parts]:
            v[p], s = P.affine(xv, values, p, cu, text)
            e[p] = (k + 2) * 2.0 ** -23 * s
            if kind == product_schedule.FP8:
                e[p] += P.cut(xv, kx, values, kws, p, cu, text)
        want, off = P.gated(act, v["_gate"], v[""], e["_gate"], e[""], True) if act else (v[""], e[""])
    near(out[:cu[-1]], want, off + HALF[dt] * (want.abs() + off), "out")


@pytest.mark.parametrize("shape", product_schedule.TOGETHER, ids=str)
def test_gradients_together(shape):
    backward_bits(shape, sum(shape[0]), True, True)


# ------------------------------------------------------------------------------------ which gradients a call forms

def backward_call(shape, dt, act, seed):
    """A backward pass of a shape on the device: form(dx, grads), and the shapes of all gradients."""
    images, text, k, n, streams, parts = shape
    cu, cud, randn, ws = on_device(shape, seed)
    ws = [{name: t.to(dt) for name, t in d.items()} for d in ws]
    x, dout, pre = randn(cu[-1], k).to(dt), randn(cu[-1], n).to(dt), randn(cu[-1], 2, n).to(dt) if act else None
    work = scratch(hilo.hilo_linear_backward_workspace_bytes(dt, cu[-1], k, n, len(images), gated=parts == 2))
    plan = hilo.linear_weights(ws)

    def form(dx, grads):
        hilo.hilo_linear_backward(plan, x, pre, dout, dx, hilo.linear_grads(grads) if grads else None, cud, text, act=ACTS[act], workspace=work)

    return form, torch.empty_like(x), ws


@pytest.mark.parametrize("shape", [([551], 0, 256, 1024, 1, 2), ([551], 0, 256, 1024, 1, 1), ([300, 70], 30, 256, 512, 2, 2), ([2000], 0, 64, 128, 1, 2),
                                   ([90, 7, 260], 11, 40, 72, 2, 1), ([1], 0, 8, 8, 1, 2)], ids=str)
def test_float32_gradients_alone(shape):
    """In float32 each gradient has the same bits whichever others a call forms."""
    form, dx, ws = backward_call(shape, torch.float32, "silu" if shape[-1] == 2 else None, 3)
    got = [{name: torch.empty_like(t) for name, t in d.items()} for d in ws]
    form(dx, got)
    alone = torch.empty_like(dx)
    form(alone, None)
    assert torch.equal(alone, dx), "dx"
    for kk, d in enumerate(got):
        for name, t in d.items():
            for with_dx in (False, True):
                one = [{name: torch.empty_like(t)} if j == kk else {} for j in range(len(got))]
                form(alone if with_dx else None, one)
                assert torch.equal(one[kk][name], t), (name, kk, with_dx)
                assert torch.equal(alone, dx), "dx"


# dx alone is cut along k there, beside the weights' gradients it is not
@pytest.mark.parametrize("shape", [([2450], 0, 7112, 472, 1, 2), ([2450], 0, 7112, 1032, 1, 1), ([2000], 0, 2056, 2056, 1, 2)], ids=str)
def test_equal_calls_give_equal_bits(shape):
    """bf16 gradients together and each kind alone: against float64, and twice the same."""
    parts = shape[-1]
    assert product_schedule.together(*shape) and product_schedule.describe(product_schedule.DX, *shape)[2] > 1
    for form_dx, form_dw in ((True, True), (True, False), (False, True)):
        backward_bits(shape, 5, form_dx, form_dw)
    form, dx, ws = backward_call(shape, torch.bfloat16, "silu" if parts == 2 else None, 4)
    for with_dx, with_dw in ((True, True), (True, False), (False, True)):
        runs = []
        for _ in range(2):
            one = [{name: torch.full_like(t, 7.0) for name, t in d.items()} for d in ws] if with_dw else None
            out = torch.full_like(dx, 7.0)
            form(out if with_dx else None, one)
            runs.append([out] + [t for d in one or [] for t in d.values()])
        assert all(torch.equal(a, b) for a, b in zip(*runs))


@pytest.mark.parametrize("T,K,N", [(2000, 128, 4112), (1300, 272, 2064), (40, 144, 4112), (300, 1040, 144)], ids=case_id)
@pytest.mark.parametrize("act", ["silu", "gelu"])
def test_codes_are_of_the_float32_values(T, K, N, act):
    """Codes out of a float32 call are those of the rows that it leaves without out_scale, bit for bit."""
    g = torch.Generator(device="cuda").manual_seed(T)
    x, cud = torch.randn(T, K, device="cuda", generator=g), torch.tensor([0, T], dtype=torch.int32, device="cuda")
    d = {"w" + p: torch.randn(N, K, device="cuda", generator=g) * K ** -0.5 for p in ("", "_gate")}
    d.update({"b" + p: torch.randn(N, device="cuda", generator=g) for p in ("", "_gate")})
    plan, work = hilo.linear_weights_fp8([hilo.quantize_block_weights(**d)]), scratch(hilo.hilo_linear_fp8_workspace_bytes(T, K, N, True))
    out, (codes, want) = torch.empty(T, N, device="cuda"), torch.empty(2, T, N, dtype=torch.uint8, device="cuda")
    scales, ks = torch.empty(2, T, hilo.scale_stride(N), dtype=torch.uint8, device="cuda")
    hilo.hilo_linear_fp8(plan, x, out, cud, act=ACTS[act], workspace=work)
    hilo.hilo_quantize_blocks(out, want, ks)
    hilo.hilo_linear_fp8(plan, x, codes, cud, act=ACTS[act], out_scale=scales, workspace=work)
    assert torch.equal(scales, ks)
    assert int((codes != want).sum()) == 0


# ------------------------------------------------------------------------ FP8: many tiles, many samples, large buffers

def codes_near(codes, scales, want, off, what):
    """Codes and scales of values `want` that are off by `off`: the scale of a largest value in that range, a code's rounding."""
    k = scales[:, :-(-want.shape[1] // 128)].to(F64) - 127
    lo, hi = (torch.stack([b.amax(1) for b in t.split(128, 1)], 1) for t in ((want.abs() - off).clamp(min=0), want.abs() + off))
    assert ((k >= P.block_exponent(lo)) & (k <= P.block_exponent(hi))).all(), what
    scale = torch.exp2(k).repeat_interleave(128, 1)[:, :want.shape[1]]
    near(P.decode(codes, scales, 1), want, off + 2.0 ** -4 * (want.abs() + off) + 2.0 ** -10 * scale, what)


def fp8_bits(shape, dt, coded, seed):
    """An FP8 product of a shape against float64."""
    images, text, k, n, streams, parts = shape
    act = "silu" if parts == 2 else None
    cu, cud, randn, ws = on_device(shape, seed)
    T = cu[-1] + BEHIND
    x, ws = randn(cu[-1], k).to(dt), [{name: t.to(dt) for name, t in d.items()} for d in ws]
    plans = [hilo.quantize_block_weights(d["w"], d["b"], d.get("w_gate"), d.get("b_gate")) for d in ws]
    out = torch.full((T, n), 7, dtype=torch.uint8 if coded else dt, device="cuda")
    os = torch.full((T, hilo.scale_stride(n)), 7, dtype=torch.uint8, device="cuda") if coded else None
    hilo.hilo_linear_fp8(hilo.linear_weights_fp8(plans), padded(x), out, cud, text, act=ACTS[act], out_scale=os,
                         workspace=scratch(hilo.hilo_linear_fp8_workspace_bytes(T, k, n, gated=parts == 2)))
    codes, scales = torch.empty_like(x, dtype=torch.uint8), torch.empty(cu[-1], hilo.scale_stride(k), dtype=torch.uint8, device="cuda")
    hilo.hilo_quantize_blocks(x, codes, scales)
    xv, kx = P.decode(codes, scales, 1), scales[:, :-(-k // 128)].to(F64) - 127
    names = ("", "_gate")[:parts]
    values = [{**d, **{"w" + p: P.decode(q["w" + p], q["s" + p], 128) for p in names}} for d, q in zip(ws, plans)]
    kws = [{"w" + p: q["s" + p][:, :-(-k // 128)].to(F64) - 127 for p in names} for q in plans]
    v, e = {}, {}
    with torch.device("cuda"):
        for p in names:
            v[p], s = P.affine(xv, values, p, cu, text)
            e[p] = (k + 2) * 2.0 ** -23 * s
            if dt is torch.bfloat16 and not coded:
                e[p] += P.cut(xv, kx, values, kws, p, cu, text)
        want, off = P.gated(act, v["_gate"], v[""], e["_gate"], e[""], True) if act else (v[""], e[""])
        assert (out[cu[-1]:] == 7).all()
        if not coded:
            return near(out[:cu[-1]], want, off + HALF[dt] * (want.abs() + off), "out")
        assert (os[cu[-1]:] == 7).all() and not os[:cu[-1], -(-n // 128):].any()
        codes_near(out[:cu[-1]], os[:cu[-1]], want, off, "codes")


# more tiles than workgroups and than two each, of one window pair and of several, odd and even, of one segment and of many
MANY = [24, 0, 61, 130, 7, 300, 1, 90] * 5
TILED = [([2000], 0, 16, 4112, 1), ([2000], 0, 128, 4112, 1), ([1900], 9, 272, 4112, 2), ([4100], 0, 512, 4112, 1), (MANY, 5, 16, 4112, 2), (MANY, 5, 400, 1040, 2),
         ([40] * 33, 0, 144, 2064, 1), ([3, 0, 66] * 12, 13, 1040, 144, 2), ([3, 0, 6] * 13, 3, 1040, 144, 2), ([1, 0] * 20, 1, 272, 528, 2)]
LEAVES = [(torch.float32, 1, False), (torch.float32, 2, False), (torch.float32, 2, True), (torch.bfloat16, 2, True), (torch.bfloat16, 1, False), (torch.bfloat16, 2, False)]


@pytest.mark.parametrize("dt,parts,coded", LEAVES, ids=case_id)
@pytest.mark.parametrize("shape", TILED, ids=lambda s: f"{len(s[0])}x{sum(s[0])}-{s[1:]}".replace(" ", ""))
def test_fp8_tiles(shape, dt, parts, coded):
    fp8_bits((*shape, parts), dt, coded, len(shape[0]) + shape[2])


@pytest.mark.parametrize("T,K,N,dt,parts,coded", [(530000, 16, 4112, torch.bfloat16, 1, False), (530000, 16, 4112, torch.bfloat16, 2, False),
                                                  (270000, 16, 4112, torch.float32, 1, False), (1050000, 16, 4112, torch.float32, 2, True),
                                                  (1050000, 4112, 16, torch.bfloat16, 1, False), (530000, 4112, 16, torch.float32, 1, False)], ids=case_id)
def test_fp8_past_32_bits(T, K, N, dt, parts, coded):
    """Rows, codes or outputs of more than 2^32 bytes: rows at both ends and in the middle against float64."""
    act = "silu" if parts == 2 else None
    g = torch.Generator(device="cuda").manual_seed(T)
    x = torch.empty(T, K, dtype=dt, device="cuda").normal_(generator=g)
    d = {"w" + p: torch.empty(N, K, device="cuda").normal_(generator=g).mul_(K ** -0.5) for p in ("", "_gate")[:parts]}
    q = hilo.quantize_block_weights(d["w"], None, d.get("w_gate"))
    codes, scales = torch.empty(T, K, dtype=torch.uint8, device="cuda"), torch.empty(T, hilo.scale_stride(K), dtype=torch.uint8, device="cuda")
    hilo.hilo_quantize_blocks(x, codes, scales)
    del x
    out = torch.empty(T, N, dtype=torch.uint8 if coded else dt, device="cuda")
    os = torch.empty(T, hilo.scale_stride(N), dtype=torch.uint8, device="cuda") if coded else None
    assert max(t.numel() * t.element_size() for t in (codes, out)) > 1 << 32 or T * K * 2 > 1 << 32  # the last of the widened rows
    cud = torch.tensor([0, T], dtype=torch.int32, device="cuda")
    hilo.hilo_linear_fp8(hilo.linear_weights_fp8([q]), codes, out, cud, x_scale=scales, out_scale=os, act=ACTS[act],
                         workspace=scratch(hilo.hilo_linear_fp8_workspace_bytes(T, K, N, gated=parts == 2)))
    values = [{"w" + p: P.decode(q["w" + p], q["s" + p], 128) for p in ("", "_gate")[:parts]}]
    kws = [{"w" + p: q["s" + p][:, :-(-K // 128)].to(F64) - 127 for p in ("", "_gate")[:parts]}]
    for a in (0, T // 2, T - 60):
        xv, kx, v, e = P.decode(codes[a:a + 60], scales[a:a + 60], 1), scales[a:a + 60, :-(-K // 128)].to(F64) - 127, {}, {}
        with torch.device("cuda"):
            for p in ("", "_gate")[:parts]:
                v[p], s = P.affine(xv, values, p, [0, 60], 0)
                e[p] = (K + 2) * 2.0 ** -23 * s
                if dt is torch.bfloat16 and not coded:
                    e[p] += P.cut(xv, kx, values, kws, p, [0, 60], 0)
            want, off = P.gated(act, v["_gate"], v[""], e["_gate"], e[""], True) if act else (v[""], e[""])
            if coded:
                codes_near(out[a:a + 60], os[a:a + 60], want, off, a)
            else:
                near(out[a:a + 60], want, off + HALF[dt] * (want.abs() + off), a)
