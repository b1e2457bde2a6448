"""The products of a feed-forward as programs use them: a block's whole feed-forward between its norms with its backward
pass and in FP8, captured into graphs, on two streams, with nothing to do, past 32-bit offsets, of many samples, and with
values that are not finite."""
import pytest
import torch

from oracle import hilo_products as P
from paper_2606_13898_amd import hilo
from test_products_gpu import ACTS, HALF, case_id, cuda, near, pack, weights

pytestmark = pytest.mark.gpu

F64, BF, F32, U8 = torch.float64, torch.bfloat16, torch.float32, torch.uint8


def cu_of(*ends):
    return torch.tensor([0, *ends], dtype=torch.int32, device="cuda")


def empty(*shape, dtype=F32):
    return torch.empty(*shape, dtype=dtype, device="cuda")


def bytes_of(n):
    return torch.empty(n, dtype=U8, device="cuda")


# ------------------------------------------------------------------------------- a block's feed-forward

@pytest.mark.parametrize("dt,images,text,D,N", [(F32, [40, 3, 100], 9, 64, 168), (BF, [40, 0, 100], 9, 128, 344), (BF, [700], 0, 256, 512)], ids=case_id)
def test_feed_forward(dt, images, text, D, N):
    """Norm, gate and up, down, gated residual and the next norm, forward and backward, against autograd in float64 by
    relative error over each tensor.  A bf16 rounding has rms 2^-8 / sqrt(3) = 2.3e-3 at most; what passes here is rounded no
    more than ten times on its way, some of it summed: 2e-2.  float32: 2^-24 a step and sums of up to 512, 1e-5."""
    g = torch.Generator().manual_seed(D + N)
    cu = pack(images, text)
    T, B = cu[-1], len(images)
    up, down = weights(g, 2, N, D, dt, True, True), weights(g, 2, D, N, dt, False, True)
    x, dx2, dh2 = torch.randn(T, D, generator=g), torch.randn(T, D, generator=g), torch.randn(T, D, generator=g).to(dt)
    mod, cud = torch.randn(B, 2, 6, D, generator=g) * 0.3, torch.tensor(cu, dtype=torch.int32, device="cuda")
    # ---- the program
    modd = mod.cuda()
    first = hilo.norms(shift=modd[:, :, 3], scale=modd[:, :, 4])
    last = hilo.norms(hilo.NORM_RMS, residual_scale=0.8, gate=modd[:, :, 5])
    wup, wdown, xd = hilo.linear_weights(cuda(up)), hilo.linear_weights(cuda(down)), x.cuda()
    h, a, y, h2 = empty(T, D, dtype=dt), empty(T, N, dtype=dt), empty(T, D, dtype=dt), empty(T, D, dtype=dt)
    pre, x2, st1, st2 = empty(T, 2, N, dtype=dt), empty(T, D), empty(T, 4), empty(T, 4)
    ws = bytes_of(max(f(dt, T, D, N, B, True) for f in (hilo.hilo_linear_workspace_bytes, hilo.hilo_linear_backward_workspace_bytes)) +
                  max(f(dt, T, N, D, B) for f in (hilo.hilo_linear_workspace_bytes, hilo.hilo_linear_backward_workspace_bytes)) +
                  hilo.hilo_norm_residual_workspace_bytes(T, B, D))
    hilo.hilo_norm_residual(first, None, xd, None, h, cud, text, stats=st1)
    hilo.hilo_linear(wup, h, a, cud, text, act=hilo.ACT_SILU, pre=pre, workspace=ws)
    hilo.hilo_linear(wdown, a, y, cud, text, workspace=ws)
    hilo.hilo_norm_residual(last, y, xd, x2, h2, cud, text, stats=st2)
    gup = [{k: torch.empty_like(v) for k, v in d.items()} for d in cuda(up)]
    gdown = [{k: torch.empty_like(v) for k, v in d.items()} for d in cuda(down)]
    dx, dy, da, dh, dx1 = empty(T, D), empty(T, D, dtype=dt), empty(T, N, dtype=dt), empty(T, D, dtype=dt), empty(T, D)
    dmod = empty(B, 2, 1, D)
    hilo.hilo_norm_residual_backward(last, dx2.cuda(), dh2.cuda(), y, x2, st2, dx, dy, hilo.norm_grads(gate=dmod[:, :, 0]), cud, text, ws)
    hilo.hilo_linear_backward(wdown, a, None, dy, da, hilo.linear_grads(gdown), cud, text, workspace=ws)
    hilo.hilo_linear_backward(wup, h, pre, da, dh, hilo.linear_grads(gup), cud, text, act=hilo.ACT_SILU, workspace=ws)
    hilo.hilo_norm_residual_backward(first, None, dh, None, xd, st1, dx1, None, None, cud, text)
    # ---- in float64, by autograd
    leaf = x.to(F64).requires_grad_()
    lup, ldown = [[{k: v.to(F64).requires_grad_() for k, v in d.items()} for d in ds] for ds in (up, down)]
    x2w, h2w, m = [], [], mod.to(F64)
    for s in range(B):
        for lo, hi, k in ((cu[s], cu[s + 1] - text, 0), (cu[s + 1] - text, cu[s + 1], 1)):
            v = leaf[lo:hi]
            n = torch.nn.functional.layer_norm(v, (D,), eps=1e-6) * (1 + m[s, k, 4]) + m[s, k, 3]
            u = n @ lup[k]["w"].T + lup[k]["b"]
            act = torch.nn.functional.silu(n @ lup[k]["w_gate"].T + lup[k]["b_gate"]) * u
            o = act @ ldown[k]["w"].T + ldown[k]["b"]
            rms = lambda t: t * torch.rsqrt((t * t).mean(1, keepdim=True) + 1e-6)  # noqa: E731
            x2w.append(0.8 * v + m[s, k, 5] * rms(o))
            h2w.append(rms(x2w[-1]))
    x2w, h2w = torch.cat(x2w), torch.cat(h2w)
    ((x2w * dx2).sum() + (h2w * dh2.to(F64)).sum()).backward()
    tol = 2e-2 if dt is BF else 1e-5

    def close(got, want, what):
        off = (got.cpu().to(F64) - want).norm() / want.norm()
        assert off <= tol, (what, float(off))

    close(x2, x2w.detach(), "x2")
    close(h2, h2w.detach(), "h2")
    close(dx + dx1, leaf.grad, "dx")
    for got, want in ((gup, lup), (gdown, ldown)):
        for k in range(2):
            for name, t in got[k].items():
                if want[k][name].grad is None or not want[k][name].grad.any():  # a stream without rows
                    assert not t.any(), f"{name} of {k}"
                else:
                    close(t, want[k][name].grad, f"{name} of {k}")


@pytest.mark.parametrize("images,text,D,N", [([5, 3], 0, 256, 528), ([30, 9], 5, 272, 400), ([300, 20, 90], 33, 528, 1040), ([1100], 0, 144, 272), ([150, 0, 40], 9, 1040, 272)], ids=case_id)
def test_fp8_feed_forward(images, text, D, N):
    """Gate and up into codes, and the down product that reads them, against the float64 product of the codes that came out."""
    g = torch.Generator().manual_seed(D + N)
    cu = pack(images, text)
    T, cud = cu[-1], cu_of(*cu[1:])
    x = torch.randn(T, D, generator=g).to(BF)
    up, down = weights(g, 2, N, D, F32, True, False), weights(g, 2, D, N, F32, False, False)
    q = lambda ds: hilo.linear_weights_fp8([hilo.quantize_block_weights(**{k: v for k, v in d.items() if v is not None}) for d in cuda(ds)])  # noqa: E731
    wup, wdown = q(up), q(down)
    h, hs, y = empty(T, N, dtype=U8), empty(T, hilo.scale_stride(N), dtype=U8), empty(T, D, dtype=BF)
    ws = bytes_of(max(hilo.hilo_linear_fp8_workspace_bytes(T, D, N, True), hilo.hilo_linear_fp8_workspace_bytes(T, N, D)))
    hilo.hilo_linear_fp8(wup, x.cuda(), h, cud, text, out_scale=hs, act=hilo.ACT_GELU, workspace=ws)
    hilo.hilo_linear_fp8(wdown, h, y, cud, text, x_scale=hs, workspace=ws)
    hv = P.decode(h.cpu(), hs.cpu(), 1)
    exact = [{"w": P.quantize(d["w"].to(F64), 128)[0], "b": None} for d in down]
    kw = [{"w": P.quantize(d["w"].to(F64), 128)[1]} for d in down]
    want, s = P.affine(hv, exact, "", cu, text)
    kx = hs[:, :-(-N // 128)].cpu().to(F64) - 127
    off = (N + 2) * 2.0 ** -23 * s + P.cut(hv, kx, exact, kw, "", cu, text)
    near(y, want, off + HALF[BF] * (want.abs() + off), "y")


# ---------------------------------------------------------------------------------- graphs, streams

def replays(body, inputs, outputs, rounds=3):
    """body() captured once, then replayed on fresh inputs with eager work in between: equal bits to eager calls."""
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        body()
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        body()
    for r in range(rounds):
        g = torch.Generator(device="cuda").manual_seed(r)
        for t in inputs:
            t.copy_(torch.randn(t.shape, generator=g, device="cuda"))
        for t in outputs:
            t.zero_()
        graph.replay()
        torch.cuda.synchronize()
        got = [t.clone() for t in outputs]
        for t in outputs:
            t.zero_()
        body()
        torch.cuda.synchronize()
        for i, (a, b) in enumerate(zip(got, outputs)):
            assert torch.equal(a, b), f"replay {r}, output {i}"
            assert a.float().abs().max() > 0


def training(T, K, N, dt, act, text=0, ends=None):
    """A forward and backward pass of a product: the call, its inputs and its outputs."""
    g = torch.Generator().manual_seed(T)
    gate = act is not None
    ws = weights(g, 2, N, K, dt, gate, True)
    plan, cud = hilo.linear_weights(cuda(ws)), cu_of(*(ends or [T]))
    x, dout, out = empty(T, K, dtype=dt).normal_(), empty(T, N, dtype=dt).normal_(), empty(T, N, dtype=dt)
    pre, dx = empty(T, 2, N, dtype=dt) if gate else None, empty(T, K, dtype=dt)
    grads = cuda(ws)
    plan_grads = hilo.linear_grads(grads if text else grads[:1])
    B = len(ends or [T])
    work = bytes_of(max(f(dt, T, K, N, B, gate) for f in (hilo.hilo_linear_workspace_bytes, hilo.hilo_linear_backward_workspace_bytes)))

    def body(stream=None):
        hilo.hilo_linear(plan, x, out, cud, text, act=ACTS[act], pre=pre, workspace=work, stream=stream)
        hilo.hilo_linear_backward(plan, x, pre, dout, dx, plan_grads, cud, text, act=ACTS[act], workspace=work, stream=stream)

    outs = [out, dx] + ([pre] if gate else []) + [t for d in (grads if text else grads[:1]) for t in d.values() if t is not None]
    return body, [x, dout], outs


# few rows, tiles of each size, cut along k (a fixup launch) and whole, float32 with and without partial sums
@pytest.mark.parametrize("T,K,N,dt,act,text,ends", [
    (3, 256, 264, BF, "silu", 0, None), (300, 2056, 264, BF, "gelu", 5, [100, 300]), (1000, 512, 1032, BF, "silu", 0, None),
    (2100, 1024, 2048, BF, None, 64, [2100]), (600, 8192, 512, BF, None, 0, None), (70, 264, 72, F32, "gelu", 0, None),
    (551, 256, 1024, F32, "silu", 64, [551])], ids=case_id)
def test_training_graph(T, K, N, dt, act, text, ends):
    body, inputs, outputs = training(T, K, N, dt, act, text, ends)
    replays(body, inputs, outputs)


@pytest.mark.parametrize("T,K,N,dt,act,coded", [
    (4, 512, 272, BF, "silu", False), (40, 512, 272, BF, "silu", True), (40, 512, 272, F32, "gelu", False), (300, 1040, 528, BF, "gelu", True), (200, 1040, 272, BF, "silu", True),
    (900, 4112, 400, BF, None, False), (2000, 528, 2048, BF, "silu", False), (700, 272, 1040, F32, "gelu", False), (200, 4112, 64, F32, None, False)], ids=case_id)
def test_fp8_graph(T, K, N, dt, act, coded):
    d = {"w": empty(N, K).normal_(), "b": empty(N, dtype=dt).normal_()}
    if act:
        d.update(w_gate=empty(N, K).normal_().mul_(K ** -0.5), b_gate=empty(N, dtype=dt).normal_())
    plan, cud, x = hilo.linear_weights_fp8([hilo.quantize_block_weights(**d)]), cu_of(T // 3, T), empty(T, K, dtype=dt).normal_()
    out = empty(T, N, dtype=U8 if coded else dt)
    scale = empty(T, hilo.scale_stride(N), dtype=U8) if coded else None
    ws = bytes_of(hilo.hilo_linear_fp8_workspace_bytes(T, K, N, act is not None))
    replays(lambda: hilo.hilo_linear_fp8(plan, x, out, cud, out_scale=scale, act=ACTS[act], workspace=ws), [x], [out] + ([scale] if coded else []))


def test_two_streams():
    """Two passes at once, each with buffers and a workspace of its own, on current streams and on one given: the bits of one
    after the other."""
    a, _, outs_a = training(1500, 512, 1032, BF, "silu", 30, [700, 1500])
    b, _, outs_b = training(700, 2048, 520, BF, None)
    a(), b()
    torch.cuda.synchronize()
    want = [t.clone() for t in outs_a + outs_b]
    s, t = torch.cuda.Stream(), torch.cuda.Stream()
    for r in range(3):
        for o in outs_a + outs_b:
            o.zero_()
        torch.cuda.synchronize()
        with torch.cuda.stream(s):
            a()
        b(stream=t)
        torch.cuda.synchronize()
        for i, (x, y) in enumerate(zip(outs_a + outs_b, want)):
            assert torch.equal(x, y), (r, i)


# ------------------------------------------------------------------------------- ends of the ranges

@pytest.mark.parametrize("dt", [BF, F32], ids=case_id)
@pytest.mark.parametrize("rows", [0, 10, 200])
def test_no_rows_in_use(dt, rows):
    """Buffers of `rows` rows none of which is in use: outputs are left alone, gradients are zero."""
    K, N, cud = 64, 136, cu_of(0, 0)
    g = torch.Generator().manual_seed(1)
    w = cuda(weights(g, 2, N, K, dt, True, True))
    plan, x, nan = hilo.linear_weights(w), empty(rows, K, dtype=dt), float("nan")
    x.fill_(nan)
    out, pre, dx = empty(rows, N, dtype=dt).fill_(7), empty(rows, 2, N, dtype=dt).fill_(7), empty(rows, K, dtype=dt).fill_(7)
    ws = bytes_of(max(f(dt, rows, K, N, 2, True) for f in (hilo.hilo_linear_workspace_bytes, hilo.hilo_linear_backward_workspace_bytes)))
    hilo.hilo_linear(plan, x, out, cud, act=hilo.ACT_GELU, pre=pre, workspace=ws)
    for shared in (False, True):
        got = [{k: torch.full_like(v, 7.0) for k, v in d.items()} for d in (w[:1] if shared else w)]
        hilo.hilo_linear_backward(plan, x, empty(rows, 2, N, dtype=dt).fill_(nan), empty(rows, N, dtype=dt).fill_(nan), dx, hilo.linear_grads(got), cud,
                                  act=hilo.ACT_GELU, workspace=ws)
        assert not any(t.any() for d in got for t in d.values())
    codes, scales = empty(rows, N, dtype=U8).fill_(7), empty(rows, hilo.scale_stride(N), dtype=U8).fill_(7)
    k8, n8 = 64, 144
    d = {k: empty(n8, k8).normal_() for k in ("w", "w_gate")}
    w8, h8, s8 = hilo.linear_weights_fp8([hilo.quantize_block_weights(**d)]), empty(rows, n8, dtype=U8).fill_(7), empty(rows, 4, dtype=U8).fill_(7)
    hilo.hilo_linear_fp8(w8, x, h8, cud, out_scale=s8, act=hilo.ACT_GELU, workspace=bytes_of(hilo.hilo_linear_fp8_workspace_bytes(rows, k8, n8, True)))
    for t in (out, pre, dx, h8, s8):
        assert (t == 7).all()


@pytest.mark.parametrize("dt", [BF, F32], ids=case_id)
def test_many_samples(dt):
    """4096 samples, most of a row, some empty, some longer: forward and backward."""
    g = torch.Generator().manual_seed(2)
    n = torch.randint(0, 3, (4096,), generator=g)
    n[torch.randint(0, 4096, (3,), generator=g)] = 150
    cu, K, N = pack(n.tolist(), 1), 40, 72
    T = cu[-1]
    ws, x = weights(g, 2, N, K, dt, True, True), torch.randn(T, K, generator=g).to(dt)
    dout, pre = torch.randn(T, N, generator=g).to(dt), torch.randn(T, 2, N, generator=g).to(dt)
    plan, cud, out = hilo.linear_weights(cuda(ws)), cu_of(*cu[1:]), empty(T, N, dtype=dt)
    work = bytes_of(max(f(dt, T, K, N, 4096, True) for f in (hilo.hilo_linear_workspace_bytes, hilo.hilo_linear_backward_workspace_bytes)))
    hilo.hilo_linear(plan, x.cuda(), out, cud, 1, act=hilo.ACT_SILU, workspace=work)
    dx, got = empty(T, K, dtype=dt), cuda(ws)
    hilo.hilo_linear_backward(plan, x.cuda(), pre.cuda(), dout.cuda(), dx, hilo.linear_grads(got), cud, 1, act=hilo.ACT_SILU, workspace=work)
    ulp = 2.0 ** -23
    (u, su), (v, sv) = (P.affine(x.to(F64), ws, p, cu, 1) for p in ("", "_gate"))
    want, off = P.gated("silu", v, u, (K + 2) * ulp * sv, (K + 2) * ulp * su, dt is BF)
    near(out, want, off + HALF[dt] * (want.abs() + off), "out")
    (wx, bx), grads = P.backward(x.to(F64), ws, pre.to(F64), dout.to(F64), "silu", cu, 1, HALF[dt], False)
    near(dx, wx, bx, "dx")
    for k in range(2):
        for name, t in got[k].items():
            near(t, *grads[k][name], name)


def test_offsets_past_32_bits():
    """Buffers of more than 2^32 bytes, the rows in use at their end and start: tiles, few rows' lookups and gradients."""
    T, K, N = 530000, 16, 4096 + 8
    x, out, pre = empty(T, K, dtype=BF).normal_(), empty(T, N, dtype=BF), empty(T, 2, N, dtype=BF)
    w = [{k: empty(N, K, dtype=BF).normal_() for k in ("w", "w_gate")}]
    plan, cud = hilo.linear_weights(w), cu_of(T)
    ws = bytes_of(hilo.hilo_linear_backward_workspace_bytes(BF, T, K, N, 1, True))
    hilo.hilo_linear(plan, x, out, cud, act=hilo.ACT_SILU, pre=pre, workspace=ws)
    for a, b in ((0, 50), (T // 2, T // 2 + 50), (T - 50, T)):
        xd, wd = x[a:b].double(), {k: v.double() for k, v in w[0].items()}
        u, v = xd @ wd["w"].T, xd @ wd["w_gate"].T
        su, sv = xd.abs() @ wd["w"].abs().T, xd.abs() @ wd["w_gate"].abs().T
        want, off = P.gated("silu", v, u, (K + 2) * 2.0 ** -23 * sv, (K + 2) * 2.0 ** -23 * su, True)
        near(out[a:b], want.cpu(), (off + HALF[BF] * (want.abs() + off)).cpu(), "out")
    # gradients of a dout that is zero but for a few rows at both ends: those rows' sums
    dout, dx = torch.zeros_like(out), empty(T, K, dtype=BF)
    rows = torch.tensor([0, 1, T // 2, T - 2, T - 1], device="cuda")
    dout[rows] = torch.randn(5, N, device="cuda").to(BF)
    got = [{k: torch.empty_like(v) for k, v in w[0].items()}]
    hilo.hilo_linear_backward(plan, x, pre, dout, dx, hilo.linear_grads(got), cud, act=hilo.ACT_SILU, workspace=ws)
    sub = [t[rows].cpu().to(F64) for t in (x, pre, dout)]
    (wx, bx), grads = P.backward(sub[0], [{k: v.cpu() for k, v in w[0].items()}], sub[1], sub[2], "silu", [0, 5], 0, HALF[BF], True)
    near(dx[rows], wx, bx, "dx")
    mask = torch.ones(T, dtype=torch.bool, device="cuda")
    mask[rows] = False
    assert not dx[mask].any()
    for name, t in got[0].items():
        near(t, *grads[0][name], name)


@pytest.mark.parametrize("dt", [BF, F32], ids=case_id)
@pytest.mark.parametrize("T", [20, 300])
def test_values_that_are_not_finite(dt, T):
    """A row of x that holds NaN or an infinity makes its own outputs so and no others; codes of it are NaN."""
    K, N, bad = 272, 144, [3, 17]
    x, w = empty(T, K, dtype=dt).normal_(), [{k: empty(N, K, dtype=dt).normal_() for k in ("w", "w_gate")}]
    x[bad[0], 200], x[bad[1], 5] = float("nan"), float("inf")
    out, cud, others = empty(T, N, dtype=dt), cu_of(T), [i for i in range(T) if i not in bad]
    ws = bytes_of(max(hilo.hilo_linear_workspace_bytes(dt, T, K, N, 1, True), hilo.hilo_linear_fp8_workspace_bytes(T, K, N, True)))
    hilo.hilo_linear(hilo.linear_weights(w), x, out, cud, act=hilo.ACT_SILU, workspace=ws)
    assert out[others].isfinite().all() and not out[bad].isfinite().any()
    w8 = hilo.linear_weights_fp8([hilo.quantize_block_weights(w[0]["w"], None, w[0]["w_gate"])])
    hilo.hilo_linear_fp8(w8, x, out, cud, act=hilo.ACT_SILU, workspace=ws)
    assert out[others].isfinite().all() and out[bad].isnan().all()
    h, s = empty(T, N, dtype=U8), empty(T, hilo.scale_stride(N), dtype=U8)
    hilo.hilo_linear_fp8(w8, x, h, cud, out_scale=s, act=hilo.ACT_SILU, workspace=ws)
    v = P.decode(h.cpu(), s.cpu(), 1)
    assert v[others].isfinite().all() and v[bad].isnan().all()
    # and read again as codes: FP8 tiles and the others
    w2 = hilo.linear_weights_fp8([hilo.quantize_block_weights(empty(K, N).normal_())])
    y = empty(T, K, dtype=dt)
    hilo.hilo_linear_fp8(w2, h, y, cud, x_scale=s, workspace=bytes_of(hilo.hilo_linear_fp8_workspace_bytes(T, N, K)))
    assert y[others].isfinite().all() and y[bad].isnan().all()


@pytest.mark.parametrize("act", ["silu", "gelu"])
@pytest.mark.parametrize("dt", [BF, F32], ids=case_id)
def test_far_gates(act, dt):
    """Gates far out: act(g) is 0 or g, its slope 0 or 1, and nothing overflows on the way."""
    far = torch.tensor([1e4, -1e4, 1e15, -1e15, 3e30, -3e30, 100.0, -100.0], device="cuda")
    T, K, N, cud = 1, 8, 8, cu_of(1)
    w = {"w": torch.zeros(N, K), "b": torch.full((N,), 2.0), "w_gate": torch.zeros(N, K), "b_gate": far.cpu()}
    plan = hilo.linear_weights(cuda([{k: v.to(dt) for k, v in w.items()}]))
    x, out, pre = torch.ones(T, K, dtype=dt, device="cuda"), empty(T, N, dtype=dt), empty(T, 2, N, dtype=dt)
    ws = bytes_of(max(f(dt, T, K, N, 1, True) for f in (hilo.hilo_linear_workspace_bytes, hilo.hilo_linear_backward_workspace_bytes)))
    hilo.hilo_linear(plan, x, out, cud, act=ACTS[act], pre=pre, workspace=ws)
    g = far.to(dt).float()
    assert torch.equal(out[0].float(), torch.where(g > 0, 2 * g, torch.zeros_like(g)))
    dout, db = torch.ones(T, N, dtype=dt, device="cuda"), [{"b": empty(N, dtype=dt), "b_gate": empty(N, dtype=dt)}]
    hilo.hilo_linear_backward(plan, x, pre, dout, None, hilo.linear_grads(db), cud, act=ACTS[act], workspace=ws)
    assert torch.equal(db[0]["b_gate"].float(), 2.0 * (g > 0)) and torch.equal(db[0]["b"].float(), torch.where(g > 0, g, torch.zeros_like(g)))


# T, N and whether codes leave, for each form of an FP8 product: few rows with and without quantisation in the product, FP8 tiles,
# widened rows, float32 tiles cut along k
FORMS = [(BF, 1, 144, False), (BF, 4, 144, False), (BF, 4, 144, True), (BF, 16, 144, False), (BF, 40, 144, False), (F32, 4, 144, False), (F32, 40, 144, True),
         (BF, 300, 144, False), (F32, 300, 1552, False), (BF, 300, 784, True), (F32, 300, 784, True), (F32, 300, 144, False), (BF, 100, 144, True)]


def gate_and_up(dt, N, K, **kw):
    d = hilo.quantize_block_weights(empty(N, K).normal_(), empty(N, dtype=dt).normal_(), empty(N, K).normal_(), empty(N, dtype=dt).normal_())
    return dict(d, **kw)


def gated_rows(plan, x, dt, T, K, N, coded, **kw):
    """Outputs of a product with a gate in float64, of codes what they stand for."""
    out, scale = empty(T, N, dtype=U8 if coded else dt), empty(T, hilo.scale_stride(N), dtype=U8) if coded else None
    hilo.hilo_linear_fp8(plan, x, out, cu_of(T), act=hilo.ACT_SILU, out_scale=scale, workspace=bytes_of(hilo.hilo_linear_fp8_workspace_bytes(T, K, N, True)), **kw)
    return P.decode(out.cpu(), scale.cpu(), 1) if coded else out.cpu().to(F64)


@pytest.mark.parametrize("bad", [float("nan"), float("inf"), -float("inf")])
@pytest.mark.parametrize("dt,T,N,coded", FORMS, ids=case_id)
def test_blocks_that_are_not_finite(dt, T, N, coded, bad):
    """A block of x that holds NaN or an infinity has NaN for codes and scale: the row's outputs are NaN in every form."""
    K, row = 272, T // 2
    x = empty(T, K, dtype=dt).normal_()
    x[row, 128:256] = 0
    x[row, 200] = bad
    v = gated_rows(hilo.linear_weights_fp8([gate_and_up(dt, N, K)]), x, dt, T, K, N, coded)
    others = [i for i in range(T) if i != row]
    assert v[row].isnan().all() and v[others].isfinite().all()


@pytest.mark.parametrize("dt,T,N,coded", FORMS, ids=case_id)
def test_scales_of_nan(dt, T, N, coded):
    """A scale of 255 makes its block NaN whatever its codes are, zeros too: of a row its outputs, of W those of its 128 columns."""
    K = 272
    codes, scales = empty(T, K, dtype=U8), empty(T, hilo.scale_stride(K), dtype=U8)
    hilo.hilo_quantize_blocks(empty(T, K, dtype=dt).normal_(), codes, scales)
    d = gate_and_up(dt, N, K)
    good = gated_rows(hilo.linear_weights_fp8([d]), codes, dt, T, K, N, coded, x_scale=scales)
    assert good.isfinite().all()
    for zero in (False, True):
        c, s, row = codes.clone(), scales.clone(), T // 2
        s[row, 1] = 255
        if zero:
            c[row, 128:256] = 0
        v = gated_rows(hilo.linear_weights_fp8([d]), c, dt, T, K, N, coded, x_scale=s)
        others = [i for i in range(T) if i != row]
        assert v[row].isnan().all(), ("x", zero)
        assert torch.equal(v[others], good[others])
        for part in ("", "_gate"):
            e = dict(d, **{k + part: d[k + part].clone() for k in ("w", "s")})
            e["s" + part][0, 2] = 255  # of the last block, 16 wide
            if zero:
                e["w" + part][:128, 256:] = 0
            v = gated_rows(hilo.linear_weights_fp8([e]), codes, dt, T, K, N, coded, x_scale=scales)
            assert v[:, :128].isnan().all(), ("w" + part, zero)
            assert torch.equal(v[:, 128:], good[:, 128:])


@pytest.mark.parametrize("rows,K,N", [(3000, 1040, 272), (5000, 144, 2064), (300, 4112, 528)], ids=case_id)
@pytest.mark.parametrize("dt", [BF, F32], ids=case_id)
def test_few_rows_of_large_buffers(dt, rows, K, N):
    """Buffers of many rows of which few are in use, as where only the device knows how many a selection left: the plans go by
    the buffers, the sums by the rows, and what lies behind is left alone."""
    g = torch.Generator().manual_seed(rows)
    cu, text = pack([30, 0, 24], 5), 5
    T, cud, ulp = cu[-1], cu_of(*cu[1:]), 2.0 ** -23
    tail = lambda t, v: torch.cat([t, torch.full((rows - T, *t.shape[1:]), v, dtype=t.dtype)]).cuda()  # noqa: E731
    ws, nan = weights(g, 2, N, K, dt, True, True), float("nan")
    x, dout, pre = (torch.randn(T, *s, generator=g).to(dt) for s in ((K,), (N,), (2, N)))
    plan, out, dx, got = hilo.linear_weights(cuda(ws)), empty(rows, N, dtype=dt).fill_(7), empty(rows, K, dtype=dt).fill_(7), cuda(ws)
    work = bytes_of(max(f(dt, rows, K, N, 3, True) for f in (hilo.hilo_linear_workspace_bytes, hilo.hilo_linear_backward_workspace_bytes))).fill_(0xff)
    hilo.hilo_linear(plan, tail(x, nan), out, cud, text, act=hilo.ACT_SILU, workspace=work)
    hilo.hilo_linear_backward(plan, tail(x, nan), tail(pre, nan), tail(dout, nan), dx, hilo.linear_grads(got), cud, text, act=hilo.ACT_SILU, workspace=work)
    (u, su), (v, sv) = (P.affine(x.to(F64), ws, p, cu, text) for p in ("", "_gate"))
    want, off = P.gated("silu", v, u, (K + 2) * ulp * sv, (K + 2) * ulp * su, dt is BF)
    near(out[:T], want, off + HALF[dt] * (want.abs() + off), "out")
    (wx, bx), grads = P.backward(x.to(F64), ws, pre.to(F64), dout.to(F64), "silu", cu, text, HALF[dt], False)
    near(dx[:T], wx, bx, "dx")
    for k in range(2):
        for name, t in got[k].items():
            near(t, *grads[k][name], f"{name} of {k}")
    assert (out[T:] == 7).all() and (dx[T:] == 7).all()
    # FP8, rows and codes out, against the same rows in buffers that they fill, within the form's float32 sums
    q = [hilo.quantize_block_weights(d["w"], d["b"], d["w_gate"], d["b_gate"]) for d in cuda([{k: t.to(F32 if k[0] == "w" else dt) for k, t in d.items()} for d in ws])]
    w8 = hilo.linear_weights_fp8(q)
    xq, kx = P.quantize(x.to(F64), 1)
    exact, kw = [{} for _ in ws], [{} for _ in ws]
    for k in range(2):
        for p in ("", "_gate"):
            exact[k]["w" + p], kw[k]["w" + p] = P.quantize(ws[k]["w" + p].to(F64), 128)
            exact[k]["b" + p] = ws[k]["b" + p]
    v, e = {}, {}
    for p in ("", "_gate"):
        v[p], s = P.affine(xq, exact, p, cu, text)
        e[p] = (K + 2) * ulp * s + (P.cut(xq, kx, exact, kw, p, cu, text) if dt is BF else 0)
    want, off = P.gated("silu", v["_gate"], v[""], e["_gate"], e[""], True)
    work = bytes_of(hilo.hilo_linear_fp8_workspace_bytes(rows, K, N, True)).fill_(0xff)
    out.fill_(7)
    hilo.hilo_linear_fp8(w8, tail(x, nan), out, cud, text, act=hilo.ACT_SILU, workspace=work)
    near(out[:T], want, off + HALF[dt] * (want.abs() + off), "FP8 out")
    h, hs = empty(rows, N, dtype=U8).fill_(9), empty(rows, hilo.scale_stride(N), dtype=U8).fill_(9)
    hilo.hilo_linear_fp8(w8, tail(x, nan), h, cud, text, act=hilo.ACT_SILU, out_scale=hs, workspace=work)
    scale = torch.exp2(hs[:T, :-(-N // 128)].cpu().to(F64) - 127).repeat_interleave(128, 1)[:, :N]
    near(P.decode(h[:T].cpu(), hs[:T].cpu(), 1), want, off + 2.0 ** -4 * (want.abs() + off) + 2.0 ** -10 * scale, "codes")
    assert (out[T:] == 7).all() and (h[T:] == 9).all() and (hs[T:] == 9).all()


@pytest.mark.parametrize("dt,T,N,whole", [(BF, 4, 16, False), (BF, 40, 16, False), (F32, 40, 16, False), (F32, 300, 16, False), (F32, 300, 4112, False), (BF, 300, 16, True)],
                         ids=case_id)
def test_values_that_float32_does_not_hold(dt, T, N, whole):
    """Codes of 2^127, 2^128 and 2^135 times 2^-100: bf16 out above 64 rows multiplies them as they are, others as infinities."""
    K = 128
    codes, scales = empty(T, K, dtype=U8).fill_(0), empty(T, 4, dtype=U8).fill_(127)
    codes[:, 0] = 0x38  # 1
    for row, (code, scale) in enumerate(((0x70, 247), (0x78, 247), (0x78, 254))):  # 128 and 256
        codes[row, 0], scales[row, 0] = code, scale
    w = {"w": empty(N, K, dtype=U8).fill_(0x38), "s": empty(-(-N // 128), 4, dtype=U8).fill_(27)}
    out = empty(T, N, dtype=dt)
    hilo.hilo_linear_fp8(hilo.linear_weights_fp8([w]), codes, out, cu_of(T), x_scale=scales, workspace=bytes_of(hilo.hilo_linear_fp8_workspace_bytes(T, K, N)))
    inf = float("inf")
    for row, v in enumerate((2.0 ** 27, 2.0 ** 28 if whole else inf, 2.0 ** 35 if whole else inf, 2.0 ** -100)):
        assert (out[row] == v).all(), row
