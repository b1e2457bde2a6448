"""The products of a feed-forward on the host: what the library and the binding refuse before anything is enqueued, and the
float64 oracle against other ways to the same values (CPU only)."""
import ctypes
import gc
import math
import os
import random
import subprocess
import weakref

import product_schedule
import pytest
import torch

from oracle import hilo_products as P
from paper_2606_13898_amd import build, hilo
from test_operators import DEVICE, DTYPE, F, NULL, PARAM, SHAPE, WORKSPACE, OnDevice, built, no_gpu

F64 = torch.float64
G = 1 << 40  # bytes of workspace, enough for anything


def pair(struct, **kw):
    """Two of `struct`, every field F but those in kw (one value, or one for each stream)."""
    arr = (struct * 2)()
    for k in range(2):
        for name, _ in struct._fields_:
            v = kw.get(name, F)
            setattr(arr[k], name, v[k] if isinstance(v, tuple) else v)
    return arr


def plain(struct, **kw):
    return pair(struct, **dict(dict(w_gate=None, b_gate=None, **({"s_gate": None} if struct is hilo.hilo_linear_w_fp8 else {})), **kw))


GATED = hilo.hilo_linear_w
SILU, GELU, NONE = hilo.ACT_SILU, hilo.ACT_GELU, hilo.ACT_NONE


# ---------------------------------------------------------------------------------------- refusals

def linear(w=None, dtype=hilo.BF16, x=F, out=F, pre=None, rows=100, k=64, n=64, act=SILU, batch=1, text=0, cu=F, ws=F * 16, bytes=G):
    w = pair(hilo.hilo_linear_w) if w is None else w
    return hilo.lib().hilo_linear(dtype, w, x, out, pre, rows, k, n, act, batch, text, cu, ws, bytes, None)


COMMON = [(dict(dtype=2), DTYPE), (dict(rows=-1), SHAPE), (dict(rows=1 << 24), SHAPE), (dict(k=0), SHAPE), (dict(k=65544), SHAPE),
          (dict(n=0), SHAPE), (dict(n=65544), SHAPE), (dict(batch=0), SHAPE), (dict(batch=4097), SHAPE), (dict(text=-1), SHAPE),
          (dict(batch=2, text=51), SHAPE), (dict(act=3), PARAM), (dict(act=-1), PARAM), (dict(act=NONE), PARAM), (dict(cu=None), NULL),
          (dict(x=F + 8), PARAM), (dict(ws=F + 128), PARAM)]


@built
@pytest.mark.parametrize("kw,status", COMMON + [
    (dict(k=60), SHAPE), (dict(n=60), SHAPE), (dict(x=None), NULL), (dict(out=None), NULL), (dict(out=F + 8), PARAM),
    (dict(pre=F + 8), PARAM), (dict(ws=None), NULL), (dict(bytes=1000), WORKSPACE), (dict(rows=0, x=None, out=None), 0)], ids=str)
def test_linear_refusals(kw, status):
    assert linear(**kw) == status


@built
@pytest.mark.parametrize("w,kw,status", [
    (dict(w=None), {}, NULL), (dict(w=(F, None)), dict(text=1), NULL), (dict(w=(F, None)), dict(rows=0), 0), (dict(w=F + 8), {}, PARAM),
    (dict(b=F + 2), {}, PARAM), (dict(w_gate=F + 8), {}, PARAM), (dict(b_gate=F + 8), {}, PARAM),
    (dict(w_gate=(F, None)), dict(text=1), NULL), (dict(w_gate=(None, F)), dict(text=1, act=NONE), NULL),
    (dict(w_gate=None), {}, PARAM), (dict(w_gate=None), dict(act=NONE, pre=F), PARAM)], ids=str)
def test_linear_weight_refusals(w, kw, status):
    assert linear(pair(hilo.hilo_linear_w, **w), **kw) == status


def backward(w=None, g=None, dtype=hilo.BF16, x=F, pre=F, dout=F, dx=F, rows=100, k=64, n=64, act=SILU, batch=1, text=0, cu=F,
             ws=F * 16, bytes=G):
    w = pair(hilo.hilo_linear_w) if w is None else w
    g = pair(hilo.hilo_linear_grads) if g is None else g
    return hilo.lib().hilo_linear_backward(dtype, w, x, pre, dout, dx, g or None, rows, k, n, act, batch, text, cu, ws, bytes, None)


@built
@pytest.mark.parametrize("kw,status", COMMON + [
    (dict(k=60), SHAPE), (dict(n=60), SHAPE), (dict(x=None), NULL), (dict(dout=None), NULL), (dict(pre=None), NULL), (dict(pre=F + 8), PARAM),
    (dict(dout=F + 8), PARAM), (dict(dx=F + 8), PARAM), (dict(ws=None), NULL), (dict(bytes=1000), WORKSPACE),
    (dict(rows=0, x=None, dout=None, pre=None, g=False), 0)], ids=str)
def test_backward_refusals(kw, status):
    assert backward(**kw) == status


@built
@pytest.mark.parametrize("g,status", [(dict(w=F + 8), PARAM), (dict(b=F + 8), PARAM), (dict(w_gate=(None, F + 8)), PARAM), (dict(b_gate=F + 4), PARAM)], ids=str)
def test_backward_gradient_refusals(g, status):
    assert backward(g=pair(hilo.hilo_linear_grads, **g)) == status
    # without a gate: none of its gradients
    w = plain(hilo.hilo_linear_w)
    assert backward(w, plain(hilo.hilo_linear_grads, w_gate=(None, F)), act=NONE) == PARAM
    assert backward(w, plain(hilo.hilo_linear_grads, b_gate=F), act=NONE) == PARAM


@built
@pytest.mark.parametrize("args,status", [
    ((2, F, 4, 64, 1, None, F, F), DTYPE), ((1, None, 4, 64, 1, None, F, F), NULL), ((1, F, 4, 64, 1, None, None, F), NULL),
    ((1, F, 4, 64, 1, None, F, None), NULL), ((1, F, -1, 64, 1, None, F, F), SHAPE), ((1, F, 1 << 24, 64, 1, None, F, F), SHAPE),
    ((1, F, 4, 8, 1, None, F, F), SHAPE), ((1, F, 4, 72, 1, None, F, F), SHAPE), ((1, F, 4, 65552, 1, None, F, F), SHAPE),
    ((1, F, 4, 64, 0, None, F, F), PARAM), ((1, F, 4, 64, 64, None, F, F), PARAM), ((1, F + 8, 4, 64, 1, None, F, F), PARAM),
    ((1, F, 4, 64, 1, None, F + 4, F), PARAM), ((1, None, 0, 64, 128, None, None, None), 0)], ids=str)
def test_quantize_refusals(args, status):
    assert hilo.lib().hilo_quantize_blocks(*args, None) == status


def fp8(w=None, dtype=hilo.BF16, x=F, xs=F, out=F, os=None, rows=100, k=64, n=64, act=SILU, batch=1, text=0, cu=F, ws=F * 16, bytes=G):
    w = pair(hilo.hilo_linear_w_fp8) if w is None else w
    return hilo.lib().hilo_linear_fp8(dtype, w, x, xs, out, os, rows, k, n, act, batch, text, cu, ws, bytes, None)


@built
@pytest.mark.parametrize("kw,status", COMMON + [
    (dict(k=72), SHAPE), (dict(n=72), SHAPE), (dict(x=None), NULL), (dict(out=None), NULL), (dict(out=F + 8), PARAM), (dict(xs=F + 4), PARAM),
    (dict(os=F + 4), PARAM), (dict(ws=None), NULL), (dict(bytes=1000), WORKSPACE), (dict(rows=0, x=None, out=None), 0)], ids=str)
def test_fp8_refusals(kw, status):
    assert fp8(**kw) == status


@built
@pytest.mark.parametrize("w,kw,status", [
    (dict(w=None), {}, NULL), (dict(s=None), {}, NULL), (dict(s_gate=None), {}, NULL), (dict(s=(F, None)), dict(text=1), NULL),
    (dict(w=F + 8), {}, PARAM), (dict(s=F + 4), {}, PARAM), (dict(s_gate=F + 4), {}, PARAM), (dict(b=F + 8), {}, PARAM),
    (dict(w_gate=None), dict(act=NONE, os=F), PARAM), (dict(w_gate=(F, None)), dict(text=1), NULL)], ids=str)
def test_fp8_weight_refusals(w, kw, status):
    assert fp8(pair(hilo.hilo_linear_w_fp8, **w), **kw) == status


@built
@no_gpu
def test_good_calls_reach_the_device():
    assert linear() == linear(pre=F, text=50) == linear(plain(hilo.hilo_linear_w), act=NONE) == linear(act=GELU) == DEVICE
    assert linear(pair(hilo.hilo_linear_w, b=None, b_gate=None), rows=64, ws=None, bytes=0) == DEVICE  # few rows need no workspace
    assert linear(pair(hilo.hilo_linear_w, w=(F, None), w_gate=(F, None))) == DEVICE                   # stream 1 is not looked at
    assert backward() == backward(g=False) == backward(dx=None, text=50) == backward(rows=0, x=None, dout=None, pre=None) == DEVICE
    assert backward(plain(hilo.hilo_linear_w), plain(hilo.hilo_linear_grads), act=NONE, pre=None) == DEVICE
    assert backward(g=pair(hilo.hilo_linear_grads, w=None, w_gate=None), x=None) == DEVICE
    assert fp8() == fp8(xs=None) == fp8(os=F) == fp8(plain(hilo.hilo_linear_w_fp8), act=NONE, text=50) == DEVICE
    assert hilo.lib().hilo_quantize_blocks(0, F, 4, 64, 128, None, F, F, None) == DEVICE


@built
def test_workspace_bytes():
    L = hilo.lib()
    for bad in ((2, 8, 64, 64, 1, 0), (1, -1, 64, 64, 1, 0), (1, 8, 60, 64, 1, 0), (1, 8, 64, 60, 1, 0), (1, 8, 64, 64, 0, 0), (1, 8, 64, 64, 4097, 0)):
        assert L.hilo_linear_workspace_bytes(*bad) == 0 and L.hilo_linear_backward_workspace_bytes(*bad) == 0
    for bad in ((-1, 64, 64, 0), (8, 72, 64, 0), (8, 64, 72, 0), (8, 65552, 64, 0)):
        assert L.hilo_linear_fp8_workspace_bytes(*bad) == 0
    assert hilo.hilo_linear_workspace_bytes(torch.bfloat16, 64, 1024, 1024, 1, True) == 0
    # more of anything never needs less
    for dt in (torch.float32, torch.bfloat16):
        for gated in (False, True):
            sizes = [hilo.hilo_linear_backward_workspace_bytes(dt, r, 256, 512, 2, gated) for r in (65, 1000, 20000)]
            assert sizes == sorted(sizes) and sizes[0] > 0
    for f in (hilo.hilo_linear_workspace_bytes, hilo.hilo_linear_backward_workspace_bytes):
        assert f(torch.float16, 64, 64, 64, 1) == 0 and f(torch.bfloat16, 64, (1 << 32) + 64, 64, 1) == f(torch.bfloat16, 64, 64, 64, 1 << 33) == 0
    assert hilo.hilo_linear_fp8_workspace_bytes(64, (1 << 32) + 64, 64) == 0


# ----------------------------------------------------------------------------------------- binding

BF, F32, U8, I32 = torch.bfloat16, torch.float32, torch.uint8, torch.int32


def weights(n=16, k=32, dt=BF, gate=True, dev=0, **kw):
    d = {"w": OnDevice(dt, n, k, dev=dev), "b": OnDevice(dt, n, dev=dev)}
    if gate:
        d.update(w_gate=OnDevice(dt, n, k, dev=dev), b_gate=OnDevice(dt, n, dev=dev))
    return dict(d, **kw)


@built
@pytest.mark.parametrize("kw", [dict(w=None), dict(w=OnDevice(BF, 16)), dict(w=OnDevice(torch.float16, 16, 32)), dict(w_gate=OnDevice(BF, 16, 40)),
                                dict(w_gate=OnDevice(F32, 16, 32)), dict(b=OnDevice(F32, 16)), dict(b=OnDevice(BF, 17)), dict(b_gate=OnDevice(BF, 16, 1)),
                                dict(w=OnDevice(BF, 16, 32, dev=1)), dict(w=OnDevice(BF, 16, 32, contiguous=False)), dict(w=OnDevice(BF, 16, 32, dev=-1))], ids=str)
def test_weights_refuse(kw):
    with pytest.raises(ValueError):
        hilo.linear_weights([weights(**kw)])
    with pytest.raises(ValueError):
        hilo.linear_weights([weights(), weights(**kw)])
    with pytest.raises(ValueError):
        hilo.linear_weights([])


def call(f, **kw):
    """hilo_linear (f 0), its backward pass (1) or the FP8 product (2) of 8 rows on device 0 with kw changed."""
    a = dict(x=OnDevice(BF, 8, 32), out=OnDevice(BF, 8, 16), pre=OnDevice(BF, 8, 2, 16), dx=OnDevice(BF, 8, 32), cu=OnDevice(I32, 2), text=0, act=SILU,
             ws=OnDevice(U8, 1 << 30), xs=OnDevice(U8, 8, 4), os=OnDevice(U8, 8, 4), grads=None)
    a.update(kw)
    if f == 0:
        return hilo.hilo_linear(hilo.linear_weights([weights()]), a["x"], a["out"], a["cu"], a["text"], act=a["act"], pre=a["pre"], workspace=a["ws"], stream=0)
    if f == 1:
        g = hilo.linear_grads([weights()]) if a["grads"] is None else a["grads"]()
        return hilo.hilo_linear_backward(hilo.linear_weights([weights()]), a["x"], a["pre"], a["out"], a["dx"], g, a["cu"], a["text"], act=a["act"],
                                         workspace=a["ws"], stream=0)
    w = weights(dt=U8, b=OnDevice(BF, 16), b_gate=None, s=OnDevice(U8, 1, 4), s_gate=OnDevice(U8, 1, 4))
    return hilo.hilo_linear_fp8(hilo.linear_weights_fp8([w]), a["x"], a["out"], a["cu"], a["text"], x_scale=a["xs"], out_scale=a["os"], act=a["act"],
                                workspace=a["ws"], stream=0)


@built
@pytest.mark.parametrize("f,kw", [
    (0, dict(x=OnDevice(BF, 8, 40))), (0, dict(x=OnDevice(BF, 9, 32))), (0, dict(x=OnDevice(F32, 8, 32))), (0, dict(x=OnDevice(BF, 8, 32, dev=1))),
    (0, dict(x=OnDevice(BF, 8, 32, contiguous=False))), (0, dict(out=OnDevice(BF, 8, 24))), (0, dict(out=OnDevice(BF, 8, 16, dev=-1))),
    (0, dict(out=OnDevice(BF, 8, 16, dev=1))), (0, dict(pre=OnDevice(BF, 8, 32))), (0, dict(cu=OnDevice(torch.int64, 2))), (0, dict(cu=OnDevice(I32, 1))),
    (0, dict(ws=OnDevice(U8, 64, dev=1))), (0, dict(ws=OnDevice(U8, 64, contiguous=False))),
    (1, dict(x=OnDevice(BF, 8, 16))), (1, dict(pre=OnDevice(BF, 8, 16))), (1, dict(out=OnDevice(BF, 8, 32))), (1, dict(dx=OnDevice(BF, 8, 16))),
    (1, dict(grads=lambda: hilo.linear_grads([weights(k=40)]))), (1, dict(grads=lambda: hilo.linear_grads([weights(dt=F32)]))),
    (1, dict(grads=lambda: hilo.linear_grads([{"b": OnDevice(BF, 24)}]))), (1, dict(grads=lambda: hilo.linear_grads([{"b": OnDevice(BF, 16, dev=1)}]))),
    (2, dict(x=OnDevice(BF, 8, 32))), (2, dict(x=OnDevice(U8, 8, 32), xs=OnDevice(U8, 8, 1))), (2, dict(x=OnDevice(U8, 8, 32), out=OnDevice(BF, 8, 16))),
    (2, dict(x=OnDevice(U8, 8, 32), out=OnDevice(U8, 8, 16), os=None)), (2, dict(x=OnDevice(F32, 8, 32), xs=None, out=OnDevice(U8, 8, 16)))], ids=str)
def test_binding_refuses(f, kw, monkeypatch):
    monkeypatch.setattr(hilo, "_current_device", lambda: 0)
    with pytest.raises(ValueError):
        call(f, **kw)


@built
@pytest.mark.parametrize("f", [0, 1, 2])
@pytest.mark.parametrize("kw,status", [(dict(text=1 << 32), SHAPE), (dict(text=-1), SHAPE), (dict(act=1 << 32), PARAM), (dict(act=-1), PARAM)], ids=str)
def test_binding_keeps_sizes(f, kw, status, monkeypatch):
    monkeypatch.setattr(hilo, "_current_device", lambda: 0)
    with pytest.raises(hilo.HiloError) as e:
        call(f, **kw)
    assert e.value.status == status


@built
def test_fp8_weights_refuse():
    w = dict(w=OnDevice(U8, 16, 32), s=OnDevice(U8, 1, 4))
    for bad in (dict(w, s=None), dict(w, s=OnDevice(U8, 1, 8)), dict(w, s=OnDevice(F32, 1, 4)), dict(w, w_gate=OnDevice(U8, 16, 32)), dict(w, w=OnDevice(BF, 16, 32)),
                dict(w, b=OnDevice(torch.float16, 16))):
        with pytest.raises(ValueError):
            hilo.linear_weights_fp8([bad])
    with pytest.raises(hilo.HiloError):
        hilo.hilo_quantize_blocks(OnDevice(BF, 8, 32), OnDevice(U8, 8, 32), OnDevice(U8, 8, 4), 2)
    for codes, scales in ((OnDevice(U8, 8, 16), OnDevice(U8, 8, 4)), (OnDevice(U8, 8, 32), OnDevice(U8, 8, 1)), (OnDevice(torch.int8, 8, 32), OnDevice(U8, 8, 4))):
        with pytest.raises(ValueError):
            hilo.hilo_quantize_blocks(OnDevice(BF, 8, 32), codes, scales)


@built
@pytest.mark.parametrize("of,d", [(hilo.linear_weights, weights), (hilo.linear_grads, weights),
                                  (hilo.linear_weights_fp8, lambda: weights(dt=U8, b=OnDevice(BF, 16), b_gate=None, s=OnDevice(U8, 1, 4), s_gate=OnDevice(U8, 1, 4)))])
def test_tensors_are_kept(of, d):
    """Weights and gradients keep their tensors, not the caller's dicts, which may change afterwards."""
    ds = [d(), d()]
    kept = [weakref.ref(t) for e in ds for t in e.values() if t is not None]
    arr = of(ds)
    ds[0].clear()
    ds[1].update(w=None, b=OnDevice(BF, 16))
    gc.collect()
    assert all(r() is not None for r in kept) and arr is not None


@built
def test_host_tensors_are_refused():
    x = torch.zeros(8, 32, dtype=BF)
    with pytest.raises(ValueError):
        hilo.linear_weights([{"w": x}])
    with pytest.raises(ValueError):
        hilo.hilo_quantize_blocks(x, x, x)


# ------------------------------------------------------------------------------------------ oracle

@pytest.mark.parametrize("act", [None, "silu", "gelu"])
@pytest.mark.parametrize("shared", [False, True])
def test_oracle_backward_is_the_slope(act, shared):
    """The oracle's gradients against central differences of its forward pass."""
    g = torch.Generator().manual_seed(5)
    cu, text, k, n, step = [0, 4, 6, 9], 2, 3, 4, 1e-5
    parts = ("", "_gate") if act else ("",)
    ws = [{name + p: torch.randn(*((n, k) if name == "w" else (n,)), generator=g, dtype=F64) for p in parts for name in ("w", "b")}
          for _ in range(1 if shared else 2)]
    x, dout = torch.randn(9, k, generator=g, dtype=F64), torch.randn(9, n, generator=g, dtype=F64)

    def value(x, ws):
        u = P.affine(x, ws, "", cu, text)[0]
        if act:
            v = P.affine(x, ws, "_gate", cu, text)[0]
            u = P.act_slope(act, v)[0] * u
        return (u * dout).sum().item()

    pre = torch.stack([P.affine(x, ws, p, cu, text)[0] for p in ("_gate", "")], 1) if act else None
    (dx, _), grads = P.backward(x, ws, pre, dout, act, cu, text, 0.0, shared)

    def slope(t):
        d = torch.zeros_like(t)
        for i in range(t.numel()):
            old = t.view(-1)[i].item()
            t.view(-1)[i] = old + step
            up = value(x, ws)
            t.view(-1)[i] = old - step
            d.view(-1)[i] = (up - value(x, ws)) / (2 * step)
            t.view(-1)[i] = old
        return d

    torch.testing.assert_close(dx, slope(x), rtol=1e-6, atol=1e-7)
    for d, got in zip(ws, grads):
        for name, t in d.items():
            torch.testing.assert_close(got[name][0], slope(t), rtol=1e-6, atol=1e-7, msg=name)


def test_oracle_quantize():
    """Codes by hand, and those of torch's conversion."""
    v, k = P.quantize(torch.tensor([[448.0, 1.0, 17.0, 0.0], [449.0, 1.0, 0.0, -3.3]], dtype=F64), 1)
    assert k.tolist() == [[0], [1]] and v.tolist() == [[448.0, 1.0, 16.0, 0.0], [448.0, 1.0, 0.0, -3.25]]
    assert P.quantize(torch.zeros(3, 20, dtype=F64), 128)[1].tolist() == [[0]]
    x = torch.randn(300, 272, generator=torch.Generator().manual_seed(6))
    for rows in (1, 128):
        v, k = P.quantize(x.double(), rows)
        scale = torch.exp2(k).repeat_interleave(rows, 0)[:300].repeat_interleave(128, 1)[:, :272]
        assert torch.equal((x / scale.float()).to(torch.float8_e4m3fn).double() * scale, v)
        top = torch.nn.functional.pad(x.abs(), (0, 112, 0, -300 % rows)).view(-1, rows, 3, 128).amax((1, 3)).double()
        assert (448 * torch.exp2(k) >= top).all() and (448 * torch.exp2(k - 1) < top).all()


@pytest.mark.parametrize("act", ["silu", "gelu"])
def test_oracle_activations(act):
    g = torch.linspace(-30, 30, 241, dtype=F64)
    want = torch.nn.functional.silu(g) if act == "silu" else torch.nn.functional.gelu(g, approximate="tanh")
    torch.testing.assert_close(P.act_slope(act, g)[0], want, rtol=1e-12, atol=1e-14)
    assert P.act_slope(act, g)[1].abs().max() <= 1.13


# ------------------------------------------------------------------------------------------ plans

@pytest.mark.parametrize("kind, images, text, k, n, streams, parts, plan", product_schedule.SHAPES, ids=str)
def test_plan_of_shape(kind, images, text, k, n, streams, parts, plan):
    assert product_schedule.describe(kind, images, text, k, n, streams, parts, 3) == plan


def test_shapes_reach_every_plan():
    got = {(kind, parts, plan[0], plan[2] > 1) for kind, *_, parts, plan in product_schedule.SHAPES}
    assert got == {(kind, parts, tile, cut) for kind in range(4) for parts in (1, 2) for tile in product_schedule.TILES[kind] for cut in (False, True)}
    assert all(product_schedule.together(*shape, 3) for shape in product_schedule.TOGETHER)


@pytest.fixture(scope="module")
def library_plans(tmp_path_factory):
    """The library's plans of calls, by its own sources compiled for the host."""
    try:
        hipcc = build.hipcc()
    except RuntimeError:
        pytest.skip("no hipcc")
    exe = str(tmp_path_factory.mktemp("plans") / "plans")
    # the kernels stay without device code, which nothing here launches
    subprocess.run([hipcc, f"--offload-arch={build.ARCH}", "--offload-host-only", "-O1", "-std=c++17", "-w", "-I", build.CSRC, "-I", os.path.join(build.ROOT, "include"),
                    os.path.join(os.path.dirname(__file__), "product_plans.hip"), "-o", exe, "-Wl,--unresolved-symbols=ignore-all"], check=True, timeout=300)

    def plans(calls):
        """calls: (kind, image rows, text rows, in, out, streams, parts), 3 rows more in the buffers; kind 4: one launch for all gradients."""
        lines = []
        for kind, images, text, k, n, streams, parts in calls:
            segments, rows = product_schedule.segments(images, text, streams == 1), sum(images) + text * len(images) + 3
            if kind == 4:
                seen = len(images), text, 0
            else:
                nk = {product_schedule.OUT: -(-k // 64), product_schedule.DX: parts * -(-n // 64), product_schedule.FP8: -(-k // 128),
                      product_schedule.DW: max(sum(-(-m // 64) for m, s in segments if s == t) for t in range(streams))}[kind]
                seen = nk, *(sum(-(-m // bm) for m, _ in segments) for bm in (256, 128))
            lines.append(" ".join(map(str, (kind, rows, k, n, parts, streams, *seen))))
        out = subprocess.run([exe], input="\n".join(lines), capture_output=True, text=True, check=True, timeout=60).stdout.splitlines()
        assert len(out) == len(calls)
        return [tuple(map(int, line.split())) for line in out]

    return plans


def random_call(rng, kind):
    size = lambda lo, hi: int(lo * (hi / lo) ** rng.random())  # noqa: E731
    step, text = 16 if kind == product_schedule.FP8 else 8, rng.choice((0, size(1, 300)))
    images = [size(1, 9000) for _ in range(rng.randint(1, 4))]
    images[0] += 64
    return kind, images, text, step * size(1, 16384 // step), step * size(1, 16384 // step), 2 if text else 1, rng.randint(1, 2)


def test_model_is_the_library(library_plans):
    """product_schedule.py's plans are the library's: of its shapes, and of calls all over the range."""
    rng = random.Random(7)
    calls = [call[:7] for call in product_schedule.SHAPES] + [random_call(rng, i % 4) for i in range(2000)]
    for call, (tile, tiles, pieces) in zip(calls, library_plans(calls)):
        assert product_schedule.describe(*call, 3) == (product_schedule.TILES[call[0]][tile], tiles, pieces), call
    calls = [(4, *shape) for shape in product_schedule.TOGETHER] + [random_call(rng, 4) for _ in range(1000)]
    for call, (one,) in zip(calls, library_plans(calls)):
        assert product_schedule.together(*call[1:], 3) == bool(one), call
