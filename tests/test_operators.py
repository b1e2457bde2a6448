"""The rotary, sandwich-norm and int8 operators on the host: what the library and the binding refuse before anything is
enqueued, and the float64 oracle against other ways to the same values (CPU only)."""
import ctypes
import gc
import os
import re
import weakref

import numpy as np
import pytest
import torch

import linear_schedule
import norm_schedule
from oracle import hilo_operators as Q
from paper_2606_13898_amd import hilo

built = pytest.mark.skipif(not os.path.exists(hilo.LIB_PATH), reason="libhilo.so not built")
F = 0x1000  # aligned, never dereferenced: a refusal, or the missing device, ends the call
NULL, SHAPE, DTYPE, PARAM, WORKSPACE, DEVICE = 1, 2, 3, 4, 5, 6
no_gpu = pytest.mark.skipif(torch.cuda.is_available(), reason="a call that is not refused would run")


# ---------------------------------------------------------------------------------------- refusals

def rope(r=None, dtype=hilo.BF16, x=F, ldx=256, pos=F, rows=4, out=F, ldo=256, **kw):
    r = hilo.rotary(2, 128, (16, 24, 24)) if r is None else r
    for k, v in kw.items():
        if k in ("pairs", "base"):
            getattr(r, k)[0] = v
        else:
            setattr(r, k, v)
    return hilo.lib().hilo_rope(dtype, ctypes.byref(r), x, ldx, pos, rows, None, 0, out, ldo, None)


@built
@pytest.mark.parametrize("kw,status", [
    (dict(dtype=2), DTYPE), (dict(x=None), NULL), (dict(pos=None), NULL), (dict(out=None), NULL), (dict(heads=0), SHAPE),
    (dict(head_dim=127), SHAPE), (dict(head_dim=258, ldx=1000, ldo=1000), SHAPE), (dict(axes=0), SHAPE), (dict(axes=5), SHAPE),
    (dict(flags=4), PARAM), (dict(pairs=-1), PARAM), (dict(pairs=17), SHAPE), (dict(base=0.0), PARAM),
    (dict(base=float("nan")), PARAM), (dict(base=float("inf")), PARAM), (dict(rows=-1), SHAPE), (dict(rows=1 << 24), SHAPE),
    (dict(ldx=255), SHAPE), (dict(ldo=255, out=F * 2), SHAPE), (dict(ldo=300), PARAM), (dict(x=F + 1), PARAM),
    (dict(pos=F + 2), PARAM), (dict(out=F + 3), PARAM), (dict(heads=1 << 20, ldx=1 << 27, ldo=1 << 27), SHAPE), (dict(rows=0), 0)])
def test_rope_refusals(kw, status):
    assert rope(**kw) == status


@built
def test_rope_refuses_no_pairs():
    assert rope(hilo.rotary(2, 128, (0, 0))) == SHAPE
    with pytest.raises(ValueError):
        hilo.rotary(1, 64, (1, 1, 1, 1, 1))
    with pytest.raises(ValueError):
        hilo.rotary(1, 64, (16, 16), (100.0,))


@built
def test_token_positions_refusals():
    f = lambda s, *a: hilo.lib().hilo_token_positions(ctypes.byref(s), *a, None)  # noqa: E731
    s = hilo.hilo_shape(1, 1, 4, 4, 2, 64, 1, 64, 64, hilo.BF16)
    for i in (0, 1, 2, 3, 4, 6):
        a = [F] * 7
        a[i] = None
        assert f(s, *a) == NULL
    s.grid_w = 3
    assert f(s, *[F] * 7) == SHAPE


def norm(dtype=hilo.BF16, y=F, x=F, x_out=F, h=F, h_scale=None, stats=None, rows=8, dim=64, batch=2, text=1, cu=F, **kw):
    n = hilo.hilo_norms(hilo.NORM_LAYER, 1e-6, 1.0, 6 * 64, F, F, F)
    for k, v in kw.items():
        if k in ("post_gain", "pre_gain"):
            getattr(n, k)[1] = v
        else:
            setattr(n, k, v)
    return hilo.lib().hilo_norm_residual(dtype, ctypes.byref(n), y, x, x_out, h, h_scale, stats, rows, dim, batch, text, cu, None)


BAD_NORMS = [(dict(dtype=7), DTYPE), (dict(dim=0), SHAPE), (dict(dim=66), SHAPE), (dict(dim=8196), SHAPE), (dict(rows=-1), SHAPE),
             (dict(rows=1 << 24), SHAPE), (dict(batch=0), SHAPE), (dict(text=-1), SHAPE), (dict(text=5), SHAPE), (dict(kind=2), PARAM),
             (dict(eps=-1.0), PARAM), (dict(eps=float("nan")), PARAM), (dict(residual_scale=float("inf")), PARAM),
             (dict(mod_stride=60), PARAM), (dict(mod_stride=66), PARAM), (dict(gate=F + 4), PARAM), (dict(scale=F + 8), PARAM),
             (dict(pre_gain=F + 4), PARAM), (dict(cu=None), NULL)]


@built
@pytest.mark.parametrize("kw,status", BAD_NORMS + [
    (dict(x=None), NULL), (dict(y=None), NULL), (dict(x_out=None), NULL), (dict(y=None, x_out=None, h=None), NULL),
    (dict(h=None, h_scale=F), NULL), (dict(x=F + 8), PARAM), (dict(x_out=F + 4), PARAM), (dict(y=F + 4), PARAM),
    (dict(h=F + 4), PARAM), (dict(h=F + 2, h_scale=F), PARAM), (dict(stats=F + 8), PARAM), (dict(dtype=hilo.F32, y=F + 8), PARAM),
    (dict(rows=0, text=0), 0), (dict(rows=0, text=0, x=None, y=None, x_out=None, h=None), 0)])
def test_norm_refusals(kw, status):
    assert norm(**kw) == status


def norm_back(dtype=hilo.BF16, dx_out=F, dh=F, y=F, x_out=F, stats=F, dx=F, dy=F, rows=8, dim=64, batch=2, text=1, cu=F,
              ws=F, ws_bytes=1 << 40, grads=True, grad_stride=192, grad_gate=F, grad_gain=F, **kw):
    n = hilo.hilo_norms(hilo.NORM_LAYER, 1e-6, 1.0, 6 * 64, F, F, F)
    for k, v in kw.items():
        if k in ("post_gain", "pre_gain"):
            getattr(n, k)[1] = v
        else:
            setattr(n, k, v)
    g = hilo.hilo_norm_grads(grad_stride, grad_gate, F, F)
    g.pre_gain[0] = grad_gain
    return hilo.lib().hilo_norm_residual_backward(dtype, ctypes.byref(n), dx_out, dh, y, x_out, stats, dx, dy,
                                                  ctypes.byref(g) if grads else None, rows, dim, batch, text, cu, ws, ws_bytes, None)


@built
@pytest.mark.parametrize("kw,status", BAD_NORMS + [
    (dict(stats=None), NULL), (dict(dx=None), NULL), (dict(dy=None), NULL), (dict(y=None), NULL), (dict(dh=None, y=None, dy=None), NULL),
    (dict(x_out=None), NULL), (dict(ws=None), NULL), (dict(ws_bytes=10), WORKSPACE), (dict(ws=F + 4), PARAM), (dict(dx=F + 4), PARAM),
    (dict(dy=F + 4), PARAM), (dict(dh=F + 2), PARAM), (dict(stats=F + 4), PARAM), (dict(dx_out=F + 4), PARAM),
    (dict(grad_stride=60), PARAM), (dict(grad_stride=70), PARAM), (dict(grad_gate=F + 4), PARAM), (dict(grad_gain=F + 4), PARAM),
    (dict(rows=0, text=0, grads=False), 0), (dict(rows=0, text=0, ws=None), NULL),
    (dict(rows=0, text=0, grads=False, ws=None, dx=None, dy=None, stats=None, dh=None, y=None, x_out=None), 0)])
def test_norm_backward_refusals(kw, status):
    assert norm_back(**kw) == status


@built
@pytest.mark.parametrize("args,status", [
    ((3, F, 4, 64, None, F, F), DTYPE), ((0, F, -1, 64, None, F, F), SHAPE), ((0, F, 4, 0, None, F, F), SHAPE),
    ((0, F, 4, 72, None, F, F), SHAPE), ((0, F, 4, 65552, None, F, F), SHAPE), ((0, F, 1 << 24, 64, None, F, F), SHAPE),
    ((0, None, 4, 64, None, F, F), NULL), ((0, F, 4, 64, None, None, F), NULL), ((0, F, 4, 64, None, F, None), NULL),
    ((0, F + 8, 4, 64, None, F, F), PARAM), ((0, F, 4, 64, None, F + 4, F), PARAM), ((0, F, 4, 64, None, F, F + 2), PARAM),
    ((0, F, 0, 64, None, F, F), 0)])
def test_quantize_refusals(args, status):
    assert hilo.lib().hilo_quantize_rows_i8(*args, None) == status


def linear(dtype=hilo.BF16, w0=(F, F, F), w1=(F, F, F), x=F, x_scale=None, out=F, rows=8, k=64, n=64, act=0, batch=2, text=1, cu=F,
           ws=F, ws_bytes=1 << 40):
    w = (hilo.hilo_linear_w_i8 * 2)(hilo.hilo_linear_w_i8(*w0), hilo.hilo_linear_w_i8(*w1))
    return hilo.lib().hilo_linear_i8(dtype, w, x, x_scale, out, rows, k, n, act, batch, text, cu, ws, ws_bytes, None)


@built
@pytest.mark.parametrize("kw,status", [
    (dict(dtype=2), DTYPE), (dict(rows=-1), SHAPE), (dict(rows=1 << 24), SHAPE), (dict(batch=0), SHAPE), (dict(text=-1), SHAPE),
    (dict(text=5), SHAPE), (dict(k=0), SHAPE), (dict(k=72), SHAPE), (dict(k=65552), SHAPE), (dict(n=0), SHAPE), (dict(n=66), SHAPE),
    (dict(n=1 << 24), SHAPE), (dict(n=(1 << 24) - 4, rows=(1 << 24) - 1), SHAPE), (dict(batch=(1 << 20) + 1, rows=1 << 23), SHAPE),
    (dict(batch=4097, rows=8194), SHAPE), (dict(batch=4096, rows=4095), SHAPE),
    (dict(act=2), PARAM), (dict(x=None), NULL), (dict(out=None), NULL), (dict(cu=None), NULL),
    (dict(ws=None), NULL), (dict(w0=(None, F, F)), NULL), (dict(w1=(F, None, F)), NULL), (dict(w0=(F + 8, F, F)), PARAM),
    (dict(w1=(F, F + 4, F)), PARAM), (dict(w0=(F, F, F + 4)), PARAM), (dict(x=F + 8), PARAM), (dict(x_scale=F + 2), PARAM),
    (dict(out=F + 4), PARAM), (dict(ws=F + 16), PARAM), (dict(ws_bytes=100), WORKSPACE), (dict(rows=0, text=0), 0),
    (dict(rows=0, text=0, x=None, out=None, ws=None, ws_bytes=0), 0)])
def test_linear_refusals(kw, status):
    assert linear(**kw) == status


@built
@no_gpu
def test_good_calls_reach_the_device():
    """Without a GPU every well-formed call ends with the device's status, also with what may be left out."""
    assert rope() == rope(ldo=512, out=2 * F) == rope(x=F + 2, out=F + 4, pos=F + 4) == DEVICE
    assert norm() == norm(gate=None, shift=None, scale=None, mod_stride=0) == norm(y=None, x_out=None) == norm(h=None) == DEVICE
    assert norm(h_scale=F, stats=F) == norm_back() == norm_back(dx_out=None) == norm_back(dh=None, x_out=None) == DEVICE
    assert norm_back(y=None, dy=None) == norm_back(grads=False, ws=None, ws_bytes=0) == norm_back(rows=0, text=0) == DEVICE
    assert linear() == linear(w1=(None, None, None), text=0) == linear(w0=(F, F, None), x_scale=F) == DEVICE
    assert hilo.lib().hilo_quantize_rows_i8(1, F, 4, 64, F, F, F, None) == DEVICE


@built
def test_workspace_bytes():
    assert hilo.hilo_linear_i8_workspace_bytes(-1, 64) == hilo.hilo_linear_i8_workspace_bytes(4, 24) == 0
    assert hilo.hilo_linear_i8_workspace_bytes(100, 64) >= 100 * 64 + 400
    # partial tiles only where K may be cut: longer than 64 steps of 128, and more rows than the narrow tiles take
    whole, cut = (hilo.hilo_linear_i8_workspace_bytes(100, k) - 100 * k for k in (8192, 8208))
    assert whole < 1 << 16 and cut >= 256 * 3 * 256 * 256 * 4
    assert hilo.hilo_linear_i8_workspace_bytes(64, 8208) < 1 << 20
    assert hilo.hilo_norm_residual_workspace_bytes(8, 0, 64) == hilo.hilo_norm_residual_workspace_bytes(8, 1, 66) == 0
    small, large = (hilo.hilo_norm_residual_workspace_bytes(r, 3, 256) for r in (1, 4000))
    assert 0 < small < large


@built
def test_binding_refuses():
    """Host tensors, and handles whose tensors do not fit together."""
    x, cu = torch.zeros(4, 64), torch.zeros(2, dtype=torch.int32)
    with pytest.raises(ValueError, match="device"):
        hilo.hilo_rope(hilo.rotary(1, 64, (32,)), x, torch.zeros(4, 1), x)
    with pytest.raises(ValueError, match="device"):
        hilo.hilo_norm_residual(hilo.norms(), x, x, x, x, cu)
    with pytest.raises(ValueError, match="device"):
        hilo.hilo_norm_residual_backward(hilo.norms(), x, x, x, x, torch.zeros(4, 4), x, x, None, cu)
    with pytest.raises(ValueError, match="device"):
        hilo.hilo_quantize_rows_i8(x, x.to(torch.int8), torch.zeros(4))
    with pytest.raises(ValueError, match="device"):
        hilo.linear_weights_i8([{"w": x.to(torch.int8), "s": torch.zeros(4), "b": None}])
    with pytest.raises(ValueError, match="gate"):
        hilo.norms(gate=torch.zeros(1, 2, 64, dtype=torch.bfloat16))
    with pytest.raises(ValueError, match="gate"):
        hilo.norms(gate=torch.zeros(2, 64))
    with pytest.raises(ValueError, match="post_gain"):
        hilo.norms(post_gain=torch.zeros(2, 64, dtype=torch.bfloat16))


class OnDevice:
    """What the binding looks at of a tensor on a device: it has no memory, and a call that is not refused ends without one."""
    is_cuda = True

    def __init__(self, dtype, *shape, dev=0, contiguous=True):
        self.dtype, self.shape, self.dev, self.contiguous = dtype, torch.Size(shape), dev, contiguous
        self.device = torch.device("cuda", dev) if dev >= 0 else torch.device("cpu")

    def __repr__(self):
        return f"{self.dtype}{list(self.shape)} on {self.device}{'' if self.contiguous else ', strided'}"

    def dim(self):
        return len(self.shape)

    def numel(self):
        return self.shape.numel()

    def get_device(self):
        return self.dev

    def is_contiguous(self):
        return self.contiguous

    def element_size(self):
        return self.dtype.itemsize

    def data_ptr(self):
        return F


def _position_args(**changed):
    """hilo_token_positions of 2 samples of 3 grids of 4 x 6 patches and 5 text rows; `changed` by name."""
    i, f = torch.int32, torch.float32
    a = dict(fine_idx=OnDevice(i, 6, 24), pool_idx=OnDevice(i, 6, 6), counts=OnDevice(i, 6, 2), cu_seqlens=OnDevice(i, 3),
             seg_off=OnDevice(i, 6), text_pos=OnDevice(f, 5, 3), pos=OnDevice(f, 2 * (3 * 30 + 5), 3))
    return [hilo.hilo_shape(2, 3, 4, 6, 5, 64, 1, 64, 64, hilo.BF16), *dict(a, **changed).values()]


@built
@pytest.mark.parametrize("changed", [
    dict(pos=OnDevice(torch.float32, 190, 2)), dict(pos=OnDevice(torch.float32, 189, 3)), dict(pos=OnDevice(torch.float32, 570)),
    dict(pos=OnDevice(torch.bfloat16, 190, 3)), dict(pos=OnDevice(torch.float32, 190, 3, contiguous=False)),
    dict(pos=OnDevice(torch.float32, 190, 3, dev=-1)), dict(pos=OnDevice(torch.float32, 190, 3, dev=1)),
    dict(fine_idx=OnDevice(torch.int64, 6, 24)), dict(fine_idx=OnDevice(torch.int32, 5, 24)), dict(pool_idx=OnDevice(torch.int32, 6, 5)),
    dict(pool_idx=OnDevice(torch.int32, 6, 6, dev=1)), dict(counts=OnDevice(torch.int32, 12)), dict(counts=OnDevice(torch.int32, 6, 1)),
    dict(cu_seqlens=OnDevice(torch.int32, 2)), dict(cu_seqlens=OnDevice(torch.int64, 3)), dict(seg_off=OnDevice(torch.int32, 2)),
    dict(text_pos=OnDevice(torch.float32, 4, 3)), dict(text_pos=OnDevice(torch.float64, 5, 3)),
    dict(text_pos=OnDevice(torch.float32, 5, 3, contiguous=False))], ids=str)
def test_token_positions_binding_refuses(changed):
    """Tensors that the kernel would read or write past their ends, or as what they are not."""
    with pytest.raises(ValueError):
        hilo.hilo_token_positions(*_position_args(**changed), stream=0)


@built
def test_token_positions_binding_status():
    with pytest.raises(hilo.HiloError) as e:
        hilo.hilo_token_positions(*_position_args(pos=None), stream=0)
    assert e.value.status == NULL
    args = _position_args()
    args[0].grid_w = 5
    with pytest.raises(hilo.HiloError) as e:
        hilo.hilo_token_positions(*args, stream=0)
    assert e.value.status == SHAPE


def _cuts_to(good):
    """A size that 32 bits would cut to `good`."""
    return (1 << 32) + good


@built
@pytest.mark.parametrize("dim,text", [(_cuts_to(64), 0), (1 << 31, 0), (64, _cuts_to(1)), (64, -1)])
def test_norm_binding_keeps_sizes(dim, text, monkeypatch):
    """Sizes past 32 bits are refused, and not taken for what is left of them."""
    monkeypatch.setattr(hilo, "_current_device", lambda: 0)
    x, cu, stats = OnDevice(torch.float32, 8, dim), OnDevice(torch.int32, 2), OnDevice(torch.float32, 8, 4)
    for call in (lambda: hilo.hilo_norm_residual(hilo.norms(), x, x, x, x, cu, text, stream=0),
                 lambda: hilo.hilo_norm_residual_backward(hilo.norms(), x, x, x, x, stats, x, x, None, cu, text, stream=0)):
        with pytest.raises(hilo.HiloError) as e:
            call()
        assert e.value.status == SHAPE


@built
@pytest.mark.parametrize("k,n,text,act,status", [(_cuts_to(64), 64, 0, 0, SHAPE), (64, _cuts_to(64), 0, 0, SHAPE), (64, 64, _cuts_to(1), 0, SHAPE),
                                                 (64, 64, -1, 0, SHAPE), (64, 64, 0, _cuts_to(1), PARAM), (64, 64, 0, -1, PARAM)])
def test_linear_binding_keeps_sizes(k, n, text, act, status, monkeypatch):
    monkeypatch.setattr(hilo, "_current_device", lambda: 0)
    f = torch.float32
    w = hilo.linear_weights_i8([{"w": OnDevice(torch.int8, n, k), "s": OnDevice(f, n)}])
    with pytest.raises(hilo.HiloError) as e:
        hilo.hilo_linear_i8(w, OnDevice(f, 8, k), OnDevice(f, 8, n), OnDevice(torch.int32, 2), text, act=act,
                            workspace=OnDevice(torch.uint8, 1 << 30), stream=0)
    assert e.value.status == status


@built
def test_handles_keep_sizes():
    for bad in (lambda: hilo.rotary(_cuts_to(1), 64, (32,)), lambda: hilo.rotary(1, _cuts_to(64), (32,)),
                lambda: hilo.rotary(1, 64, (_cuts_to(32),)), lambda: hilo.rotary(1, 64, (32,), flags=_cuts_to(1)),
                lambda: hilo.norms(_cuts_to(1))):
        with pytest.raises(ValueError, match="32 bits"):
            bad()
    assert hilo.hilo_linear_i8_workspace_bytes(8, _cuts_to(64)) == 0
    assert hilo.hilo_norm_residual_workspace_bytes(8, _cuts_to(1), 64) == hilo.hilo_norm_residual_workspace_bytes(8, 1, _cuts_to(64)) == 0


# ------------------------------------------------------------------------------------------ oracle

@pytest.mark.parametrize("rms", [False, True])
def test_oracle_backward_is_the_slope(rms):
    """Every gradient of the oracle against central differences of its forward pass."""
    rng = np.random.default_rng(1)
    cu, text, D, alpha, step = np.array([0, 3, 3, 7]), 0, 6, 0.8, 1e-5
    for text, cu in ((0, cu), (2, np.array([0, 3, 5, 9]))):
        T, B = cu[-1], len(cu) - 1
        v = dict(y=rng.standard_normal((T, D)), x=rng.standard_normal((T, D)), gate=rng.standard_normal((B, 2, D)),
                 shift=rng.standard_normal((B, 2, D)), scale=rng.standard_normal((B, 2, D)),
                 post_gain=rng.standard_normal((2, D)), pre_gain=rng.standard_normal((2, D)))
        cx, ch = rng.standard_normal((T, D)), rng.standard_normal((T, D))

        def value(v):
            xo, h, _ = Q.norm_residual(cu=cu, text_len=text, rms=rms, eps=1e-3, alpha=alpha, **v)
            return (xo * cx).sum() + (h * ch).sum()

        xo = Q.norm_residual(cu=cu, text_len=text, rms=rms, eps=1e-3, alpha=alpha, **v)[0]
        dx, dy, sums = Q.norm_residual_backward(cx, ch, v["y"], xo, cu, text, rms, 1e-3, alpha, v["gate"], v["scale"],
                                                v["post_gain"], v["pre_gain"])
        for name, got in dict(sums, x=dx, y=dy).items():
            want = np.zeros_like(v[name])
            for i in np.ndindex(want.shape):
                d = np.zeros_like(want)
                d[i] = step
                want[i] = (value(dict(v, **{name: v[name] + d})) - value(dict(v, **{name: v[name] - d}))) / (2 * step)
            np.testing.assert_allclose(got, want, rtol=1e-6, atol=1e-6, err_msg=name)


@pytest.mark.parametrize("rms", [False, True])
def test_oracle_norm_against_torch(rms):
    x = torch.from_numpy(np.random.default_rng(2).standard_normal((5, 12)))
    want = x * torch.rsqrt((x * x).mean(1, keepdim=True) + 1e-6) if rms else torch.nn.functional.layer_norm(x, (12,), eps=1e-6)
    np.testing.assert_allclose(Q.norm(x.numpy(), rms, 1e-6)[0], want.numpy(), rtol=1e-12, atol=1e-12)


@pytest.mark.parametrize("adjacent", [False, True])
@pytest.mark.parametrize("one_spectrum", [False, True])
def test_oracle_rope(adjacent, one_spectrum):
    """Turns are products with unit complex numbers; they keep lengths, and scores depend on differences of positions."""
    rng = np.random.default_rng(3)
    pairs, base = (2, 3, 1), [100.0, 10.0, 3.0]
    q, k = rng.standard_normal((1, 14)), rng.standard_normal((1, 14))
    pos, gap = rng.uniform(0, 50, (4, 3)), np.array([[1.5, -2.0, 7.0]])
    turn = lambda v, p: Q.rope(v, p, 1, pairs, base, adjacent, one_spectrum)  # noqa: E731
    scores = [(turn(q, p[None] + gap) @ turn(k, p[None]).T).item() for p in pos]
    np.testing.assert_allclose(scores, scores[0], rtol=0, atol=1e-11)
    x = rng.standard_normal((4, 14))
    y = turn(x, pos)
    np.testing.assert_allclose(np.linalg.norm(y, axis=1), np.linalg.norm(x, axis=1), rtol=1e-13)
    np.testing.assert_array_equal(y[:, 12:], x[:, 12:])
    at = (lambda v: v[:, 0:12:2] + 1j * v[:, 1:12:2]) if adjacent else (lambda v: v[:, :6] + 1j * v[:, 6:12])
    freq = [100.0 ** (-j / 6) for j in range(6)] if one_spectrum else [1, 100 ** -.5, 1, 10 ** (-1 / 3), 10 ** (-2 / 3), 1]
    t = pos[:, [0, 0, 1, 1, 1, 2]] * np.array(freq)
    np.testing.assert_allclose(at(y), at(x) * np.exp(1j * t), rtol=0, atol=1e-12)
    np.testing.assert_allclose(Q.rope(y, pos, 1, pairs, base, adjacent, one_spectrum, True), x, rtol=0, atol=1e-13)


def test_oracle_int8():
    """Codes by hand; the product against whole-number loops."""
    codes, scale = Q.quantize_rows_i8(np.array([[127.0, -63.5, 0.5, 1.5], [0, 0, 0, 0], [1e-3, -1e-3, 4e-4, 0]], np.float32))
    assert codes.tolist() == [[127, -64, 0, 2], [0, 0, 0, 0], [127, -127, 51, 0]] and scale[0] == 1.0 and scale[1] == 0
    rng = np.random.default_rng(4)
    a, cu = rng.integers(-127, 128, (5, 7)).astype(np.int8), np.array([0, 2, 5])
    w = [{"w": rng.integers(-127, 128, (3, 7)).astype(np.int8), "s": rng.uniform(0, 1, 3), "b": rng.uniform(0, 1, 3)} for _ in range(2)]
    s = rng.uniform(0, 1, 5)
    out, _ = Q.linear_i8(a, s, w, cu, 1)
    for m in range(5):
        k = 1 if m in (1, 4) else 0
        for n in range(3):
            acc = sum(int(a[m, i]) * int(w[k]["w"][n, i]) for i in range(7))
            assert abs(out[m, n] - (acc * s[m] * w[k]["s"][n] + w[k]["b"][n])) < 1e-9


# ---------------------------------------------------------------------------------------- schedule

@pytest.mark.parametrize("shape,plan", linear_schedule.SHAPES, ids=str)
def test_linear_plans(shape, plan):
    """The shapes of the GPU tests reach the plans that they are there for."""
    assert linear_schedule.describe(*shape) == plan


def test_linear_plans_cut_no_tile_of_short_k():
    """Up to 64 steps of 128 every tile runs whole, so such a call has no partial tiles and no second launch."""
    rng = np.random.default_rng(3)
    for _ in range(3000):
        text = int(rng.choice([0, 1, 77, 300]))
        lens = [int(n) + text for n in rng.integers(1, 4000, rng.choice([1, 2, 8]))]
        K, N = 16 * int(rng.integers(1, 513)), 4 * int(rng.integers(1, 3000))
        plan = linear_schedule.describe(lens, text, K, N, bool(rng.integers(2)))
        assert plan[0] == "small" or (plan[2] == 1 and plan[4] == 0), (lens, text, K, N, plan)


def test_norm_forms_are_the_launchers():
    """The widths of norm_schedule.FORMS are those that the launchers go by, forward and backward."""
    source = open(os.path.join(os.path.dirname(hilo.__file__), "csrc", "norm.hip")).read()
    for macro in ("HILO_NR", "HILO_NB"):
        found = re.findall(r"if \(p\.D <= (\d+)\) %s\((\d), (\d)\);" % macro, source)
        last = re.findall(r"else %s\((\d), (\d)\);" % macro, source)
        assert [tuple(map(int, f)) for f in found] + [(8192, *map(int, last[-1]))] == norm_schedule.FORMS


@pytest.mark.parametrize("shapes,workers", [(norm_schedule.FORWARD, norm_schedule.workers), (norm_schedule.BACKWARD, norm_schedule.back_workers)],
                         ids=["forward", "backward"])
def test_norm_shapes_share_rows(shapes, workers):
    """Every form, at both ends of its widths, with shares of several rows, some of which cross into the next segment.
    Backward: no sum is longer than the tolerances of its test allow."""
    reached, back = {}, workers is norm_schedule.back_workers
    for D, rows in shapes:
        lens, P = norm_schedule.lens(rows), workers(rows + 2, D)
        most, crossing, met = norm_schedule.describe(lens, norm_schedule.TEXT, P)
        several = 9 if back and norm_schedule.form(D)[0] == 1 else 3
        assert sum(lens) == rows > P and most >= several and crossing >= 2 and met >= 2, (D, rows, most, crossing, met)
        reached.setdefault(norm_schedule.form(D), set()).add(D)
        if back:
            assert norm_schedule.longest_sum(lens, norm_schedule.TEXT, D, P) <= 80
    for low, (top, W, NV) in zip([0] + [f[0] for f in norm_schedule.FORMS], norm_schedule.FORMS):
        assert {low + 4, top} <= reached[W, NV]
    assert len({workers(rows + 2, D) for D, rows in shapes}) >= 3


def test_linear_plans_with_gelu():
    """With GELU, whose tiles cost more, the same shapes reach whole tiles of every size, cut ones of both and the small ones."""
    kinds = {(p[0], p[0] != "small" and p[2] > 1, p[0] != "small" and p[4] > 0)
             for p in (linear_schedule.describe(*shape, True) for shape, _ in linear_schedule.SHAPES)}
    assert kinds == {("small", False, False), (128, False, False), (192, False, False), (256, False, False), (192, True, False),
                     (192, True, True), (256, True, True)}


@built
def test_tensors_are_kept():
    """int8 weights and norms' gains keep their tensors, not the caller's dicts and lists, which may change afterwards."""
    w = [dict(w=OnDevice(torch.int8, 16, 32), s=OnDevice(torch.float32, 16), b=OnDevice(torch.float32, 16)) for _ in range(2)]
    gains, slopes = [[OnDevice(torch.float32, 32), OnDevice(torch.float32, 32)] for _ in range(2)]
    kept = [weakref.ref(t) for d in w for t in d.values()] + [weakref.ref(t) for t in gains + slopes]
    made = hilo.linear_weights_i8(w), hilo.norms(post_gain=gains), hilo.norm_grads(pre_gain=slopes)
    w[0].clear()
    w[1].update(b=None)
    gains[:] = slopes[:] = [None, None]
    gc.collect()
    assert all(r() is not None for r in kept) and made
