"""The products of a feed-forward, their gradients and the block-scaled FP8 form in float64, from their definitions
(include/hilo.h: hilo_linear, hilo_linear_backward, hilo_quantize_blocks, hilo_linear_fp8), with what a float32 sum of the
same products may be off by."""
import math

import torch

F64 = torch.float64


def segments(cu, text_len):
    """(first row, end, stream) of every sample's image and text rows."""
    for lo, hi in zip(cu[:-1], cu[1:]):
        yield lo, hi - text_len, 0
        yield hi - text_len, hi, 1


def of_stream(ds, k):
    return ds[min(k, len(ds) - 1)]


def act_slope(name, g):
    """act(g), act'(g) and the exponent's argument z."""
    if name == "silu":
        z, dz = g, torch.ones_like(g)
    else:
        c = 2.0 * math.sqrt(2.0 / math.pi)
        z, dz = c * (g + 0.044715 * g ** 3), c * (1.0 + 3 * 0.044715 * g ** 2)
    p = torch.sigmoid(z)
    q = torch.sigmoid(-z)
    return g * p, p + g * p * q * dz, z


def affine(x, d, part, cu, text_len, of=lambda d, name: d[name].to(F64)):
    """x w^T + b by stream, and the sum of the magnitudes that went into each value."""
    n = of(of_stream([d] if isinstance(d, dict) else d, 0), "w" + part).shape[0]
    v, s = torch.zeros(x.shape[0], n, dtype=F64), torch.zeros(x.shape[0], n, dtype=F64)
    for a, b, k in segments(cu, text_len):
        e = of_stream(d, k)
        w, bias = of(e, "w" + part), e.get("b" + part)
        v[a:b] = x[a:b] @ w.T
        s[a:b] = x[a:b].abs() @ w.abs().T
        if bias is not None:
            v[a:b] += bias.to(F64)
            s[a:b] += bias.to(F64).abs()
    return v, s


def gated(act, g, u, eg, eu, fast):
    """act(g) u, and how far off it is with g and u off by eg and eu: |act'| <= 1.13; the exponential's argument is rounded a
    few times (z 2^-22), it and the reciprocal are off by some ulps (fast) or one, products by one."""
    a, _, z = act_slope(act, g)
    rel = ((8 if fast else 6) + 6 * z.abs().clamp(max=200)) * 2.0 ** -24
    off = 1.13 * eg * (u.abs() + eu) + a.abs() * eu + (a * u).abs() * rel
    return a * u, off


def backward(x, weights, pre, dout, act, cu, text_len, half, shared):
    """dx, gradients by stream and, beside each, its bound: values of dg and du off by `half` of themselves (their rounding)
    and by what the activation's arithmetic loses, then a float32 sum, then a rounding by half."""
    T = x.shape[0]
    if act is None:
        parts = {"": (dout, torch.zeros_like(dout))}
    else:
        g, u = pre[:, 0], pre[:, 1]
        a, slope, z = act_slope(act, g)
        # p, 1 - p and their products: relative to |p| + |g p q z'|
        rel = (16 + 12 * z.abs().clamp(max=200)) * 2.0 ** -24
        big = slope.abs() + (slope - a / torch.where(g == 0, torch.ones_like(g), g)).abs() * 2 + 2.0 ** -24
        parts = {"": (dout * a, (dout * a).abs() * rel), "_gate": (dout * u * slope, (dout * u).abs() * big * rel)}
    ulp = 2.0 ** -24
    dx, bx = torch.zeros_like(x), torch.zeros_like(x)
    streams = 1 if shared else 2
    grads = [{} for _ in range(streams)]
    rows = [torch.zeros(T, dtype=torch.bool) for _ in range(streams)]
    for a, b, k in segments(cu, text_len):
        rows[0 if shared else k][a:b] = True
        for part, (d, e) in parts.items():
            w = of_stream(weights, k)["w" + part].to(F64)
            terms = 2 * w.shape[0] + 8
            dx[a:b] += d[a:b] @ w
            bx[a:b] += (d[a:b].abs() * (half + terms * ulp) + e[a:b] * (1 + half)) @ w.abs()
    bx += dx.abs() * half
    for k in range(streams):
        r = rows[k]
        for part, (d, e) in parts.items():
            terms = int(r.sum()) + 16
            off = d[r].abs() * (half + terms * ulp) + e[r] * (1 + half)
            w, b = d[r].T @ x[r], d[r].sum(0)
            grads[k]["w" + part] = (w, off.T @ x[r].abs() + w.abs() * half)
            grads[k]["b" + part] = (b, off.sum(0) + b.abs() * half)
    return (dx, bx), grads


# ------------------------------------------------------------------------------------------- FP8 blocks

def cut(x, k, ws, kws, part, cu, text_len):
    """What the FP8 matrix instruction may cut: of each group of eight products, all but the one with the largest exponents are
    cut below 2^-13 of its power of two, which is at most the product of the group's largest magnitudes (those of numbers
    below 2^-6 of the scale count as that).  x, ws: values; k, kws: their blocks' exponents."""
    def tops(v, e):
        v = torch.maximum(v.abs(), torch.exp2(e - 6.0))
        return torch.nn.functional.pad(v, (0, -v.shape[1] % 8)).unflatten(1, (-1, 8)).amax(2)

    n = ws[0]["w" + part].shape[0]
    out, tx = torch.zeros(x.shape[0], n, dtype=F64), tops(x, k.repeat_interleave(128, 1)[:, :x.shape[1]])
    for a, b, s in segments(cu, text_len):
        w, e = of_stream(ws, s)["w" + part], of_stream(kws, s)["w" + part]
        tw = tops(w, e.repeat_interleave(128, 0)[:n].repeat_interleave(128, 1)[:, :w.shape[1]])
        out[a:b] = 7 * 2.0 ** -13 * tx[a:b] @ tw.T
    return out

def block_exponent(top):
    """The least k with 448 2^k >= top, at least -127; 0 where top is 0."""
    k = torch.zeros_like(top)
    some = top > 0
    t = torch.where(some, top, torch.ones_like(top))
    k = torch.floor(torch.log2(t / 448.0)) - 1
    for _ in range(3):
        k = torch.where(448.0 * torch.exp2(k) < t, k + 1, k)
    return torch.where(some, k.clamp(min=-127), torch.zeros_like(k))


def quantize(x, block_rows):
    """Values of the codes of x (float64), and the exponents [row blocks][column blocks]."""
    r, c = x.shape
    nr, nc = -(-r // block_rows), -(-c // 128)
    values, k = torch.zeros_like(x), torch.zeros(nr, nc, dtype=F64)
    for j in range(nc):
        for i in range(nr) if block_rows > 1 else [slice(None)]:
            at = (slice(i * block_rows, (i + 1) * block_rows) if block_rows > 1 else i, slice(128 * j, 128 * j + 128))
            b = x[at]
            top = b.abs().amax() if block_rows > 1 else b.abs().amax(1)
            e = block_exponent(top)
            k[i, j] = e
            scale = torch.exp2(e) if block_rows > 1 else torch.exp2(e)[:, None]
            v = b / scale
            step = torch.exp2(torch.frexp(v).exponent.to(F64) - 4.0).clamp(min=2.0 ** -9)
            values[at] = torch.round(v / step) * step * scale
    return values, k


def decode(codes, scales, block_rows):
    """Values of uint8 codes and E8M0 bytes."""
    v = codes.view(torch.float8_e4m3fn).to(F64)
    s = scales.to(F64) - 127.0
    s = torch.where(s == 128.0, torch.full_like(s, float("nan")), torch.exp2(s))
    s = s.repeat_interleave(block_rows, 0)[:v.shape[0]].repeat_interleave(128, 1)[:, :v.shape[1]]
    return v * s
