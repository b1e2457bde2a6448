"""Plain float64 forms of the rotary, sandwich-norm and int8 operators (numpy, one row or segment at a time): the test
oracle of hilo_rope, hilo_token_positions, hilo_norm_residual (and its backward pass), hilo_quantize_rows_i8 and
hilo_linear_i8.  Shares no code with the GPU path."""
import numpy as np


def segments(cu, text_len):
    """(first row, end, sample, stream) of every segment, empty ones too."""
    out = []
    for s in range(len(cu) - 1):
        lo, hi = int(cu[s]), int(cu[s + 1])
        out += [(lo, hi - text_len, s, 0), (hi - text_len, hi, s, 1)]
    return out


# ------------------------------------------------------------------------------------------ rotary

def rope_angles(pos, pairs, base, one_spectrum=False):
    """[rows][n] angles in radians."""
    n, cols, j = sum(pairs), [], 0
    bases = [base] * len(pairs) if np.isscalar(base) else list(base)
    for a, m in enumerate(pairs):
        for i in range(m):
            w = float(bases[0]) ** (-j / n) if one_spectrum else float(bases[a]) ** (-i / m)
            cols.append(np.asarray(pos, np.float64)[:, a] * w)
            j += 1
    return np.stack(cols, 1)


def rope(x, pos, heads, pairs, base=10000.0, adjacent=False, one_spectrum=False, backward=False):
    """x [rows][heads * hd] -> the same, every head's first 2 n columns turned pair by pair."""
    rows, n = x.shape[0], sum(pairs)
    y = np.array(x, np.float64).reshape(rows, heads, -1)
    t = rope_angles(pos, pairs, base, one_spectrum)
    for j in range(n):
        p, q = (2 * j, 2 * j + 1) if adjacent else (j, j + n)
        c, s = np.cos(t[:, j])[:, None], np.sin(t[:, j])[:, None]
        s = -s if backward else s
        u, v = y[:, :, p].copy(), y[:, :, q].copy()
        y[:, :, p], y[:, :, q] = u * c - v * s, v * c + u * s
    return y.reshape(rows, -1)


def token_positions(batch, images, grid_w, text_len, fine_idx, pool_idx, counts, text_pos=None):
    """[tokens][3] (time, height, width) of a compressed sequence, sample after sample."""
    rows = []
    for s in range(batch):
        for i in range(images):
            g = s * images + i
            for k in range(counts[g][0]):
                rows.append((i, *divmod(int(fine_idx[g][k]), grid_w)))
            for k in range(counts[g][1]):
                bi, bj = divmod(int(pool_idx[g][k]), grid_w // 2)
                rows.append((i, 2 * bi + 0.5, 2 * bj + 0.5))
        rows += [tuple(text_pos[t]) if text_pos is not None else (0, 0, 0) for t in range(text_len)]
    return np.array(rows, np.float64).reshape(-1, 3)


# ------------------------------------------------------------------------------------------- norms

def norm(v, rms, eps):
    """(normalised rows, mean, 1 / deviation)."""
    m = np.zeros(len(v)) if rms else v.mean(1)
    d = v - m[:, None]
    r = 1.0 / np.sqrt((d * d).mean(1) + eps)
    return d * r[:, None], m, r


def _vec(v, s, k, default):
    return default if v is None else np.asarray(v[s][k], np.float64)


def _gain(v, k):
    return 1.0 if v is None else np.asarray(v[k], np.float64)


def norm_residual(y, x, cu, text_len, rms=False, eps=1e-6, alpha=1.0, gate=None, shift=None, scale=None,
                  post_gain=None, pre_gain=None):
    """(x_out, h, stats) in float64; y None: x_out is x."""
    x_out, h = np.array(x, np.float64), np.zeros(x.shape)
    stats = np.zeros((len(x), 4))
    for a, b, s, k in segments(cu, text_len):
        if y is not None:
            u, stats[a:b, 0], stats[a:b, 1] = norm(np.asarray(y[a:b], np.float64), rms, eps)
            x_out[a:b] = alpha * x_out[a:b] + _vec(gate, s, k, 1.0) * (u * _gain(post_gain, k))
        v, stats[a:b, 2], stats[a:b, 3] = norm(x_out[a:b], rms, eps)
        h[a:b] = v * _gain(pre_gain, k) * (1.0 + _vec(scale, s, k, 0.0)) + _vec(shift, s, k, 0.0)
    return x_out, h, stats


def norm_residual_backward(dx_out, dh, y, x_out, cu, text_len, rms=False, eps=1e-6, alpha=1.0, gate=None, scale=None,
                           post_gain=None, pre_gain=None):
    """dx, dy and the sums: dict of gate, shift, scale [batch][2][dim] and post_gain, pre_gain [2][dim]."""
    T, D = x_out.shape
    dx, dy = np.zeros((T, D)), np.zeros((T, D))
    sums = {k: np.zeros((len(cu) - 1, 2, D)) for k in ("gate", "shift", "scale")}
    sums |= {k: np.zeros((2, D)) for k in ("post_gain", "pre_gain")}

    def through(n, v, r):
        n = n - v * (n * v).mean(1)[:, None] - (0.0 if rms else n.mean(1)[:, None])
        return r[:, None] * n

    for a, b, s, k in segments(cu, text_len):
        g = np.zeros((b - a, D)) if dx_out is None else np.array(dx_out[a:b], np.float64)
        if dh is not None:
            d = np.asarray(dh[a:b], np.float64)
            v, _, r = norm(np.asarray(x_out[a:b], np.float64), rms, eps)
            one, pre = 1.0 + _vec(scale, s, k, 0.0), _gain(pre_gain, k)
            g += through(d * one * pre, v, r)
            sums["shift"][s, k], sums["scale"][s, k] = d.sum(0), (d * v * pre).sum(0)
            sums["pre_gain"][k] += (d * v * one).sum(0)
        dx[a:b] = g * (1.0 if y is None else alpha)
        if y is not None:
            u, _, r = norm(np.asarray(y[a:b], np.float64), rms, eps)
            gt, post = _vec(gate, s, k, 1.0), _gain(post_gain, k)
            dy[a:b] = through(g * gt * post, u, r)
            sums["gate"][s, k] = (g * u * post).sum(0)
            sums["post_gain"][k] += (g * u * gt).sum(0)
    return dx, dy, sums


# --------------------------------------------------------------------------------------------- int8

def quantize_rows_i8(x):
    """(codes, scales) of float32 rows; every step one float32 operation, as the codes are defined."""
    x = np.asarray(x, np.float32)
    top = np.abs(x).max(1)
    ok = top >= np.float32(2.0 ** -120)
    inv = np.zeros_like(top)
    inv[ok] = (np.float32(1.0) / top[ok]) * np.float32(127.0)
    codes = np.rint(np.clip(x * inv[:, None], -127, 127).astype(np.float32))
    return codes.astype(np.int8), np.where(ok, top / np.float32(127.0), np.float32(0)).astype(np.float32)


def gelu_tanh(u):
    return 0.5 * u * (1.0 + np.tanh(np.sqrt(2.0 / np.pi) * (u + 0.044715 * u ** 3)))


def linear_i8(codes, a_scale, w, cu, text_len, gelu=False):
    """w: per stream {"w", "s", "b"}; int64 sums, then float64.  Also the largest part of what was added up."""
    T, N = codes.shape[0], w[0]["w"].shape[0]
    out, size = np.zeros((T, N)), np.zeros((T, N))
    for a, b, _, k in segments(cu, text_len):
        if a == b:
            continue
        acc = codes[a:b].astype(np.float64) @ w[k]["w"].astype(np.float64).T  # whole numbers below 2^53
        v = acc * np.asarray(a_scale[a:b], np.float64)[:, None] * np.asarray(w[k]["s"], np.float64)
        size[a:b] = np.abs(v)
        if w[k]["b"] is not None:
            v = v + np.asarray(w[k]["b"], np.float64)
            size[a:b] += np.abs(np.asarray(w[k]["b"], np.float64))
        out[a:b] = gelu_tanh(v) if gelu else v
    return out, size
