"""The operators on feature rows from their definitions, in 64 bits on the CPU: root-mean-square norm, short causal
convolution, selective scan, and their gradients by the formulas.  Written for clarity, a row or a tap at a time.

Every function takes arrays of any float type, widens them and returns float64.  With `magnitude=True` the sums are formed
from the absolute values of their terms: the scale that rounding errors of those sums are relative to.
"""
import numpy as np

E4M3_MAX = 448.0


def _f64(a):
    return None if a is None else np.asarray(a, np.float64)


def sigmoid(x):
    x = _f64(x)
    e = np.exp(-np.abs(x))
    return np.where(x >= 0, 1.0 / (1.0 + e), e / (1.0 + e))


def softplus(x):
    x = _f64(x)
    return np.maximum(x, 0.0) + np.log1p(np.exp(-np.abs(x)))


def silu(x):
    return x * sigmoid(x)


def dsilu(x):
    s = sigmoid(x)
    return s * (1.0 + x * (1.0 - s))


# ---- norm ----

def rms_norm(x, residual=None, weight=None, eps=1e-6):
    """(sum, y, rstd)."""
    s = _f64(x) if residual is None else _f64(x) + _f64(residual)
    rstd = 1.0 / np.sqrt(np.mean(s * s, axis=1) + eps)
    y = s * rstd[:, None] * (1.0 if weight is None else _f64(weight))
    return s, y, rstd


def block_scales(y, q_block):
    """max |y| / 448 of every block of q_block columns (0: of the row)."""
    y = np.abs(_f64(y))
    width = q_block or y.shape[1]
    return np.stack([y[:, i:i + width].max(axis=1) / E4M3_MAX for i in range(0, y.shape[1], width)], axis=1)


def round_e4m3(v):
    """v rounded to the nearest e4m3 number (3 bits behind the point, exponents from -6, ties to even), |v| <= 464."""
    v = _f64(v)
    _, e = np.frexp(np.where(v == 0, 1.0, v))
    step = np.exp2(np.maximum(e - 1, -6) - 3)
    return np.rint(v / step) * step


def rms_norm_backward(s, rstd, dy, weight=None, dsum=None, magnitude=False):
    """(ds, dweight)."""
    f = np.abs if magnitude else lambda v: v
    s, rstd, dy = f(_f64(s)), _f64(rstd)[:, None], f(_f64(dy))
    w = np.ones(s.shape[1]) if weight is None else f(_f64(weight))
    second = s * rstd ** 3 * np.mean(s * w * dy, axis=1, keepdims=True)
    ds = rstd * w * dy + second if magnitude else rstd * w * dy - second
    if dsum is not None:
        ds = ds + f(_f64(dsum))
    return ds, np.sum(dy * s * rstd, axis=0)


# ---- sequences ----

def spans(row_offsets, row_lengths=None):
    off = np.asarray(row_offsets, np.int64)
    return [(int(off[i]), int(off[i + 1] if row_lengths is None else off[i] + row_lengths[i])) for i in range(len(off) - 1)]


def _extended(x, state, taps):
    before = np.zeros((taps - 1, x.shape[1])) if state is None else _f64(state)
    return np.concatenate([before, x])


def short_conv(row_offsets, x, weight, bias=None, act="silu", state_in=None, row_lengths=None, magnitude=False):
    """(y [rows][dim], NaN in rows of no sequence; state [n_seq][taps-1][dim]).  magnitude: the sums of absolute values instead of y."""
    f = np.abs if magnitude else lambda v: v
    x, w = f(_f64(x)), f(_f64(weight))
    taps = w.shape[1]
    y, states = np.full(x.shape, np.nan), []
    for i, (a, b) in enumerate(spans(row_offsets, row_lengths)):
        rows = _extended(x[a:b], None if state_in is None else f(_f64(state_in[i])), taps)
        p = np.zeros((b - a, x.shape[1]))
        for k in range(taps):
            p += w[:, k] * rows[k:k + b - a]
        if bias is not None:
            p += f(_f64(bias))
        y[a:b] = silu(p) if act == "silu" and not magnitude else p
        states.append(rows[len(rows) - (taps - 1):])
    return y, np.stack(states) if states else np.zeros((0, taps - 1, x.shape[1]))


def short_conv_backward(row_offsets, x, weight, dy, bias=None, act="silu", state_in=None, row_lengths=None, magnitude=False):
    """(dx, dweight, dbias); state_in is a constant."""
    f = np.abs if magnitude else lambda v: v
    x, w, dy = _f64(x), _f64(weight), _f64(dy)
    dim, taps = w.shape
    dx, dw, db = np.full(x.shape, np.nan), np.zeros((dim, taps)), np.zeros(dim)
    for i, (a, b) in enumerate(spans(row_offsets, row_lengths)):
        rows = _extended(x[a:b], None if state_in is None else state_in[i], taps)
        n = b - a
        p = sum(w[:, k] * rows[k:k + n] for k in range(taps)) + (0.0 if bias is None else _f64(bias))
        dp = dy[a:b] * (dsilu(p) if act == "silu" else 1.0)
        if magnitude:                    # an error of p moves dp by at most half of it
            dp = np.abs(dp) + (0.5 * np.abs(dy[a:b]) * (sum(np.abs(w[:, k] * rows[k:k + n]) for k in range(taps)) + np.abs(p)) if act == "silu" else 0.0)
        drows = np.zeros(rows.shape)
        for k in range(taps):
            drows[k:k + n] += f(w[:, k]) * dp
            dw[:, k] += np.sum(dp * f(rows[k:k + n]), axis=0)
        db += dp.sum(axis=0)
        dx[a:b] = drows[taps - 1:]
    return dx, dw, db


def _per_channel(x, n_group, dim, n):
    return np.repeat(_f64(x).reshape(-1, n_group, n), dim // n_group, axis=1)


def scan(row_offsets, u, delta, a, b, c, skip=None, z=None, delta_bias=None, act="softplus", n_group=1, state_in=None,
         row_lengths=None, magnitude=False, keep=None):
    """(y, states).  `keep`: a dict that gets each sequence's h with the state before it first, [rows + 1][dim][n]."""
    f = np.abs if magnitude else lambda v: v
    u, a = f(_f64(u)), _f64(a)
    dim, n = a.shape
    raw = _f64(delta) + (0.0 if delta_bias is None else _f64(delta_bias))
    step = softplus(raw) if act == "softplus" else raw
    bs, cs = f(_per_channel(b, n_group, dim, n)), f(_per_channel(c, n_group, dim, n))
    y, states = np.full(u.shape, np.nan), []
    for i, (lo, hi) in enumerate(spans(row_offsets, row_lengths)):
        h = np.zeros((dim, n)) if state_in is None else f(_f64(state_in[i]))
        hs = [h]
        for t in range(lo, hi):
            h = np.exp(step[t][:, None] * a) * h + (f(step[t]) * u[t])[:, None] * bs[t]
            hs.append(h)
            y[t] = np.sum(cs[t] * h, axis=1)
        states.append(h)
        if keep is not None:
            keep[i] = np.stack(hs)
    y = y + (0.0 if skip is None else f(_f64(skip)) * u)
    if z is not None:
        y = y * f(silu(_f64(z)))
    return y, np.stack(states) if states else np.zeros((0, dim, n))


def scan_backward(row_offsets, u, delta, a, b, c, dy, skip=None, z=None, delta_bias=None, act="softplus", n_group=1, state_in=None,
                  row_lengths=None, magnitude=False):
    """Gradients as a dict: du, ddelta, db, dc, da, dskip, ddelta_bias and, with a gate, dz; state_in is a constant."""
    f = np.abs if magnitude else lambda v: v
    keep = {}
    scan(row_offsets, u, delta, a, b, c, None, None, delta_bias, act, n_group, state_in, row_lengths, magnitude, keep)
    u, a, dy = f(_f64(u)), _f64(a), f(_f64(dy))
    rows, dim = u.shape
    n = a.shape[1]
    raw = _f64(delta) + (0.0 if delta_bias is None else _f64(delta_bias))
    step, slope = (softplus(raw), sigmoid(raw)) if act == "softplus" else (raw, np.ones(raw.shape))
    bs, cs = f(_per_channel(b, n_group, dim, n)), f(_per_channel(c, n_group, dim, n))
    sk = np.zeros(dim) if skip is None else f(_f64(skip))
    dp = dy if z is None else dy * f(silu(_f64(z)))
    nan = lambda *s: np.full(s, np.nan)          # noqa: E731
    o = dict(du=nan(rows, dim), ddelta=nan(rows, dim), db=nan(rows, n_group * n), dc=nan(rows, n_group * n), da=np.zeros((dim, n)),
             dskip=np.zeros(dim), ddelta_bias=np.zeros(dim))
    if z is not None:
        o["dz"] = nan(rows, dim)
        zz, sz = _f64(z), sigmoid(z)
        dsl = sz * (1.0 + np.abs(zz) * (1.0 - sz)) if magnitude else dsilu(zz)      # (its two terms cancel near z = -1.28)
    for i, (lo, hi) in enumerate(spans(row_offsets, row_lengths)):
        carried = np.zeros((dim, n))
        for t in range(hi - 1, lo - 1, -1):
            h, before = keep[i][t - lo + 1], keep[i][t - lo]
            e = np.exp(step[t][:, None] * a)
            g = cs[t] * dp[t][:, None] + carried
            carried = e * g
            gb = np.sum(g * bs[t], axis=1)
            dstep = np.sum(g * f(a) * e * before, axis=1) + u[t] * gb
            o["da"] += carried * before * f(step[t])[:, None]
            o["du"][t] = f(step[t]) * gb + sk * dp[t]
            o["ddelta"][t] = dstep * slope[t]
            o["db"][t] = np.sum((g * (f(step[t]) * u[t])[:, None]).reshape(n_group, -1, n), axis=1).reshape(-1)
            o["dc"][t] = np.sum((dp[t][:, None] * h).reshape(n_group, -1, n), axis=1).reshape(-1)
            o["dskip"] += dp[t] * u[t]
            o["ddelta_bias"] += o["ddelta"][t]
            if z is not None:
                o["dz"][t] = dy[t] * (np.sum(cs[t] * h, axis=1) + sk * u[t]) * dsl[t]
    return o
