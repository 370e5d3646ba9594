"""Seeded random sizes, types, layouts and options of the operators on feature rows against the 64-bit oracle."""
import random

import numpy as np
import pytest
import torch

from oracle import rows_oracle as R
from paper_1912_11040_amd import binding
from tests import test_gpu_scan as S
from tests import test_gpu_short_conv as C
from tests.rows_parity import TYPES, near, out_matrix, surroundings_untouched, wide

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def aug():
    with binding.Augmenter(0) as a:
        yield a


def _size(r, most):
    """1 .. most, spread over the logarithm, powers of two and their neighbours often."""
    n = int(round(most ** r.random()))
    if r.random() < 0.4:
        n = (1 << (n.bit_length() - 1)) + r.choice([-1, 0, 0, 1])
    return max(1, min(most, n))


def _lengths(r, rows):
    n = _size(r, 12)
    return [0 if r.random() < 0.15 else _size(r, max(1, rows // n)) for _ in range(n)]


def _layout(r):
    pad = r.choice([0, 0, 1, 5, 64])
    return dict(pad=pad, shift=r.randint(0, pad), behind=r.choice([0, 2]), gaps=r.random() < 0.3)


@pytest.mark.parametrize("seed", range(30))
def test_scan(aug, seed):
    r = random.Random(seed)
    n, g = r.choice([16, 16, _size(r, 128)]), r.choice([1, 1, 2, 3, 5])
    dim, lengths, name = g * _size(r, 160 // g), _lengths(r, 900), r.choice(list(TYPES))
    kw = dict(_layout(r), gate=r.random() < 0.6, plain=r.random() < 0.2)
    print(f"  {name} dim {dim} states {n} groups {g} lengths {lengths} {kw}", flush=True)
    off, lens, t, state, dy = S._inputs(lengths, dim, n, g, TYPES[name], seed, **kw)
    st = state if r.random() < 0.5 else None
    rows, pad, shift = len(dy), kw["pad"], kw["shift"]
    y, out = out_matrix(rows, dim, TYPES[name], pad, shift), torch.full_like(state, float("nan"))
    aug.aug_scan_batch(off, **t, y_out=y, n_group=g, state_in=st, state_out=out, row_lengths=lens)
    args = dict(n_group=g, state_in=None if st is None else wide(st), row_lengths=lens, **S._wide(t))
    want, mag = R.scan(off, **args), R.scan(off, **args, magnitude=True)
    terms = S._terms(lengths, n)
    near(y, want[0], mag[0], terms, "y")
    near(out, want[1], mag[1], terms, "state")
    widths = dict(du=dim, ddelta=dim, db=g * n, dc=g * n, **(dict(dz=dim) if "z" in t else {}))
    got = {k: out_matrix(rows, w, TYPES[name], pad, shift) for k, w in widths.items()}
    got.update({k: torch.full(s, float("nan"), device="cuda") for k, s in dict(da=(dim, n), dskip=(dim,), ddelta_bias=(dim,)).items()})
    aug.aug_scan_backward_batch(off, **t, dy=dy, n_group=g, state_in=st, row_lengths=lens, **{k + "_out": v for k, v in got.items()})
    want, mag = (R.scan_backward(off, dy=wide(dy), magnitude=m, **args) for m in (False, True))
    for k, v in got.items():
        near(v, want[k], mag[k], 2 * terms + (sum(lengths) if k not in widths else dim // g if k in ("db", "dc") else 0), k)
        assert k not in widths or surroundings_untouched(v)


@pytest.mark.parametrize("seed", range(20))
def test_short_conv(aug, seed):
    r = random.Random(100 + seed)
    dim, taps, lengths, name, kw = _size(r, 1200), r.randint(1, 8), _lengths(r, 1500), r.choice(list(TYPES)), _layout(r)
    act = r.choice(["silu", "none"])
    print(f"  {name} dim {dim} taps {taps} {act} lengths {lengths} {kw}", flush=True)
    off, lens, x, w, bias, state, dy = C._inputs(lengths, dim, taps, TYPES[name], seed, **kw)
    st, b = state if r.random() < 0.6 else None, bias if r.random() < 0.6 else None
    y, out = out_matrix(len(x), dim, TYPES[name], kw["pad"], kw["shift"]), torch.full_like(state, float("nan"))
    aug.aug_short_conv_batch(off, x, w, y, bias=b, activation=act, state_in=st, state_out=out, row_lengths=lens)
    args = (off, wide(x), wide(w))
    rest = dict(bias=C._n(b), act=act, state_in=C._n(st), row_lengths=lens)
    want = R.short_conv(*args, **rest)
    near(y, want[0], R.short_conv(*args, **rest, magnitude=True)[0], taps + 12, "y")
    assert np.array_equal(wide(out), want[1].reshape(wide(out).shape)) and surroundings_untouched(y)
    dx, dw, db = torch.full_like(y, 7.0), torch.empty_like(w), torch.empty_like(bias)
    aug.aug_short_conv_backward_batch(off, x, w, dy, bias=b, activation=act, state_in=st, dx_out=dx, dweight_out=dw, dbias_out=db, row_lengths=lens)
    want, mag = (R.short_conv_backward(*args, wide(dy), magnitude=m, **rest) for m in (False, True))
    near(dx, want[0], mag[0], 2 * taps + 16, "dx")
    near(dw, want[1], mag[1], taps + 16 + sum(lengths), "dweight")
    near(db, want[2], mag[2], taps + 16 + sum(lengths), "dbias")


@pytest.mark.parametrize("seed", range(20))
def test_norm(aug, seed):
    r = random.Random(200 + seed)
    dim, name, q_block = _size(r, 9000), r.choice(list(TYPES)), r.choice([0, 16, 32, 64, 128, 256, 512])
    rows, kw = _size(r, 200000 // dim + 1), _layout(r)
    print(f"  {name} {rows} x {dim} q_block {q_block} {kw}", flush=True)
    g = torch.Generator("cuda").manual_seed(seed)
    made = lambda: out_matrix(rows, dim, TYPES[name], kw["pad"], kw["shift"])          # noqa: E731
    x, res, dy, dsum = (made().copy_(torch.randn(rows, dim, device="cuda", generator=g)) for _ in range(4))
    w = 1 + 0.3 * torch.randn(dim, device="cuda", generator=g)
    s, y, rstd = made(), made(), torch.empty(rows, device="cuda")
    q = out_matrix(rows, dim, torch.float8_e4m3fn, kw["pad"], kw["shift"])
    scale = torch.empty(rows, -(-dim // (q_block or dim)), device="cuda")
    aug.aug_rms_norm_batch(x, w, residual=res, sum_out=s, y_out=y, rstd_out=rstd, q_out=q, scale_out=scale, q_block=q_block)
    ws, wy, wr = R.rms_norm(wide(x), wide(res), wide(w))
    terms = dim / 2 + 16
    near(s, ws, np.abs(ws), 1, "sum")
    near(y, wy, np.abs(wy), terms, "y")
    near(rstd, wr, wr, terms, "rstd")
    want = R.block_scales(wy, q_block)
    near(scale, want, want, terms + 2, "scale")
    by = np.repeat(wide(scale), q_block or dim, axis=1)[:, :dim]
    v = np.divide(wy, by, out=np.zeros_like(wy), where=by > 0)          # 0 where the scale is 0
    assert np.all(np.abs(wide(q.float()) - v) <= np.maximum(2.0 ** -4 * np.abs(v), 2.0 ** -10) + (terms + 4) * 2.0 ** -24 * np.abs(v))
    dx, dw = made(), torch.empty(dim, device="cuda")
    aug.aug_rms_norm_backward_batch(s, rstd, dy, w, dsum=dsum, dx_out=dx, dweight_out=dw)
    args = (wide(s), wide(rstd), wide(dy), wide(w), wide(dsum))
    want, mag = R.rms_norm_backward(*args), R.rms_norm_backward(*args, magnitude=True)
    near(dx, want[0], mag[0], dim + 16, "dx")
    near(dw, want[1], mag[1], rows + 16, "dweight")
    assert all(surroundings_untouched(m) for m in (s, y, q, dx))
