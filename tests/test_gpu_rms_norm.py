"""aug_rms_norm_batch and its gradients against the 64-bit oracle, through the C ABI."""
import numpy as np
import pytest
import torch

from oracle import rows_oracle as R
from paper_1912_11040_amd import binding
from tests.rows_parity import TYPES, matrix, near, out_matrix, surroundings_untouched, wide

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def aug():
    with binding.Augmenter(0) as a:
        yield a


def _inputs(rows, dim, dtype, seed, pad=0, shift=0):
    rng = np.random.default_rng(seed)
    x = rng.standard_normal((rows, dim)) * np.exp(rng.standard_normal((rows, 1)))
    return (matrix(x, dtype, pad, shift), matrix(rng.standard_normal((rows, dim)), dtype, pad, shift),
            torch.from_numpy(1 + 0.2 * rng.standard_normal(dim)).float().cuda())


# A row's sum of squares has `dim` positive terms: in any order at most dim + 8 roundings; half of that is in its root.
def _terms(dim):
    return dim / 2 + 16


SIZES = [(1, 1), (3, 7), (5, 40), (4, 64), (17, 100), (2, 128), (3, 129), (9, 512), (5, 1001), (33, 1024), (3, 1500), (6, 2048), (3, 4100),
         (2, 8192), (2, 16384), (700, 72)]


@pytest.mark.parametrize("name", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("rows,dim", SIZES)
def test_norm(aug, rows, dim, name):
    dtype, pad, shift = TYPES[name], (5, 3, 8)[dim % 3], (2, 0, 8)[rows % 3]
    shift = min(shift, pad)
    for with_residual in (True, False):
        x, res, w = _inputs(rows, dim, dtype, dim + rows, pad, shift)
        res, weight = (res, w) if with_residual else (None, None)
        s_out, y_out = out_matrix(rows, dim, dtype, pad, shift), out_matrix(rows, dim, dtype, pad, shift)
        rstd = torch.empty(rows, device="cuda")
        aug.aug_rms_norm_batch(x, weight, residual=res, eps=1e-5, sum_out=s_out, y_out=y_out, rstd_out=rstd)
        s, y, r = R.rms_norm(wide(x), None if res is None else wide(res), None if weight is None else wide(weight), 1e-5)
        near(s_out, s, np.abs(s), 1, "sum")
        near(y_out, y, np.abs(y), _terms(dim), "y")
        near(rstd, r, np.abs(r), _terms(dim), "rstd")
        assert surroundings_untouched(s_out) and surroundings_untouched(y_out)


@pytest.mark.parametrize("name", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("rows,dim,q_block", [(3, 40, 0), (3, 40, 16), (5, 100, 32), (4, 1024, 128), (3, 1001, 128), (2, 2048, 0), (9, 500, 64),
                                              (3, 4100, 512), (2, 16384, 256), (2, 16383, 0), (700, 72, 16), (5, 48, 512)])
def test_norm_in_8_bits(aug, rows, dim, q_block, name):
    x, res, w = _inputs(rows, dim, TYPES[name], 3 * dim + rows, pad=dim % 4)
    x[0] = 0
    res[0] = 0                                            # a row of zeros: scales of zero
    width = q_block or dim
    q = out_matrix(rows, dim, torch.float8_e4m3fn, dim % 3)
    scale = torch.empty(rows, -(-dim // width), device="cuda")
    y_out = out_matrix(rows, dim, TYPES[name])
    aug.aug_rms_norm_batch(x, w, residual=res, q_out=q, scale_out=scale, q_block=q_block, y_out=y_out)
    _, y, _ = R.rms_norm(wide(x), wide(res), wide(w))
    near(y_out, y, np.abs(y), _terms(dim), "y")
    near(scale, R.block_scales(y, q_block), R.block_scales(y, q_block), _terms(dim) + 2, "scale")
    assert surroundings_untouched(q)
    # by the scales that came out: at most half a step of e4m3 off, 2^-4 of the value, or 2^-10 (a step of the smallest ones is 2^-9)
    per_column = np.repeat(wide(scale), width, axis=1)[:, :dim]
    v = np.divide(y, per_column, out=np.zeros_like(y), where=per_column > 0)
    got = wide(q.float())
    assert np.all(np.abs(got - v) <= np.maximum(2.0 ** -4 * np.abs(v), 2.0 ** -10) + (_terms(dim) + 4) * 2.0 ** -24 * np.abs(v))
    assert np.all(got[0] == 0) and np.all(wide(scale)[0] == 0)
    # and not just near: all but those within the rounding of v of a tie are the nearest
    exact = R.round_e4m3(np.clip(v, -448, 448))
    lo, hi = (R.round_e4m3(np.clip(v * (1 + s * (_terms(dim) + 4) * 2.0 ** -24), -448, 448)) for s in (-1, 1))
    assert np.all((got == exact) | (got == lo) | (got == hi))


def test_norm_marks_blocks_that_hold_no_numbers(aug):
    x = torch.randn(4, 96, device="cuda")
    x[1, 40], x[2, 90], x[3, 5] = float("nan"), float("inf"), 1e30
    q, scale = out_matrix(4, 96, torch.float8_e4m3fn), torch.empty(4, 3, device="cuda")
    aug.aug_rms_norm_batch(x, None, q_out=q, scale_out=scale, q_block=32)
    sc = wide(scale)
    assert np.isfinite(sc[0]).all() and np.isnan(sc[1]).all()          # a NaN is in the whole row's sum of squares
    assert np.isnan(sc[2][2]) and np.all(sc[2][:2] == 0)               # the root of infinity: zeros, and infinity times zero
    assert np.isnan(wide(q.float())[1]).all() and np.isfinite(wide(q.float())[0]).all()


@pytest.mark.parametrize("dim", [64, 1001, 2048])
def test_norm_in_place(aug, dim):
    for out in ("x", "residual"):
        x, res, w = _inputs(6, dim, torch.bfloat16, dim)
        s, y = out_matrix(6, dim, torch.bfloat16), out_matrix(6, dim, torch.bfloat16)
        aug.aug_rms_norm_batch(x, w, residual=res, sum_out=s, y_out=y)
        s_at, y_at = (x, res) if out == "x" else (res, x)
        aug.aug_rms_norm_batch(x, w, residual=res, sum_out=s_at, y_out=y_at)
        assert torch.equal(s_at, s) and torch.equal(y_at, y)


@pytest.mark.parametrize("name", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("rows,dim", SIZES + [(2500, 130), (5000, 24)])
def test_norm_gradients(aug, rows, dim, name):
    dtype, pad = TYPES[name], dim % 5
    x, dsum, w = _inputs(rows, dim, dtype, dim + 2 * rows, pad)
    dy = matrix(np.random.default_rng(rows).standard_normal((rows, dim)), dtype, pad)
    for full in (True, False):
        weight, extra = (w, dsum) if full else (None, None)
        _, _, r = R.rms_norm(wide(x))
        rstd = torch.from_numpy(r).float().cuda()
        dx, dw = out_matrix(rows, dim, dtype, pad), torch.full((dim,), float("nan"), device="cuda")
        aug.aug_rms_norm_backward_batch(x, rstd, dy, weight, dsum=extra, dx_out=dx, dweight_out=dw)
        args = (wide(x), wide(rstd), wide(dy), None if weight is None else wide(weight), None if extra is None else wide(extra))
        want, mag = R.rms_norm_backward(*args), R.rms_norm_backward(*args, magnitude=True)
        near(dx, want[0], mag[0], dim + 16, "dx")
        near(dw, want[1], mag[1], rows + 16, "dweight")
        assert surroundings_untouched(dx)
        again = torch.empty_like(dw)
        aug.aug_rms_norm_backward_batch(x, rstd, dy, weight, dsum=extra, dx_out=dy, dweight_out=again)       # in dy's place
        assert torch.equal(dy, dx) and torch.equal(again, dw)
        dy = matrix(np.random.default_rng(rows + 1).standard_normal((rows, dim)), dtype, pad)


def test_norm_of_no_rows(aug):
    dw = torch.full((8,), 3.0, device="cuda")
    e = torch.empty(0, 8, device="cuda")
    aug.aug_rms_norm_batch(e, None, y_out=e)
    aug.aug_rms_norm_backward_batch(e, torch.empty(0, device="cuda"), e, None, dx_out=e, dweight_out=dw)
    assert float(dw.abs().max()) == 0.0
