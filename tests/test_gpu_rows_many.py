"""The operators on feature rows at sizes where a group of threads goes through several rows, blocks or streams one after another, and where blocks of
rows are long: what the large calls spend their time in, against the 64-bit oracle.  Sizes follow from the number of compute units."""
import numpy as np
import pytest
import torch

from oracle import rows_oracle as R
from paper_1912_11040_amd import binding
from tests import test_gpu_scan as S
from tests import test_gpu_short_conv as C
from tests.rows_parity import TYPES, near, out_matrix, wide

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def aug():
    with binding.Augmenter(0) as a:
        yield a


@pytest.fixture(scope="module")
def units():
    return torch.cuda.get_device_properties(0).multi_processor_count


# ---- norm: rows of a group, rows of sums ----

@pytest.mark.parametrize("dim,rows_a_unit,name,q_block", [
    (40, 600, "bf16", 16), (200, 150, "f32", 0), (500, 150, "f16", 64), (600, 40, "bf16", 0), (600, 40, "f32", 128), (2048, 70, "bf16", 128),
    (2500, 20, "f16", 0), (4096, 20, "bf16", 512), (5000, 10, "f32", 0), (9000, 9, "bf16", 256), (16383, 9, "f16", 0)])
def test_norm_of_many_rows(aug, units, dim, rows_a_unit, name, q_block):
    rows = rows_a_unit * units + 3
    g = torch.Generator("cuda").manual_seed(dim)
    x, res = (torch.randn(rows, dim, device="cuda", generator=g).to(TYPES[name]) for _ in range(2))
    if name != "f16":                                     # rows that take another path, between the others
        x[::97, 0] = 1e30
    w = 1 + 0.3 * torch.randn(dim, device="cuda", generator=g)
    s, y, rstd = torch.empty_like(x), torch.empty_like(x), torch.empty(rows, device="cuda")
    q, width = torch.empty(rows, dim, dtype=torch.float8_e4m3fn, device="cuda"), q_block or dim
    scale = torch.empty(rows, -(-dim // width), device="cuda")
    aug.aug_rms_norm_batch(x, w, residual=res, sum_out=s, y_out=y, rstd_out=rstd, q_out=q, scale_out=scale, q_block=q_block)
    ws, wy, wr = R.rms_norm(wide(x), wide(res), wide(w))
    terms = dim / 2 + 16
    near(s, ws, np.abs(ws), 1, "sum")
    near(y, wy, np.abs(wy), terms, "y")
    near(rstd, wr, wr, terms, "rstd")
    want = R.block_scales(wy, q_block)
    near(scale, want, want, terms + 2, "scale")
    by = np.repeat(wide(scale), width, axis=1)[:, :dim]
    v = wy / by
    assert np.all(np.abs(wide(q.float()) - v) <= np.maximum(2.0 ** -4 * np.abs(v), 2.0 ** -10) + (terms + 4) * 2.0 ** -24 * np.abs(v))


@pytest.mark.parametrize("dim,rows_a_unit,name", [(40, 150, "bf16"), (300, 40, "f32"), (700, 20, "f16"), (1001, 20, "f32"), (1500, 10, "bf16"), (2500, 6, "f32"),
                                                  (5000, 3, "bf16"), (9000, 3, "f16")])
def test_norm_gradients_of_many_rows(aug, units, dim, rows_a_unit, name):
    rows = rows_a_unit * units + 3
    g = torch.Generator("cuda").manual_seed(dim)
    x, dy, dsum = (torch.randn(rows, dim, device="cuda", generator=g).to(TYPES[name]) for _ in range(3))
    w = 1 + 0.3 * torch.randn(dim, device="cuda", generator=g)
    rstd = torch.from_numpy(R.rms_norm(wide(x))[2]).float().cuda()
    dx, dw = torch.empty_like(x), torch.empty(dim, device="cuda")
    aug.aug_rms_norm_backward_batch(x, rstd, dy, w, dsum=dsum, dx_out=dx, dweight_out=dw)
    args = (wide(x), wide(rstd), wide(dy), wide(w), wide(dsum))
    want, mag = R.rms_norm_backward(*args), R.rms_norm_backward(*args, magnitude=True)
    near(dx, want[0], mag[0], dim + 16, "dx")
    near(dw, want[1], mag[1], rows + 16, "dweight")


# ---- short convolution: the gradients of the taps over a run of blocks ----

@pytest.mark.parametrize("dim,n_seq,longest,taps,name", [(1280, 200, 130, 4, "f16"), (1281, 220, 90, 3, "f32"), (40, 1700, 40, 4, "f32"),
                                                         (39, 1600, 60, 7, "bf16"), (2048, 150, 100, 2, "bf16")])
def test_convolution_gradients_of_many_blocks(aug, units, dim, n_seq, longest, taps, name):
    lengths = np.random.default_rng(dim).integers(0, longest, n_seq)
    across = 1
    while across < 64 and 2 * across < dim:
        across *= 2
    assert n_seq > 1.3 * -(-4 * units // -(-dim // (2 * across)))       # blocks, at least one a sequence, and runs of them
    off, _, x, w, bias, state, dy = C._inputs(lengths, dim, taps, TYPES[name], dim)
    for act, b, st in (("silu", bias, state), ("none", None, None)):
        dx, dw, db = torch.full_like(dy, 7.0), torch.empty_like(w), torch.empty_like(bias)
        aug.aug_short_conv_backward_batch(off, x, w, dy, bias=b, activation=act, state_in=st, dx_out=dx, dweight_out=dw, dbias_out=db)
        args = (off, wide(x), wide(w), wide(dy), C._n(b), act, C._n(st))
        want, mag = R.short_conv_backward(*args), R.short_conv_backward(*args, magnitude=True)
        near(dx, want[0], mag[0], 2 * taps + 16, "dx")
        near(dw, want[1], mag[1], taps + 16 + lengths.sum(), "dweight")
        near(db, want[2], mag[2], taps + 16 + lengths.sum(), "dbias")


# ---- scan ----

def _some(t, channels):
    """The call's arguments for some of its channels, in 64 bits (one group of b and c)."""
    return {k: wide(v)[:, channels] if k in ("u", "delta", "z") else wide(v)[channels] if k in ("a", "skip", "delta_bias") else wide(v) for k, v in t.items()}


def _forward(aug, lengths, dim, n, g, name, seed, channels=None):
    off, _, t, state, _ = S._inputs(lengths, dim, n, g, TYPES[name], seed)
    y, out = torch.full_like(t["u"], 7.0), torch.empty_like(state)
    aug.aug_scan_batch(off, **t, y_out=y, n_group=g, state_in=state, state_out=out)
    pick = slice(None) if channels is None else channels
    args = dict(n_group=g, state_in=wide(state)[:, pick], **_some(t, pick))
    want, mag = R.scan(off, **args), R.scan(off, **args, magnitude=True)
    near(y[:, pick], want[0], mag[0], S._terms(lengths, n), "y")
    near(out[:, pick], want[1], mag[1], S._terms(lengths, n), "state")


@pytest.mark.parametrize("rows,name", [(2100, "bf16"), (4200, "f32"), (8300, "f16"), (16500, "f32")])
def test_scan_in_long_blocks(aug, units, rows, name):
    """Blocks of 128 to 1024 rows: a sequence that a few groups cannot walk alone, and a short one behind it."""
    g = units // 2                                        # as many tiles of channels
    _forward(aug, [rows, 70], g, 16, g, name, rows)


@pytest.mark.parametrize("dim,n,name", [(2048, 16, "bf16"), (2000, 16, "f32"), (2048, 4, "f16"), (520, 64, "bf16"), (300, 128, "f32")])
def test_scan_of_few_long_sequences(aug, dim, n, name):
    channels = np.unique(np.r_[0, 1, 63, 64, dim // 2, dim - 64:dim])
    _forward(aug, [4000, 3977, 4000, 17] if n < 64 else [1500, 1477], dim, n, 1, name, dim + n, channels)


@pytest.mark.parametrize("dim,n,name", [(1024, 16, "bf16"), (1000, 16, "f32"), (1024, 11, "f16"), (1024, 2, "f32"), (512, 64, "bf16")])
def test_scan_of_many_whole_sequences(aug, dim, n, name):
    """Sequences of several hundred rows, left whole."""
    lengths = np.linspace(200, 600, 60).astype(int)[np.random.default_rng(n).permutation(60)].tolist()
    channels = np.unique(np.r_[0, 1, 63, 64, dim // 2, dim - 40:dim])
    _forward(aug, lengths, dim, n, 1, name, dim + n, channels)


@pytest.mark.parametrize("n_seq,dim,n,name", [(512, 1024, 16, "bf16"), (700, 1000, 11, "f32"), (3000, 2048, 16, "f16"), (900, 512, 64, "bf16"), (4000, 1024, 3, "f32")])
def test_steps_of_many_streams(aug, n_seq, dim, n, name):
    """Several streams to a group."""
    off, _, t, state, _ = S._inputs([1] * n_seq, dim, n, 1, TYPES[name], n_seq)
    y, out = torch.full_like(t["u"], 7.0), torch.empty_like(state)
    aug.aug_scan_step(**t, state_in=state, state_out=out, y_out=y)
    pick = np.unique(np.r_[0, 1, 63, 64, dim // 2, dim - 5:dim])
    args = dict(state_in=wide(state[:, torch.from_numpy(pick).cuda()]), **_some(t, pick))
    want, mag = R.scan(off, **args), R.scan(off, **args, magnitude=True)
    near(y[:, pick], want[0], mag[0], S._terms([1], n), "y")
    near(out[:, pick], want[1], mag[1], S._terms([1], n), "state")


@pytest.mark.parametrize("dim,n,g,rows,name", [(4096, 16, 1, 1500, "bf16"), (192, 11, 64, 2600, "f32"), (4096, 8, 1, 1500, "f32"), (128, 64, 64, 2300, "f16"),
                                               (128, 20, 64, 2300, "bf16"), (128, 128, 64, 1200, "f32")])
def test_scan_gradients_of_many_blocks(aug, units, dim, n, g, rows, name):
    """Runs of several blocks, joined and not: every gradient."""
    lengths = []
    r = np.random.default_rng(dim + n)
    while sum(lengths) < rows:
        lengths.append(int(r.choice([0, 1, r.integers(2, 30), r.integers(30, 200), r.integers(200, 500)])))
    block = 32 if n <= 64 else 16
    tiles = g * -(-dim // g // (64 if n <= 16 else 32 if n <= 64 else 16))
    assert sum(-(-k // block) for k in lengths) > 1.3 * -(-8 * units // tiles)
    off, _, t, state, dy = S._inputs(lengths, dim, n, g, TYPES[name], dim + n)
    got = {"d" + k: torch.full(t[k].shape, 7.0, dtype=dy.dtype, device="cuda") for k in ("u", "delta", "b", "c", "z")}
    got.update(da=torch.empty_like(t["a"]), dskip=torch.empty(dim, device="cuda"), ddelta_bias=torch.empty(dim, device="cuda"))
    aug.aug_scan_backward_batch(off, **t, dy=dy, n_group=g, state_in=state, **{k + "_out": v for k, v in got.items()})
    args = dict(n_group=g, state_in=wide(state), dy=wide(dy), **S._wide(t))
    want, mag = R.scan_backward(off, **args), R.scan_backward(off, **args, magnitude=True)
    for k, v in got.items():
        over = sum(lengths) if k in ("da", "dskip", "ddelta_bias") else dim // g if k in ("db", "dc") else 0
        near(v, want[k], mag[k], 2 * S._terms(lengths, n) + over, k)
    only = torch.empty_like(got["da"])                    # and a call that asks for one of them: the same sums
    aug.aug_scan_backward_batch(off, **t, dy=dy, n_group=g, state_in=state, da_out=only)
    assert torch.equal(only, got["da"])
