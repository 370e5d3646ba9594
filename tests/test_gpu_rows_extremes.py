"""The operators on feature rows where 32 bits end: infinite steps, inputs that are no numbers, growing states, rows beyond the range of their
squares.  What the definition keeps finite stays finite, and what it makes infinite is infinite."""
import numpy as np
import pytest
import torch

from oracle import rows_oracle as R
from paper_1912_11040_amd import binding
from tests import test_gpu_scan as S
from tests.rows_parity import TYPES, half_step, wide

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def aug():
    with binding.Augmenter(0) as a:
        yield a


def agrees(got, want, mag, terms, name):
    """got is want to within its rounding where want is finite, the same infinity where it is one, and no number where it is none."""
    g = wide(got).reshape(want.shape)
    finite = np.isfinite(want)
    assert np.isfinite(mag[finite]).all(), f"{name}: the bound says nothing"
    # 32-bit numbers below 2^-126 are multiples of 2^-149: a rounding among them is off by 2^-150 at most, and decays of at most one, the only
    # ones that lead there, do not enlarge it.
    tol = half_step(got.dtype) * np.abs(want) * (1 + 2.0 ** -7) + terms * (2.0 ** -24 * mag + 2.0 ** -150)
    if got.dtype == torch.float16:
        tol = tol + 2.0 ** -25           # half a step of that type's
    with np.errstate(invalid="ignore"):
        bad = np.where(finite, ~(np.abs(g - want) <= tol), np.where(np.isnan(want), np.isfinite(g), g != want))
    assert not bad.any(), f"{name}: {bad.sum()} of {bad.size} off, first at {tuple(np.argwhere(bad)[0])}: {g[bad][0]!r} for {want[bad][0]!r}"


def _gradients(aug, off, t, dy, g, state, softplus=True):
    like = dict(du="u", ddelta="delta", db="b", dc="c", dz="z")
    out = {k: torch.full(t[v].shape, 7.0, dtype=dy.dtype, device="cuda") for k, v in like.items() if v in t}
    out.update(da=torch.empty_like(t["a"]), dskip=torch.empty_like(t["a"][:, 0]), ddelta_bias=torch.empty_like(t["a"][:, 0]))
    aug.aug_scan_backward_batch(off, **t, dy=dy, n_group=g, softplus=softplus, state_in=state, **{k + "_out": v for k, v in out.items()})
    return out


# ---- a step that is infinite: the state forgets, and the gradient stops there ----

@pytest.mark.parametrize("name", ["f16", "f32"])
@pytest.mark.parametrize("n", [1, 2, 3, 5, 7, 8, 11, 16, 17, 33, 65, 100, 128])
@pytest.mark.parametrize("lengths,last", [([21, 13, 4], True), ([30, 300, 9], False)])
def test_infinite_step(aug, lengths, last, n, name):
    """One channel's step is infinite in one row of the second sequence.  The rows before it (their gradients too), the other channels and the
    other sequences are those of the definition, whatever the number of states; in that row the output is infinite."""
    dim, g, d = 70, 2, 41
    off, _, t, state, dy = S._inputs(lengths, dim, n, g, TYPES[name], 300 + n)
    at = int(off[2]) - 1 if last else int(off[1]) + lengths[1] // 2
    t["delta"][at, d] = float("inf")
    for k in ("u", "b", "c", "z"):                        # one sign, so that the definition's output there is an infinity
        t[k][at] = t[k][at].abs() + 0.125
    args = dict(n_group=g, state_in=wide(state), **_wide(t))
    y, out = torch.empty_like(dy), torch.empty_like(state)
    aug.aug_scan_batch(off, **t, y_out=y, n_group=g, state_in=state, state_out=out)
    with np.errstate(all="ignore"):
        want, mag = R.scan(off, **args), R.scan(off, **args, magnitude=True)
        gwant, gmag = (R.scan_backward(off, dy=wide(dy), magnitude=m, **args) for m in (False, True))
    got = _gradients(aug, off, t, dy, g, state)
    assert want[0][at, d] == np.inf and np.isfinite(gwant["du"][at - 1, d])
    # Behind that row its channel holds infinities, which are lost where a decay is too small for 32 bits: not compared, nor what sums over
    # them (db and dc of its group's states from that row on, the channel's parameters).
    behind = np.zeros(len(dy), bool)
    behind[at + 1:int(off[2])] = True
    terms = S._terms(lengths, n)

    def compare(what, k, ref, bound, extra):
        ref, bound = ref.copy(), bound.copy()
        g_ = wide(what).copy().reshape(ref.shape)
        if k in ("y", "du", "ddelta", "dz"):
            skip = np.zeros(ref.shape, bool)
            skip[behind, d] = True
            skip[at, d] = k != "y"
        elif k in ("db", "dc"):
            skip = np.zeros(ref.shape, bool)
            skip[at:int(off[2]), (d // (dim // g)) * n:(d // (dim // g) + 1) * n] = True
        else:
            skip = np.zeros(ref.shape, bool)
            if k == "state":
                skip[1, d] = True
            else:
                skip[d] = True
        for v in (ref, bound, g_):
            v[skip] = 1.0
        agrees(torch.from_numpy(g_).to(what.dtype), ref, bound, extra, k)

    compare(y, "y", want[0], mag[0], terms)
    compare(out, "state", want[1], mag[1], terms)
    for k, v in got.items():
        over = sum(lengths) if k in ("da", "dskip", "ddelta_bias") else dim // g if k in ("db", "dc") else 0
        compare(v, k, gwant[k], gmag[k], 2 * terms + over)


def _wide(t):
    return {k: wide(v) for k, v in t.items()}


# ---- states that grow beyond 32 bits inside a block of rows, where nothing is that grows, or next to nothing ----

def _growing(dim, n, softplus, seed):
    """A sequence of 150 rows in blocks of 32 or fewer: in rows 32 to 45 every state of the even channels grows by e^93 in all, more than the largest
    32-bit number.  The input is zero up to row 95 and dy from row 32 on."""
    off, _, t, _, dy = S._inputs([150, 40], dim, n, 1, torch.float32, seed, gate=False)
    dy[32:150] = 0
    t["u"][:96] = 0
    t["a"][::2] = 0.5 if softplus else -0.5
    t["delta"] = -t["delta"].abs() - 2 if softplus else t["delta"].abs() * 0.1
    t["delta_bias"] = torch.zeros(dim, device="cuda")
    t["delta"][32:46, ::2] = 12.0 if softplus else -12.0
    t["delta"][36, ::2] = 30.0 if softplus else -30.0
    return off, t, dy


# the roundings of a decay's argument, its step's and its rate's among them, are relative to the argument: six of |step a| in every row
GROWN = 6 * 93


@pytest.mark.parametrize("softplus", [True, False])
@pytest.mark.parametrize("n", [3, 16, 64, 100])
@pytest.mark.parametrize("row,value", [(47, 0.0), (47, 1e-30)])
def test_gradients_through_growing_decays(aug, row, value, n, softplus):
    """The gradient that a block hands to the rows before it is zero times e^93, or 1e-30 times that."""
    dim = 24
    off, t, dy = _growing(dim, n, softplus, 50 + n)
    dy[row] = value
    args = dict(act="softplus" if softplus else "none", **_wide(t))
    want, mag = (R.scan_backward(off, dy=wide(dy), magnitude=m, **args) for m in (False, True))
    got = _gradients(aug, off, t, dy, 1, None, softplus)
    for k, v in got.items():
        over = 190 if k in ("da", "dskip", "ddelta_bias") else dim if k in ("db", "dc") else 0
        agrees(v, want[k], mag[k], 2 * S._terms([150], n) + over + GROWN, k)


@pytest.mark.parametrize("rows", [150, 1200])
@pytest.mark.parametrize("n", [3, 16, 64, 100])
def test_states_and_gradients_through_blocks_that_grow(aug, n, rows):
    """A block of rows that multiplies states by e^93: a state of 1e-30 that comes into it, and a gradient of 1e-30 that comes in from behind,
    are within 32 bits behind it.  Few blocks are joined one after another, many by several groups of lanes."""
    dim = 24
    off, _, t, _, dy = S._inputs([rows, 40], dim, n, 1, torch.float32, 70 + n, gate=False)
    dy[:], t["u"][:rows] = 0, 0
    t["u"][3], dy[rows - 9] = 1e-30, 1e-30
    t["a"][::2], t["delta_bias"] = 0.5, torch.zeros(dim, device="cuda")
    t["delta"][:rows, ::2] = -20.0
    t["delta"][64:78, ::2] = 12.0                         # in blocks of 64 rows the second one, in smaller ones alone in one too
    t["delta"][68, ::2] = 30.0
    args = _wide(t)
    terms = S._terms([rows], n) + GROWN
    # The even channels' state is 2e-9 times 1e-30 times b before it grows, and a rounding among numbers below 2^-126 is that of 2^-126: the bound
    # counts step u and step u b of that row as no smaller.
    least = dict(args, u=args["u"].copy(), b=args["b"].copy())
    least["u"][3] = np.maximum(args["u"][3], 2.0 ** -126 / R.softplus(args["delta"][3]))
    least["b"][3] = np.maximum(np.abs(args["b"][3]), 1.0)
    want, mag = R.scan(off, **args), R.scan(off, **least, magnitude=True)
    y, out = torch.empty_like(dy), torch.empty(2, dim, n, device="cuda")
    aug.aug_scan_batch(off, **t, y_out=y, state_out=out)
    agrees(y, want[0], mag[0], terms, "y")
    agrees(out, want[1], mag[1], terms, "state")
    want, mag = R.scan_backward(off, dy=wide(dy), **args), R.scan_backward(off, dy=wide(dy), magnitude=True, **least)
    for k, v in _gradients(aug, off, t, dy, 1, None).items():
        over = rows + 40 if k in ("da", "dskip", "ddelta_bias") else dim if k in ("db", "dc") else 0
        agrees(v, want[k], mag[k], 2 * terms + over, k)


# ---- what is no number in a sequence's last row ----

@pytest.mark.parametrize("name", ["bf16", "f32"])
@pytest.mark.parametrize("value", [float("nan"), float("inf")])
@pytest.mark.parametrize("lengths,n", [([13], 16), ([40, 21, 3], 11), ([131, 65], 8), ([33, 7], 64), ([17, 30], 128)])
def test_last_rows_state_has_no_part_in_the_rates_gradient(aug, lengths, n, value, name):
    """An input that is no number in a sequence's last row reaches that row's state, which no row follows: the gradient by the rates has the states
    before each row only, and stays what it is."""
    dim, g = 68, 2
    off, _, t, state, dy = S._inputs(lengths, dim, n, g, TYPES[name], 90 + n)
    for i in range(len(lengths)):
        t["u"][int(off[i + 1]) - 1, 5 + i] = value
    args = dict(n_group=g, state_in=wide(state), **_wide(t))
    with np.errstate(invalid="ignore"):
        want, mag = (R.scan_backward(off, dy=wide(dy), magnitude=m, **args) for m in (False, True))
    got = _gradients(aug, off, t, dy, g, state)
    assert np.isfinite(want["da"]).all() and not np.isfinite(want["dskip"]).all()
    agrees(got["da"], want["da"], mag["da"], 2 * S._terms(lengths, n) + sum(lengths), "da")
    agrees(got["du"], want["du"], mag["du"], 2 * S._terms(lengths, n), "du")


# ---- rows whose squares are beyond 32 bits, and rows beyond whose squares nothing is ----

LOUD = [1e30, 3e38, 2e19, 1.0, 3e16]
QUIET = [1e-17, 1e-23, 1e-30, 1.0, 3e-38, 1e-41, 0.0]


def _rows_of(dim, levels, dtype, seed):
    """Rows of values between 2^-6 of a level and it, one of them the level itself, in the type and in 64 bits."""
    rng = np.random.default_rng(seed)
    v = rng.uniform(2.0 ** -6, 1.0, (len(levels), dim)) * rng.choice([-1.0, 1.0], (len(levels), dim))
    v[:, dim // 2] = 1.0
    x = torch.from_numpy(v * np.array(levels)[:, None]).to(dtype)
    assert torch.isfinite(x).all()
    return x.cuda()


@pytest.mark.parametrize("name", ["bf16", "f32"])
@pytest.mark.parametrize("dim,q_block", [(1, 0), (40, 16), (100, 0), (500, 64), (1001, 128), (3000, 0), (4100, 512), (9000, 0), (16384, 256)])
@pytest.mark.parametrize("levels,eps", [(LOUD, 1e-6), (LOUD, 0.0), (LOUD, 1e38), (QUIET, 0.0), (QUIET, 1e-38), (QUIET, 1e-30), (QUIET, 1e-6)])
def test_norm_beyond_the_range_of_squares(aug, levels, eps, dim, q_block, name):
    dtype = TYPES[name]
    x = _rows_of(dim, levels, dtype, dim)
    w = torch.linspace(0.5, 1.5, dim, device="cuda")
    rows, width = len(levels), q_block or dim
    y, q = torch.empty_like(x), torch.empty(rows, dim, dtype=torch.float8_e4m3fn, device="cuda")
    scale, rstd = torch.empty(rows, -(-dim // width), device="cuda"), torch.empty(rows, device="cuda")
    aug.aug_rms_norm_batch(x, w, eps=eps, y_out=y, q_out=q, scale_out=scale, rstd_out=rstd, q_block=q_block)
    with np.errstate(divide="ignore", invalid="ignore"):
        # (eps as the call gets it)
        _, want, r = R.rms_norm(wide(x), None, wide(w), float(np.float32(eps)))
    # a reciprocal root beyond 32 bits is infinite, one below 2^-126 has the step of those
    r = np.where(r > np.finfo(np.float32).max, np.inf, r)
    terms = dim / 2 + 16
    agrees(rstd, r, np.abs(r), terms, "rstd")
    agrees(y, want, np.abs(want), terms, "y")
    if levels[-1] == 0.0 and eps == 0.0:
        want = want[:-1]                                  # (zero by zero)
        assert np.isnan(wide(scale)[-1]).all()
    n = len(want)
    scales = R.block_scales(want, q_block)
    agrees(scale[:n], scales, scales, terms + 2, "scale")
    by = np.repeat(wide(scale)[:n], width, axis=1)[:, :dim]
    v = np.divide(want, by, out=np.zeros_like(want), where=by >= 2.0 ** -126)
    seen = by >= 2.0 ** -126                              # (scales of at least the smallest normal number)
    got = wide(q.float())[:n]
    assert np.all(np.abs(got - v)[seen] <= (np.maximum(2.0 ** -4 * np.abs(v), 2.0 ** -10) + (terms + 4) * 2.0 ** -24 * np.abs(v))[seen])


@pytest.mark.parametrize("name", ["bf16", "f32"])
def test_norm_of_a_row_with_one_loud_value(aug, name):
    """One value of 1e30 among ordinary ones: the row's scale is that value's, and no other row's."""
    x = torch.randn(4, 96, device="cuda").to(TYPES[name])
    x[3, 5] = 1e30
    y, q, scale, rstd = torch.empty_like(x), torch.empty(4, 96, dtype=torch.float8_e4m3fn, device="cuda"), torch.empty(4, 3, device="cuda"), torch.empty(4, device="cuda")
    aug.aug_rms_norm_batch(x, None, y_out=y, q_out=q, scale_out=scale, rstd_out=rstd, q_block=32)
    _, want, r = R.rms_norm(wide(x))
    agrees(rstd, r, r, 64, "rstd")
    agrees(y, want, np.abs(want), 64, "y")
    agrees(scale, R.block_scales(want, 32), R.block_scales(want, 32), 66, "scale")
    assert wide(q.float())[3, 5] == 448.0 and wide(y)[3, 5] > 9.7


@pytest.mark.parametrize("name", ["bf16", "f32"])
@pytest.mark.parametrize("dim", [1, 40, 500, 1001, 3000, 9000])
def test_norm_gradients_of_loud_and_quiet_rows(aug, dim, name):
    """Rows of 1e30 to 1e-30, whose reciprocal roots' third powers are beyond 32 bits: both terms of the gradient are there."""
    levels = [1e30, 3e18, 1e13, 1e6, 1.0, 1e-6, 1e-13, 1e-20, 1e-30]
    x = _rows_of(dim, levels, TYPES[name], dim)
    dy = _rows_of(dim, [1.0] * len(levels), TYPES[name], dim + 1)
    w = torch.linspace(0.5, 1.5, dim, device="cuda")
    rstd = torch.from_numpy(R.rms_norm(wide(x), eps=0.0)[2]).float().cuda()
    dx, dw = torch.empty_like(x), torch.empty_like(w)
    aug.aug_rms_norm_backward_batch(x, rstd, dy, w, dx_out=dx, dweight_out=dw)
    args = (wide(x), wide(rstd), wide(dy), wide(w))
    want, mag = R.rms_norm_backward(*args), R.rms_norm_backward(*args, magnitude=True)
    agrees(dx, want[0], mag[0], dim + 16, "dx")
    agrees(dw, want[1], mag[1], len(levels) + 16, "dweight")


@pytest.mark.parametrize("name", ["bf16", "f32"])
@pytest.mark.parametrize("dim,q_block", [(40, 16), (100, 0), (1001, 128), (4100, 0)])
@pytest.mark.parametrize("level", [1e-39, 1e-40, 1e-41, 3e-42, 3e-43, 1e-44])
def test_scales_below_the_normal_numbers(aug, level, dim, q_block, name):
    """Outputs so small that their scale is one of few bits: it is none less than the block's largest value over 448, so that codes are numbers."""
    x = _rows_of(dim, [1.0, 1.0], TYPES[name], dim)
    w = torch.full((dim,), level, device="cuda")
    q, width = torch.empty(2, dim, dtype=torch.float8_e4m3fn, device="cuda"), q_block or dim
    scale = torch.empty(2, -(-dim // width), device="cuda")
    aug.aug_rms_norm_batch(x, w, q_out=q, scale_out=scale, q_block=q_block)
    _, want, _ = R.rms_norm(wide(x), None, wide(w))
    exact, got = R.block_scales(want, q_block), wide(scale)
    # y is off by half a step of 2^-149 and 64 + dim / 2 roundings, the quotient is rounded up
    tol = 2.0 ** -150 / 448 + (dim / 2 + 64) * 2.0 ** -24 * exact
    assert np.all(got >= exact - tol) and np.all(got <= exact + tol + 2.0 ** -149)
    by = np.repeat(got, width, axis=1)[:, :dim]
    v, codes = np.divide(want, by, out=np.zeros_like(want), where=by > 0), wide(q.float())
    assert np.isfinite(codes).all()
    off = np.divide(2.0 ** -150, by, out=np.zeros_like(want), where=by > 0) + (dim / 2 + 64) * 2.0 ** -24 * np.abs(v)
    assert np.all(np.abs(codes - v) <= np.maximum(2.0 ** -4 * (np.abs(v) + off), 2.0 ** -10) + off)


# ---- steps of both signs, all values well within 32 bits ----

def _signed(lengths, dim, n, g, dtype, seed):
    off, _, t, state, dy = S._inputs(lengths, dim, n, g, dtype, seed, plain=True)
    t["a"] = t["a"] * (1.5 / t["a"].abs().max())          # so that a row's decay is e^3 at most, and a long sequence's product e^20
    t["delta"] = t["delta"] * 0.5
    return off, t, state, dy


@pytest.mark.parametrize("name", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("n_seq,dim,n,g", [(4, 10, 128, 5), (9, 66, 100, 3), (33, 64, 64, 1), (5, 40, 16, 1), (7, 20, 3, 2)])
def test_streams_with_steps_of_both_signs(aug, n_seq, dim, n, g, name):
    off, t, state, _ = _signed([1] * n_seq, dim, n, g, TYPES[name], 7 * n_seq + n)
    y, out = torch.empty_like(t["u"]), torch.empty_like(state)
    aug.aug_scan_step(**t, state_in=state, state_out=out, y_out=y, n_group=g, softplus=False)
    args = dict(n_group=g, state_in=wide(state), act="none", **_wide(t))
    want, mag = R.scan(off, **args), R.scan(off, **args, magnitude=True)
    assert mag[0].max() < 6e4 and mag[1].max() < 6e4      # every element is compared, in every type
    agrees(y, want[0], mag[0], S._terms([1], n) + 18, "y")             # (six of the decay's argument, which is 3 at most)
    agrees(out, want[1], mag[1], S._terms([1], n) + 18, "state")


@pytest.mark.parametrize("name", ["bf16", "f32"])
@pytest.mark.parametrize("lengths,dim,n,g", [([70, 5, 33], 72, 16, 1), ([300], 66, 11, 3), ([100, 40], 24, 128, 2), ([64, 64], 64, 64, 1)])
def test_gradients_with_steps_of_both_signs(aug, lengths, dim, n, g, name):
    off, t, state, dy = _signed(lengths, dim, n, g, TYPES[name], dim + n)
    args = dict(n_group=g, state_in=wide(state), act="none", **_wide(t))
    want, mag = R.scan(off, **args), R.scan(off, **args, magnitude=True)
    argument = 6 * max(np.abs(args["delta"][a:b, :, None] * args["a"][None]).sum(0).max() for a, b in R.spans(off) if b > a)
    terms = S._terms(lengths, n) + argument
    y, out = torch.empty_like(dy), torch.empty_like(state)
    aug.aug_scan_batch(off, **t, y_out=y, n_group=g, softplus=False, state_in=state, state_out=out)
    agrees(y, want[0], mag[0], terms, "y")
    agrees(out, want[1], mag[1], terms, "state")
    want, mag = (R.scan_backward(off, dy=wide(dy), magnitude=m, **args) for m in (False, True))
    for k, v in _gradients(aug, off, t, dy, g, state, softplus=False).items():
        over = sum(lengths) if k in ("da", "dskip", "ddelta_bias") else dim // g if k in ("db", "dc") else 0
        agrees(v, want[k], mag[k], 2 * terms + over, k)


@pytest.mark.parametrize("n", [3, 11, 16, 64, 128])
@pytest.mark.parametrize("value", [float("nan"), 1e30])
def test_gradients_behind_a_step_that_is_no_number(aug, value, n):
    """A step of NaN makes NaN of its channel's gradients in every row before it, also where no gradient comes from behind; a step that forgets the state makes
    zeros of what comes from behind."""
    dim = 20
    off, _, t, state, dy = S._inputs([150, 9], dim, n, 1, torch.float32, 110 + n)
    dy[60:150] = 0
    t["delta"][100, 7] = value
    args = dict(state_in=wide(state), **_wide(t))
    with np.errstate(all="ignore"):
        want, mag = (R.scan_backward(off, dy=wide(dy), magnitude=m, **args) for m in (False, True))
    assert np.isnan(want["du"][:101, 7]).all() == np.isnan(value)
    got = _gradients(aug, off, t, dy, 1, state)
    for k in ("du", "ddelta"):
        ref, bound, g = want[k].copy(), mag[k].copy(), wide(got[k]).copy()
        for v in (ref, bound, g):
            v[100:150, 7] = 1.0                           # (there and behind it the states are beyond 32 bits, or NaN)
        agrees(torch.from_numpy(g).float(), ref, bound, 2 * S._terms([150], n), k)
