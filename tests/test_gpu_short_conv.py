"""aug_short_conv_batch, its gradients and its form for streams against the 64-bit oracle, through the C ABI."""
import numpy as np
import pytest
import torch

from oracle import rows_oracle as R
from paper_1912_11040_amd import binding
from tests.rows_parity import TYPES, UNTOUCHED, matrix, near, out_matrix, surroundings_untouched, wide

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def aug():
    with binding.Augmenter(0) as a:
        yield a


def _inputs(lengths, dim, taps, dtype, seed, pad=0, shift=0, behind=0, gaps=False):
    """A batch with `behind` rows behind the last sequence; with gaps, a padded layout."""
    rng = np.random.default_rng(seed)
    lengths = np.asarray(lengths, np.int64)
    slots = lengths + (rng.integers(0, 4, len(lengths)) if gaps else 0)
    off = np.concatenate([[0], np.cumsum(slots)]).astype(np.int64)
    rows = int(off[-1]) + behind
    x = matrix(rng.standard_normal((rows, dim)), dtype, pad, shift)
    inside = np.zeros(rows, bool)
    for a, n in zip(off, lengths):
        inside[a:a + n] = True
    x[torch.from_numpy(~inside).cuda()] = float("nan")                # never read
    w = torch.from_numpy(rng.standard_normal((dim, taps))).float().cuda()
    bias = torch.from_numpy(rng.standard_normal(dim)).float().cuda()
    state = torch.from_numpy(rng.standard_normal((len(lengths), taps - 1, dim))).to(dtype).cuda()
    dy = matrix(rng.standard_normal((rows, dim)), dtype, pad, shift)
    dy[torch.from_numpy(~inside).cuda()] = float("nan")
    return off, lengths if gaps else None, x, w, bias, state, dy


RAGGED = [5, 0, 1, 70, 2, 3, 0, 131, 64, 65]
CASES = [([1], 1, 1, {}), ([1], 40, 4, {}), ([3, 0, 2], 8, 4, {}), (RAGGED, 40, 4, dict(behind=3)), (RAGGED, 64, 3, dict(gaps=True, behind=2)),
         (RAGGED, 65, 2, dict(pad=3)), (RAGGED, 100, 8, dict(pad=7, shift=3)), (RAGGED, 520, 4, dict(pad=520, gaps=True)), ([700], 16, 5, {}),
         ([300, 2], 1030, 4, dict(pad=2, shift=1)), ([1] * 90, 72, 6, {}), ([2049, 17], 24, 7, {})]


def _n(t):
    return None if t is None else wide(t)


@pytest.mark.parametrize("name", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("lengths,dim,taps,kw", CASES)
def test_short_conv(aug, lengths, dim, taps, kw, name):
    off, lens, x, w, bias, state, _ = _inputs(lengths, dim, taps, TYPES[name], dim + taps, **kw)
    for act, b, st in (("silu", bias, state), ("none", None, None), ("silu", None, state)):
        y = out_matrix(len(x), dim, TYPES[name], kw.get("pad", 0), kw.get("shift", 0))
        st_out = torch.full_like(state, float("nan"))
        aug.aug_short_conv_batch(off, x, w, y, bias=b, activation=act, state_in=st, state_out=st_out, row_lengths=lens)
        args = (off, _n(x), _n(w), _n(b), act, _n(st), lens)
        want, want_state = R.short_conv(*args)
        near(y, want, R.short_conv(*args, magnitude=True)[0], taps + 12, "y")
        assert np.array_equal(wide(st_out), want_state.reshape(wide(st_out).shape))
        assert surroundings_untouched(y)
        if st is not None:                                            # in place, the same bits
            y2, st2 = torch.empty_like(y), st.clone()
            aug.aug_short_conv_batch(off, x, w, y2, bias=b, activation=act, state_in=st2, state_out=st2, row_lengths=lens)
            assert torch.equal(st2, st_out)


@pytest.mark.parametrize("name", ["bf16", "f32"])
def test_pieces_and_streams_join_to_the_whole(aug, name):
    off, _, x, w, bias, state, _ = _inputs([23], 72, 4, TYPES[name], 5)
    whole, end = torch.empty_like(x), torch.empty_like(state)
    aug.aug_short_conv_batch(off, x, w, whole, bias=bias, state_in=state, state_out=end)
    st, parts = state.clone(), []
    for a, b in ((0, 1), (1, 3), (3, 4), (4, 20)):
        y = torch.empty_like(x[a:b])
        aug.aug_short_conv_batch([0, b - a], x[a:b], w, y, bias=bias, state_in=st, state_out=st)
        parts.append(y)
    for t in range(20, 23):
        y = x[t:t + 1].clone()
        aug.aug_short_conv_step(y, w, st, st, y, bias=bias)           # y in x's place
        parts.append(y)
    assert torch.equal(torch.cat(parts), whole) and torch.equal(st, end)


@pytest.mark.parametrize("name", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("n_seq,dim,taps", [(1, 1, 1), (1, 40, 4), (7, 65, 2), (33, 1024, 4), (3, 1030, 8), (300, 24, 3)])
def test_short_conv_of_streams(aug, n_seq, dim, taps, name):
    off, _, x, w, bias, state, _ = _inputs([1] * n_seq, dim, taps, TYPES[name], n_seq + dim, pad=dim % 3)
    y, out = out_matrix(n_seq, dim, TYPES[name], 2, 1), torch.full_like(state, float("nan"))
    for act, b in (("silu", bias), ("none", None)):
        aug.aug_short_conv_step(x, w, state, out, y, bias=b, activation=act)
        args = (off, _n(x), _n(w), _n(b), act, _n(state))
        want, want_state = R.short_conv(*args)
        near(y, want, R.short_conv(*args, magnitude=True)[0], taps + 12, "y")
        assert np.array_equal(wide(out), want_state.reshape(wide(out).shape)) and surroundings_untouched(y)


@pytest.mark.parametrize("name", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("lengths,dim,taps,kw", CASES)
def test_short_conv_gradients(aug, lengths, dim, taps, kw, name):
    off, lens, x, w, bias, state, dy = _inputs(lengths, dim, taps, TYPES[name], 2 * dim + taps, **kw)
    for act, b, st in (("silu", bias, state), ("none", None, None)):
        dx = out_matrix(len(x), dim, TYPES[name], kw.get("pad", 0), kw.get("shift", 0))
        dw, db = torch.full_like(w, float("nan")), torch.full((dim,), float("nan"), device="cuda")
        aug.aug_short_conv_backward_batch(off, x, w, dy, bias=b, activation=act, state_in=st, dx_out=dx, dweight_out=dw, dbias_out=db,
                                          row_lengths=lens)
        args = (off, _n(x), _n(w), _n(dy), _n(b), act, _n(st), lens)
        want, mag = R.short_conv_backward(*args), R.short_conv_backward(*args, magnitude=True)
        rows = sum(lengths)
        near(dx, want[0], mag[0], 2 * taps + 16, "dx")
        near(dw, want[1], mag[1], taps + 16 + rows, "dweight")
        near(db, want[2], mag[2], taps + 16 + rows, "dbias")
        assert surroundings_untouched(dx)
        dw2, db2 = torch.empty_like(dw), torch.empty_like(db)
        aug.aug_short_conv_backward_batch(off, x, w, dy, bias=b, activation=act, state_in=st, dweight_out=dw2, dbias_out=db2, row_lengths=lens)
        assert torch.equal(dw, dw2) and torch.equal(db, db2)          # without dx, and again: the same bits


def test_sequences_keep_to_themselves(aug):
    """NaN and infinity of one sequence reach no other one, and nothing before them."""
    off, _, x, w, bias, state, dy = _inputs([70, 66, 5], 40, 4, torch.float32, 9)
    y0, y1 = torch.empty_like(x), torch.empty_like(x)
    aug.aug_short_conv_batch(off, x, w, y0, bias=bias, state_in=state)
    x[off[1] + 30] = float("nan")
    dy[off[1] + 30] = float("inf")
    state[2] = float("nan")
    aug.aug_short_conv_batch(off, x, w, y1, bias=bias, state_in=state)
    same = torch.ones(len(x), dtype=torch.bool, device="cuda")
    same[off[1] + 30:off[1] + 34] = False
    same[off[2]:off[2] + 3] = False
    assert torch.equal(y0[same], y1[same]) and bool(y1[~same].isnan().all())


def test_gradients_of_empty_sequences_are_zeros(aug):
    dw, db = torch.full((8, 4), 3.0, device="cuda"), torch.full((8,), 3.0, device="cuda")
    e, w = torch.empty(0, 8, device="cuda"), torch.randn(8, 4, device="cuda")
    for off in ([0], [0, 0, 0]):
        dw.fill_(UNTOUCHED), db.fill_(UNTOUCHED)
        aug.aug_short_conv_backward_batch(off, e, w, e, dx_out=e, dweight_out=dw, dbias_out=db)
        assert float(dw.abs().max()) == 0.0 and float(db.abs().max()) == 0.0
    state = torch.randn(2, 3, 8, device="cuda")
    out = torch.empty_like(state)
    aug.aug_short_conv_batch([0, 0, 0], e, w, e, state_in=state, state_out=out)
    assert torch.equal(out, state)
