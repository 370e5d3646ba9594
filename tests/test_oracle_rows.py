"""Pins of the oracle of the operators on feature rows: closed forms, and gradients against differences.  CPU only."""
import numpy as np
import pytest
import torch

from oracle import rows_oracle as R


def test_norm_of_a_constant_row_is_the_weight():
    w = np.array([1.0, -2.0, 0.5])
    s, y, rstd = R.rms_norm(np.full((2, 3), 3.0), np.full((2, 3), 1.0), w, eps=0.0)
    np.testing.assert_allclose(s, 4.0)
    np.testing.assert_allclose(y, np.tile(w, (2, 1)))
    np.testing.assert_allclose(rstd, 0.25)


def test_e4m3_rounding_is_torchs():
    v = np.concatenate([np.linspace(-460, 460, 4001), np.geomspace(1e-4, 448, 999), [0.0, 2.0 ** -10, 3 * 2.0 ** -10, 464.0]])
    ref = torch.from_numpy(v).float().to(torch.float8_e4m3fn).double().numpy()
    np.testing.assert_array_equal(R.round_e4m3(v.astype(np.float32)), ref)


def test_convolution_is_numpys_and_pieces_join():
    rng = np.random.default_rng(0)
    x, w = rng.standard_normal((19, 3)), rng.standard_normal((3, 4))
    y, state = R.short_conv([0, 19], x, w, act="none")
    for d in range(3):
        np.testing.assert_allclose(y[:, d], np.convolve(x[:, d], w[d, ::-1])[:19], atol=1e-12)
    y1, s1 = R.short_conv([0, 2], x[:2], w, act="none")
    y2, s2 = R.short_conv([0, 17], x[2:], w, act="none", state_in=s1)
    np.testing.assert_allclose(np.concatenate([y1, y2]), y)
    np.testing.assert_array_equal(s2, state)


def test_scan_of_constant_steps_is_a_geometric_sum():
    # step 0.5, rate -0.2, unit inputs: h_t = 0.5 (1 - q^t) / (1 - q), q = exp(-0.1)
    t, one = 30, np.ones((30, 1))
    y, state = R.scan([0, t], one, 0.5 * one, np.array([[-0.2]]), one, 2 * one, act="none")
    q = np.exp(-0.1)
    np.testing.assert_allclose(y[:, 0], 2 * 0.5 * (1 - q ** np.arange(1, t + 1)) / (1 - q))
    np.testing.assert_allclose(state[0, 0, 0], y[-1, 0] / 2)


def _case(seed, n_group=2, gate=True):
    rng = np.random.default_rng(seed)
    rows, dim, n = 9, 4, 3
    off = np.array([0, 5, 5, 9])
    k = dict(u=rng.standard_normal((rows, dim)), delta=rng.standard_normal((rows, dim)), a=-rng.uniform(0.2, 2, (dim, n)),
             b=rng.standard_normal((rows, n_group * n)), c=rng.standard_normal((rows, n_group * n)), skip=rng.standard_normal(dim),
             delta_bias=rng.standard_normal(dim))
    if gate:
        k["z"] = rng.standard_normal((rows, dim))
    return off, k, dict(n_group=n_group, state_in=rng.standard_normal((3, dim, n))), rng.standard_normal((rows, dim))


def _difference(f, args, name, dy, h=1e-6):
    out = np.zeros_like(args[name])
    for i in np.ndindex(out.shape):
        v = {s: dict(args, **{name: args[name].copy()}) for s in (1, -1)}
        for s in v:
            v[s][name][i] += s * h
        out[i] = np.sum((f(**v[1]) - f(**v[-1])) * dy) / (2 * h)
    return out


@pytest.mark.parametrize("gate,act", [(True, "softplus"), (False, "softplus"), (True, "none")])
def test_scan_gradients_are_differences(gate, act):
    off, k, rest, dy = _case(3, gate=gate)
    g = R.scan_backward(off, dy=dy, act=act, **k, **rest)
    for name in k:
        want = _difference(lambda **v: R.scan(off, act=act, **v, **rest)[0], k, name, dy)
        np.testing.assert_allclose(g["d" + name], want, rtol=1e-6, atol=1e-7, err_msg=name)


@pytest.mark.parametrize("act", ["silu", "none"])
def test_convolution_gradients_are_differences(act):
    rng = np.random.default_rng(5)
    off = np.array([0, 1, 1, 8])
    k = dict(x=rng.standard_normal((8, 3)), weight=rng.standard_normal((3, 4)), bias=rng.standard_normal(3))
    st, dy = rng.standard_normal((3, 3, 3)), rng.standard_normal((8, 3))
    got = R.short_conv_backward(off, dy=dy, act=act, state_in=st, **k)
    for name, g in zip(k, got):
        want = _difference(lambda **v: R.short_conv(off, act=act, state_in=st, **v)[0], k, name, dy)
        np.testing.assert_allclose(g, want, rtol=1e-6, atol=1e-8, err_msg=name)


def test_norm_gradients_are_differences():
    rng = np.random.default_rng(6)
    k = dict(x=rng.standard_normal((4, 5)), weight=rng.standard_normal(5))
    dy, dsum = rng.standard_normal((4, 5)), rng.standard_normal((4, 5))
    rstd = R.rms_norm(**k)[2]
    ds, dw = R.rms_norm_backward(k["x"], rstd, dy, k["weight"], dsum)
    f = lambda **v: R.rms_norm(**v)[1]           # noqa: E731
    np.testing.assert_allclose(ds - dsum, _difference(f, k, "x", dy), rtol=1e-6, atol=1e-8)
    np.testing.assert_allclose(dw, _difference(f, k, "weight", dy), rtol=1e-6, atol=1e-8)


def test_magnitudes_bound_the_results():
    off, k, rest, dy = _case(8)
    g, m = R.scan_backward(off, dy=dy, **k, **rest), R.scan_backward(off, dy=dy, magnitude=True, **k, **rest)
    for name in g:
        assert np.all(m[name] >= np.abs(g[name]) - 1e-12), name
