"""The operators on feature rows as they are used: behind the front end, one after another and back, as streams, in graphs, on other streams,
in matrices beyond 2^31 elements, between the library's other calls."""
import numpy as np
import pytest
import torch

from oracle import aug_oracle as O
from oracle import rows_oracle as R
from paper_1912_11040_amd import binding
from paper_1912_11040_amd import workloads as W
from tests.parity import dev
from tests.rows_parity import UNTOUCHED, near, wide

pytestmark = pytest.mark.gpu

FE = W.FrontendConfig()
DIM, N, TAPS = FE.n_mel, 16, 4                       # the features themselves are the channels


class Block:
    """Norm, short convolution, a product that makes step, b and c, the scan, on the front end's rows."""

    def __init__(self, dtype, seed=0):
        g = torch.Generator("cuda").manual_seed(seed)
        r = lambda *s, scale=1.0: scale * torch.randn(s, device="cuda", generator=g)          # noqa: E731
        self.dtype = dtype
        self.norm_w, self.conv_w, self.conv_b = 1 + r(DIM, scale=0.2), r(DIM, TAPS, scale=0.5), r(DIM, scale=0.2)
        self.project = r(DIM, DIM + 2 * N, scale=DIM ** -0.5)
        self.a, self.skip, self.bias = -torch.exp(r(DIM, N, scale=0.5)), r(DIM), r(DIM, scale=0.5) - 2

    def buffers(self, rows, n_seq):
        e = lambda *s, t=self.dtype: torch.full(s, UNTOUCHED, dtype=t, device="cuda")        # noqa: E731
        f = torch.float32
        return dict(x=e(rows, DIM), sum=e(rows, DIM), norm=e(rows, DIM), rstd=e(rows, t=f), conv=e(rows, DIM), made=e(rows, DIM + 2 * N),
                    y=e(rows, DIM), conv_state=e(n_seq, TAPS - 1, DIM), state=e(n_seq, DIM, N, t=f),
                    du=e(rows, DIM), dmade=e(rows, DIM + 2 * N), dz=e(rows, DIM), da=e(DIM, N, t=f), dskip=e(DIM, t=f), dbias=e(DIM, t=f),
                    dnorm=e(rows, DIM), dconv_w=e(DIM, TAPS, t=f), dconv_b=e(DIM, t=f), dx=e(rows, DIM), dnorm_w=e(DIM, t=f))

    def scan_args(self, b):
        return dict(u=b["conv"], delta=b["made"][:, :DIM], a=self.a, b=b["made"][:, DIM:DIM + N], c=b["made"][:, DIM + N:], skip=self.skip,
                    z=b["norm"], delta_bias=self.bias)

    def forward(self, aug, b, off, residual, lengths=None):
        aug.aug_rms_norm_batch(b["x"], self.norm_w, residual=residual, sum_out=b["sum"], y_out=b["norm"], rstd_out=b["rstd"])
        aug.aug_short_conv_batch(off, b["norm"], self.conv_w, b["conv"], bias=self.conv_b, state_out=b["conv_state"], row_lengths=lengths)
        torch.matmul(b["conv"].float(), self.project, out=self._made(b))
        b["made"].copy_(self._made(b))
        aug.aug_scan_batch(off, **self.scan_args(b), y_out=b["y"], state_out=b["state"], row_lengths=lengths)

    def _made(self, b):
        if "made32" not in b:
            b["made32"] = torch.empty(b["made"].shape, device="cuda")
        return b["made32"]

    def backward(self, aug, b, off, dy, lengths=None):
        m = b["dmade"]
        aug.aug_scan_backward_batch(off, **self.scan_args(b), dy=dy, du_out=b["du"], ddelta_out=m[:, :DIM], db_out=m[:, DIM:DIM + N],
                                    dc_out=m[:, DIM + N:], dz_out=b["dz"], da_out=b["da"], dskip_out=b["dskip"], ddelta_bias_out=b["dbias"],
                                    row_lengths=lengths)
        aug.aug_short_conv_backward_batch(off, b["norm"], self.conv_w, b["du"], bias=self.conv_b, dx_out=b["dnorm"], dweight_out=b["dconv_w"],
                                          dbias_out=b["dconv_b"], row_lengths=lengths)
        aug.aug_rms_norm_backward_batch(b["sum"], b["rstd"], b["dnorm"], self.norm_w, dsum=b["dz"], dx_out=b["dx"], dweight_out=b["dnorm_w"])


def _utterances(lens, seed):
    rng = np.random.default_rng(seed)
    off = np.concatenate([[0], np.cumsum(lens)]).astype(np.int64)
    frames = np.array([O.frame_count(int(n), FE.win, FE.hop) for n in lens], np.int64)
    return off, dev(rng.standard_normal(int(off[-1])).astype(np.float32)), dev(rng.uniform(0.8, 1.2, len(lens)).astype(np.float32)), frames


@pytest.mark.parametrize("padded", [False, True])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_from_waveforms_to_gradients(dtype, padded):
    """Each step against the oracle on what the step before it gave."""
    off, wave, alpha, frames = _utterances([16000, 399, 8000, 25000, 700], 3)
    foff = np.arange(6) * int(frames.max() + 2) if padded else np.concatenate([[0], np.cumsum(frames)])
    lengths = frames if padded else None
    rows, blk = int(foff[-1]), Block(dtype)
    inside = np.zeros(rows, bool)
    for a, n in zip(foff, frames):
        inside[a:a + n] = True
    b = blk.buffers(rows, 5)
    feats = torch.empty(rows, DIM, device="cuda")
    with binding.Augmenter(0) as aug:
        aug.aug_vtlp_mel_batch(off, wave, alpha, FE, foff, feats)
        b["x"].copy_(feats)
        residual = (torch.randn(rows, DIM, device="cuda") * 0.5).to(dtype)
        dy = torch.randn(rows, DIM, device="cuda").to(dtype)
        blk.forward(aug, b, foff, residual, lengths)
        if padded:                                    # the norm knows of no sequences; what it makes of the other rows is not read
            b["norm"][torch.from_numpy(~inside).cuda()] = float("nan")
        blk.backward(aug, b, foff, dy, lengths)
        torch.cuda.synchronize()
    longest = int(frames.max())
    s, y, rstd = R.rms_norm(wide(b["x"]), wide(residual), wide(blk.norm_w))
    near(b["sum"], s, np.abs(s), 1, "sum")
    near(b["norm"][torch.from_numpy(inside).cuda()], y[inside], np.abs(y[inside]), DIM / 2 + 16, "norm")
    k = dict(bias=wide(blk.conv_b), row_lengths=lengths)
    args = (foff, wide(b["norm"]), wide(blk.conv_w))
    near(b["conv"], R.short_conv(*args, **k)[0], R.short_conv(*args, **k, magnitude=True)[0], TAPS + 12, "conv")
    sa = {n: wide(v) for n, v in blk.scan_args(b).items()}
    want, mag = R.scan(foff, **sa, row_lengths=lengths), R.scan(foff, **sa, row_lengths=lengths, magnitude=True)
    terms = 64 + 6 * longest + N
    near(b["y"], want[0], mag[0], terms, "y")
    near(b["state"], want[1], mag[1], terms, "state")
    want, mag = (R.scan_backward(foff, dy=wide(dy), **sa, row_lengths=lengths, magnitude=f) for f in (False, True))
    m = b["dmade"]
    for name, got in dict(du=b["du"], ddelta=m[:, :DIM], db=m[:, DIM:DIM + N], dc=m[:, DIM + N:], dz=b["dz"], da=b["da"], dskip=b["dskip"],
                          ddelta_bias=b["dbias"]).items():
        near(got, want[name], mag[name], 2 * terms + (rows if name in ("da", "dskip", "ddelta_bias") else DIM), name)
    args = (foff, wide(b["norm"]), wide(blk.conv_w), wide(b["du"]))
    want, mag = R.short_conv_backward(*args, **k), R.short_conv_backward(*args, **k, magnitude=True)
    near(b["dnorm"], want[0], mag[0], 2 * TAPS + 16, "dnorm")
    near(b["dconv_w"], want[1], mag[1], TAPS + 16 + rows, "dconv_w")
    near(b["dconv_b"], want[2], mag[2], TAPS + 16 + rows, "dconv_b")
    args = (wide(b["sum"]), wide(b["rstd"]), wide(b["dnorm"]), wide(blk.norm_w), wide(b["dz"]))
    want, mag = R.rms_norm_backward(*args), R.rms_norm_backward(*args, magnitude=True)
    near(b["dx"], want[0], mag[0], DIM + 16, "dx")
    near(b["dnorm_w"], want[1], mag[1], rows + 16, "dnorm_w")


def test_streams_give_what_the_batch_gives():
    """Three utterances row by row, as a server gets them, against the batch."""
    dtype, rows, blk = torch.float32, 20, Block(torch.float32, 4)
    off = np.arange(4) * rows
    b = blk.buffers(3 * rows, 3)
    b["x"].normal_()
    conv_state, state = torch.zeros(3, TAPS - 1, DIM, device="cuda"), torch.zeros(3, DIM, N, device="cuda")
    with binding.Augmenter(0) as aug:
        blk.forward(aug, b, off, None)
        s = blk.buffers(3, 3)
        for t in range(rows):
            s["x"].copy_(b["x"].view(3, rows, DIM)[:, t])
            aug.aug_rms_norm_batch(s["x"], blk.norm_w, sum_out=s["sum"], y_out=s["norm"])
            aug.aug_short_conv_step(s["norm"], blk.conv_w, conv_state, conv_state, s["conv"], bias=blk.conv_b)
            assert torch.equal(s["conv"], b["conv"].view(3, rows, DIM)[:, t])
            s["made"].copy_(b["made"].view(3, rows, -1)[:, t])           # (a product of other sizes may round otherwise)
            aug.aug_scan_step(**blk.scan_args(s), state_in=state, state_out=state, y_out=s["y"])
            sa = {n: wide(v) for n, v in blk.scan_args(b).items()}
            if t == 0:
                want, mag = R.scan(off, **sa), R.scan(off, **sa, magnitude=True)
            pick = np.arange(3) * rows + t
            near(s["y"], want[0][pick], mag[0][pick], 64 + 6 * rows + N, "y")
        assert torch.equal(conv_state, b["conv_state"])
        near(state, want[1], mag[1], 64 + 6 * rows + N, "state")


@pytest.mark.parametrize("lens", [[40, 7, 90], [700]])
def test_captured_calls_replay(lens):
    """Forward and backward, recorded once; replays on new inputs, eager calls of the same context with the same sequences, synchronisations
    and another context's calls between them, each against the eager result."""
    off = np.concatenate([[0], np.cumsum(lens)]).astype(np.int64)
    rows, blk = int(off[-1]), Block(torch.float32, 5)
    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(stream), binding.Augmenter(0) as aug, binding.Augmenter(0) as other:
        b, e = blk.buffers(rows, len(lens)), blk.buffers(rows, len(lens))
        dy = torch.randn(rows, DIM, device="cuda")
        b["x"].normal_()

        def both(a, into):
            a.aug_rms_norm_batch(into["x"], blk.norm_w, sum_out=into["sum"], y_out=into["norm"], rstd_out=into["rstd"])
            a.aug_short_conv_batch(off, into["norm"], blk.conv_w, into["conv"], bias=blk.conv_b, state_out=into["conv_state"])
            a.aug_scan_batch(off, **blk.scan_args(into), y_out=into["y"], state_out=into["state"])
            blk.backward(a, into, off, dy)
            a.aug_scan_step(**{k: v[:len(lens)] if v.shape[0] == rows else v for k, v in blk.scan_args(into).items()}, state_in=into["state"],
                            state_out=into["state"], y_out=into["made"][:len(lens), :DIM])

        for into in (b, e):
            into["made"].normal_()
        both(aug, b)
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=stream):
            both(aug, b)
        names = [n for n in b if n != "made32"]
        for i in range(4):
            made = torch.randn(rows, DIM + 2 * N, device="cuda")
            x = torch.randn(rows, DIM, device="cuda")
            for into in (b, e):
                into["x"].copy_(x)
                into["made"].copy_(made)
            graph.replay()
            if i % 2:
                torch.cuda.synchronize()
            both(aug if i < 2 else other, e)
            torch.cuda.synchronize()
            for n in names:
                assert torch.equal(b[n].nan_to_num(), e[n].nan_to_num()), (i, n)
        del graph
        torch.cuda.synchronize()


def test_capture_needs_a_call_before_it():
    blk, stream = Block(torch.float32, 6), torch.cuda.Stream()
    off = np.array([0, 50])
    with torch.cuda.stream(stream), binding.Augmenter(0) as aug:
        b = blk.buffers(50, 1)
        b["norm"].normal_()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=stream):
            b["sum"].copy_(b["norm"])
            with pytest.raises(binding.AugError) as err:
                aug.aug_short_conv_batch(off, b["norm"], blk.conv_w, b["conv"])
        assert err.value.code == binding.AUG_ERR_UNSUPPORTED and "captured" in str(err.value)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(b["sum"], b["norm"]) and bool((b["conv"] == UNTOUCHED).all())
        aug.aug_short_conv_batch(off, b["norm"], blk.conv_w, b["conv"])                      # and the context works on
        torch.cuda.synchronize()
        assert bool((b["conv"] != UNTOUCHED).any())
        del graph


def test_other_calls_between():
    """Front-end calls, other sequences and other operators between two calls of the same sequences change nothing."""
    off, wave, alpha, frames = _utterances([9000, 4000], 7)
    foff = np.concatenate([[0], np.cumsum(frames)])
    blk = Block(torch.float32, 8)
    with binding.Augmenter(0) as aug:
        b = blk.buffers(int(foff[-1]), 2)
        b["x"].normal_()
        blk.forward(aug, b, foff, None)
        first = {n: b[n].clone() for n in ("y", "state", "conv_state", "norm")}
        feats, feats2 = torch.empty(int(foff[-1]), DIM, device="cuda"), torch.empty(int(foff[-1]), DIM, device="cuda")
        aug.aug_vtlp_mel_batch(off, wave, alpha, FE, foff, feats)
        for lens in ([5], [1] * 100, [300, 0, 2]):
            o = np.concatenate([[0], np.cumsum(lens)])
            c = blk.buffers(int(o[-1]), len(lens))
            c["x"].normal_()
            blk.forward(aug, c, o, None)
            blk.backward(aug, c, o, torch.randn(int(o[-1]), DIM, device="cuda"))
        blk.forward(aug, b, foff, None)
        aug.aug_vtlp_mel_batch(off, wave, alpha, FE, foff, feats2)
        torch.cuda.synchronize()
        for n, v in first.items():
            assert torch.equal(b[n], v), n
        assert torch.equal(feats, feats2)


def test_times_by_stage():
    blk = Block(torch.float32, 9)
    with binding.Augmenter(0) as aug:
        b = blk.buffers(64, 1)
        b["x"].normal_()
        aug.aug_profile_enable(True)
        blk.forward(aug, b, [0, 64], None)
        blk.backward(aug, b, [0, 64], b["y"].clone())
        t = aug.aug_profile_read()
    assert [t[k][1] for k in ("norm", "short_conv", "scan")] == [2, 2, 2] and all(t[k][0] > 0 for k in ("norm", "short_conv", "scan"))


def test_current_device_and_errors_leave_the_context_usable():
    blk = Block(torch.float32, 10)
    with binding.Augmenter(0) as aug:
        b = blk.buffers(8, 1)
        b["x"].normal_()
        with pytest.raises(binding.AugError) as err:
            aug.aug_rms_norm_batch(b["x"], blk.norm_w, y_out=b["norm"], q_block=24)
        assert err.value.code == binding.AUG_ERR_INVALID_ARG and bool((b["norm"] == UNTOUCHED).all())
        with pytest.raises(ValueError, match="cpu"):
            aug.aug_rms_norm_batch(b["x"].cpu(), None, y_out=b["norm"])
        with pytest.raises(binding.AugError, match="overlaps"):
            aug.aug_short_conv_batch([0, 8], b["x"], blk.conv_w, b["x"])
        aug.aug_rms_norm_batch(b["x"], blk.norm_w, y_out=b["norm"])
        assert torch.cuda.current_device() == 0
        torch.cuda.synchronize()
        assert bool((b["norm"] != UNTOUCHED).any())


def test_matrices_beyond_2_to_31_elements():
    """The last rows of matrices whose elements are numbered past 32 bits, against the same rows by themselves."""
    rows, ld, dim, n = 70000, 40000, 64, 4
    base = torch.empty(rows * ld, dtype=torch.bfloat16, device="cuda").view(rows, ld)
    cols = [base[:, i * dim:(i + 1) * dim] for i in range(9)]
    for c in cols[:5]:
        c.copy_(torch.randn(rows, dim, device="cuda"))
    u, delta, z, dy, bc = cols[:5]
    small = [c.contiguous() for c in (u, delta, z, dy, bc)]
    a, w = -torch.rand(dim, n, device="cuda") - 0.1, torch.randn(dim, 4, device="cuda")
    off = [0, 100, rows - 300, rows]
    with binding.Augmenter(0) as aug:
        for x, args in (((u, delta, z, dy, bc), cols[5:]), (small, [torch.empty(rows, dim, dtype=torch.bfloat16, device="cuda") for _ in range(4)])):
            o1, o2, o3, o4 = args
            rstd = torch.empty(rows, device="cuda")
            aug.aug_rms_norm_batch(x[0], None, residual=x[1], y_out=o1, rstd_out=rstd)
            aug.aug_short_conv_batch(off, x[0], w, o2)
            aug.aug_scan_batch(off, x[0], x[1], a, x[4][:, :n], x[4][:, n:2 * n], o3, z=x[2])
            aug.aug_scan_backward_batch(off, x[0], x[1], a, x[4][:, :n], x[4][:, n:2 * n], x[3], z=x[2], du_out=o4)
            kept = [t.clone() for t in (o1, o2, o3, o4, rstd)]
            aug.aug_short_conv_backward_batch(off, x[0], w, x[3], dx_out=o1)
            aug.aug_rms_norm_backward_batch(x[0], rstd, x[3], None, dx_out=o2)
            kept += [o1.clone(), o2.clone()]
            torch.cuda.synchronize()
            if x is small:
                for i, (p, q) in enumerate(zip(first, kept)):
                    assert torch.equal(p, q), i
            first = kept


def test_two_contexts_on_two_streams():
    """The same work at once in two contexts, each on a stream of its own, against one alone."""
    off = np.array([0, 300, 301, 900])
    rows, blk = 900, Block(torch.float32, 11)
    with binding.Augmenter(0) as aug:
        want = blk.buffers(rows, 3)
        want["x"].normal_()
        want["made"].normal_()
        dy = torch.randn(rows, DIM, device="cuda")

        def work(a, b):
            a.aug_rms_norm_batch(b["x"], blk.norm_w, sum_out=b["sum"], y_out=b["norm"], rstd_out=b["rstd"])
            a.aug_short_conv_batch(off, b["norm"], blk.conv_w, b["conv"], bias=blk.conv_b, state_out=b["conv_state"])
            a.aug_scan_batch(off, **blk.scan_args(b), y_out=b["y"], state_out=b["state"])
            blk.backward(a, b, off, dy)

        work(aug, want)
    sides = []
    for _ in range(2):
        b = blk.buffers(rows, 3)
        b["x"].copy_(want["x"])
        b["made"].copy_(want["made"])
        stream = torch.cuda.Stream()
        sides.append((stream, binding.Augmenter(0, stream), b))
    torch.cuda.synchronize()
    for _ in range(5):
        for stream, a, b in sides:
            work(a, b)
    torch.cuda.synchronize()
    for _, a, b in sides:
        a.close()
        for n in want:
            assert torch.equal(b[n].nan_to_num(), want[n].nan_to_num()), n


def test_as_many_sequences_as_there_may_be():
    """65535 sequences of one row or none, against the formulas of a single row."""
    n_seq, dim, n = 65535, 9, 3
    lengths = (np.arange(n_seq) % 5 != 2).astype(np.int64)
    off = np.concatenate([[0], np.cumsum(lengths)])
    rows, r = int(off[-1]), lambda *s: torch.randn(*s, device="cuda")          # noqa: E731
    x, delta, b, c, dy, w = r(rows, dim), r(rows, dim), r(rows, n), r(rows, n), r(rows, dim), r(dim, 4)
    a, state, cstate = -torch.rand(dim, n, device="cuda"), r(n_seq, dim, n), r(n_seq, 3, dim)
    y, yc, du, dxc = (torch.empty_like(x) for _ in range(4))
    out, cout, da = torch.empty_like(state), torch.empty_like(cstate), torch.empty_like(a)
    with binding.Augmenter(0) as aug:
        aug.aug_scan_batch(off, x, delta, a, b, c, y, state_in=state, state_out=out)
        aug.aug_scan_backward_batch(off, x, delta, a, b, c, dy, state_in=state, du_out=du, da_out=da)
        aug.aug_short_conv_batch(off, x, w, yc, activation="none", state_in=cstate, state_out=cout)
        aug.aug_short_conv_backward_batch(off, x, w, dy, activation="none", state_in=cstate, dx_out=dxc)
        torch.cuda.synchronize()
    has = torch.from_numpy(lengths > 0).cuda()
    f = lambda t: t.double()          # noqa: E731
    step, h0 = torch.nn.functional.softplus(f(delta)), f(state)[has]
    e = torch.exp(step[:, :, None] * f(a))
    h = e * h0 + (step * f(x))[:, :, None] * f(b)[:, None]
    g = f(dy)[:, :, None] * f(c)[:, None]

    def close(got, want, mag):          # 80 roundings of the terms' magnitudes
        assert bool(((f(got) - want).abs() <= 80 * 2.0 ** -24 * mag).all())

    mag = e * h0.abs() + (step * f(x).abs())[:, :, None] * f(b).abs()[:, None]
    close(out[has], h, mag)
    assert torch.equal(out[~has], state[~has]) and torch.equal(cout[~has], cstate[~has])
    close(y, (h * f(c)[:, None]).sum(2), (mag * f(c).abs()[:, None]).sum(2))
    close(du, step * (g * f(b)[:, None]).sum(2), step * (g * f(b)[:, None]).abs().sum(2))
    terms = g * e * h0 * step[:, :, None]
    assert bool(((f(da) - terms.sum(0)).abs() <= (80 + 2048) * 2.0 ** -24 * terms.abs().sum(0)).all())      # as many blocks in a run, at most
    p = torch.cat([f(cstate)[has], f(x)[:, None]], 1) * f(w).t()
    close(yc, p.sum(1), p.abs().sum(1))
    assert torch.equal(cout[has], torch.cat([cstate[has][:, 1:], x[:, None]], 1))
    close(dxc, f(dy) * f(w)[:, 3], (f(dy) * f(w)[:, 3]).abs())


@pytest.mark.parametrize("dim,n,g", [(32768, 2, 1), (32768, 2, 4096), (8192, 128, 2)])
def test_as_many_channels_as_there_may_be(dim, n, g):
    off, rows = np.array([0, 2, 2, 5]), 5
    r = np.random.default_rng(12)
    t = {k: dev(r.standard_normal((rows, w)).astype(np.float32)).bfloat16() for k, w in dict(u=dim, delta=dim, b=g * n, c=g * n).items()}
    t["a"] = dev(-np.exp(r.uniform(-2, 1, (dim, n))).astype(np.float32))
    dy, w = dev(r.standard_normal((rows, dim)).astype(np.float32)).bfloat16(), dev(r.standard_normal((dim, 3)).astype(np.float32))
    y, yc, dx = (torch.empty_like(dy) for _ in range(3))
    state = torch.empty(3, dim, n, device="cuda")
    grads = dict(du=torch.empty_like(dy), ddelta=torch.empty_like(dy), db=torch.empty_like(t["b"]), dc=torch.empty_like(t["c"]),
                 da=torch.empty_like(t["a"]))
    dw = torch.empty_like(w)
    with binding.Augmenter(0) as aug:
        aug.aug_scan_batch(off, **t, y_out=y, n_group=g, state_out=state)
        aug.aug_scan_backward_batch(off, **t, dy=dy, n_group=g, **{k + "_out": v for k, v in grads.items()})
        aug.aug_short_conv_batch(off, t["u"], w, yc)
        aug.aug_short_conv_backward_batch(off, t["u"], w, dy, dx_out=dx, dweight_out=dw)
        torch.cuda.synchronize()
    ws = {k: wide(v) for k, v in t.items()}
    want, mag = R.scan(off, n_group=g, **ws), R.scan(off, n_group=g, magnitude=True, **ws)
    near(y, want[0], mag[0], 64 + 6 * 3 + n, "y")
    near(state, want[1], mag[1], 64 + 6 * 3 + n, "state")
    want, mag = (R.scan_backward(off, n_group=g, dy=wide(dy), magnitude=m, **ws) for m in (False, True))
    for k, v in grads.items():
        near(v, want[k], mag[k], 2 * (64 + 6 * 3 + n) + (dim // g if k in ("db", "dc") else rows), k)
    args = (off, wide(t["u"]), wide(w))
    near(yc, R.short_conv(*args)[0], R.short_conv(*args, magnitude=True)[0], 3 + 12, "conv")
    want, mag = R.short_conv_backward(*args, wide(dy)), R.short_conv_backward(*args, wide(dy), magnitude=True)
    near(dx, want[0], mag[0], 6 + 16, "dx")
    near(dw, want[1], mag[1], 3 + 16 + rows, "dw")
