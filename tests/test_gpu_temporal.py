"""The causal convolution over time and the selective state-space scan, forward and backward, against the oracle in 64 bits.

Tolerances.  An output is rounded to its type once, half a step of it: eps / 2 of its value.  Ahead of that sums and states are fp32: every
term passes `depth` roundings of 2^-24 of its magnitude at most, so the error stays below depth 2^-24 M with M the same result formed
from absolute values.  Convolution: w + 1 roundings of the sum (twice, going back), the sigmoid's exponential with its argument's rounding
(|a| < 16 here) and reciprocal: 40.  Scan: step size and gate 16 each, 4 states and 2 exchanges per sum, and 4 per timestep that a state is carried through: 64 + 4 T.  And a
decay exp(-u), u = step size times |a|, has the relative error of u in its exponent: the sum delta + dt_bias is rounded (|.| < 8 where both
are there: 8 2^-24 of a small step size), the step size is formed in a dozen roundings, the product with a log2(e) in two: 22 2^-24 u.  Carried
over any number of steps it changes a term X exp(-u) by 22 2^-24 X u exp(-u), and u exp(-u) = u exp(-u / 8) exp(-7 u / 8) <= (8 / e)
exp(-7 u / 8): 65 2^-24 of the term with 7/8 of its exponent, which is what M is formed with.  64 + 65 + 4 T in all.  Errors are as often up
as down, so that in the 2-norm 8 sqrt(depth) of them have to do."""
import numpy as np
import pytest
import torch

import paper_2109_07893_amd as dg
from oracle import temporal as tp

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
F32, BF16 = torch.float32, torch.bfloat16
NAN = float("nan")


def close(got, want, mag, depth, what):
    dtype = got.dtype
    half = torch.finfo(dtype).eps / 2
    got, want, mag = got.detach().cpu().double().numpy(), np.asarray(want, dtype=np.float64), np.asarray(mag, dtype=np.float64)
    assert got.shape == want.shape, (what, got.shape, want.shape)
    assert np.isfinite(got).all(), what
    step = depth * 2.0 ** -24 * mag
    err = np.abs(got - want)
    bad = err > half * (np.abs(want) + step) + step + 1e-38
    assert not bad.any(), f"{what}: {int(bad.sum())} of {bad.size} off, worst {err[bad].max():.3e} at {np.argwhere(bad)[0]}"
    norm = np.linalg.norm
    assert norm(err) <= half * norm(want) + 8 * depth ** 0.5 * 2.0 ** -24 * norm(mag) + 1e-38, (what, norm(err), norm(want))


def np64(t):
    return None if t is None else t.detach().cpu().double().numpy()


def cuda(t):
    return None if t is None else t.to(DEV)


class Conv:
    """Inputs of a convolution, made on the CPU from a seed."""

    def __init__(self, T, n, f, w, dtype, seed=0, silu=True, bias=True, before=True, lengths=None):
        g = torch.Generator().manual_seed(seed)
        s = lambda *shape: torch.randn(shape, generator=g)  # noqa: E731
        self.T, self.n, self.f, self.w, self.silu = T, n, f, w, silu
        self.x, self.taps = s(T, n, f).to(dtype), s(w, f)
        self.bias, self.before = s(f) if bias else None, s(w - 1, n, f).to(dtype) if before else None
        self.g_y, self.after = s(T, n, f).to(dtype), s(w - 1, n, f).to(dtype)
        self.lengths = None if lengths is None else torch.tensor(lengths, dtype=torch.int32)

    def poison(self):
        """Not-a-number wherever a sequence has no timestep."""
        if self.lengths is not None:
            gone = torch.arange(self.T)[:, None] >= self.lengths.clamp(0, self.T)[None, :]
            self.x[gone], self.g_y[gone] = NAN, NAN
        return self

    def forward(self, in_place=False):
        x = cuda(self.x)
        y = torch.full_like(x, NAN)
        before = cuda(self.before)
        after = before if in_place else torch.full((self.w - 1, self.n, self.f), NAN, dtype=x.dtype, device=DEV)
        dg.causal_conv(x, cuda(self.taps), cuda(self.bias), y, silu=self.silu, x_before=before, x_after=after, lengths=cuda(self.lengths))
        return y, after

    def backward(self, accumulate=False, after=True, start=0.0):
        x = cuda(self.x)
        out = dict(dx=torch.full_like(x, NAN), dx_before=torch.full((self.w - 1, self.n, self.f), NAN, dtype=x.dtype, device=DEV),
                   dtaps=torch.full((self.w, self.f), start, device=DEV), dbias=torch.full((self.f,), start, device=DEV) if self.bias is not None else None)
        ws = torch.full((dg.causal_conv_backward_workspace(self.T, self.n, self.f, self.w),), 255, dtype=torch.uint8, device=DEV)
        dg.causal_conv_backward(x, cuda(self.taps), cuda(self.bias), cuda(self.g_y), out["dx"], out["dtaps"], out["dbias"], ws, silu=self.silu, x_before=cuda(self.before),
                                dx_after=cuda(self.after) if after else None, dx_before=out["dx_before"], lengths=cuda(self.lengths), accumulate=accumulate)
        return out

    def oracle(self):
        a = dict(x=np64(self.x), taps=np64(self.taps), bias=np64(self.bias), act=self.silu, x_before=np64(self.before), lengths=None if self.lengths is None else self.lengths.numpy())
        return a

    def check(self, in_place=False, back=True):
        a = self.oracle()
        y, after = self.forward(in_place)
        want, want_after = tp.causal_conv(**a)
        mags = {k: np.abs(v) if k in ("x", "taps", "bias", "x_before") and v is not None else v for k, v in a.items()}
        mag, _ = tp.causal_conv(**dict(mags, act=False))
        close(y, want, mag, 40, "y")
        assert np.array_equal(np64(after), want_after), "x_after"
        if not back:
            return
        for after_grad in (True, False):
            got = self.backward(after=after_grad)
            h = dict(a, g_y=np64(self.g_y), dx_after=np64(self.after) if after_grad else None)
            want, mag = tp.causal_conv_backward(**h), tp.causal_conv_backward(magnitudes=True, **h)
            for k, v in got.items():
                if v is not None:
                    close(v, want[k], mag[k], 40 if k.startswith("dx") else 40 + 64, k)


# sizes: one frame, fewer frames than taps, around the frames fetched together, a piece of the time axis and its border, odd widths
@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("T,n,f,w", [(1, 1, 16, 4), (1, 37, 64, 4), (2, 5, 48, 4), (3, 300, 16, 2), (4, 7, 80, 3), (5, 33, 128, 4), (16, 3, 32, 2), (17, 2, 144, 3),
                                     (33, 1, 16, 4), (130, 2, 48, 4), (200, 1, 2064, 3), (7, 3, 16384, 2)])
def test_conv(T, n, f, w, dtype):
    Conv(T, n, f, w, dtype, seed=T + n + f).check()


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("w", [2, 3, 4])
@pytest.mark.parametrize("T", [1, 3, 21, 70])
def test_conv_lengths(T, w, dtype):
    """Sequences without a timestep, with fewer than there are taps, whole, and with lengths outside of 0 .. T."""
    Conv(T, 9, 32, w, dtype, seed=w, lengths=[0, 1, 2, 3, T, T - 1, T + 5, -4, T // 2]).poison().check()


@pytest.mark.parametrize("silu,bias,before", [(False, True, True), (True, False, False), (False, False, True)])
def test_conv_without(silu, bias, before):
    Conv(19, 11, 64, 4, F32, silu=silu, bias=bias, before=before).check()


@pytest.mark.parametrize("T", [1, 2, 40])
@pytest.mark.parametrize("lengths", [None, [0, 1, 2, 40, 1]])
def test_conv_state_in_place(T, lengths):
    Conv(T, 5, 16, 4, BF16, lengths=lengths).check(in_place=True, back=False)


def test_conv_steps_are_the_series():
    """Timestep by timestep with the state rolled on in place: the series bit for bit."""
    c = Conv(9, 41, 48, 4, BF16)
    y, after = c.forward()
    x, state = cuda(c.x), cuda(c.before)
    for t in range(c.T):
        one = torch.empty_like(x[:1])
        dg.causal_conv(x[t:t + 1], cuda(c.taps), cuda(c.bias), one, silu=True, x_before=state, x_after=state)
        assert torch.equal(one[0], y[t]), t
    assert torch.equal(state, after)


def test_conv_accumulates_and_repeats():
    c = Conv(50, 200, 64, 4, F32)
    a, b, more = c.backward(), c.backward(), c.backward(accumulate=True, start=1000.0)
    assert all(torch.equal(a[k], b[k]) for k in a)
    for k in ("dtaps", "dbias"):
        assert torch.equal(more[k], (a[k].double() + 1000.0).float()) or (more[k] - a[k] - 1000.0).abs().max() <= 1000.0 * 2 ** -23


class Scan:
    def __init__(self, T, n, f, N, dtype, seed=0, z=True, d=True, dt_bias=True, before=True, lengths=None):
        g = torch.Generator().manual_seed(seed)
        s = lambda *shape: torch.randn(shape, generator=g)  # noqa: E731
        self.T, self.n, self.f, self.N = T, n, f, N
        self.x, self.delta, self.bc, self.g_y = s(T, n, f).to(dtype), s(T, n, f).to(dtype), s(T, n, 2 * N).to(dtype), s(T, n, f).to(dtype)
        self.z = s(T, n, f).to(dtype) if z else None
        self.a = -torch.arange(1, N + 1).float() * torch.exp(0.3 * s(f, N))
        self.d, self.dt_bias = s(f) if d else None, s(f) - 3.0 if dt_bias else None
        self.h_before, self.dh_after = s(n, f, N) if before else None, s(n, f, N) if before else None
        self.lengths = None if lengths is None else torch.tensor(lengths, dtype=torch.int32)

    def poison(self):
        if self.lengths is not None:
            gone = torch.arange(self.T)[:, None] >= self.lengths.clamp(0, self.T)[None, :]
            for t in (self.x, self.delta, self.bc, self.z, self.g_y):
                if t is not None:
                    t[gone] = NAN
        return self

    def inputs(self):
        return {k: cuda(getattr(self, k)) for k in ("x", "delta", "bc", "a", "z", "d", "dt_bias", "lengths")}

    def forward(self, in_place=False, keep=True):
        i = self.inputs()
        y, before = torch.full_like(i["x"], NAN), cuda(self.h_before)
        after = before if in_place else torch.full((self.n, self.f, self.N), NAN, device=DEV)
        kept = torch.full((dg.selective_scan_checkpoints(self.T, self.n, self.f, self.N),), NAN, device=DEV) if keep else None
        ws = torch.full((dg.selective_scan_workspace(self.T, self.n, self.f, self.N),), 255, dtype=torch.uint8, device=DEV)
        dg.selective_scan(y=y, ws=ws, h_before=before, h_after=after, checkpoints=kept, **i)
        return y, after, kept

    def backward(self, kept, accumulate=False, start=0.0, dh_before=True):
        i = self.inputs()
        out = dict(dx=torch.full_like(i["x"], NAN), ddelta=torch.full_like(i["x"], NAN), dbc=torch.full_like(i["bc"], NAN), dz=torch.full_like(i["x"], NAN) if self.z is not None else None,
                   da=torch.full((self.f, self.N), start, device=DEV), dd=torch.full((self.f,), start, device=DEV) if self.d is not None else None,
                   ddt_bias=torch.full((self.f,), start, device=DEV) if self.dt_bias is not None else None,
                   dh_before=torch.full((self.n, self.f, self.N), NAN, device=DEV) if dh_before else None)
        ws = torch.full((dg.selective_scan_backward_workspace(self.T, self.n, self.f, self.N),), 255, dtype=torch.uint8, device=DEV)
        dg.selective_scan_backward(g_y=cuda(self.g_y), checkpoints=kept, ws=ws, dh_after=cuda(self.dh_after), accumulate=accumulate, **i, **out)
        return out

    def oracle(self):
        a = {k: np64(getattr(self, k)) for k in ("x", "delta", "bc", "a", "z", "d", "dt_bias", "h_before")}
        return dict(a, lengths=None if self.lengths is None else self.lengths.numpy())

    def check(self, back=True):
        a, depth = self.oracle(), 129 + 4 * self.T
        y, after, kept = self.forward(keep=back)
        want, want_after, _ = tp.selective_scan(**a)
        mag, mag_after, _ = tp.selective_scan(magnitudes=True, **a)
        close(y, want, mag, depth, "y")
        close(after, want_after, mag_after, depth, "h_after")
        if not back:
            return
        got = self.backward(kept)
        h = dict(a, g_y=np64(self.g_y), dh_after=np64(self.dh_after))
        want, mag = tp.selective_scan_backward(**h), tp.selective_scan_backward(magnitudes=True, **h)
        for k, v in got.items():
            if v is not None:
                close(v, want[k], mag[k], depth + self.f if k == "dbc" else depth + 32 if k in ("da", "dd", "ddt_bias") else depth, k)


# sizes: single timesteps, around a group of four, a tile of sixteen and two of them; widths of one wavefront's channels, odd multiples, more
# than one workgroup; enough rows for workgroups that go round
@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("N", [8, 16, 32])
@pytest.mark.parametrize("T,n,f", [(1, 1, 16), (1, 9, 128), (2, 3, 16), (3, 2, 32), (4, 5, 48), (5, 1, 16), (15, 3, 64), (16, 2, 16), (17, 9, 32), (33, 2, 80)])
def test_scan(T, n, f, N, dtype):
    Scan(T, n, f, N, dtype, seed=T + n + f + N).check()


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("T,n,f,N", [(20, 2, 144, 16), (18, 3, 400, 8), (9, 1, 2064, 32), (6, 700, 16, 16), (2, 1500, 128, 16), (2, 1, 16384, 8), (17, 1, 15984, 8)])
def test_scan_wide_and_many(T, n, f, N, dtype):
    Scan(T, n, f, N, dtype, seed=f).check()


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("N", [8, 16, 32])
@pytest.mark.parametrize("T,n,f", [(128, 1, 16), (1000, 1, 32), (515, 2, 144), (300, 3, 48)])
def test_scan_in_pieces(T, n, f, N, dtype):
    """Few sequences, many timesteps: the time axis is shared out."""
    Scan(T, n, f, N, dtype, seed=T).check()


@pytest.mark.parametrize("N", [8, 32])
def test_scan_very_long(N):
    """Thousands of pieces, joined in runs of many."""
    Scan(70_001, 1, 16, N, F32, seed=N).check()


@pytest.mark.parametrize("N", [8, 16, 32])
@pytest.mark.parametrize("T", [1, 6, 16, 37, 400])
def test_scan_lengths(T, N):
    Scan(T, 9, 32, N, F32, seed=N, lengths=[0, 1, T, T - 1, T + 9, -3, T // 2, T // 3, min(T, 17)]).poison().check()


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("N", [8, 16, 32])
@pytest.mark.parametrize("T", [2, 8, 9, 12, 13, 48, 49])
def test_scan_lengths_around_tiles(T, N, dtype):
    """Where tiles of eight timesteps give way to those of sixteen, either way and in either type; widths of more than one workgroup too."""
    lengths = [0, T, 1, 8, T - 1, T // 2, 9]
    Scan(T, 7, 48, N, dtype, seed=T + N, lengths=lengths).poison().check()
    Scan(T, 7, 160, N, dtype, seed=T + N, lengths=lengths, z=False).poison().check()


@pytest.mark.parametrize("T", [5, 400])
@pytest.mark.parametrize("z,d,dt_bias,before", [(False, True, True, True), (True, False, True, False), (True, True, False, True), (False, False, False, False)])
def test_scan_without(T, z, d, dt_bias, before):
    Scan(T, 4, 16, 16, F32, z=z, d=d, dt_bias=dt_bias, before=before).check()


@pytest.mark.parametrize("T,n,f", [(1, 13, 64), (20, 5, 16), (700, 1, 16)])
def test_scan_state_in_place(T, n, f):
    s = Scan(T, n, f, 16, BF16)
    y, after, _ = s.forward()
    y1, after1, _ = s.forward(in_place=True, keep=False)
    assert torch.equal(y, y1) and torch.equal(after, after1)


def test_scan_steps_are_the_series():
    """Timestep by timestep with the state in place: the series bit for bit (it is not cut into pieces at this size)."""
    s = Scan(11, 6, 48, 16, BF16)
    y, after, _ = s.forward()
    i, h = s.inputs(), cuda(s.h_before)
    ws = torch.empty(dg.selective_scan_workspace(1, s.n, s.f, s.N), dtype=torch.uint8, device=DEV)
    for t in range(s.T):
        one = torch.empty_like(i["x"][:1])
        cut = {k: v[t:t + 1] if k in ("x", "delta", "bc", "z") else v for k, v in i.items()}
        dg.selective_scan(y=one, ws=ws, h_before=h, h_after=h, **cut)
        assert torch.equal(one[0], y[t]), t
    assert torch.equal(h, after)


@pytest.mark.parametrize("T,n", [(40, 30), (600, 1)])
def test_scan_accumulates_and_repeats(T, n):
    s = Scan(T, n, 32, 16, F32)
    y, after, kept = s.forward()
    y2, after2, kept2 = s.forward()
    assert torch.equal(y, y2) and torch.equal(after, after2) and torch.equal(kept, kept2)
    a, b, more = s.backward(kept), s.backward(kept), s.backward(kept, accumulate=True, start=100.0)
    assert all(torch.equal(a[k], b[k]) for k in a)
    for k in ("da", "dd", "ddt_bias"):
        assert (more[k].double() - a[k].double() - 100.0).abs().max() <= (100.0 + a[k].abs().max().item()) * 2 ** -23
    assert torch.equal(s.backward(kept, dh_before=False)["dx"], a["dx"])


@pytest.mark.parametrize("T,cut", [(50, 16), (50, 33), (400, 300)])
def test_scan_blocks_chain(T, cut):
    """A series in two blocks, the state handed over and its gradient back, against the whole."""
    s = Scan(T, 5, 32, 16, F32)
    y, after, kept = s.forward()
    whole = s.backward(kept)

    def block(lo, hi):
        b = Scan(hi - lo, 5, 32, 16, F32)
        for k in ("x", "delta", "bc", "z", "g_y"):
            setattr(b, k, getattr(s, k)[lo:hi].clone())
        for k in ("a", "d", "dt_bias", "h_before", "dh_after"):
            setattr(b, k, getattr(s, k))
        return b

    first, second = block(0, cut), block(cut, T)
    y1, h1, kept1 = first.forward()
    second.h_before = h1.cpu()
    y2, h2, kept2 = second.forward()
    b2 = second.backward(kept2)
    first.dh_after = b2["dh_before"].cpu()
    b1 = first.backward(kept1)
    a = s.oracle()
    h = dict(a, g_y=np64(s.g_y), dh_after=np64(s.dh_after))
    want, mag = tp.selective_scan_backward(**h), tp.selective_scan_backward(magnitudes=True, **h)
    depth = 129 + 4 * T
    close(torch.cat([y1, y2]), tp.selective_scan(**a)[0], tp.selective_scan(magnitudes=True, **a)[0], depth, "y")
    for k in ("dx", "ddelta", "dbc", "dz"):
        close(torch.cat([b1[k], b2[k]]), want[k], mag[k], depth + 32, k)
    close(b1["da"] + b2["da"], want["da"], mag["da"], depth + 32, "da")
    close(b1["dh_before"], want["dh_before"], mag["dh_before"], depth, "dh_before")
    assert torch.equal(h2, after) or T > 128


@pytest.mark.parametrize("delta", [-100.0, -30.0, -12.0, 0.0, 15.0, 60.0])
def test_scan_step_sizes(delta):
    """softplus far from the middle: tiny steps keep their digits, large ones are the argument itself."""
    s = Scan(7, 3, 16, 8, F32, dt_bias=False)
    s.delta = s.delta + delta
    s.a = s.a * (0.01 if delta > 10 else 1.0)
    s.check()


@pytest.mark.parametrize("T", [600, 5000])
def test_scan_growing_states(T):
    """a > 0, where the growth across a piece of the time axis is beyond fp32 and no state is: zero until the last timesteps (from behind:
    until the first ones), which are what they are on their own."""
    n, f, N, few = 1, 32, 8, 6
    s = Scan(T, n, f, N, F32, d=False, dt_bias=False, before=False)
    s.a, s.dh_after = 0.1 * s.a.abs(), None                       # up to e^6 or so a timestep
    s.x[:-few], s.g_y[few:] = 0.0, 0.0

    def part(lo, hi):
        b = Scan(few, n, f, N, F32, d=False, dt_bias=False, before=False)
        b.x, b.delta, b.bc, b.z, b.g_y = (t[lo:hi].clone() for t in (s.x, s.delta, s.bc, s.z, s.g_y))
        b.a, b.dh_after = s.a, None
        return b

    y, after, kept = s.forward()
    y1, after1, _ = part(T - few, T).forward()
    assert not y[:-few].any() and torch.equal(y[-few:], y1) and torch.equal(after, after1)
    got = s.backward(kept)
    first = part(0, few)
    want = first.backward(first.forward()[2])
    for k in ("dx", "ddelta", "dbc", "dz"):
        assert torch.isfinite(got[k]).all() and torch.equal(got[k][:few], want[k]) and not got[k][few:].any(), k
    assert torch.equal(got["dh_before"], want["dh_before"])


@pytest.mark.parametrize("T", [5, 400])
def test_scan_no_state_kept(T):
    """a of minus infinity: what a timestep finds is forgotten; a sequence without a timestep keeps its state."""
    s = Scan(T, 3, 16, 8, F32, lengths=[0, T, 1])
    s.a[:, ::2] = -float("inf")
    y, after, _ = s.forward(keep=False)
    assert torch.equal(after[0], cuda(s.h_before)[0]) and torch.isfinite(y).all() and torch.isfinite(after).all()


def test_scan_infinite_values_stay_where_they_are():
    """An infinity or a NaN in one sequence, or in a channel of it, does not reach another."""
    s = Scan(21, 4, 32, 16, F32)
    clean, _, _ = s.forward()
    s.x[3, 1, 5], s.x[4, 2, 7] = float("inf"), NAN
    y, after, _ = s.forward()
    touched = torch.zeros_like(y, dtype=torch.bool)
    touched[3:, 1, 5] = touched[4:, 2, 7] = True
    assert torch.equal(y[~touched], clean[~touched]) and not torch.isfinite(y[touched]).any()


def test_offsets_beyond_32_bits():
    """Frames of more than 2^31 elements: the last sequences as in a small call."""
    T, n, f, N, tail = 9, (1 << 21) + 3, 128, 8, 5
    assert T * n * f > 1 << 31
    make = lambda width: torch.empty((T, n, width), dtype=BF16, device=DEV).normal_()  # noqa: E731
    x, delta, bc = make(f), make(f), make(2 * N)
    a, h = -torch.rand((f, N), device=DEV) - 0.1, torch.zeros((n, f, N), device=DEV)
    ws = torch.empty(dg.selective_scan_workspace(T, n, f, N), dtype=torch.uint8, device=DEV)
    y = torch.empty_like(x)
    cut = [t[:, -tail:].contiguous() for t in (x, delta, bc)]
    y1, h1 = torch.empty_like(cut[0]), torch.empty((tail, f, N), device=DEV)
    dg.selective_scan(x, delta, bc, a, y, ws, h_after=h)
    dg.selective_scan(*cut, a, y1, ws, h_after=h1)
    assert torch.equal(y[:, -tail:], y1) and torch.equal(h[-tail:], h1)
    back = []
    for q, g in (((x, delta, bc), y), (cut, y1)):                 # y as the gradient, then everything back
        rows = q[0].shape[1]
        kept = torch.empty(dg.selective_scan_checkpoints(T, rows, f, N), device=DEV)
        ws = torch.empty(max(dg.selective_scan_workspace(T, rows, f, N), dg.selective_scan_backward_workspace(T, rows, f, N)), dtype=torch.uint8, device=DEV)
        dg.selective_scan(*q, a, torch.empty_like(q[0]), ws, checkpoints=kept)
        out = [torch.empty_like(t) for t in q]
        dg.selective_scan_backward(*q, a, g, kept, *out, torch.empty_like(a), ws)
        back.append([t[:, -tail:].clone() for t in out])
        del kept, ws, out
    assert all(torch.equal(p, q) for p, q in zip(*back))
    del h, back
    taps = torch.randn((4, f), device=DEV)
    dg.causal_conv(x, taps, None, y, silu=True)
    dg.causal_conv(cut[0], taps, None, y1, silu=True)
    assert torch.equal(y[:, -tail:], y1)
    ws = torch.empty(dg.causal_conv_backward_workspace(T, n, f, 4), dtype=torch.uint8, device=DEV)
    dx, dtaps, dx1 = torch.empty_like(x), torch.empty_like(taps), torch.empty_like(y1)
    dg.causal_conv_backward(x, taps, None, delta, dx, dtaps, None, ws, silu=True)
    dg.causal_conv_backward(cut[0], taps, None, cut[1], dx1, dtaps, None, ws, silu=True)
    assert torch.equal(dx[:, -tail:], dx1)


def test_another_stream_and_a_graph():
    """Calls on a stream of their own, then recorded and replayed between eager work; every replay against the eager result."""
    s, c = Scan(300, 2, 32, 16, F32), Conv(40, 3, 32, 4, F32)
    i = s.inputs()
    ws = torch.empty(max(dg.selective_scan_workspace(s.T, s.n, s.f, s.N), dg.selective_scan_backward_workspace(s.T, s.n, s.f, s.N)), dtype=torch.uint8, device=DEV)
    kept = torch.empty(dg.selective_scan_checkpoints(s.T, s.n, s.f, s.N), device=DEV)
    y, g_y = torch.empty_like(i["x"]), cuda(s.g_y)
    out = {k: torch.empty_like(i[k[1:]]) for k in ("dx", "ddelta", "dbc", "dz", "da", "dd", "ddt_bias")}
    cx, ctaps, cy, cdx, cg = cuda(c.x), cuda(c.taps), torch.empty_like(cuda(c.x)), torch.empty_like(cuda(c.x)), cuda(c.g_y)
    cdt, cws = torch.empty_like(ctaps), torch.empty(dg.causal_conv_backward_workspace(c.T, c.n, c.f, c.w), dtype=torch.uint8, device=DEV)

    def work():
        dg.causal_conv(cx, ctaps, None, cy, silu=True)
        dg.causal_conv_backward(cx, ctaps, None, cg, cdx, cdt, None, cws, silu=True)
        dg.selective_scan(y=y, ws=ws, checkpoints=kept, **i)
        dg.selective_scan_backward(g_y=g_y, checkpoints=kept, ws=ws, **i, **out)
        return [y, cy, cdx, cdt] + list(out.values())

    eager = [t.clone() for t in work()]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        results = work()
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(eager, results))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        work()
    for _ in range(3):
        for t in results:
            t.zero_()
        ws.fill_(7)
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(eager, results))
        s.forward()


def test_two_streams_and_two_graphs():
    """Two series at once, each on a stream and in a workspace of its own; then a graph of each over ONE workspace, replayed in turn."""
    runs = [Scan(300, 2, 48, 16, F32, seed=1), Scan(500, 1, 32, 8, BF16, seed=2)]
    size = max(max(dg.selective_scan_workspace(s.T, s.n, s.f, s.N), dg.selective_scan_backward_workspace(s.T, s.n, s.f, s.N)) for s in runs)
    spaces = [torch.empty(size, dtype=torch.uint8, device=DEV) for _ in runs]

    def prepared(s):
        i = s.inputs()
        out = {k: torch.empty_like(i[k[1:]]) for k in ("dx", "ddelta", "dbc", "dz", "da", "dd", "ddt_bias")}
        return i, out, torch.empty_like(i["x"]), torch.empty(dg.selective_scan_checkpoints(s.T, s.n, s.f, s.N), device=DEV), cuda(s.g_y)

    sets = [prepared(s) for s in runs]

    def work(k, ws):
        i, out, y, kept, g_y = sets[k]
        dg.selective_scan(y=y, ws=ws, checkpoints=kept, **i)
        dg.selective_scan_backward(g_y=g_y, checkpoints=kept, ws=ws, **i, **out)

    for k in range(2):
        work(k, spaces[k])
    eager = [[y.clone()] + [t.clone() for t in out.values()] for _, out, y, _, _ in sets]
    streams = [torch.cuda.Stream() for _ in runs]

    def check():
        torch.cuda.synchronize()
        for want, (_, out, y, _, _) in zip(eager, sets):
            assert all(torch.equal(a, b) for a, b in zip(want, [y] + list(out.values())))
            for t in [y] + list(out.values()):
                t.zero_()
        torch.cuda.synchronize()

    check()
    for _ in range(3):
        for k, st in enumerate(streams):
            with torch.cuda.stream(st):
                work(k, spaces[k])
        check()
    graphs = [torch.cuda.CUDAGraph() for _ in runs]
    for k, graph in enumerate(graphs):
        with torch.cuda.graph(graph):
            work(k, spaces[0])
    for _ in range(3):
        for graph in graphs:
            graph.replay()
        check()


class Forgetful(Scan):
    """Every second state with a of minus infinity, which 64 bits are given as -1e30: exp(-1e30 dt) = 0 there for every step size met."""

    def __init__(self, *args, **kw):
        super().__init__(*args, **kw)
        self.a[:, ::2] = -float("inf")

    def oracle(self):
        a = super().oracle()
        return dict(a, a=np.where(np.isinf(a["a"]), -1e30, a["a"]))


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("N", [8, 16, 32])
@pytest.mark.parametrize("T,n,f", [(1, 7, 32), (5, 7, 32), (13, 7, 48), (50, 7, 160), (400, 3, 16)])
def test_scan_no_state_kept_going_back(T, n, f, N, dtype):
    """... and its gradients: what a timestep finds has none, a sequence without a timestep hands its gradient on as it is."""
    lengths = [0, T, 1, T - 1, T // 2, 2, T][:n]
    s = Forgetful(T, n, f, N, dtype, seed=T + N, lengths=lengths).poison()
    s.check()
    got = s.backward(s.forward()[2])
    assert torch.equal(got["dh_before"][0].cpu(), s.dh_after[0])


def test_scan_all_states_forgotten():
    """No sequence of different lengths, and growth without bound where no timestep follows."""
    s = Forgetful(21, 4, 32, 16, F32)
    s.a[:] = -float("inf")
    s.check()
    s = Scan(21, 4, 32, 16, F32, lengths=[0, 0, 0, 0])
    s.a[:] = float("inf")
    y, after, kept = s.forward()
    got = s.backward(kept)
    assert not y.any() and torch.equal(after.cpu(), s.h_before) and torch.equal(got["dh_before"].cpu(), s.dh_after)
    assert not any(got[k].any() for k in got if k != "dh_before")


def carried(step, a):
    """How many timesteps' roundings a state carries with it, at most.  k timesteps' stay with a term that has decayed by exp(-u), u = the sum of step
    size times |a| over them, and M holds exp(-7/8 u) of it: k exp(-u / 8) of M.  The largest over all stretches of the series, from
    those of 1, 2, 4, ... timesteps: one of up to 2 k contains one of k."""
    slowest = np.abs(a).min(1)[None, None, :]
    total = np.concatenate([np.zeros((1,) + step.shape[1:]), np.cumsum(step, 0)])
    most, k = 2.0, 1
    while k < len(total):
        least = (total[k:] - total[:-k]) * slowest
        most = max(most, float((2 * k * np.exp(-least.min(0) / 8)).max()))
        k *= 2
    return min(most, len(step))


@pytest.mark.parametrize("T,n,f,N", [(70_001, 1, 16, 8), (9000, 2, 16, 32), (20_000, 1, 32, 16)])
def test_scan_long_as_its_states_last(T, n, f, N):
    """Hundreds of pieces against a bound that goes by how long a state lasts and not by how long the series is.  Ahead of it as above, 64 and 65, and
    what pieces add: the decay across one has its step sizes added up (a lane's, up to 36 of them here; in a run of pieces 16 more and 5 over
    the runs, roundings of a positive sum all of them) and its product taken once more, 60 2^-24 of its exponent: 60 8 / e = 177 more."""
    s = Scan(T, n, f, N, F32, seed=T)
    a = s.oracle()
    depth = 64 + 65 + 177 + 4 * carried(tp.softplus(a["delta"] + a["dt_bias"]), a["a"])
    assert depth < 129 + T                                        # four times as close as by the series' length, at least
    y, after, kept = s.forward()
    want, want_after, _ = tp.selective_scan(**a)
    mag, mag_after, _ = tp.selective_scan(magnitudes=True, **a)
    close(y, want, mag, depth, "y")
    close(after, want_after, mag_after, depth, "h_after")
    got = s.backward(kept)
    h = dict(a, g_y=np64(s.g_y), dh_after=np64(s.dh_after))
    want, mag = tp.selective_scan_backward(**h), tp.selective_scan_backward(magnitudes=True, **h)
    for k in ("dx", "ddelta", "dbc", "dz", "dh_before"):
        close(got[k], want[k], mag[k], 2 * depth + f, k)          # a state and a gradient that were carried meet
