"""Pins of the temporal layer's oracle: hand-worked values, finite differences, the hand-over between blocks, sequences of
different lengths against sequences cut to their length."""
import numpy as np
import pytest

from oracle import temporal as tp


def data(seed, T=5, n=3, f=4, N=3, w=3):
    r = np.random.default_rng(seed)
    s = lambda *shape: r.standard_normal(shape)  # noqa: E731
    return dict(x=s(T, n, f), delta=s(T, n, f), bc=s(T, n, 2 * N), z=s(T, n, f), a=-np.exp(s(f, N)), d=s(f), dt_bias=s(f), h_before=s(n, f, N)), \
        dict(x=s(T, n, f), taps=s(w, f), bias=s(f), x_before=s(w - 1, n, f)), dict(y=s(T, n, f), h=s(n, f, N), after=s(w - 1, n, f))


def test_conv_by_hand():
    x = np.array([1.0, 2.0, 4.0]).reshape(3, 1, 1)
    y, after = tp.causal_conv(x, np.array([[1.0], [10.0], [100.0]]), np.array([0.5]), x_before=np.array([7.0, 8.0]).reshape(2, 1, 1))
    assert y.ravel().tolist() == [1 + 80 + 700 + 0.5, 2 + 10 + 800 + 0.5, 4 + 20 + 100 + 0.5]
    assert after.ravel().tolist() == [2.0, 4.0]
    y, after = tp.causal_conv(x, np.ones((3, 1)), x_before=np.array([7.0, 8.0]).reshape(2, 1, 1), lengths=[1])
    assert y.ravel().tolist() == [16.0, 0.0, 0.0] and after.ravel().tolist() == [8.0, 1.0]
    assert np.isclose(tp.causal_conv(x, np.array([[1.0], [0.0]]), act=True)[0][1, 0, 0], 2 / (1 + np.exp(-2)))


def test_scan_by_hand():
    """softplus(log(e - 1)) = 1; a = -log 2 halves the state with every step of size 1."""
    one = np.log(np.e - 1)
    x, bc = np.array([1.0, 3.0]).reshape(2, 1, 1), np.array([[2.0, 5.0], [1.0, 10.0]]).reshape(2, 1, 2)
    y, h, _ = tp.selective_scan(x, np.full((2, 1, 1), one), bc, np.array([[-np.log(2.0)]]), d=np.array([100.0]), h_before=np.full((1, 1, 1), 8.0))
    assert np.allclose(y.ravel(), [(4 + 2) * 5 + 100, (3 + 3) * 10 + 300]) and np.allclose(h, 6)


@pytest.mark.parametrize("lengths", [None, [5, 2, 0]])
def test_scan_gradients_are_differences(lengths):
    s, _, g = data(1)

    def loss(p):
        y, h, _ = tp.selective_scan(lengths=lengths, **p)
        return (y * g["y"]).sum() + (h * g["h"]).sum()

    out = tp.selective_scan_backward(g_y=g["y"], dh_after=g["h"], lengths=lengths, **s)
    r = np.random.default_rng(3)
    for name in s:
        by = r.standard_normal(s[name].shape)
        eps = 1e-6
        diff = (loss(dict(s, **{name: s[name] + eps * by})) - loss(dict(s, **{name: s[name] - eps * by}))) / (2 * eps)
        assert np.isclose(diff, (out["d" + name] * by).sum(), rtol=1e-6, atol=1e-7), name


@pytest.mark.parametrize("lengths", [None, [5, 1, 0]])
@pytest.mark.parametrize("act", [False, True])
def test_conv_gradients_are_differences(lengths, act):
    _, s, g = data(2)

    def loss(p):
        y, after = tp.causal_conv(act=act, lengths=lengths, **p)
        return (y * g["y"]).sum() + (after * g["after"]).sum()

    out = tp.causal_conv_backward(g_y=g["y"], dx_after=g["after"], act=act, lengths=lengths, **s)
    r = np.random.default_rng(4)
    for name in s:
        by = r.standard_normal(s[name].shape)
        eps = 1e-6
        diff = (loss(dict(s, **{name: s[name] + eps * by})) - loss(dict(s, **{name: s[name] - eps * by}))) / (2 * eps)
        assert np.isclose(diff, (out["d" + name] * by).sum(), rtol=1e-6, atol=1e-7), name


def test_blocks_chain():
    s, c, g = data(5, T=7)
    y, h, _ = tp.selective_scan(**s)
    cut = lambda p, a, b: {k: v[a:b] if k in ("x", "delta", "bc", "z") else v for k, v in p.items()}  # noqa: E731
    y1, h1, _ = tp.selective_scan(**cut(s, 0, 3))
    y2, h2, _ = tp.selective_scan(**dict(cut(s, 3, 7), h_before=h1))
    assert np.allclose(np.concatenate([y1, y2]), y) and np.allclose(h2, h)
    whole = tp.selective_scan_backward(g_y=g["y"], dh_after=g["h"], **s)
    back2 = tp.selective_scan_backward(g_y=g["y"][3:], dh_after=g["h"], **dict(cut(s, 3, 7), h_before=h1))
    back1 = tp.selective_scan_backward(g_y=g["y"][:3], dh_after=back2["dh_before"], **cut(s, 0, 3))
    assert np.allclose(np.concatenate([back1["dx"], back2["dx"]]), whole["dx"]) and np.allclose(back1["da"] + back2["da"], whole["da"])
    y, after = tp.causal_conv(act=True, **c)
    y1, a1 = tp.causal_conv(act=True, **cut(c, 0, 1))
    y2, a2 = tp.causal_conv(act=True, **dict(cut(c, 1, 7), x_before=a1))
    assert np.allclose(np.concatenate([y1, y2]), y) and np.allclose(a2, after)


def test_lengths_cut():
    s, c, _ = data(6)
    y, h, _ = tp.selective_scan(lengths=[5, 2, 0], **s)
    short = {k: v[:2, 1:2] if k in ("x", "delta", "bc", "z") else v[1:2] if k == "h_before" else v for k, v in s.items()}
    y1, h1, _ = tp.selective_scan(**short)
    assert np.allclose(y[:2, 1], y1[:, 0]) and not y[2:, 1].any() and np.allclose(h[1], h1[0])
    assert not y[:, 2].any() and np.array_equal(h[2], s["h_before"][2])
