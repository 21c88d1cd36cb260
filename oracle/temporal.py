"""The temporal layer's operators in 64 bits, timestep by timestep, from their definitions (numpy): the causal convolution over time, the
selective state-space scan, and their adjoints.  Frames are [T, n, f]; `lengths` [n]: sequence v has timesteps 0 .. lengths[v]-1.
With `magnitudes` every product enters with its absolute value and decays are exp(7/8 of their exponent), which bounds what a relative
error of that exponent does (u exp(-u) <= 2.95 exp(-7 u / 8)): what the rounding errors of a result are measured against."""
import numpy as np


def sigmoid(v):
    e = np.exp(-np.abs(v))
    return np.where(v >= 0, 1.0, e) / (1.0 + e)


def softplus(v):
    return np.maximum(v, 0.0) + np.log1p(np.exp(-np.abs(v)))


def silu(v):
    return v * sigmoid(v)


def silu_slope(v):
    s = sigmoid(v)
    return s * (1.0 + v * (1.0 - s))


def _there(lengths, T, n):
    last = np.full(n, T) if lengths is None else np.clip(np.asarray(lengths), 0, T)
    return last, (np.arange(T)[:, None] < last[None, :])[:, :, None]


def causal_conv(x, taps, bias=None, act=False, x_before=None, lengths=None):
    """(y, x_after)"""
    T, n, f = x.shape
    w = taps.shape[0]
    last, there = _there(lengths, T, n)
    frames = np.concatenate([np.zeros((w - 1, n, f)) if x_before is None else x_before, x])
    a = np.zeros((T, n, f)) if bias is None else np.broadcast_to(bias, (T, n, f)).copy()
    with np.errstate(invalid="ignore"):
        for t in range(T):
            for j in range(w):
                a[t] += taps[j] * frames[w - 1 + t - j]
        y = np.where(there, silu(a) if act else a, 0.0)
    after = np.stack([np.stack([frames[last[v] + j, v] for v in range(n)]) for j in range(w - 1)])
    return y, after


def causal_conv_backward(x, taps, g_y, bias=None, act=False, x_before=None, dx_after=None, lengths=None, magnitudes=False):
    """dict(dx, dx_before, dtaps, dbias)"""
    T, n, f = x.shape
    w = taps.shape[0]
    last, there = _there(lengths, T, n)
    frames = np.concatenate([np.zeros((w - 1, n, f)) if x_before is None else x_before, x])
    frames[w - 1:] = np.where(there, frames[w - 1:], 0.0)
    g = np.where(there, g_y, 0.0)
    if magnitudes:
        frames, g, taps, bias = np.abs(frames), np.abs(g), np.abs(taps), None if bias is None else np.abs(bias)
    if act:
        a = sum(taps[j] * frames[w - 1 - j:w - 1 - j + T] for j in range(w)) + (0.0 if bias is None else bias)
        g = np.where(there, g * (1.1 + a if magnitudes else silu_slope(a)), 0.0)     # |silu'| <= 1.1, |silu''| <= 1/2
    if magnitudes:
        dx_after = None if dx_after is None else np.abs(dx_after)
    dx, dtaps = np.zeros_like(frames), np.zeros_like(taps)
    for t in range(T):
        for j in range(w):
            dx[w - 1 + t - j] += taps[j] * g[t]
            dtaps[j] += (g[t] * frames[w - 1 + t - j]).sum(0)
    if dx_after is not None:
        for v in range(n):
            for j in range(w - 1):
                dx[last[v] + j, v] += dx_after[j, v]
    return dict(dx=dx[w - 1:], dx_before=dx[:w - 1], dtaps=dtaps, dbias=g.sum((0, 1)))


def selective_scan(x, delta, bc, a, z=None, d=None, dt_bias=None, h_before=None, lengths=None, magnitudes=False):
    """(y, h_after, h of every timestep [T, n, f, N])"""
    T, n, f = x.shape
    N = a.shape[1]
    _, there = _there(lengths, T, n)
    with np.errstate(invalid="ignore", over="ignore"):
        x = np.where(there, x, 0.0)
        step = np.where(there, softplus(delta + (0.0 if dt_bias is None else dt_bias)), 0.0)
        b, c = np.where(there, bc[:, :, :N], 0.0), np.where(there, bc[:, :, N:], 0.0)
        gate = 1.0 if z is None else np.where(there, silu(z), 0.0)
    d = np.zeros(f) if d is None else d
    h = np.zeros((n, f, N)) if h_before is None else h_before.copy()
    if magnitudes:
        x, b, c, gate, d, h = np.abs(x), np.abs(b), np.abs(c), np.abs(gate), np.abs(d), np.abs(h)
    y, states = np.zeros((T, n, f)), np.zeros((T, n, f, N))
    for t in range(T):
        h = np.exp((0.875 if magnitudes else 1.0) * step[t][..., None] * a) * h + (step[t] * x[t])[..., None] * b[t][:, None, :]
        states[t] = h
        y[t] = (h * c[t][:, None, :]).sum(-1) + d * x[t]
    return np.where(there, y * gate, 0.0), h, states


def selective_scan_backward(x, delta, bc, a, g_y, z=None, d=None, dt_bias=None, h_before=None, dh_after=None, lengths=None, magnitudes=False):
    """dict(dx, ddelta, dbc, dz, da, dd, ddt_bias, dh_before)"""
    T, n, f = x.shape
    N = a.shape[1]
    _, there = _there(lengths, T, n)
    x, g = np.where(there, x, 0.0), np.where(there, g_y, 0.0)
    pre = np.where(there, delta + (0.0 if dt_bias is None else dt_bias), 0.0)
    step, slope = np.where(there, softplus(pre), 0.0), np.where(there, sigmoid(pre), 0.0)
    b, c = np.where(there, bc[:, :, :N], 0.0), np.where(there, bc[:, :, N:], 0.0)
    dd = np.zeros(f) if d is None else d
    start = np.zeros((n, f, N)) if h_before is None else h_before
    _, _, states = selective_scan(x, np.where(there, delta, 0.0), bc, a, None, d, dt_bias, h_before, lengths, magnitudes)
    gate, gate_slope = (1.0, 0.0) if z is None else (np.where(there, silu(z), 0.0), np.where(there, silu_slope(z), 0.0))
    signed = a
    if magnitudes:
        x, g, b, c, dd, start, signed = (np.abs(v) for v in (x, g, b, c, dd, start, a))
        gate, gate_slope = np.abs(gate), 0.0 if z is None else np.where(there, 1.1 + np.abs(z), 0.0)
        dh_after = None if dh_after is None else np.abs(dh_after)
    out = dict(dx=np.zeros_like(x), ddelta=np.zeros_like(x), dbc=np.zeros((T, n, 2 * N)), dz=np.zeros_like(x), da=np.zeros_like(a), dd=np.zeros(f), ddt_bias=np.zeros(f))
    k = np.zeros((n, f, N)) if dh_after is None else dh_after.copy()
    inner = np.stack([(states[t] * c[t][:, None, :]).sum(-1) + dd * x[t] for t in range(T)])
    out["dz"] = g * inner * gate_slope
    g = g * gate
    for t in range(T - 1, -1, -1):
        e = np.exp((0.875 if magnitudes else 1.0) * step[t][..., None] * a)
        before = start if t == 0 else states[t - 1]
        gh = k + g[t][..., None] * c[t][:, None, :]
        gb = (gh * b[t][:, None, :]).sum(-1)
        u = gh * e * before
        out["dx"][t] = dd * g[t] + step[t] * gb
        out["ddelta"][t] = ((u * signed).sum(-1) + x[t] * gb) * slope[t]
        out["dbc"][t, :, :N] = (gh * (step[t] * x[t])[..., None]).sum(1)
        out["dbc"][t, :, N:] = (states[t] * g[t][..., None]).sum(1)
        out["da"] += (u * step[t][..., None]).sum(0)
        out["dd"] += (g[t] * x[t]).sum(0)
        out["ddt_bias"] += out["ddelta"][t].sum(0)
        k = gh * e
    out["dh_before"] = k
    return out
