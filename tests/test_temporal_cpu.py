"""Refusals of the temporal layer's entry points and of the gradients' norm and clipping, before anything is enqueued (no GPU)."""
import ctypes
import os

import pytest
import torch

import paper_2109_07893_amd as dg
from paper_2109_07893_amd import binding

AT = [0x100000000 * (k + 1) for k in range(24)]   # never dereferenced: every call must fail on the host first
NULL, SHAPE, CAPACITY, OVERFLOW, ALIAS, ALIGN = -1, -2, -3, -4, -5, -7


@pytest.fixture(scope="module")
def lib():
    if not os.path.exists(dg.library_path()):
        dg.build_library()
    return dg.load_library()


def size(fn, *args):
    out = ctypes.c_size_t(0)
    return fn(*args, ctypes.byref(out)), out.value


def test_conv_refusals(lib):
    ok = dict(x=AT[0], taps=AT[1], bias=AT[2], x_before=AT[3], y=AT[4], x_after=AT[5], lengths=None, T=4, n=8, f=32, w=4, flags=8, dt=0)

    def call(**kw):
        a = dict(ok, **kw)
        return lib.dgnn_causal_conv(*a.values(), None)

    assert call(x=None) == NULL and call(taps=None) == NULL and call(y=None) == NULL
    for bad in (dict(T=0), dict(n=0), dict(f=24), dict(f=0), dict(f=16400), dict(w=1), dict(w=5), dict(flags=1), dict(dt=2)):
        assert call(**bad) == SHAPE, bad
    assert call(n=1 << 31) == OVERFLOW and call(T=1 << 30, n=1 << 20) == OVERFLOW
    assert call(x=AT[0] + 4) == ALIGN and call(x_after=AT[5] + 8) == ALIGN
    frame = 8 * 32 * 4
    assert call(y=AT[0]) == ALIAS and call(y=AT[0] + 2 * frame) == ALIAS and call(x_after=AT[0] + 3 * frame) == ALIAS
    assert call(x_after=AT[3] + frame) == ALIAS and call(x_after=AT[4]) == ALIAS and call(y=AT[3]) == ALIAS


def test_conv_backward_refusals(lib):
    rc, need = size(lib.dgnn_causal_conv_backward_workspace, 4, 8, 32, 4)
    assert rc == 0 and need > 0
    ok = dict(x=AT[0], taps=AT[1], bias=AT[2], x_before=AT[3], g_y=AT[4], dx_after=AT[5], dx=AT[6], dx_before=AT[7], dtaps=AT[8], dbias=AT[9], lengths=None,
              T=4, n=8, f=32, w=4, flags=8, accumulate=0, dt=0, ws=AT[10], wsb=need)

    def call(**kw):
        a = dict(ok, **kw)
        return lib.dgnn_causal_conv_backward(*a.values(), None)

    for name in ("x", "taps", "g_y", "dx", "dtaps", "dbias", "ws"):
        assert call(**{name: None}) == NULL, name
    assert call(w=5) == SHAPE and call(f=8) == SHAPE and call(flags=16) == SHAPE and call(dt=-1) == SHAPE
    assert call(wsb=need - 1) == CAPACITY and call(n=1 << 31) == OVERFLOW
    assert call(dx=AT[6] + 4) == ALIGN and call(g_y=AT[4] + 2) == ALIGN
    assert call(dx=AT[4]) == ALIAS and call(dx_before=AT[5]) == ALIAS and call(dx_before=AT[6]) == ALIAS and call(ws=AT[6]) == ALIAS
    assert size(lib.dgnn_causal_conv_backward_workspace, 0, 8, 32, 4)[0] == SHAPE
    assert lib.dgnn_causal_conv_backward_workspace(4, 8, 32, 4, None) == NULL


def test_scan_refusals(lib):
    rc, need = size(lib.dgnn_selective_scan_workspace, 40, 8, 32, 16)
    assert rc == 0 and need > 0
    ok = dict(x=AT[0], delta=AT[1], bc=AT[2], z=AT[3], a=AT[4], d=AT[5], dt_bias=AT[6], h_before=AT[7], y=AT[8], h_after=AT[9], checkpoints=AT[10], lengths=None,
              T=40, n=8, f=32, states=16, dt=0, ws=AT[11], wsb=need)

    def call(**kw):
        a = dict(ok, **kw)
        return lib.dgnn_selective_scan(*a.values(), None)

    for name in ("x", "delta", "bc", "a", "y", "ws"):
        assert call(**{name: None}) == NULL, name
    for bad in (dict(T=0), dict(n=-1), dict(f=40), dict(f=1 << 15), dict(states=12), dict(states=64), dict(dt=3)):
        assert call(**bad) == SHAPE, bad
    assert call(n=1 << 31) == OVERFLOW and call(T=1 << 30, n=1 << 16) == OVERFLOW
    for name in ("x", "bc", "h_before", "h_after", "checkpoints", "y", "ws"):
        assert call(**{name: ok[name] + 8}) == ALIGN, name
    assert call(y=AT[0]) == ALIAS and call(y=AT[3]) == ALIAS and call(h_after=AT[2] + 64) == ALIAS and call(checkpoints=AT[7]) == ALIAS
    assert call(h_after=AT[7] + 16) == ALIAS and call(ws=AT[8] + 16) == ALIAS and call(checkpoints=AT[9]) == ALIAS
    rc, long_need = size(lib.dgnn_selective_scan_workspace, 4096, 1, 32, 16)
    assert rc == 0 and long_need > need
    assert call(T=4096, n=1, wsb=long_need - 1) == CAPACITY
    assert size(lib.dgnn_selective_scan_checkpoints, 33, 8, 32, 16) == (0, 5 * 8 * 32 * 16 * 4)
    assert size(lib.dgnn_selective_scan_checkpoints, 33, 8, 32, 4)[0] == SHAPE and lib.dgnn_selective_scan_checkpoints(33, 8, 32, 16, None) == NULL


def test_scan_backward_refusals(lib):
    rc, need = size(lib.dgnn_selective_scan_backward_workspace, 40, 8, 32, 16)
    assert rc == 0 and need > 0
    ok = dict(x=AT[0], delta=AT[1], bc=AT[2], z=AT[3], a=AT[4], d=AT[5], dt_bias=AT[6], checkpoints=AT[7], g_y=AT[8], dh_after=AT[9], dx=AT[10], ddelta=AT[11],
              dbc=AT[12], dz=AT[13], da=AT[14], dd=AT[15], ddt_bias=AT[16], dh_before=AT[17], lengths=None, T=40, n=8, f=32, states=16, accumulate=0, dt=0, ws=AT[18],
              wsb=need)

    def call(**kw):
        a = dict(ok, **kw)
        return lib.dgnn_selective_scan_backward(*a.values(), None)

    for name in ("x", "delta", "bc", "a", "checkpoints", "g_y", "dx", "ddelta", "dbc", "dz", "da", "dd", "ddt_bias", "ws"):
        assert call(**{name: None}) == NULL, name
    assert call(z=None) == SHAPE and call(d=None) == SHAPE and call(dt_bias=None) == SHAPE       # gradients of what is not there
    assert call(states=24) == SHAPE and call(dt=2) == SHAPE and call(wsb=need - 1) == CAPACITY and call(n=1 << 31) == OVERFLOW
    for name in ("dx", "dbc", "dz", "g_y", "dh_after", "dh_before", "ws", "checkpoints"):
        assert call(**{name: ok[name] + 4}) == ALIGN, name
    assert call(dx=AT[0]) == ALIAS and call(ddelta=AT[10]) == ALIAS and call(dh_before=AT[9]) == ALIAS and call(dbc=AT[2]) == ALIAS and call(ws=AT[13]) == ALIAS


def test_most_timesteps(lib):
    """2^30 timesteps at most: positions in time are 32-bit numbers, one piece of the time axis further on too."""
    for fn, last in (("dgnn_causal_conv_backward_workspace", 4), ("dgnn_selective_scan_workspace", 8), ("dgnn_selective_scan_backward_workspace", 8),
                     ("dgnn_selective_scan_checkpoints", 8)):
        assert size(getattr(lib, fn), 1 << 30, 1, 16, last)[0] == 0 and size(getattr(lib, fn), (1 << 30) + 1, 1, 16, last)[0] == OVERFLOW, fn


class Item(ctypes.Structure):
    _fields_ = [("g", ctypes.c_void_p), ("out", ctypes.c_void_p), ("count", ctypes.c_int64), ("dt", ctypes.c_int64)]


def items(*rows):
    return (Item * len(rows))(*[Item(*r) for r in rows])


def test_clip_refusals(lib):
    rc, need = size(lib.dgnn_grad_clip_workspace, 2)
    assert rc == 0 and need > 0
    assert size(lib.dgnn_grad_clip_workspace, 0)[0] == SHAPE and lib.dgnn_grad_clip_workspace(1, None) == NULL

    def call(rows, count=None, max_norm=1.0, norm=AT[20], ws=AT[21], wsb=need):
        t = items(*rows)
        return lib.dgnn_grad_clip(len(rows) if count is None else count, ctypes.addressof(t), max_norm, norm, ws, wsb, None)

    good = [(AT[0], AT[0], 100, 0), (AT[1], AT[2], 50, 1)]
    assert lib.dgnn_grad_clip(2, None, 1.0, AT[20], AT[21], need, None) == NULL and lib.dgnn_grad_norm(2, None, AT[20], AT[21], need, None) == NULL
    assert call(good, norm=None) == NULL and call(good, ws=None) == NULL and call([(None, AT[0], 1, 0)]) == NULL and call([(AT[0], None, 1, 0)]) == NULL
    assert call(good, count=0) == SHAPE and call(good, max_norm=0.0) == SHAPE and call(good, max_norm=float("nan")) == SHAPE
    assert call([(AT[0], AT[0], -1, 0)]) == SHAPE and call([(AT[0], AT[0], 1, 2)]) == SHAPE and call([(AT[0], AT[0], 1 << 41, 0)]) == OVERFLOW
    assert call(good, wsb=need - 1) == CAPACITY
    assert call([(AT[0] + 2, AT[0] + 2, 4, 0)]) == ALIGN and call([(AT[0] + 1, AT[1], 4, 1)]) == ALIGN and call(good, ws=AT[21] + 8) == ALIGN
    # the same tensor twice, parts of each other, an output over another one's gradient, shifted against its own, over the norm, over the sums
    assert call([(AT[0], AT[0], 100, 0), (AT[0], AT[0], 100, 0)]) == ALIAS
    assert call([(AT[0], AT[0], 100, 0), (AT[0] + 396, AT[3], 100, 0), (AT[4], AT[3] + 4, 1, 0)]) == ALIAS
    assert call([(AT[0], AT[1], 100, 0), (AT[1] + 396, AT[2], 100, 0)]) == ALIAS
    assert call([(AT[0], AT[0] + 4, 100, 0)]) == ALIAS
    assert call([(AT[0], AT[20] - 8, 4, 0)]) == ALIAS and call([(AT[0], AT[21] + 64, 4, 0)]) == ALIAS and call([(AT[20], AT[1], 4, 0)]) == ALIAS
    t = items((AT[21], None, 4, 0))
    assert lib.dgnn_grad_norm(1, ctypes.addressof(t), AT[20], AT[21], need, None) == ALIAS


def test_binding_refuses():
    """Shapes, types and devices that the marshalling itself turns down."""
    x, taps, bias = torch.zeros(3, 4, 16), torch.zeros(3, 16), torch.zeros(16)
    with pytest.raises(ValueError, match="GPU"):
        dg.causal_conv(x, taps, bias, torch.zeros_like(x))
    for bad in (dict(y=torch.zeros(3, 4, 32)), dict(taps=torch.zeros(3, 8)), dict(bias=torch.zeros(8)), dict(x_before=torch.zeros(3, 4, 16)),
                dict(lengths=torch.zeros(3, dtype=torch.int32))):
        a = dict(dict(x=x, taps=taps, bias=bias, y=torch.zeros_like(x)), **bad)
        with pytest.raises(ValueError):
            dg.causal_conv(**a)
    with pytest.raises(TypeError):
        dg.causal_conv(x, taps.double(), bias, torch.zeros_like(x))
    with pytest.raises(TypeError):
        dg.causal_conv(x.half(), taps, bias, x.half())
    with pytest.raises(TypeError):
        dg.causal_conv(x, taps, bias, torch.zeros_like(x), lengths=torch.zeros(4, dtype=torch.int64))
    s = dict(x=x, delta=x, bc=torch.zeros(3, 4, 16), a=torch.zeros(16, 8), y=torch.zeros_like(x), ws=torch.zeros(256, dtype=torch.uint8))
    with pytest.raises(ValueError, match="GPU"):
        dg.selective_scan(**s)
    for bad in (dict(bc=torch.zeros(3, 4, 32)), dict(delta=torch.zeros(3, 4, 32)), dict(z=x.bfloat16()), dict(d=torch.zeros(8)), dict(h_before=torch.zeros(4, 16, 16)),
                dict(h_after=torch.zeros(4, 8, 16))):
        with pytest.raises(ValueError):
            dg.selective_scan(**dict(s, **bad))
    with pytest.raises(dg.DgnnError):
        dg.selective_scan(**dict(s, checkpoints=torch.zeros(4 * 16 * 8 - 1)))
    with pytest.raises(ValueError):
        dg.Gradients([])
    with pytest.raises(ValueError):
        dg.Gradients([torch.zeros(3)])
    assert binding.selective_scan_checkpoints(17, 2, 16, 8) == 3 * 2 * 16 * 8


def test_parameters_are_inputs_too(lib):
    """Outputs and workspaces that lie over parameters or lengths, gradients of parameters over anything; 32-bit numbers between two of them."""
    conv = dict(x=AT[0], taps=AT[1], bias=AT[2], x_before=AT[3], y=AT[4], x_after=AT[5], lengths=AT[6], T=4, n=8, f=32, w=4, flags=8, dt=0)
    need = size(lib.dgnn_causal_conv_backward_workspace, 4, 8, 32, 4)[1]
    conv_back = dict(x=AT[0], taps=AT[1], bias=AT[2], x_before=AT[3], g_y=AT[4], dx_after=AT[5], dx=AT[6], dx_before=AT[7], dtaps=AT[8], dbias=AT[9], lengths=AT[11],
                     T=4, n=8, f=32, w=4, flags=8, accumulate=0, dt=0, ws=AT[10], wsb=need)
    need = size(lib.dgnn_selective_scan_workspace, 40, 8, 32, 16)[1]
    scan = dict(x=AT[0], delta=AT[1], bc=AT[2], z=AT[3], a=AT[4], d=AT[5], dt_bias=AT[6], h_before=AT[7], y=AT[8], h_after=AT[9], checkpoints=AT[10], lengths=AT[12],
                T=40, n=8, f=32, states=16, dt=0, ws=AT[11], wsb=need)
    need = size(lib.dgnn_selective_scan_backward_workspace, 40, 8, 32, 16)[1]
    scan_back = dict(x=AT[0], delta=AT[1], bc=AT[2], z=AT[3], a=AT[4], d=AT[5], dt_bias=AT[6], checkpoints=AT[7], g_y=AT[8], dh_after=AT[9], dx=AT[10], ddelta=AT[11],
                     dbc=AT[12], dz=AT[13], da=AT[14], dd=AT[15], ddt_bias=AT[16], dh_before=AT[17], lengths=AT[19], T=40, n=8, f=32, states=16, accumulate=0, dt=0,
                     ws=AT[18], wsb=need)
    vector = 32 * 4
    sizes = dict(taps=4 * vector, dtaps=4 * vector, a=16 * vector, da=16 * vector, lengths=8 * 4)         # of the others: one number per channel
    for fn, ok, parameters, gradients, outputs in (
            (lib.dgnn_causal_conv, conv, ("taps", "bias"), (), ("y", "x_after")),
            (lib.dgnn_causal_conv_backward, conv_back, ("taps", "bias"), ("dtaps", "dbias"), ("dx", "dx_before", "ws")),
            (lib.dgnn_selective_scan, scan, ("a", "d", "dt_bias"), (), ("y", "h_after", "checkpoints", "ws")),
            (lib.dgnn_selective_scan_backward, scan_back, ("a", "d", "dt_bias"), ("da", "dd", "ddt_bias"), ("dx", "ddelta", "dbc", "dz", "dh_before", "ws"))):
        def call(**kw):
            return fn(*dict(ok, **kw).values(), None)

        for k in parameters + gradients + ("lengths",):
            for at in (ok[k] + 1, ok[k] + 2):
                assert call(**{k: at}) == ALIGN, (fn, k)
        for o in outputs:
            for k in parameters + ("lengths",):
                last = sizes.get(k, vector) - 16                  # 16 bytes inside of it, from either end
                assert call(**{o: ok[k]}) == ALIAS and call(**{o: ok[k] + last}) == ALIAS, (fn, o, k)
        inputs = [k for k in ok if k not in gradients + outputs and isinstance(ok[k], int) and ok[k] in AT]
        for k in gradients:
            for o in inputs + [o for o in outputs + gradients if o != k]:
                assert call(**{k: ok[o]}) == ALIAS and call(**{k: ok[o] - sizes.get(k, vector) + 4}) == ALIAS, (fn, k, o)
