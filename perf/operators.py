"""Operators of a temporal layer with a linear, input-gated recurrence, and of the step between its gradients and the update, as cases
that can be measured.  Frames are time-major, [T, n, f]: n sequences (vertices), f channels.

    conv   causal convolution over time, one filter of w taps per channel, with SiLU:
               a[t] = bias + sum_j taps[j] x[t - j],  y[t] = silu(a[t])
    scan   selective state-space scan, N states per channel, B and C per sequence and timestep shared by its channels:
               dt = softplus(delta + dt_bias),  h[t] = exp(dt a) h[t - 1] + dt x B[t],  y[t] = (C[t] . h[t] + d x) silu(z)
    clip   the norm over the gradients of a model, and the gradients scaled to at most max_norm

A case names its sizes in full:

    kind    conv | scan | clip
    mode    forward | step (T = 1, the state rolled on in place) | backward (conv) | train (scan: forward, then backward)
    T, n, f, dtype;  w taps (conv);  N states (scan)
    ragged  sequences of different lengths, some empty: behind its length a sequence gives zeros and keeps its state
    carry   the scan starts from a state that was handed over, and its gradient goes on to what lies before
    count, total   tensors and elements (clip);  dtype mixed: fp32 and bf16 in turn
"""
import math

import torch

own = False
DEV = "cuda:0"
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16}


def listed():
    return [
        # one new snapshot of a thousand sequences: the convolution's smallest call, its state rolled on in place
        dict(name="conv_step", kind="conv", mode="step", T=1, n=1003, f=64, w=4, dtype="bf16", ragged=False),
        # a block of sixteen snapshots of an ordinary graph, inference in bf16
        dict(name="conv_forward", kind="conv", mode="forward", T=16, n=150_001, f=64, w=4, dtype="bf16", ragged=False),
        # gradients through a longer block of wide frames, vertices that leave early
        dict(name="conv_backward", kind="conv", mode="backward", T=24, n=60_013, f=128, w=3, dtype="f32", ragged=True),
        # a handful of sequences taken one token further: launches are what counts
        dict(name="scan_step_few", kind="scan", mode="step", T=1, n=5, f=128, N=16, dtype="bf16", ragged=False, carry=True),
        # ... and all vertices of a graph one snapshot further: the state is what counts
        dict(name="scan_step", kind="scan", mode="step", T=1, n=60_013, f=64, N=16, dtype="bf16", ragged=False, carry=True),
        # a block of sixteen snapshots of an ordinary graph (recipe c2 of the benchmark at an odd size)
        dict(name="scan_forward", kind="scan", mode="forward", T=16, n=100_003, f=64, N=16, dtype="f32", ragged=False, carry=False),
        # few sequences, very long ones: the time axis is all there is to share out
        dict(name="scan_long", kind="scan", mode="forward", T=16_411, n=3, f=128, N=16, dtype="bf16", ragged=False, carry=True),
        # a training step over a block of snapshots (recipe c3's width)
        dict(name="scan_train", kind="scan", mode="train", T=16, n=50_021, f=32, N=16, dtype="f32", ragged=False, carry=True),
        # ... over a few sequences of a wide layer
        dict(name="scan_train_wide", kind="scan", mode="train", T=1025, n=4, f=1536, N=16, dtype="bf16", ragged=False, carry=False),
        # ... over sequences of different lengths, an odd width, another state size
        dict(name="scan_train_ragged", kind="scan", mode="train", T=57, n=1501, f=48, N=8, dtype="f32", ragged=True, carry=True),
        # the gradients of a small recurrent model: many tensors, few elements
        dict(name="clip_model", kind="clip", mode="forward", count=46, total=90_011, dtype="f32"),
        # ... and of one that learns a vector per vertex too
        dict(name="clip_embedding", kind="clip", mode="forward", count=9, total=400_000_011, dtype="mixed"),
    ]


# ---------------------------------------------------------------------------------------------------------- drawn cases
# the most elements T n f of a drawn case
MOST = {("conv", "forward"): 1.5e8, ("conv", "backward"): 1.5e8, ("conv", "step"): 2e7, ("scan", "forward"): 1e8, ("scan", "train"): 2.4e7, ("scan", "step"): 3.8e6}


def spread(rng, low, high):
    return int(round(2.0 ** rng.uniform(math.log2(low), math.log2(high))))


def draw(rng):
    kind, mode = rng.choice([("conv", "step"), ("conv", "forward"), ("conv", "backward"), ("scan", "step"), ("scan", "forward"),
                             ("scan", "forward"), ("scan", "train"), ("scan", "train"), ("clip", "forward")])
    if kind == "clip":
        return dict(kind=kind, mode=mode, count=spread(rng, 1, 60), total=spread(rng, 1000, 4e8), dtype=rng.choice(("f32", "bf16", "mixed")))
    c = dict(kind=kind, mode=mode, f=rng.choice((16, 32, 48, 64, 96, 128, 128, 256, 768, 1536)), dtype=rng.choice(("f32", "bf16")))
    c["T"] = 1 if mode == "step" else spread(rng, 2, 128) if rng.random() < 0.6 else spread(rng, 128, 8192)
    most = MOST[kind, mode]
    if kind == "conv":
        c["w"] = rng.choice((2, 3, 4, 4))
    else:
        c["N"] = rng.choice((8, 16, 16, 32))
        c["carry"] = mode == "step" or rng.random() < 0.5
        most = most * 16 / max(c["N"], 16)
    c["n"] = spread(rng, 1, max(2, most / (c["T"] * c["f"])))
    c["ragged"] = mode != "step" and rng.random() < 0.3
    return c


def counts_of(case):
    """Elements of every tensor of a clip case: a few large ones, many small ones, odd counts."""
    weight = [2.0 ** -(i % 12) for i in range(case["count"])]
    return [max(1, int(case["total"] * v / sum(weight))) | 1 for v in weight]


def types_of(case):
    return [TYPES[("f32", "bf16")[i % 2] if case["dtype"] == "mixed" else case["dtype"]] for i in range(case["count"])]


# ---------------------------------------------------------------------------------------------------------- preparation
def prepare(case, seed):
    g = torch.Generator(device=DEV).manual_seed(seed)
    normal = lambda *shape: torch.randn(shape, generator=g, device=DEV)  # noqa: E731
    uniform = lambda *shape: torch.rand(shape, generator=g, device=DEV)  # noqa: E731
    s = dict(case)
    if case["kind"] == "clip":
        s["grads"] = [(1e-3 * normal(count)).to(dt) for count, dt in zip(counts_of(case), types_of(case))]
        s["max_norm"] = 1.0
        if own:
            s["out"] = [torch.empty_like(x) for x in s["grads"]]
            s["gradients"] = framework().Gradients(s["grads"], s["out"])
        return s
    T, n, f, dt = case["T"], case["n"], case["f"], TYPES[case["dtype"]]
    frames = lambda width=f: normal(T, n, width).to(dt)  # noqa: E731
    s["x"] = frames()
    s["lengths"] = None
    if case["ragged"]:
        s["lengths"] = torch.where(uniform(n) < 0.06, torch.zeros(n, device=DEV), T * (0.5 + 0.5 * uniform(n))).round().to(torch.int32)
    s["g_y"] = frames() if case["mode"] in ("backward", "train") else None
    if case["kind"] == "conv":
        w = case["w"]
        s["taps"], s["bias"] = (2 * uniform(w, f) - 1) * w ** -0.5, 0.1 * normal(f)
        s["x_before"] = normal(w - 1, n, f).to(dt)
        if own and case["mode"] == "backward":
            s["ws"] = torch.empty(framework().causal_conv_backward_workspace(T, n, f, w), dtype=torch.uint8, device=DEV)
        return s
    N = case["N"]
    # steps between 0.001 and 0.1 at the bias, decays -1 .. -N with some spread, as such layers start out and stay
    step = torch.exp(math.log(1e-3) + uniform(f) * math.log(100.0))
    s["dt_bias"] = step + torch.log(-torch.expm1(-step))
    s["a"] = -torch.arange(1, N + 1, device=DEV).float() * torch.exp(0.2 * normal(f, N))
    s["d"] = 1 + 0.1 * normal(f)
    s["delta"], s["bc"], s["z"] = (0.5 * normal(T, n, f)).to(dt), frames(2 * N), frames()
    s["h_before"] = normal(n, f, N) if case["carry"] else None
    s["dh_after"] = normal(n, f, N) if case["carry"] and case["mode"] == "train" else None
    if own:
        dg = framework()
        need = dg.selective_scan_workspace(T, n, f, N)
        if case["mode"] == "train":
            need = max(need, dg.selective_scan_backward_workspace(T, n, f, N))
            s["checkpoints"] = torch.empty(dg.selective_scan_checkpoints(T, n, f, N), dtype=torch.float32, device=DEV)
        s["ws"] = torch.empty(need, dtype=torch.uint8, device=DEV)
    return s


def framework():
    import paper_2109_07893_amd
    return paper_2109_07893_amd


# ---------------------------------------------------------------------------------------------------------- plain forms
def sigmoid(x):
    return 1 / (1 + torch.exp(-x))


def softplus(x):
    return torch.where(x > 20, x, torch.log1p(torch.exp(x.clamp(max=20))))


def valid(s):
    """[T, n, 1]: whether a sequence has this timestep."""
    if s["lengths"] is None:
        return torch.ones((s["T"], s["n"], 1), dtype=torch.bool, device=DEV)
    return (torch.arange(s["T"], device=DEV)[:, None] < s["lengths"][None, :])[:, :, None]


def ends(s):
    """[w - 1, n, f]: where the last w - 1 frames of every sequence lie in (x_before, x)."""
    n, f, w = s["n"], s["f"], s["w"]
    last = torch.full((n,), s["T"], device=DEV) if s["lengths"] is None else s["lengths"].long()
    return (last[None, :] + torch.arange(w - 1, device=DEV)[:, None])[:, :, None].expand(w - 1, n, f)


def conv_plain(s):
    T, w = s["T"], s["w"]
    frames = torch.cat([s["x_before"], s["x"]]).float()
    pre = s["bias"] + sum(s["taps"][j] * frames[w - 1 - j:w - 1 - j + T] for j in range(w))
    y = torch.where(valid(s), pre * sigmoid(pre), 0.0).to(s["x"].dtype)
    return y, torch.gather(frames, 0, ends(s)).to(s["x"].dtype)


def conv_backward_plain(s):
    T, w, dt = s["T"], s["w"], s["x"].dtype
    frames = torch.cat([s["x_before"], s["x"]]).float()
    pre = s["bias"] + sum(s["taps"][j] * frames[w - 1 - j:w - 1 - j + T] for j in range(w))
    sig = sigmoid(pre)
    ga = torch.where(valid(s), s["g_y"].float() * sig * (1 + pre * (1 - sig)), 0.0)
    ahead = torch.cat([torch.zeros_like(frames[:w - 1]), ga, torch.zeros_like(frames[:w - 1])])
    dx = sum(s["taps"][j] * ahead[j:j + T + w - 1] for j in range(w))
    dtaps = torch.stack([(ga * frames[w - 1 - j:w - 1 - j + T]).sum((0, 1)) for j in range(w)])
    return dict(dx=dx[w - 1:].to(dt), dx_before=dx[:w - 1].to(dt), dtaps=dtaps, dbias=ga.sum((0, 1)))


def prefix(decay, inflow, reach=1):
    """h[t] = decay[t] h[t - 1] + inflow[t] for all t, by doubling."""
    if reach >= decay.shape[0]:
        return inflow
    inflow = torch.cat([inflow[:reach], inflow[reach:] + decay[reach:] * inflow[:-reach]])
    decay = torch.cat([decay[:reach], decay[reach:] * decay[:-reach]])
    return prefix(decay, inflow, 2 * reach)


def scan_parts(s):
    """What both directions are made of: step sizes, decays and states [T, n, f, N], and y ahead of its gate."""
    N, there = s["N"], valid(s)
    x = torch.where(there, s["x"].float(), 0.0)
    step = torch.where(there, softplus(s["delta"].float() + s["dt_bias"]), 0.0)
    b, c = s["bc"][:, :, :N].float()[:, :, None, :], s["bc"][:, :, N:].float()[:, :, None, :]
    decay = torch.exp(step[..., None] * s["a"])
    inflow = (step * x)[..., None] * b
    if s["h_before"] is not None:
        inflow[0] += decay[0] * s["h_before"]
    h = prefix(decay, inflow)
    return there, x, step, b, c, decay, h, (h * c).sum(-1) + s["d"] * x


def scan_plain(s):
    there, _, _, _, _, _, h, inner = scan_parts(s)
    z = s["z"].float()
    return torch.where(there, inner * z * sigmoid(z), 0.0).to(s["x"].dtype), h[-1]


def scan_train_plain(s):
    dt = s["x"].dtype
    there, x, step, b, c, decay, h, inner = scan_parts(s)
    z = s["z"].float()
    sig = sigmoid(z)
    y = torch.where(there, inner * z * sig, 0.0)
    g = torch.where(there, s["g_y"].float(), 0.0)
    dz = g * inner * sig * (1 + z * (1 - sig))
    g = g * z * sig
    start = torch.zeros_like(h[:1]) if s["h_before"] is None else s["h_before"][None]
    before = torch.cat([start, h[:-1]])
    inflow = g[..., None] * c
    if s["dh_after"] is not None:
        inflow[-1] += s["dh_after"]
    gh = prefix(torch.cat([decay[1:], decay[:1]]).flip(0), inflow.flip(0)).flip(0)
    through = gh * decay * before
    gb = (gh * b).sum(-1)
    dstep = (through * s["a"]).sum(-1) + gb * x
    ddelta = torch.where(there, dstep * sigmoid(s["delta"].float() + s["dt_bias"]), 0.0)
    dbc = torch.cat([(gh * (step * x)[..., None]).sum(2), (h * g[..., None]).sum(2)], -1)
    out = dict(y=y.to(dt), h_after=h[-1], dx=(s["d"] * g + step * gb).to(dt), ddelta=ddelta.to(dt), dbc=dbc.to(dt), dz=dz.to(dt),
               da=(through * step[..., None]).sum((0, 1)), dd=(g * x).sum((0, 1)), ddt_bias=ddelta.sum((0, 1)))
    if s["carry"]:
        out["dh_before"] = decay[0] * gh[0]
    return out


def clip_plain(s):
    norm = torch.stack([g.float().square().sum(dtype=torch.float64) for g in s["grads"]]).sum().sqrt()
    factor = torch.where(torch.isfinite(norm), (s["max_norm"] / (norm + 1e-6)).clamp(max=1.0), 1.0).float()
    return dict(norm=norm.float(), out=[(g.float() * factor).to(g.dtype) for g in s["grads"]])


# ---------------------------------------------------------------------------------------------------------- one pass
def run(s):
    if own:
        return run_own(s)
    kind, mode = s["kind"], s["mode"]
    if kind == "clip":
        return clip_plain(s)
    if mode == "backward":
        return conv_backward_plain(s)
    if mode == "train":
        return scan_train_plain(s)
    y, state = conv_plain(s) if kind == "conv" else scan_plain(s)
    if mode == "step":
        state = s["x_before" if kind == "conv" else "h_before"].copy_(state)
    return dict(y=y, state=state)


def run_own(s):
    dg, kind, mode = framework(), s["kind"], s["mode"]
    if kind == "clip":
        return dict(norm=s["gradients"].clip(s["max_norm"]), out=s["out"])
    x, lengths = s["x"], s["lengths"]
    if kind == "conv":
        before = s["x_before"]
        if mode == "backward":
            out = dict(dx=torch.empty_like(x), dx_before=torch.empty_like(before), dtaps=torch.empty_like(s["taps"]), dbias=torch.empty_like(s["bias"]))
            dg.causal_conv_backward(x, s["taps"], s["bias"], s["g_y"], out["dx"], out["dtaps"], out["dbias"], s["ws"], silu=True,
                                    x_before=before, dx_before=out["dx_before"], lengths=lengths)
            return out
        y, after = torch.empty_like(x), before if mode == "step" else torch.empty_like(before)
        dg.causal_conv(x, s["taps"], s["bias"], y, silu=True, x_before=before, x_after=after, lengths=lengths)
        return dict(y=y, state=after)
    a, d, dt_bias, z, before = s["a"], s["d"], s["dt_bias"], s["z"], s["h_before"]
    y = torch.empty_like(x)
    after = before if mode == "step" else torch.empty((s["n"],) + tuple(a.shape), device=DEV)
    dg.selective_scan(x, s["delta"], s["bc"], a, y, s["ws"], z=z, d=d, dt_bias=dt_bias, h_before=before, h_after=after,
                      checkpoints=s.get("checkpoints"), lengths=lengths)
    if mode != "train":
        return dict(y=y, state=after)
    out = dict(y=y, h_after=after, dx=torch.empty_like(x), ddelta=torch.empty_like(x), dbc=torch.empty_like(s["bc"]), dz=torch.empty_like(z),
               da=torch.empty_like(a), dd=torch.empty_like(d), ddt_bias=torch.empty_like(dt_bias))
    if s["carry"]:
        out["dh_before"] = torch.empty_like(after)
    dg.selective_scan_backward(x, s["delta"], s["bc"], a, s["g_y"], s["checkpoints"], out["dx"], out["ddelta"], out["dbc"], out["da"], s["ws"],
                               z=z, dz=out["dz"], d=d, dd=out["dd"], dt_bias=dt_bias, ddt_bias=out["ddt_bias"], dh_after=s["dh_after"],
                               dh_before=out.get("dh_before"), lengths=lengths)
    return out


# ---------------------------------------------------------------------------------------------------------- what a pass cannot do without
def work(case):
    if case["kind"] == "clip":
        sizes = [c * (2 if dt == torch.bfloat16 else 4) for c, dt in zip(counts_of(case), types_of(case))]
        return {"bytes": 2 * sum(sizes), "flops": 3 * sum(counts_of(case))}
    T, n, f, s = case["T"], case["n"], case["f"], 2 if case["dtype"] == "bf16" else 4
    there = 0.7 if case["ragged"] else 1.0                            # of the timesteps, about
    frame = T * n * f
    if case["kind"] == "conv":
        w = case["w"]
        edge = 2 * s * (w - 1) * n * f
        if case["mode"] == "backward":
            return {"bytes": s * frame * (1 + 2 * there) + edge, "flops": there * frame * (6 * w + 14)}
        return {"bytes": s * frame * (1 + there) + edge, "flops": there * frame * (2 * w + 5)}
    N = case["N"]
    state = 4 * n * f * N * (2 if case["carry"] else 1)
    rows = T * n * 2 * N * s
    moved, done = s * frame * (1 + 3 * there) + rows * there + state, there * frame * (7 * N + 14)
    if case["mode"] == "train":
        # going back: the inputs and g_y once more, four gradients, and the sums over time and sequences
        moved += s * frame * (3 + 4 * there) + rows * (1 + there) + (state if case["carry"] else 0)
        done += there * frame * (21 * N + 30)
    return {"bytes": moved, "flops": done}


# ---------------------------------------------------------------------------------------------------------- in 64 bits, step by step
def exact(case, seed):
    s = prepare(case, seed)
    if case["kind"] == "clip":
        norm = math.sqrt(sum(float((g.double() ** 2).sum()) for g in s["grads"]))
        return dict(norm=torch.tensor(norm, dtype=torch.float64), out=[g.double() * min(1.0, s["max_norm"] / (norm + 1e-6)) for g in s["grads"]])
    wide = {k: v.double() for k, v in s.items() if isinstance(v, torch.Tensor)}
    last = wide["lengths"] if s["lengths"] is not None else torch.full((case["n"],), float(case["T"]), device=DEV)
    return (exact_conv if case["kind"] == "conv" else exact_scan)(case, wide, last[:, None])


def exact_conv(case, s, last):
    T, w = case["T"], case["w"]
    frame = lambda t: s["x"][t] if t >= 0 else s["x_before"][w - 1 + t]  # noqa: E731
    pre = [s["bias"] + sum(s["taps"][j] * frame(t - j) for j in range(w)) for t in range(T)]
    if case["mode"] != "backward":
        y = torch.stack([torch.where(t < last, p / (1 + torch.exp(-p)), 0.0) for t, p in enumerate(pre)])
        state = torch.zeros_like(s["x_before"])
        for t in range(1 - w, T):
            for j in range(w - 1):
                state[j] = torch.where(last - (w - 1) + j == t, frame(t), state[j])
        return dict(y=y, state=state)
    dx = torch.zeros((T + w - 1,) + tuple(s["x"].shape[1:]), dtype=torch.float64, device=DEV)
    dtaps, dbias = torch.zeros_like(s["taps"]), torch.zeros_like(s["bias"])
    for t in range(T):
        sig = 1 / (1 + torch.exp(-pre[t]))
        g = torch.where(t < last, s["g_y"][t] * (sig + pre[t] * sig * (1 - sig)), 0.0)
        dbias += g.sum(0)
        for j in range(w):
            dtaps[j] += (g * frame(t - j)).sum(0)
            dx[t - j + w - 1] += s["taps"][j] * g
    return dict(dx=dx[w - 1:], dx_before=dx[:w - 1], dtaps=dtaps, dbias=dbias)


def exact_scan(case, s, last):
    T, n, f, N = case["T"], case["n"], case["f"], case["N"]
    train = case["mode"] == "train"
    if train and T * n * f * N > 1.5e9:
        return None                                                   # every state of the pass is kept in 64 bits
    h = s["h_before"].clone() if case["carry"] else torch.zeros((n, f, N), dtype=torch.float64, device=DEV)
    y, kept = torch.zeros_like(s["x"]), []
    step_of = lambda t: torch.logaddexp(s["delta"][t] + s["dt_bias"], torch.zeros((), dtype=torch.float64, device=DEV))  # noqa: E731
    gate = lambda t: s["z"][t] / (1 + torch.exp(-s["z"][t]))  # noqa: E731
    for t in range(T):
        there, step = t < last, step_of(t)
        if train:
            kept.append(h)
        new = torch.exp(step[..., None] * s["a"]) * h + (step * s["x"][t])[..., None] * s["bc"][t][:, None, :N]
        h = torch.where(there[..., None], new, h)
        y[t] = torch.where(there, ((h * s["bc"][t][:, None, N:]).sum(-1) + s["d"] * s["x"][t]) * gate(t), 0.0)
    if not train:
        return dict(y=y, state=h)
    out = dict(y=y, h_after=h, dx=torch.zeros_like(y), ddelta=torch.zeros_like(y), dbc=torch.zeros_like(s["bc"]), dz=torch.zeros_like(y),
               da=torch.zeros_like(s["a"]), dd=torch.zeros_like(s["d"]), ddt_bias=torch.zeros_like(s["dt_bias"]))
    after, carried = h, s["dh_after"] if case["carry"] else torch.zeros_like(h)
    for t in range(T - 1, -1, -1):
        there, step, x, z = t < last, step_of(t), s["x"][t], s["z"][t]
        b, c, decay = s["bc"][t][:, None, :N], s["bc"][t][:, None, N:], torch.exp(step[..., None] * s["a"])
        sig = 1 / (1 + torch.exp(-z))
        g_y = torch.where(there, s["g_y"][t], 0.0)
        out["dz"][t] = g_y * ((after * c).sum(-1) + s["d"] * x) * (sig + z * sig * (1 - sig))
        g = g_y * z * sig
        gh = torch.where(there[..., None], carried + g[..., None] * c, 0.0)
        through = gh * decay * kept[t]
        gb = (gh * b).sum(-1)
        ddelta = ((through * s["a"]).sum(-1) + gb * x) / (1 + torch.exp(-(s["delta"][t] + s["dt_bias"])))
        out["dx"][t], out["ddelta"][t] = s["d"] * g + step * gb, ddelta
        out["dbc"][t] = torch.cat([(gh * (step * x)[..., None]).sum(1), (after * g[..., None]).sum(1)], -1)
        out["da"] += (through * step[..., None]).sum(0)
        out["dd"] += (g * x).sum(0)
        out["ddt_bias"] += ddelta.sum(0)
        carried = torch.where(there[..., None], decay * gh, carried)
        after = kept[t]
        kept[t] = None
    if case["carry"]:
        out["dh_before"] = carried
    return out
