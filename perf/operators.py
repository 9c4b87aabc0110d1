"""Workloads of the gated linear recurrence and of the 4-bit gate product.

The gated linear recurrence is the LSTM cell whose gates depend on the input
alone: from pre-activations p [T, B, 4H] (gate rows i, f, g, o) and a bias b,

    c_t = sigmoid(f_t) c_{t-1} + sigmoid(i_t) tanh(g_t),   h_t = sigmoid(o_t) tanh(c_t),

with, for batches of unequal sequences, a length each: past it the state stays
and h is zero.  ``run`` cases go forward, ``train`` cases forward and back: the
gradients of p, of the state that the sequence began with and of the bias,
from those of h and of the last state.

The 4-bit product gives the gate pre-activations of N input rows,

    y[n, r] = b[r] + sum_d s[r, d // G] (q[r, d] - z[r, d // G]) x[n, d],

with q and z in 0 .. 15, two q in a byte (even d in the low half), and one
float32 scale s for each group of G columns.

``own`` false computes both with elementary torch operations, true with the
library's kernels.
"""

import math

import torch

own = False


def listed():
    return [
        # serving, one token: 32 sequences, the state carried from call to call
        dict(name="step", op="run", dtype="bf16", T=1, B=32, H=1024, ragged=False, state=True),
        # one short clip through the smallest layer; launches and latency
        dict(name="frames", op="run", dtype="f32", T=100, B=1, H=64, ragged=False, state=False),
        # throughput: 256 clips of 16 frames at once
        dict(name="clips", op="run", dtype="bf16", T=16, B=256, H=512, ragged=False, state=True),
        # a padded batch of unequal sequences, units no multiple of anything
        dict(name="ragged", op="run", dtype="f32", T=1000, B=31, H=333, ragged=True, state=True),
        # one long sequence: all the parallelism there is lies along time
        dict(name="long", op="run", dtype="bf16", T=65536, B=1, H=512, ragged=False, state=False),
        # a training step's pass on ordinary sequences
        dict(name="train", op="train", dtype="bf16", T=2048, B=8, H=1024, ragged=False, state=True),
        # and on one long sequence and a batch of unequal ones in float32
        dict(name="train long", op="train", dtype="f32", T=20000, B=1, H=512, ragged=False, state=False),
        # one token through a small layer's gates
        dict(name="token", op="q4", dtype="bf16", N=1, D=2048, R=2048, G=128),
        # one token through a very wide layer: reading the weights is all
        dict(name="token wide", op="q4", dtype="f32", N=1, D=8192, R=32768, G=128),
        # a decoding batch, finer groups
        dict(name="batch", op="q4", dtype="bf16", N=48, D=2048, R=8192, G=64),
        # the frames of one clip with the odd widths of convolutional features, finest groups
        dict(name="features", op="q4", dtype="f32", N=100, D=8256, R=256, G=32),
        # the frames of 256 clips at once: a matrix product
        dict(name="sequences", op="q4", dtype="bf16", N=4096, D=2048, R=2048, G=128),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["run", "run", "train", "q4", "q4"])
    dtype = rng.choice(["bf16", "f32"])
    if op == "q4":
        N, D, H = _log(rng, 1, 4096), _log(rng, 64, 8256), _log(rng, 24, 2048)
        while N * D * 4 * H > 4096 * 2048 * 2048:
            N = (N + 1) // 2
        return dict(op=op, dtype=dtype, N=N, D=D, R=4 * H, G=rng.choice([32, 64, 128]))
    T, B, H = _log(rng, 1, 65536), _log(rng, 1, 256), _log(rng, 24, 2048)
    most = (16 if op == "train" else 32) << 20
    while T * B * H > most:
        if B > 1 and rng.random() < 0.6:
            B = (B + 1) // 2
        else:
            T = (T + 1) // 2
    return dict(op=op, dtype=dtype, T=T, B=B, H=H, ragged=B > 1 and rng.random() < 0.4, state=rng.random() < 0.5)


def _type(case):
    return torch.bfloat16 if case["dtype"] == "bf16" else torch.float32


def _lengths(case):
    """Lengths of a padded batch, 0 .. T in equal steps (host list)."""
    T, B = case["T"], case["B"]
    return [T * b // max(1, B - 1) for b in range(B)]


def _inputs(case, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    dt = _type(case)

    def normal(*shape, sd=1.0):
        return torch.randn(*shape, generator=g, device="cuda").mul_(sd)

    if case["op"] == "q4":
        N, D, R, G = case["N"], case["D"], case["R"], case["G"]
        groups = -(-D // G)
        w = torch.zeros(R, groups * G, device="cuda")
        w[:, :D] = normal(R, D, sd=1.0 / math.sqrt(D))
        w = w.view(R, groups, G)
        lo, hi = w.amin(-1).clamp_(max=0.0), w.amax(-1).clamp_(min=0.0)
        s = ((hi - lo) / 15.0).clamp_(min=1e-8)
        z = torch.round(-lo / s).clamp_(0, 15)
        q = (torch.round(w / s[..., None]) + z[..., None]).clamp_(0, 15).to(torch.uint8).view(R, -1)[:, :D]
        if D % 2:
            q = torch.cat([q, q.new_zeros(R, 1)], 1)
        packed = (q[:, 0::2] | (q[:, 1::2] << 4)).contiguous()
        x = normal(N, D).clamp_(min=0.0).to(dt)    # half of it zeros, as after a rectifier
        return dict(q=packed, s=s, z=z.to(torch.uint8), x=x, b=normal(R, sd=0.1), y=torch.empty(N, R, device="cuda", dtype=dt))
    T, B, H = case["T"], case["B"], case["H"]
    st = dict(p=normal(T, B, 4 * H).to(dt), b=normal(4 * H, sd=0.1), c0=None, lengths=None)
    # forget gates from a few steps' memory to some hundreds
    st["b"][H:2 * H] += torch.linspace(0.5, 5.5, H, device="cuda")
    if case["state"]:
        st["c0"] = normal(B, H, sd=0.5)
    if case["ragged"]:
        order = torch.randperm(B, generator=g, device="cuda")
        st["lengths"] = torch.tensor(_lengths(case), dtype=torch.int32, device="cuda")[order].contiguous()
    st["h"] = torch.empty(T, B, H, device="cuda", dtype=dt)
    st["c"] = torch.empty(B, H, device="cuda")
    if case["op"] == "train":
        st["dh"] = normal(T, B, H).to(dt)
        st["dc"] = normal(B, H)
        st["saved"] = torch.empty(-(-T // 8), B, H, device="cuda")
        st["dp"] = torch.empty_like(st["p"])
        st["dc0"] = torch.empty(B, H, device="cuda")
        st["db"] = torch.empty(4 * H, device="cuda")
    return st


def prepare(case, seed):
    st = _inputs(case, seed)
    st["case"] = case
    if own and case["op"] == "q4":
        from paper_1905_00689_amd import binding as lib
        st["m"] = lib.approx_lstm_q4_load(st["q"], st["s"], st["z"], case["D"], case["G"])
    return st


def run(st):
    op = st["case"]["op"]
    if own:
        return _own_q4(st) if op == "q4" else _own_linear(st, op == "train")
    return _plain_q4(st) if op == "q4" else _plain_linear(st, op == "train")


def _own_q4(st):
    from paper_1905_00689_amd import binding as lib
    lib.approx_lstm_q4_run(st["m"], st["x"], st["y"], bias=st["b"])
    return {"y": st["y"]}


def _own_linear(st, train):
    from paper_1905_00689_amd import binding as lib
    if not train:
        lib.approx_lstm_linear_run(st["p"], st["h"], bias=st["b"], lengths=st["lengths"], c0=st["c0"], c_out=st["c"])
        return {"h": st["h"], "c": st["c"]}
    lib.approx_lstm_linear_run(st["p"], st["h"], bias=st["b"], lengths=st["lengths"], c0=st["c0"], c_out=st["c"],
                               c_save=st["saved"])
    lib.approx_lstm_linear_backward(st["p"], st["dh"], st["saved"], st["dp"], bias=st["b"], lengths=st["lengths"],
                                    dc_out=st["dc"], dc0=st["dc0"], dbias=st["db"])
    return {"h": st["h"], "c": st["c"], "dp": st["dp"], "dc0": st["dc0"], "db": st["db"]}


def _plain_q4(st):
    D, G = st["case"]["D"], st["case"]["G"]
    q = torch.stack([st["q"] & 15, st["q"] >> 4], -1).flatten(1)[:, :D].float()
    s = st["s"].repeat_interleave(G, 1)[:, :D]
    z = st["z"].float().repeat_interleave(G, 1)[:, :D]
    y = st["x"].float() @ ((q - z) * s).t() + st["b"]
    return {"y": y.to(st["x"].dtype)}


def _scan(a, b):
    """y_t = a_t y_{t-1} + b_t along dim 0 from y_{-1} = 0, in log2(T) doublings."""
    d = 1
    while d < len(a):
        b = torch.cat([b[:d], torch.addcmul(b[d:], a[d:], b[:-d])])
        a = torch.cat([a[:d], a[d:] * a[:-d]])
        d *= 2
    return b


def _plain_linear(st, train):
    p, dt = st["p"], st["p"].dtype
    T, B, _ = p.shape
    pi, pf, pg, po = (p.float() + st["b"]).chunk(4, -1)
    i, f, g, o = torch.sigmoid(pi), torch.sigmoid(pf), torch.tanh(pg), torch.sigmoid(po)
    c0 = st["c0"] if st["c0"] is not None else torch.zeros_like(i[0])
    u = i * g
    live = None
    if st["lengths"] is not None:
        live = (torch.arange(T, device=p.device)[:, None] < st["lengths"])[..., None]
        f, u = torch.where(live, f, 1.0), torch.where(live, u, 0.0)
    c = _scan(f, torch.cat([torch.addcmul(u[:1], f[:1], c0), u[1:]]))
    tc = torch.tanh(c)
    h = o * tc
    if live is not None:
        h = torch.where(live, h, 0.0)
    out = {"h": h.to(dt), "c": c[-1]}
    if not train:
        return out
    dh = st["dh"].float()
    e = dh * o * (1 - tc * tc)
    if live is not None:
        e = torch.where(live, e, 0.0)
    e = torch.cat([e[:-1], e[-1:] + st["dc"]]).flip(0)
    later = torch.cat([torch.ones_like(f[:1]), f[1:].flip(0)])
    d = _scan(later, e).flip(0)
    before = torch.cat([c0[None], c[:-1]])
    dp = torch.cat([d * g * i * (1 - i), d * before * f * (1 - f), d * i * (1 - g * g), dh * tc * o * (1 - o)], -1)
    if live is not None:
        dp = torch.where(live, dp, 0.0)
    out["dp"] = dp.to(dt)
    out["dc0"] = f[0] * d[0]
    out["db"] = dp.sum((0, 1), dtype=torch.float64).float()
    return out


def work(case):
    e = 2 if case["dtype"] == "bf16" else 4
    if case["op"] == "q4":
        N, D, R, G = case["N"], case["D"], case["R"], case["G"]
        groups = -(-D // G)
        return {"bytes": R * -(-D // 2) + 5 * R * groups + 4 * R + e * N * (D + R), "flops": 2 * N * D * R}
    T, B, H = case["T"], case["B"], case["H"]
    steps, rows = T * B, T * B
    if case["ragged"]:
        steps = sum(_lengths(case))
    state = 4 * B * H * (2 if case["state"] else 1) + 16 * H
    if case["op"] == "run":
        return {"bytes": e * H * (4 * steps + rows) + state, "flops": 20 * H * steps}
    return {"bytes": e * H * (5 * steps + 5 * rows) + state + 8 * B * H + 16 * H, "flops": 60 * H * steps}


def exact(case, seed):
    """The same by the definitions in float64, the recurrence one timestep after another."""
    st = _inputs(case, seed)
    if case["op"] == "q4":
        D, G, R = case["D"], case["G"], case["R"]
        w = torch.empty(R, 2 * st["q"].shape[1], dtype=torch.float64, device="cuda")
        w[:, 0::2], w[:, 1::2] = (st["q"] % 16).double(), torch.div(st["q"], 16, rounding_mode="floor").double()
        group = torch.arange(D, device="cuda") // G
        w = (w[:, :D] - st["z"].double()[:, group]) * st["s"].double()[:, group]
        return {"y": torch.addmm(st["b"].double(), st["x"].double(), w.t())}
    T, B, H = case["T"], case["B"], case["H"]
    p = st["p"].double() + st["b"].double()
    i, f, g, o = (torch.special.expit(p[..., :H]), torch.special.expit(p[..., H:2 * H]), torch.tanh(p[..., 2 * H:3 * H]),
                  torch.special.expit(p[..., 3 * H:]))
    del p
    keep = torch.ones(T, B, 1, dtype=torch.float64, device="cuda")
    if st["lengths"] is not None:
        keep = (torch.arange(T, device="cuda").view(T, 1, 1) < st["lengths"].view(1, B, 1)).double()
    f, i, o = 1 - keep * (1 - f), i * keep, o * keep
    c = torch.zeros(T + 1, B, H, dtype=torch.float64, device="cuda")
    if st["c0"] is not None:
        c[0] = st["c0"].double()
    into = i * g
    for t in range(T):
        torch.addcmul(into[t], f[t], c[t], out=c[t + 1])
    th = torch.tanh(c[1:])
    out = {"h": o * th, "c": c[T]}
    if case["op"] == "run":
        return out
    dh = st["dh"].double() * keep
    inner = dh * o * (1 - th.square())
    e = st["dc"].double()
    for t in range(T - 1, -1, -1):
        inner[t] += e
        e = f[t] * inner[t]
    dp = torch.empty(T, B, 4, H, dtype=torch.float64, device="cuda")
    dp[:, :, 0] = inner * g * i * (1 - i)
    dp[:, :, 1] = inner * c[:T] * f * (1 - f)
    dp[:, :, 2] = inner * i * (1 - g.square())
    dp[:, :, 3] = dh * th * o * (1 - o)
    out.update(dp=dp.view(T, B, 4 * H), dc0=e, db=dp.sum((0, 1)).view(4 * H))
    return out
