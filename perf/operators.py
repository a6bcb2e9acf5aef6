"""Performance cases of the sequence operators beside the neuron: layer norm over the channels, and the gated delta rule.

A case is one call (or one forward with its backward) with its sizes.  Kinds:

  norm         layer norm over the channels of x[M][C][S] (time-first tensors: M = T*N; time-last ones: S holds the time)
  norm_train   the same with its backward: gradients of the input and of the weights
  step         one time step of the gated delta rule for a batch of sequences: outputs and the updated states
  prompt       the gated delta rule over whole sequences, from a state to a state
  delta_train  the gated delta rule over whole sequences and its backward

`own` chooses between the plain forms below (elementary torch operations in 32 bits) and the package's operators.
"""
import math

import torch

own = False

EPS = 1e-5
CHUNK = 64  # steps that the plain form of the delta rule joins in one matrix product
TORCH = {"f32": torch.float32, "bf16": torch.bfloat16}
BYTES = {"f32": 4, "bf16": 2}


def _norm(name, kind, dtype, M, C, S):
    return {"name": name, "kind": kind, "dtype": dtype, "M": M, "C": C, "S": S}


def _delta(name, kind, dtype, T, N, Hk, Hv, Dk, Dv, ragged=False, state=False):
    return {"name": name, "kind": kind, "dtype": dtype, "T": T, "N": N, "Hk": Hk, "Hv": Hv, "Dk": Dk, "Dv": Dv,
            "ragged": ragged, "state": state}


def listed():
    return [
        # one arriving time step of four streams of the audio layer (512 channels): the launch is what it costs
        _norm("norm_token", "norm", "f32", 4, 512, 1),
        # the audio layer's whole batch, 250 steps x 256 samples x 512 channels, in training
        _norm("norm_train_audio", "norm_train", "f32", 64000, 512, 1),
        # event-camera planes in bf16 (30 steps x 32 samples, 64 channels, 44x44 positions): channels strided by the plane
        _norm("norm_train_event", "norm_train", "bf16", 960, 64, 1936),
        # odd widths: rows that start at no vector's border
        _norm("norm_train_odd", "norm_train", "bf16", 4811, 1001, 1),
        # time-last tensors of the long sequences: 16 samples, 1024 channels, 4096 steps innermost
        _norm("norm_time_last", "norm", "bf16", 16, 1024, 4096),
        # one stream answering step by step
        _delta("step_one", "step", "bf16", 1, 1, 4, 4, 128, 128),
        # a serving batch of 128 streams, value heads in pairs that share their keys: all states read and written
        _delta("step_batch", "step", "bf16", 1, 128, 8, 16, 128, 128),
        # a short odd prompt, from nothing to a state
        _delta("prompt_short", "prompt", "bf16", 77, 1, 8, 8, 64, 64),
        # a padded batch of requests of different lengths, each continuing its state
        _delta("prompt_ragged", "prompt", "bf16", 2000, 8, 4, 8, 128, 128, True, True),
        # one very long prompt: few heads to share the chip
        _delta("prompt_long", "prompt", "bf16", 16384, 1, 16, 16, 128, 128),
        # a training step of ordinary size
        _delta("delta_train", "delta_train", "bf16", 2048, 8, 16, 16, 128, 128),
        # the audio shape's 251 steps in f32 with head sizes that fill no tile and shared keys
        _delta("delta_train_odd", "delta_train", "f32", 251, 12, 3, 6, 48, 80),
    ]


def _log(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    kind = rng.choice(["norm", "norm_train", "norm_train", "step", "prompt", "delta_train"])
    dtype = rng.choice(["f32", "bf16"])
    if kind in ("norm", "norm_train"):
        C = _log(rng, 16, 8192)
        S = 1 if rng.random() < 0.6 else _log(rng, 2, 4096)
        top = 30_000_000 if dtype == "f32" else 60_000_000
        return {"kind": kind, "dtype": dtype, "M": _log(rng, 1, max(1, min(65536, top // (C * S)))), "C": C, "S": S}
    Hk = rng.randint(1, 16)
    Hv = Hk * rng.choice([1, 1, 2])
    Dk = rng.choice([16, 32, 48, 64, 96, 128, 128])
    Dv = rng.choice([16, 32, 64, 80, 128, 128, 200])
    case = {"kind": kind, "dtype": dtype, "T": 1, "N": 1, "Hk": Hk, "Hv": Hv, "Dk": Dk, "Dv": Dv, "ragged": False,
            "state": False}
    if kind == "step":
        case["N"] = _log(rng, 1, max(1, min(128, 32_000_000 // (Hv * Dk * Dv))))
        return case
    # tokens x value heads, kept to what the largest listed case has
    top = 250_000 if kind == "prompt" else 200_000
    case["T"] = _log(rng, 1, 16384 if kind == "prompt" else 4096)
    if dtype == "f32":
        top //= 4
    case["T"] = min(case["T"], top // Hv)
    case["N"] = _log(rng, 1, max(1, min(32, top // (Hv * case["T"]))))
    case["ragged"] = case["N"] > 1 and rng.random() < 0.5
    case["state"] = kind == "prompt" and rng.random() < 0.5
    return case


# ---------------------------------------------------------------------------
# what a program has in hand
# ---------------------------------------------------------------------------
def _inputs(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    dt = TORCH[case["dtype"]]

    def normal(*shape):
        return torch.randn(*shape, generator=gen, device="cuda")

    if case["kind"] in ("norm", "norm_train"):
        M, C, S = case["M"], case["C"], case["S"]
        # activations of a layer: a mean and a width for each channel
        x = (normal(M, C, S).mul_(0.5 + normal(C, 1).abs()).add_(0.5 * normal(C, 1))).to(dt)
        st = {"x": x, "gamma": 1 + 0.2 * normal(C), "beta": 0.2 * normal(C)}
        if case["kind"] == "norm_train":
            st["grad_y"] = normal(M, C, S).to(dt)
        return st
    T, N, Hk, Hv, Dk, Dv = (case[n] for n in ("T", "N", "Hk", "Hv", "Dk", "Dv"))

    def unit(*shape):
        x = normal(*shape)
        return (x / x.square().sum(-1, keepdim=True).sqrt().clamp_min(1e-6)).to(dt)

    # unit queries and keys, write strengths in (0, 1), decays of a head between slow (0.999) and fast (0.1) a step
    rate = torch.exp(math.log(0.002) + (math.log(1.0) - math.log(0.002)) * torch.rand(Hv, generator=gen, device="cuda"))
    st = {"q": unit(T, N, Hk, Dk), "k": unit(T, N, Hk, Dk), "v": normal(T, N, Hv, Dv).to(dt),
          "g": (-rate * torch.log1p(torch.exp(normal(T, N, Hv)))).to(dt),
          "beta": torch.sigmoid(normal(T, N, Hv)).to(dt), "lengths": None, "state": None, "grad_o": None}
    if case["kind"] == "step" or case["state"]:
        st["state"] = 0.3 * normal(N, Hv, Dk, Dv)
    if case["ragged"]:
        st["lengths"] = torch.randint(max(1, T // 3), T + 1, (N,), generator=gen, device="cuda", dtype=torch.int32)
    if case["kind"] == "delta_train":
        st["grad_o"] = normal(T, N, Hv, Dv).to(dt)
    return st


def prepare(case, seed):
    st = _inputs(case, seed)
    st["case"] = case
    st["scale"] = 1.0 / math.sqrt(case["Dk"]) if "Dk" in case else None
    return st


# ---------------------------------------------------------------------------
# plain forms
# ---------------------------------------------------------------------------
def _plain_norm(st):
    x = st["x"].float()
    mean = x.mean(1, keepdim=True)
    xc = x - mean
    rstd = 1.0 / torch.sqrt(xc.square().mean(1, keepdim=True) + EPS)
    xh = xc * rstd
    y = (xh * st["gamma"][:, None] + st["beta"][:, None]).to(st["x"].dtype)
    if "grad_y" not in st:
        return {"y": y}
    gy = st["grad_y"].float()
    a = gy * st["gamma"][:, None]
    gx = rstd * (a - a.mean(1, keepdim=True) - xh * (a * xh).mean(1, keepdim=True))
    return {"y": y, "grad_x": gx.to(st["x"].dtype), "grad_gamma": (gy * xh).sum((0, 2)), "grad_beta": gy.sum((0, 2))}


def _plain_step(st):
    case = st["case"]
    r = case["Hv"] // case["Hk"]
    q, k = (st[n][0].float().repeat_interleave(r, 1) for n in ("q", "k"))
    v, g, beta = (st[n][0].float() for n in ("v", "g", "beta"))
    state = st["state"] * torch.exp(g)[..., None, None]
    u = beta[..., None] * (v - (k[..., None] * state).sum(-2))
    state = state + k[..., None] * u[..., None, :]
    o = st["scale"] * (q[..., None] * state).sum(-2)
    return {"o": o[None].to(st["v"].dtype), "state": state}


def _unit_lower_inverse(A):
    """(I + A)^-1 of strictly lower triangles [..., L, L], L a power of two: diagonal blocks of twice the size at a time."""
    L = A.shape[-1]
    X = torch.ones(*A.shape[:-2], L, 1, 1, device=A.device)
    b = 1
    while b < L:
        n = L // (2 * b)
        low = A.unflatten(-1, (n, 2 * b)).unflatten(-3, (n, 2 * b)).diagonal(dim1=-4, dim2=-2).movedim(-1, -3)[..., b:, :b]
        first, last = X[..., 0::2, :, :], X[..., 1::2, :, :]
        corner = -(last @ (low @ first))
        X = torch.cat((torch.cat((first, torch.zeros_like(first)), -1), torch.cat((corner, last), -1)), -2)
        b *= 2
    return X.squeeze(-3)


def _plain_delta(q, k, v, g, beta, state, lengths, scale):
    """o [T, N, Hv, Dv] and the last states, from 32-bit inputs [T, N, heads, D]: chunks of steps as matrix products."""
    T, N, Hv, Dv = v.shape
    r = Hv // q.shape[2]
    q, k = q.repeat_interleave(r, 2), k.repeat_interleave(r, 2)
    if lengths is not None:  # steps behind a sequence's end write nothing and keep the state
        live = torch.arange(T, device=v.device)[:, None] < lengths[None, :]
        g, beta = (torch.where(live[..., None], x, 0.0) for x in (g, beta))
        q, k, v = (torch.where(live[..., None, None], x, 0.0) for x in (q, k, v))
    pad = -T % CHUNK

    def chunks(x):  # [chunks, N, Hv, CHUNK, ...]
        x = torch.cat((x, x.new_zeros(pad, *x.shape[1:]))) if pad else x
        return x.unflatten(0, (-1, CHUNK)).movedim(1, 3).contiguous()

    q, k, v, g, beta = (chunks(x) for x in (q, k, v, g, beta))
    G = g.double().cumsum(-1)
    M = torch.exp((G[..., :, None] - G[..., None, :]).float().tril())
    kT = k.transpose(-1, -2).contiguous()
    A = (M * (k @ kT) * beta[..., None, :]).tril(-1)
    P = (scale * M * (q @ kT) * beta[..., None, :]).tril()
    X = _unit_lower_inverse(A)
    eG = torch.exp(G).float()[..., None]
    to_end = torch.exp(G[..., -1:] - G).float() * beta
    qd, kd, kw = scale * eG * q, X @ (eG * k), (kT * to_end[..., None, :])
    v = X @ v
    last = torch.exp(G[..., -1]).float()[..., None, None]
    S = state if state is not None else v.new_zeros(N, Hv, q.shape[-1], Dv)
    o = []
    for c in range(q.shape[0]):
        u = v[c] - kd[c] @ S
        o.append(qd[c] @ S + P[c] @ u)
        S = last[c] * S + kw[c] @ u
    o = torch.stack(o).movedim(3, 1).flatten(0, 1)[:T]
    return o, S


def _plain_sequence(st):
    names = ("q", "k", "v", "g", "beta")
    dt = st["v"].dtype
    args = [st[n].float() for n in names]
    if st["grad_o"] is None:
        with torch.no_grad():
            o, S = _plain_delta(*args, st["state"], st["lengths"], st["scale"])
        return {"o": o.to(dt), "state": S}
    args = [a.detach().requires_grad_() for a in args]
    o, _ = _plain_delta(*args, st["state"], st["lengths"], st["scale"])
    grads = torch.autograd.grad(o, args, st["grad_o"].float())
    out = {"grad_" + n: x.to(dt) for n, x in zip(names, grads)}
    out["o"] = o.detach().to(dt)
    return out


# ---------------------------------------------------------------------------
# the package's operators
# ---------------------------------------------------------------------------
def _own(st):
    from paper_2501_14490_amd import mfpsn

    case = st["case"]
    if case["kind"] == "norm":
        return {"y": mfpsn.layer_norm_forward(st["x"], st["gamma"], st["beta"], EPS, axis=1)}
    if case["kind"] == "norm_train":
        y, mean, rstd = mfpsn.layer_norm_forward(st["x"], st["gamma"], st["beta"], EPS, axis=1, want_stats=True)
        gx, gg, gb = mfpsn.layer_norm_backward(st["x"], st["gamma"], mean, rstd, st["grad_y"], axis=1)
        return {"y": y, "grad_x": gx, "grad_gamma": gg, "grad_beta": gb}
    desc = mfpsn.make_delta_desc(st["q"].shape, st["v"].shape, case["dtype"], st["scale"])
    args = [st[n] for n in ("q", "k", "v", "g", "beta")]
    if case["kind"] == "step":
        o, state = mfpsn.delta_step(desc, *args, st["state"])
        return {"o": o, "state": state}
    if case["kind"] == "prompt":
        o, state = mfpsn.delta_forward(desc, *args, lengths=st["lengths"], state=st["state"], want_state=True)
        return {"o": o, "state": state}
    o, saved = mfpsn.delta_forward(desc, *args, lengths=st["lengths"], want_saved=True)
    grads = mfpsn.delta_backward(desc, *args, saved, st["grad_o"], lengths=st["lengths"])
    return {"o": o, "grad_q": grads[0], "grad_k": grads[1], "grad_v": grads[2], "grad_g": grads[3],
            "grad_beta": grads[4]}


def run(state):
    if own:
        return _own(state)
    if state["case"]["kind"] in ("norm", "norm_train"):
        with torch.no_grad():
            return _plain_norm(state)
    if state["case"]["kind"] == "step":
        with torch.no_grad():
            return _plain_step(state)
    return _plain_sequence(state)


def work(case):
    es = BYTES[case["dtype"]]
    if case["kind"] in ("norm", "norm_train"):
        n, C = case["M"] * case["C"] * case["S"], case["C"]
        if case["kind"] == "norm":  # x, gamma, beta in, y out
            return {"bytes": 2 * n * es + 8 * C, "flops": 8 * n}
        return {"bytes": 4 * n * es + 16 * C, "flops": 20 * n}  # x, grad_y in, y, grad_x out
    T, N, Hk, Hv, Dk, Dv = (case[n] for n in ("T", "N", "Hk", "Hv", "Dk", "Dv"))
    steps = T * N
    if case["ragged"]:  # lengths between a third and the whole
        steps = steps * 2 / 3
    inputs = steps * (2 * Hk * Dk + Hv * Dv + 2 * Hv) * es
    states = N * Hv * Dk * Dv * 4
    flops = steps * Hv * Dk * Dv * 6  # read by the key, write, read by the query
    if case["kind"] == "delta_train":  # inputs and grad_o in, o and the inputs' gradients out; twice the products again
        return {"bytes": 2 * inputs + 2 * T * N * Hv * Dv * es, "flops": 3 * flops}
    held = 2 if case["kind"] == "step" or case["state"] else 1
    return {"bytes": inputs + T * N * Hv * Dv * es + held * states, "flops": flops}


# ---------------------------------------------------------------------------
# the definitions in 64 bits
# ---------------------------------------------------------------------------
def _exact_norm(case, st):
    x = st["x"].double()
    gamma, beta = (st[n].double().view(1, -1, 1) for n in ("gamma", "beta"))
    C = case["C"]
    dev = x - x.sum(1, keepdim=True) / C
    s = (dev.pow(2).sum(1, keepdim=True) / C + EPS).pow(-0.5)
    out = {"y": dev * s * gamma + beta}
    if case["kind"] == "norm":
        return out
    gy = st["grad_y"].double()
    out["grad_gamma"] = (gy * dev * s).sum(2).sum(0)
    out["grad_beta"] = gy.sum(2).sum(0)
    d = gy * gamma
    # derivative of dev * s, s = (mean dev^2 + eps)^-1/2, and of dev = x - mean x
    d = d * s - dev * s.pow(3) * (d * dev).sum(1, keepdim=True) / C
    out["grad_x"] = d - d.sum(1, keepdim=True) / C
    return out


def _exact_delta(case, st):
    T, N, Hv, Dk, Dv = (case[n] for n in ("T", "N", "Hv", "Dk", "Dv"))
    r = Hv // case["Hk"]
    q, k = (st[n].double().repeat_interleave(r, 2) for n in ("q", "k"))
    v, g, beta = (st[n].double() for n in ("v", "g", "beta"))
    scale = st["scale"]
    live = torch.ones(T, N, dtype=torch.bool, device="cuda")
    if st["lengths"] is not None:
        live = torch.arange(T, device="cuda")[:, None] < st["lengths"][None, :]
    live = live.double()[:, :, None, None]
    S = torch.zeros(N, Hv, Dk, Dv, dtype=torch.float64, device="cuda")
    if st["state"] is not None:
        S = S + st["state"].double()

    def advance(S, t):
        """S_t and the residual v_t - e^g S_{t-1}^T k_t."""
        kept = S * torch.exp(g[t])[..., None, None]
        res = v[t] - torch.matmul(k[t][..., None, :], kept).squeeze(-2)
        new = kept + k[t][..., :, None] * (beta[t][..., None] * res)[..., None, :]
        return S + live[t][..., None] * (new - S), res

    every = 64
    o, marks = torch.zeros(T, N, Hv, Dv, dtype=torch.float64, device="cuda"), []
    for t in range(T):
        if t % every == 0 and case["kind"] == "delta_train":
            marks.append(S)
        S, _ = advance(S, t)
        o[t] = live[t] * scale * torch.matmul(q[t][..., None, :], S).squeeze(-2)
    if case["kind"] != "delta_train":
        return {"o": o, "state": S}
    go = st["grad_o"].double() * live
    gq, gk, gv, gg, gb = (torch.zeros_like(x) for x in (q, k, v, g, beta))
    dS = torch.zeros_like(S)
    for m in reversed(range(len(marks))):
        span = range(m * every, min(T, (m + 1) * every))
        S, before = marks[m], []
        for t in span:
            before.append(S)
            S, res = advance(S, t)
            before[-1] = (before[-1], res, S)
        for t in reversed(span):
            old, res, new = before.pop()
            alive = live[t][..., 0]
            decay = torch.exp(g[t])[..., None, None]
            gq[t] = scale * torch.matmul(new, go[t][..., None]).squeeze(-1)
            dS = dS + scale * q[t][..., :, None] * go[t][..., None, :]
            write = torch.matmul(k[t][..., None, :], dS).squeeze(-2)  # gradient of beta * res
            gb[t] = alive * (write * res).sum(-1)
            dres = beta[t][..., None] * write
            gv[t] = live[t] * dres
            gk[t] = live[t] * (torch.matmul(dS, (beta[t][..., None] * res)[..., None]).squeeze(-1)
                               - torch.matmul(old * decay, dres[..., None]).squeeze(-1))
            kept = dS - k[t][..., :, None] * dres[..., None, :]  # gradient of e^g S_{t-1}
            gg[t] = alive * (kept * old * decay).sum((-1, -2))
            dS = dS + live[t][..., None] * (kept * decay - dS)

    def shared(x):
        return x.unflatten(2, (case["Hk"], r)).sum(3)

    return {"o": o, "grad_q": shared(gq), "grad_k": shared(gk), "grad_v": gv, "grad_g": gg, "grad_beta": gb}


def exact(case, seed):
    """What run() returns, from the definitions: every time step by itself, in 64 bits."""
    st = prepare(case, seed)
    with torch.no_grad():
        if case["kind"] in ("norm", "norm_train"):
            return _exact_norm(case, st)
        return _exact_delta(case, st)
