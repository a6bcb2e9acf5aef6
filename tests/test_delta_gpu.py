"""The gated delta rule against its definition in 64 bits, step by step, on the GPU through the C ABI.

Bounds, in the 2-norm of an output over all its values (B times the norm of what is expected):
  f32   every value goes through at most 8 products in a row of at most 128 terms (the inverse's, the residuals', the
        output's; twice for gradients).  A product's float sum is off by about sqrt(128) 2^-24 of the norms of its
        factors, which cancellation makes at most sqrt(128) more of the result: 8 * 128 * 2^-24, rounded up to 1e-4.
  bf16  one half step, 2^-8, for each rounding to 16 bits on the way: o has four (state, residuals, P, the stored o);
        grad_v five (state's gradient, dO is exact, P, r', X, the stored value); grad_q, grad_k six (both states, r,
        E or F, dV, the stored value); grad_g and grad_beta eight (the same, as differences of two such sums).
        States and their gradients are float: the forward's has the float bound (its products take all 24 bits); the
        gradient of the first state is made of grad_v's roundings.
Single values: 40 times that bound times the larger of their size and the output's root mean square."""
import math

import pytest

import sequence_reference as ref

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")
if not torch.cuda.is_available():
    pytest.skip("no GPU", allow_module_level=True)

from paper_2501_14490_amd import mfpsn  # noqa: E402  (loads libmfpsn.so or raises)

DEV = torch.device("cuda:0")
DT = {"f32": torch.float32, "bf16": torch.bfloat16}
HALF = 2.0 ** -8
F32 = 1e-4
BOUND = {"f32": dict.fromkeys(("o", "state", "q", "k", "v", "g", "beta", "state_in"), F32),
         "bf16": {"o": 4 * HALF, "state": F32, "q": 6 * HALF, "k": 6 * HALF, "v": 5 * HALF,
                  "g": 8 * HALF, "beta": 8 * HALF, "state_in": 5 * HALF}}
NAMES = ("q", "k", "v", "g", "beta")


def make(T, N, Hk, Hv, Dk, Dv, dtype, seed=0, lengths=None, rate=0.3):
    """CPU tensors in the storage type: unit keys and queries, strengths in (0, 1), decays of about `rate` a step."""
    gen = torch.Generator().manual_seed(seed)

    def normal(*shape):
        return torch.randn(*shape, generator=gen)

    def unit(*shape):
        x = normal(*shape)
        return x / x.norm(dim=-1, keepdim=True).clamp_min(1e-6)

    c = {"q": unit(T, N, Hk, Dk), "k": unit(T, N, Hk, Dk), "v": normal(T, N, Hv, Dv),
         "g": -rate * torch.rand(T, N, Hv, generator=gen) * 2, "beta": torch.sigmoid(normal(T, N, Hv)),
         "grad_o": normal(T, N, Hv, Dv)}
    c = {n: t.to(DT[dtype]) for n, t in c.items()}
    c["state"], c["grad_state"] = 0.5 * normal(N, Hv, Dk, Dv), 0.5 * normal(N, Hv, Dk, Dv)
    c["lengths"] = torch.tensor(lengths, dtype=torch.int32) if lengths is not None else None
    c["scale"], c["dtype"] = 1.0 / math.sqrt(Dk), dtype
    return c


def dev(t):
    return t.to(DEV) if t is not None else None


def near(got, want, bound, what, terms=0.0):
    """terms: the norm of what `want` is a sum of, where its terms cancel"""
    got = got.double().cpu()
    assert got.shape == want.shape, what
    assert torch.isfinite(got).all(), f"{what} is not finite"
    if want.numel() == 0:
        return
    off, norm = (got - want), max(want.norm().item(), terms)
    assert off.norm().item() <= bound * norm + 1e-30, f"{what}: off by {off.norm().item() / max(norm, 1e-30):.3g}, bound {bound:.3g}"
    rms = norm / math.sqrt(want.numel())
    worst = (off.abs() / want.abs().clamp_min(rms + 1e-30)).max().item()
    assert worst <= 40 * bound, f"{what}: one value off by {worst:.3g}"


def forward(c, ins=None, state=True, **more):
    ins = ins or [dev(c[n]) for n in NAMES]
    desc = mfpsn.make_delta_desc(ins[0].shape, ins[2].shape, c["dtype"], c["scale"])
    return desc, ins, mfpsn.delta_forward(desc, *ins, lengths=dev(c["lengths"]), state=dev(c["state"]) if state else None,
                                          want_state=True, **more)


def check(c, state=True, grad_state=True, ins=None, cancels=False):
    """Forward (saving and not saving) and backward of case c."""
    b = BOUND[c["dtype"]]
    args = [c[n].double() for n in NAMES]
    o64, S64, g64 = ref.delta_grads(*args, c["scale"], torch.where(torch.isfinite(c["grad_o"]), c["grad_o"], 0.0).double(),
                                    c["state"].double() if state else None, c["lengths"],
                                    c["grad_state"].double() if grad_state else None)
    desc, ins, (o, S) = forward(c, ins, state)
    near(o, o64, b["o"], "o, nothing saved")
    near(S, S64, b["state"], "state, nothing saved")
    _, _, (o, S, saved) = forward(c, ins, state, want_saved=True)
    near(o, o64, b["o"], "o")
    near(S, S64, b["state"], "state")
    got = mfpsn.delta_backward(desc, *ins, saved, dev(c["grad_o"]), dev(c["lengths"]),
                               dev(c["grad_state"]) if grad_state else None, want_grad_state=True)
    torch.cuda.synchronize()
    for n, x, y in zip(NAMES, got, g64):
        terms = g64[0].norm().item() + g64[1].norm().item() if cancels and n == "g" else 0.0
        near(x, y if y is not None else torch.zeros_like(x, dtype=torch.float64, device="cpu"), b[n], "grad_" + n, terms)
    if state:
        near(got[5], g64[5], b["state_in"], "grad_state_in")


# lengths around the chunk, from one step on
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("T", [1, 2, 7, 8, 9, 15, 31, 33, 63, 64, 65, 127, 128, 130, 200])
def test_lengths(T, dtype):
    check(make(T, 2, 2, 2, 64, 32, dtype, seed=T))


# head sizes and shares: smallest, odd, not filling a tile, largest
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("Hk,Hv,Dk,Dv", [(1, 1, 1, 1), (1, 2, 5, 7), (3, 3, 16, 16), (2, 6, 48, 80), (1, 1, 65, 33),
                                         (1, 2, 96, 40), (2, 2, 127, 129), (1, 1, 128, 256), (1, 4, 128, 17),
                                         (1, 1, 64, 200)])
def test_heads(Hk, Hv, Dk, Dv, dtype):
    check(make(90, 1, Hk, Hv, Dk, Dv, dtype, seed=Dk + Dv))
    check(make(5, 2, Hk, Hv, Dk, Dv, dtype, seed=Dk + Dv + 1), state=False, grad_state=False)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_long_sequence_and_slow_decay(dtype):
    check(make(1000, 1, 1, 2, 64, 64, dtype, seed=3, rate=0.004))
    check(make(600, 1, 1, 1, 128, 128, dtype, seed=4, rate=0.004), state=False, grad_state=False)


# long enough, and of few enough heads, for the sequence to be cut into segments whose states are joined: ends within a
# segment, sequences that end before most segments, keys and values of one and of several tiles, states in and out
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("T,N,Hk,Hv,Dk,Dv,lengths", [(4200, 1, 1, 1, 16, 24, None), (5000, 3, 1, 2, 20, 70, [5000, 130, 0]),
                                                     (4161, 1, 1, 2, 128, 16, None), (2049, 2, 2, 2, 40, 33, [2049, 700]),
                                                     (1985, 4, 8, 8, 16, 70, None), (1024, 1, 1, 1, 128, 128, None),
                                                     (2048, 5, 4, 8, 16, 70, [2048, 5, 2047, 900, 0]),
                                                     (4100, 3, 16, 16, 16, 70, None)])
def test_segments_of_a_long_sequence(T, N, Hk, Hv, Dk, Dv, lengths, dtype):
    c = make(T, N, Hk, Hv, Dk, Dv, dtype, seed=T, lengths=lengths, rate=0.003)
    if lengths:
        for n in range(N):
            for name in NAMES:
                c[name][lengths[n]:, n] = float("nan")
    o64, S64 = ref.delta(*[c[n].double() for n in NAMES], c["scale"], c["state"].double(), c["lengths"])
    desc, ins, (o, S) = forward(c)
    plain = mfpsn.make_delta_desc((T, 1000, Hk, Dk), (T, 1000, Hv, Dv), dtype)  # (too many heads: not cut)
    assert mfpsn.mfpsn_delta_workspace_size(desc) > mfpsn.mfpsn_delta_workspace_size(plain) / 1000 * N
    near(o, o64, BOUND[dtype]["o"], "o")
    near(S, S64, BOUND[dtype]["state"], "state")
    # the state behind the sequences in the array of the one before them
    state, again = dev(c["state"]).clone(), torch.empty_like(o)
    work = torch.empty(mfpsn.mfpsn_delta_workspace_size(desc), dtype=torch.uint8, device=DEV)
    mfpsn.mfpsn_delta_forward(desc, *[dev(c[n]) for n in NAMES], dev(c["lengths"]) if lengths else None, state, again, state,
                              None, work, None)
    torch.cuda.synchronize()
    assert torch.equal(again, o) and torch.equal(state, S)


# the backward of such sequences: the gradients of the states between the segments, joined in reverse
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("T,N,Hk,Hv,Dk,Dv,lengths", [(1100, 1, 1, 2, 64, 70, None), (2049, 3, 1, 2, 20, 40, [2049, 130, 0]),
                                                     (1500, 2, 2, 2, 128, 128, [1500, 700]), (4100, 1, 1, 1, 16, 16, None)])
def test_gradients_of_a_long_sequence(T, N, Hk, Hv, Dk, Dv, lengths, dtype):
    c = make(T, N, Hk, Hv, Dk, Dv, dtype, seed=T, lengths=lengths, rate=0.01)
    if lengths:
        for n in range(N):
            for name in NAMES + ("grad_o",):
                c[name][lengths[n]:, n] = float("nan")
    check(c)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("T,lengths", [(150, [150, 0, 1, 64, 65, 149]), (6, [6, 0, 3, 1, 5, 2]), (70, [0, 0, 0, 0, 0, 0]),
                                       (64, [64, 200, -3, 63, 1, 32])])
def test_ragged_batches_read_nothing_behind_their_ends(T, lengths, dtype):
    c = make(T, 6, 1, 2, 32, 48, dtype, seed=T, lengths=lengths)
    for n in range(6):
        for name in NAMES + ("grad_o",):
            c[name][max(0, lengths[n]):, n] = float("nan") if n % 2 else float("inf")
    check(c)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_steps_that_forget_everything_or_write_nothing(dtype):
    """g = -inf (and far below where exp is 0), beta = 0, and decays that differ by thousands within a chunk."""
    c = make(140, 2, 1, 2, 32, 32, dtype, seed=11)
    c["g"][[0, 17, 18, 64, 100]] = float("-inf")
    c["g"][40] = -5000.0
    c["g"][[70, 71], 0] = -90.0
    c["beta"][[3, 64, 90]] = 0.0
    c["beta"][20:24] = 1.0
    args = [c[n].double() for n in NAMES]
    b = BOUND[dtype]
    # (the definition's derivative by g at -inf is a limit, 0; autograd's would be nan: e^-1e6 is as zero)
    args[3] = args[3].clamp_min(-1e6)
    o64, S64, g64 = ref.delta_grads(*args, c["scale"], c["grad_o"].double(), c["state"].double(), None,
                                    c["grad_state"].double())
    desc, ins, (o, S, saved) = forward(c, want_saved=True)
    got = mfpsn.delta_backward(desc, *ins, saved, dev(c["grad_o"]), None, dev(c["grad_state"]), True)
    near(o, o64, b["o"], "o")
    near(S, S64, b["state"], "state")
    for n, x, y in zip(NAMES + ("state_in",), got, g64):
        near(x, y, b[n], "grad_" + n)
    short = {n: (t[:8] if n in NAMES else t) for n, t in c.items()}
    o64, S64 = ref.delta(*[a[:8] for a in args], c["scale"], c["state"].double())
    _, _, (o, S) = forward(short)
    near(o, o64, b["o"], "o of a short sequence")
    near(S, S64, b["state"], "state of a short sequence")


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_equal_keys(dtype):
    """The same key at every step, written with full strength and no decay: A is all ones below its diagonal, the
    powers of which reach 10^18 in a chunk while the inverse stays within 1.

    Every step then overwrites all that the one before it wrote, so grad_g is exactly 0: its terms cancel.  They are
    q.dq and k.dk of the steps (g enters as e^G at every q and k), with unit q and k at most |dq| and |dk|: a sum of
    terms is as exact as its terms, so its bound goes by the norm of grad_q and grad_k."""
    c = make(100, 1, 1, 1, 16, 16, dtype, seed=2)
    key = torch.zeros(16)
    key[3] = 1.0
    c["k"][:] = key.to(DT[dtype])
    c["q"][:] = key.to(DT[dtype])
    c["beta"][:] = 1.0
    c["g"][:] = 0.0
    check(c, state=False, grad_state=False, cancels=True)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("shift", [0, 1])
def test_slices_of_one_projection(dtype, shift):
    """q, k and v as slices of one [T, N, q + k + v] tensor; with `shift`, starting at no vector."""
    T, N, Hk, Hv, Dk, Dv = 70, 3, 2, 4, 24, 40
    c = make(T, N, Hk, Hv, Dk, Dv, dtype, seed=9)
    width = 2 * Hk * Dk + Hv * Dv + shift
    both = torch.full((T, N, width), float("nan"), dtype=DT[dtype], device=DEV)
    at = shift
    ins = []
    for n, H, D in (("q", Hk, Dk), ("k", Hk, Dk), ("v", Hv, Dv)):
        part = both[:, :, at:at + H * D]
        part.copy_(c[n].flatten(2))
        ins.append(part.unflatten(2, (H, D)))
        assert not ins[-1].is_contiguous()
        at += H * D
    check(c, ins=ins + [dev(c["g"]), dev(c["beta"])])


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("Hk,Hv,Dk,Dv", [(1, 2, 5, 7), (2, 4, 128, 128), (1, 1, 64, 250)])
def test_steps_one_by_one(Hk, Hv, Dk, Dv, dtype):
    """DeltaState over a sequence: the definition's outputs, and its state in float throughout."""
    T, N = 12, 3
    c = make(T, N, Hk, Hv, Dk, Dv, dtype, seed=Dk)
    args = [c[n].double() for n in NAMES]
    o64, S64 = ref.delta(*args, c["scale"], c["state"].double())
    desc = mfpsn.make_delta_desc(c["q"].shape, c["v"].shape, dtype, c["scale"])
    st = mfpsn.DeltaState(desc, dev(c["state"]).clone())
    ins = [dev(c[n]) for n in NAMES]
    o = torch.stack([st.step(*(x[t] for x in ins)) for t in range(T)])
    # a step's roundings are float's, and one of the stored o
    near(o, o64, F32 + (HALF if dtype == "bf16" else 0), "o")
    near(st.state, S64, F32, "state")
    # a step that writes a new state leaves the old one, and takes none for zeros
    one = [x[:1] for x in ins]
    before = dev(c["state"]).clone()
    first, new = mfpsn.delta_step(desc, *one, before)
    assert torch.equal(before, dev(c["state"])) and torch.equal(first[0], o[0])
    zero, _ = mfpsn.delta_step(desc, *one, None)
    want, _ = mfpsn.delta_step(desc, *one, torch.zeros_like(before))
    assert torch.equal(zero, want)


def test_prompt_then_steps():
    """A state that delta_forward left goes on step by step as the whole sequence would."""
    T, cut = 90, 77
    c = make(T, 2, 2, 4, 64, 64, "bf16", seed=21)
    ins = [dev(c[n]) for n in NAMES]
    desc = mfpsn.make_delta_desc((cut, 2, 2, 64), (cut, 2, 4, 64), "bf16", c["scale"])
    o, S = mfpsn.delta_forward(desc, *(x[:cut] for x in ins), want_state=True)
    st = mfpsn.DeltaState(desc, S)
    rest = [st.step(*(x[t] for x in ins)) for t in range(cut, T)]
    o64, S64 = ref.delta(*[c[n].double() for n in NAMES], c["scale"])
    near(torch.cat((o, torch.stack(rest))), o64, BOUND["bf16"]["o"], "o")
    near(st.state, S64, BOUND["bf16"]["state"], "state")


@pytest.mark.parametrize("T", [5, 70])
def test_state_updated_in_place(T):
    c = make(T, 2, 1, 2, 64, 40, "f32", seed=1)
    desc, ins, (o, S) = forward(c)
    state = dev(c["state"]).clone()
    o2 = torch.empty_like(o)
    ws = torch.empty(max(16, mfpsn.mfpsn_delta_workspace_size(desc)), dtype=torch.uint8, device=DEV)
    mfpsn.mfpsn_delta_forward(desc, *ins, None, state, o2, state, None, ws)
    torch.cuda.synchronize()
    assert torch.equal(o, o2) and torch.equal(S, state)


def test_empty_sequences_and_batches():
    c = make(0, 2, 1, 2, 16, 16, "f32")
    desc, ins, (o, S, saved) = forward(c, want_saved=True)
    assert o.numel() == 0 and torch.equal(S.cpu(), c["state"])
    got = mfpsn.delta_backward(desc, *ins, saved, dev(c["grad_o"]), None, dev(c["grad_state"]), True)
    assert torch.equal(got[5].cpu(), c["grad_state"])
    c = make(5, 0, 1, 2, 16, 16, "f32")
    desc, ins, (o, S, saved) = forward(c, want_saved=True)
    got = mfpsn.delta_backward(desc, *ins, saved, dev(c["grad_o"]), None, dev(c["grad_state"]), True)
    assert all(t.numel() == 0 for t in got) and S.numel() == 0


def test_same_bits_on_repeats_with_garbage_workspaces_and_another_stream():
    c = make(150, 3, 1, 2, 64, 96, "bf16", seed=6, lengths=[150, 20, 128])
    desc, ins, _ = forward(c)
    go, gs, le, st = dev(c["grad_o"]), dev(c["grad_state"]), dev(c["lengths"]), dev(c["state"])

    def run(fill):
        ws = torch.full((mfpsn.mfpsn_delta_backward_workspace_size(desc),), fill, dtype=torch.uint8, device=DEV)
        saved = torch.full((mfpsn.mfpsn_delta_saved_size(desc),), fill, dtype=torch.uint8, device=DEV)
        o, S = (torch.empty(c["v"].shape, dtype=torch.bfloat16, device=DEV), torch.empty_like(st))
        mfpsn.mfpsn_delta_forward(desc, *ins, le, st, o, S, saved, None)
        return (o, S, *mfpsn.delta_backward(desc, *ins, saved, go, le, gs, True, workspace=ws))

    want = run(0)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        again = run(255)  # (all NaN)
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(want, again))


def test_graph_replays():
    """Prompt, training step and single step captured; two graphs in turn, each with its own workspaces."""
    graphs = []
    for T in (100, 70):
        c = make(T, 2, 2, 2, 32, 32, "bf16", seed=T)
        ins = [dev(c[n]) for n in NAMES]
        desc = mfpsn.make_delta_desc(ins[0].shape, ins[2].shape, "bf16", c["scale"])
        go, st = dev(c["grad_o"]), dev(c["state"])

        def run(desc=desc, ins=ins, go=go, st=st):
            o, S = mfpsn.delta_forward(desc, *ins, state=st, want_state=True)
            o2, saved = mfpsn.delta_forward(desc, *ins, state=st, want_saved=True)
            step = mfpsn.delta_step(desc, *(x[:1] for x in ins), S)
            return (o, S, o2, *step, *mfpsn.delta_backward(desc, *ins, saved, go))

        want = run()
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            got = run()
        graphs.append((graph, want, got, run))  # (run holds the inputs)
    for _ in range(3):
        for graph, want, got, _ in graphs:
            for t in got:
                t.zero_()
            torch.cuda.synchronize()
            graph.replay()
            (got[0].float() * 2).sum().item()
        torch.cuda.synchronize()
        for graph, want, got, _ in graphs:
            for i, (a, b) in enumerate(zip(want, got)):
                assert torch.equal(a, b), i


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_autograd_of_other_strides_and_broadcast_inputs(dtype):
    """Batch-first and broadcast inputs give the bits of their dense copies, and a broadcast input the sum of them."""
    c = make(70, 3, 2, 4, 24, 40, dtype, seed=21)
    go = dev(c["grad_o"])
    batch_first = [dev(c[n]).transpose(0, 1).contiguous().requires_grad_() for n in NAMES]
    o, _ = mfpsn.DeltaFunction.apply(*[t.transpose(0, 1) for t in batch_first], c["scale"])
    o.backward(go)
    dense = [dev(c[n]).requires_grad_() for n in NAMES]
    want, _ = mfpsn.DeltaFunction.apply(*dense, c["scale"])
    want.backward(go)
    assert torch.equal(o, want)
    for x, y in zip(batch_first, dense):
        assert torch.equal(x.grad, y.grad.transpose(0, 1))
    k = dev(c["k"])[:, :, :1].detach().requires_grad_()
    beta = dev(c["beta"])[:, :1, :1].detach().requires_grad_()
    ins = [dense[0].detach(), k.expand(70, 3, 2, 24), dense[2].detach(), dense[3].detach(), beta.expand(70, 3, 4)]
    mfpsn.DeltaFunction.apply(*ins, c["scale"])[0].backward(go)
    whole = [t.detach().clone().requires_grad_() for t in ins]
    mfpsn.DeltaFunction.apply(*whole, c["scale"])[0].backward(go)
    assert torch.equal(k.grad, whole[1].grad.sum(2, keepdim=True))
    # (torch sums the two axes in an order of its own: 11 additions of the type's half step)
    near_sum = whole[4].grad.double().sum((1, 2), keepdim=True)
    step = 11 * torch.finfo(beta.dtype).eps / 2 * whole[4].grad.double().abs().sum((1, 2), keepdim=True) + 1e-30
    assert ((beta.grad.double() - near_sum).abs() <= step).all()


def test_second_derivatives_are_refused():
    c = make(20, 1, 1, 1, 16, 16, "f32", seed=3)
    leaves = [dev(c[n]).requires_grad_() for n in NAMES]
    o, _ = mfpsn.DeltaFunction.apply(*leaves, c["scale"])
    (first,) = torch.autograd.grad((o * o).sum(), leaves[:1], create_graph=True)
    with pytest.raises(RuntimeError):
        first.sum().backward()
    x = torch.randn(4, 8, 1, device=DEV, requires_grad=True)
    y = mfpsn.LayerNormFunction.apply(x, None, None, 1e-5, 1)
    (first,) = torch.autograd.grad((y * y).sum(), x, create_graph=True)
    with pytest.raises(RuntimeError):
        first.sum().backward()


def test_autograd_and_differences():
    """DeltaFunction's gradients, against the definition's and against differences of the kernels' own forward."""
    c = make(75, 2, 1, 2, 16, 24, "f32", seed=13, lengths=[75, 40])
    leaves = [dev(c[n]).requires_grad_() for n in NAMES]
    state = dev(c["state"]).requires_grad_()
    go, gs, le = dev(c["grad_o"]), dev(c["grad_state"]), dev(c["lengths"])
    o, S = mfpsn.DeltaFunction.apply(*leaves, c["scale"], state, le)
    torch.autograd.backward((o, S), (go, gs))
    _, _, g64 = ref.delta_grads(*[c[n].double() for n in NAMES], c["scale"], c["grad_o"].double(), c["state"].double(),
                                c["lengths"], c["grad_state"].double())
    for n, x, y in zip(NAMES + ("state_in",), leaves + [state], g64):
        near(x.grad, y, BOUND["f32"][n], "grad_" + n)
    h = 2e-3
    gen = torch.Generator().manual_seed(5)
    for i, leaf in enumerate(leaves + [state]):
        d = torch.randn(leaf.shape, generator=gen).to(DEV)
        f = []
        for s in (1, -1):
            moved = [x.detach() + (s * h * d if j == i else 0) for j, x in enumerate(leaves + [state])]
            with torch.no_grad():
                o, S = mfpsn.DeltaFunction.apply(*moved[:5], c["scale"], moved[5], le)
            f.append((o.double() * go).sum().item() + (S.double() * gs).sum().item())
        slope, along = (f[0] - f[1]) / (2 * h), (leaf.grad.double() * d).sum().item()
        # h^2 of the third derivative, and 1e-6 of the outputs' norm over h
        size = leaf.grad.double().norm().item()
        assert abs(slope - along) <= 0.02 * size + 0.02, (i, slope, along)


def test_only_the_output_or_only_the_state_has_a_gradient():
    c = make(20, 1, 1, 1, 16, 16, "f32", seed=3)
    for which in (0, 1):
        leaves = [dev(c[n]).requires_grad_() for n in NAMES]
        out = mfpsn.DeltaFunction.apply(*leaves, c["scale"])
        (out[which] * (dev(c["grad_o"]) if which == 0 else dev(c["grad_state"]))).sum().backward()
        zero = torch.zeros_like(c["grad_o"])
        _, _, g64 = ref.delta_grads(*[c[n].double() for n in NAMES], c["scale"],
                                    (c["grad_o"] if which == 0 else zero).double(), None, None,
                                    c["grad_state"].double() if which else None)
        for n, x, y in zip(NAMES, leaves, g64):
            if y is not None and y.abs().max() > 0:
                near(x.grad, y, F32, "grad_" + n)
            else:
                assert not x.grad.any()


def test_refusals():
    c = make(9, 2, 1, 2, 16, 16, "f32")
    desc, ins, (o, S, saved) = forward(c, want_saved=True)
    st = dev(c["state"])
    with pytest.raises(TypeError):
        mfpsn.delta_forward(desc, *[x.bfloat16() for x in ins])
    with pytest.raises(ValueError):
        mfpsn.delta_forward(desc, ins[0][:8], *ins[1:])
    with pytest.raises(ValueError):
        mfpsn.delta_forward(desc, ins[0].transpose(0, 1).contiguous().transpose(0, 1), *ins[1:])
    with pytest.raises(ValueError):
        mfpsn.delta_forward(desc, *ins[:4], ins[4].cpu())
    with pytest.raises(ValueError):
        mfpsn.delta_forward(desc, *ins, state=st[:1])
    with pytest.raises(TypeError):
        mfpsn.delta_forward(desc, *ins, state=st.bfloat16())
    with pytest.raises(TypeError):
        mfpsn.delta_forward(desc, *ins, lengths=torch.zeros(2, dtype=torch.int64, device=DEV))
    with pytest.raises(ValueError):
        mfpsn.delta_forward(desc, *ins, lengths=torch.zeros(3, dtype=torch.int32, device=DEV))
    with pytest.raises(ValueError):
        mfpsn.delta_backward(desc, *ins, saved, dev(c["grad_o"])[:1])
    with pytest.raises(mfpsn.MfpsnError):
        mfpsn.delta_backward(desc, *ins, saved[:-16], dev(c["grad_o"]))
    with pytest.raises(ValueError):
        mfpsn.delta_step(desc, *ins, st)
    with pytest.raises(ValueError):
        mfpsn.make_delta_desc((3, 2, 1, 4), (4, 2, 1, 4))
    for shape in ((9, 2, 1, 129), (9, 2, 3, 16)):
        with pytest.raises((mfpsn.MfpsnError, ValueError)):
            bad = mfpsn.make_delta_desc(shape, (9, 2, 2, 16))
            mfpsn.mfpsn_delta_workspace_size(bad)
    for kw in ({"dtype": "q8_8"}, {"scale": float("nan")}):
        with pytest.raises(mfpsn.MfpsnError):
            mfpsn.mfpsn_delta_workspace_size(mfpsn.make_delta_desc((9, 2, 1, 16), (9, 2, 2, 16), **kw))
