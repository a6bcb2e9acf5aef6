"""The sequence operators with the neuron, as a network has them: norm over the channels, gated delta rule, norm over
each head's values, spiking neuron; trained through autograd and fed step by step."""
import pytest

import sequence_reference as ref

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")
if not torch.cuda.is_available():
    pytest.skip("no GPU", allow_module_level=True)

from paper_2501_14490_amd import mfpsn  # noqa: E402  (loads libmfpsn.so or raises)

DEV = torch.device("cuda:0")
T, N, C, Hk, Hv, Dk, Dv, K, D = 70, 3, 48, 2, 4, 16, 12, 4, 2


def parameters(dtype):
    gen = torch.Generator().manual_seed(0)

    def normal(*shape):
        return torch.randn(*shape, generator=gen)

    p = {"gamma": 1 + 0.1 * normal(C), "beta": 0.1 * normal(C), "w": normal(C, 2 * Hk * Dk + Hv * Dv + 2 * Hv) / C ** 0.5,
         "gamma2": 1 + 0.1 * normal(Dv), "beta2": 0.1 * normal(Dv), "taps": normal(Hv * Dv, K), "bias": 0.1 * normal(Hv * Dv)}
    x = normal(T, N, C).to(dtype)
    return x, {n: t.to(DEV) for n, t in p.items()}


def projected(h, w, dtype):
    """q, k, v (slices of one product, queries and keys scaled to at most unit length), g, beta."""
    y = torch.matmul(h.float(), w)
    qk, v, g, b = y.split([2 * Hk * Dk, Hv * Dv, Hv, Hv], -1)
    qk = qk.unflatten(-1, (2, Hk, Dk))
    qk = (qk / qk.norm(dim=-1, keepdim=True)).to(dtype)
    both = torch.cat((qk.flatten(-3), v.to(dtype)), -1)
    q, k, v = both.split([Hk * Dk, Hk * Dk, Hv * Dv], -1)
    return (q.unflatten(-1, (Hk, Dk)), k.unflatten(-1, (Hk, Dk)), v.unflatten(-1, (Hv, Dv)),
            (-torch.log1p(torch.exp(g))).to(dtype).contiguous(), torch.sigmoid(b).to(dtype).contiguous())


def block(x, p, dtype):
    h = mfpsn.LayerNormFunction.apply(x, p["gamma"], p["beta"], 1e-5, 2)
    o, state = mfpsn.DeltaFunction.apply(*projected(h, p["w"], dtype))
    y = mfpsn.LayerNormFunction.apply(o, p["gamma2"], p["beta2"], 1e-5, 3)
    spikes = mfpsn.MfPSNFunction.apply(y.flatten(2), p["taps"], p["bias"], K, D, 0.5, "sigmoid", 4.0, 0, 7)
    return spikes, y, state


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_training_step(dtype):
    x, p = parameters(dtype)
    leaves = {n: t.clone().requires_grad_() for n, t in p.items()}
    xd = x.to(DEV).requires_grad_()
    spikes, y, state = block(xd, leaves, dtype)
    assert set(spikes.float().unique().tolist()) == {0.0, 1.0}
    gen = torch.Generator().manual_seed(1)
    gs = torch.randn(spikes.shape, generator=gen).to(DEV).to(dtype)
    spikes.backward(gs)
    # the neuron's own gradient by its input, then the block's from the definitions in 64 bits
    yl = y.detach().flatten(2).requires_grad_()
    mfpsn.MfPSNFunction.apply(yl, p["taps"], p["bias"], K, D, 0.5, "sigmoid", 4.0, 0, 7).backward(gs)
    l64 = {n: t.double().cpu().requires_grad_() for n, t in p.items()}
    x64 = x.double().requires_grad_()
    h, _, _ = ref.layer_norm(x64, l64["gamma"], l64["beta"], 1e-5, 2)
    yy = torch.matmul(h, l64["w"])
    qk, v, g, b = yy.split([2 * Hk * Dk, Hv * Dv, Hv, Hv], -1)
    qk = qk.unflatten(-1, (2, Hk, Dk))
    qk = qk / qk.norm(dim=-1, keepdim=True)
    o, S = ref.delta(qk[..., 0, :, :], qk[..., 1, :, :], v.unflatten(-1, (Hv, Dv)), -torch.log1p(torch.exp(g)),
                     torch.sigmoid(b), Dk ** -0.5)
    out, _, _ = ref.layer_norm(o, l64["gamma2"], l64["beta2"], 1e-5, 3)
    out.backward(yl.grad.double().cpu().view(out.shape))
    # f32: the products' bound, twice (norm over few values); bf16: the stored h, projections, o and y, the products'
    # six roundings, and the norm's division by a standard deviation that they move as well
    bound = 5e-4 if dtype == torch.float32 else 16 * 2.0 ** -8
    for n in ("gamma", "beta", "w", "gamma2", "beta2"):
        a, b = leaves[n].grad.double().cpu(), l64[n].grad
        assert (a - b).norm() <= bound * b.norm(), (n, ((a - b).norm() / b.norm()).item())
    a, b = xd.grad.double().cpu(), x64.grad
    assert (a - b).norm() <= bound * b.norm(), ("x", ((a - b).norm() / b.norm()).item())
    bound = 2e-4 if dtype == torch.float32 else 10 * 2.0 ** -8
    assert (state.double().cpu() - S).norm() <= bound * S.norm()


def test_step_by_step_is_the_whole_sequence():
    """Norms, delta rule and neuron one time step after another: the whole sequence's values up to rounding, and
    spikes wherever the potential is not within that of the threshold."""
    x, p = parameters(torch.float32)
    x = x.to(DEV)
    with torch.no_grad():
        spikes, y, state = block(x, p, torch.float32)
        h = mfpsn.layer_norm_forward(x, p["gamma"], p["beta"])
        ins = projected(h, p["w"], torch.float32)
        desc = mfpsn.make_delta_desc(ins[0].shape, ins[2].shape, "f32")
        memory = mfpsn.DeltaState(desc, device=DEV)
        ndesc = mfpsn.make_desc((T, N, Hv * Dv), K, D, "f32", "sigmoid", 4.0, 0.5, 0, 0, 7)
        sign, shift = mfpsn.quantize(p["taps"], 0, 7)
        neuron = mfpsn.StreamState(ndesc, (N, Hv * Dv), sign, shift, p["bias"])
        _, H = mfpsn.forward(ndesc, y.flatten(2).contiguous(), sign, shift, p["bias"], want_h=True)
        for t in range(T):
            ht = mfpsn.layer_norm_forward(x[t], p["gamma"], p["beta"], axis=1)
            assert torch.equal(ht, h[t])
            o = memory.step(*(z[t] for z in ins))
            yt = mfpsn.layer_norm_forward(o, p["gamma2"], p["beta2"], axis=2)
            assert (yt - y[t]).norm() <= 5e-4 * y[t].norm()
            st, ht = neuron.step(yt.flatten(1), want_h=True)
            clear = (H[t] - 0.5).abs() > 0.01
            assert torch.equal(st[clear].float(), spikes[t][clear])
        assert (memory.state - state).norm() <= 1e-4 * state.norm()
