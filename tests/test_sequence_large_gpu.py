"""Layer norm and the gated delta rule on tensors of more than 4 GiB: what lies behind a 32-bit offset has the bits that
it has in a call of its own."""
import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")
if not torch.cuda.is_available():
    pytest.skip("no GPU", allow_module_level=True)

from paper_2501_14490_amd import mfpsn  # noqa: E402  (loads libmfpsn.so or raises)

DEV = torch.device("cuda:0")


def normal(*shape):
    return torch.empty(shape, dtype=torch.bfloat16, device=DEV).normal_()


@pytest.fixture(autouse=True)
def room():
    """The tests hold up to 70 GB, and give them back."""
    torch.cuda.empty_cache()
    if torch.cuda.mem_get_info(DEV)[0] < 100 << 30:
        pytest.skip("less than 100 GiB of the GPU's memory are free")
    yield
    torch.cuda.empty_cache()


@pytest.mark.parametrize("M,C,S", [(9000001, 255, 1), (1100001, 2048, 1), (120001, 10001, 2), (70001, 48, 701)])
def test_layer_norm_behind_4_gib(M, C, S):
    x, gy, gamma, beta = normal(M, C, S), normal(M, C, S), torch.randn(C, device=DEV), torch.randn(C, device=DEV)
    assert x.numel() * 2 > 1 << 32
    y, mean, rstd = mfpsn.layer_norm_forward(x, gamma, beta, axis=1, want_stats=True)
    gx = mfpsn.layer_norm_backward(x, gamma, mean, rstd, gy, axis=1, want_weights=False)
    n = 64
    y1, mean1, rstd1 = mfpsn.layer_norm_forward(x[-n:].clone(), gamma, beta, axis=1, want_stats=True)
    gx1 = mfpsn.layer_norm_backward(x[-n:].clone(), gamma, mean1, rstd1, gy[-n:].clone(), axis=1, want_weights=False)
    torch.cuda.synchronize()
    assert torch.equal(mean[-n:], mean1) and torch.equal(rstd[-n:], rstd1)
    assert torch.equal(y[-n:], y1) and torch.equal(gx[-n:], gx1)


def test_delta_rule_behind_4_gib():
    """Two halves, the second from the first one's state and the first with the second one's gradient of it, give the
    bits of the whole: both cut the steps into the same chunks."""
    T, half, H, D = 132096, 66048, 128, 128  # (half: a multiple of the chunks' 64 steps)
    q, k, v, go = normal(T, 1, H, D), normal(T, 1, H, D).mul_(D ** -0.5), normal(T, 1, H, D), normal(T, 1, H, D)
    assert q.numel() * 2 > 1 << 32
    g, beta = -0.1 * normal(T, 1, H).abs(), normal(T, 1, H).sigmoid()
    ins = [q, k, v, g, beta]
    desc = mfpsn.make_delta_desc(q.shape, v.shape, "bf16")
    part = mfpsn.make_delta_desc((half, 1, H, D), (half, 1, H, D), "bf16")
    first, second = [t[:half] for t in ins], [t[half:] for t in ins]
    o, S, saved = mfpsn.delta_forward(desc, *ins, want_state=True, want_saved=True)
    grads = mfpsn.delta_backward(desc, *ins, saved, go)
    del saved
    o1, S1, saved1 = mfpsn.delta_forward(part, *first, want_state=True, want_saved=True)
    o2, S2, saved2 = mfpsn.delta_forward(part, *second, state=S1, want_state=True, want_saved=True)
    assert torch.isfinite(S).all() and torch.equal(S, S2)
    assert torch.equal(o[:half], o1) and torch.equal(o[half:], o2)
    *grads2, gs = mfpsn.delta_backward(part, *second, saved2, go[half:], want_grad_state=True)
    grads1 = mfpsn.delta_backward(part, *first, saved1, go[:half], grad_state=gs)
    for whole, a, b in zip(grads, grads1, grads2):
        assert torch.equal(whole[half:], b) and torch.equal(whole[:half], a)
