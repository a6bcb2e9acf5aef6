"""Layer norm over the channels against its definition in 64 bits, on the GPU through the C ABI.

Bounds, per element, with e = 2^-24 (a float rounding) and n the additions that one float sum chains (a lane's own
elements, at most max(32, C/16), then at most 10 joins of lanes and waves):
  mean        off by at most n e mean|x| + e |mean|
  xh          off by rstd times that, and (n/2 + 6) e relative (the variance's sum enters by its square root)
  y           gamma xh + beta: two roundings more, and the storage type's half step
  grad_x      r (a - mean a - xh mean(a xh)): the errors of its three terms, each sum n + 4 roundings
  weights     sums of M S terms, chained at most M S / 1024 + 80 long (at the sizes below)
"""
import numpy as np
import pytest

import sequence_reference as ref

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")
if not torch.cuda.is_available():
    pytest.skip("no GPU", allow_module_level=True)

from paper_2501_14490_amd import mfpsn  # noqa: E402  (loads libmfpsn.so or raises)

DEV = torch.device("cuda:0")
E = 2.0 ** -24
HALF = {torch.float32: 2.0 ** -24, torch.bfloat16: 2.0 ** -8}
DT = {"f32": torch.float32, "bf16": torch.bfloat16}


def make(M, C, S, dtype, seed, mean=0.5, affine=True):
    gen = torch.Generator().manual_seed(seed)
    x = (mean + torch.randn(M, C, S, generator=gen)).to(DT[dtype])
    gy = torch.randn(M, C, S, generator=gen).to(DT[dtype])
    gamma, beta = (1 + 0.3 * torch.randn(C, generator=gen), torch.randn(C, generator=gen)) if affine else (None, None)
    return x, gy, gamma, beta


def check(M, C, S, dtype, seed=0, mean=0.5, affine=True, eps=1e-5, place=lambda t: t.to(DEV)):
    x, gy, gamma, beta = make(M, C, S, dtype, seed, mean, affine)
    args = [place(x)] + [t.to(DEV) if t is not None else None for t in (gamma, beta)]
    y, mu, rstd = mfpsn.layer_norm_forward(*args, eps, axis=1, want_stats=True)
    gx, gg, gb = mfpsn.layer_norm_backward(args[0], args[1], mu, rstd, place(gy), axis=1)
    torch.cuda.synchronize()
    x64, g64 = x.double(), gy.double()
    gam = gamma.double().view(1, -1, 1) if affine else torch.ones(1, C, 1, dtype=torch.float64)
    bet = beta.double().view(1, -1, 1) if affine else torch.zeros(1, C, 1, dtype=torch.float64)
    leaf = x64.clone().requires_grad_()
    gl, bl = (t.flatten().clone().requires_grad_() for t in (gam, bet))
    want, m64, r64 = ref.layer_norm(leaf, gl, bl, eps, 1)
    wx, wg, wb = torch.autograd.grad((want * g64).sum(), (leaf, gl, bl))
    want, m64, r64 = want.detach(), m64.detach(), r64.detach()
    half = HALF[DT[dtype]]
    n = max(32, C // 16) + 10
    n2 = M * S // 1024 + 80
    xh = (x64 - m64) * r64
    e_mean = n * E * x64.abs().mean(1, keepdim=True) + E * m64.abs()
    e_xh = r64 * e_mean + xh.abs() * (n / 2 + 6) * E

    def near(got, expect, bound, what):
        off = (got.double().cpu().reshape(expect.shape) - expect).abs() - bound
        assert torch.isfinite(got).all(), what
        assert (off <= 0).all(), f"{what}: {off.max().item():.3g} over its bound"

    near(mu, m64, e_mean, "mean")
    near(rstd, r64, r64 * (n / 2 + 4) * E, "rstd")
    near(y, want, gam.abs() * e_xh + 3 * E * (want.abs() + bet.abs()) + half * want.abs() + 1e-30, "y")
    a = g64 * gam
    ma, mh = a.mean(1, keepdim=True), (a * xh).mean(1, keepdim=True)
    e_mh = (n + 4) * E * (a * xh).abs().mean(1, keepdim=True) + (a.abs() * e_xh).mean(1, keepdim=True)
    e_gx = r64 * (2 * E * a.abs() + (n + 4) * E * a.abs().mean(1, keepdim=True) + xh.abs() * e_mh + e_xh * mh.abs()
                  + 3 * E * (a.abs() + ma.abs() + (xh * mh).abs())) + wx.abs() * ((n / 2 + 6) * E + half)
    near(gx, wx, e_gx * 1.01 + 1e-30, "grad_x")
    near(gg, wg, (g64.abs() * e_xh).sum((0, 2)) + n2 * E * (g64 * xh).abs().sum((0, 2)) + 1e-30, "grad_gamma")
    near(gb, wb, n2 * E * g64.abs().sum((0, 2)) + 1e-30, "grad_beta")
    return y, gx, gg, gb


# channels contiguous: a wave, four waves and more than a block a row; odd widths; one row, one channel
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("M,C", [(1, 1), (3, 2), (5, 7), (9, 64), (33, 100), (7, 256), (130, 257), (17, 512), (4, 1001),
                                 (70, 1024), (6, 2047), (5, 2048), (3, 4100), (2, 8192), (3, 9001), (2, 20000)])
def test_rows(M, C, dtype):
    check(M, C, 1, dtype, seed=M * 31 + C)


# planes: columns that fill no tile, widths of vectors and odd ones, channels beyond the registers
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("M,C,S", [(1, 1, 2), (2, 3, 5), (4, 64, 36), (3, 65, 49), (1, 256, 100), (2, 257, 7), (2, 1000, 12),
                                   (1, 1024, 33), (1, 1025, 8), (1, 2500, 3), (130, 5, 2), (600, 16, 4)])
def test_planes(M, C, S, dtype):
    check(M, C, S, dtype, seed=M + C + S)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_many_rows_for_each_block(dtype):
    check(20000, 24, 1, dtype)  # more rows than the blocks of the backward take at once
    check(3, 8, 40000, dtype)
    check(40, 8, 7001, dtype)
    check(3, 20, 100000, dtype)


@pytest.mark.parametrize("S", [1, 6])
def test_without_weights_and_with_a_large_mean(S):
    check(11, 96, S, "f32", affine=False)
    check(11, 96, S, "f32", mean=3000.0)  # the variance is no difference of large sums


@pytest.mark.parametrize("C,S", [(64, 1), (64, 8)])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_tensors_that_start_at_no_vector(C, S, dtype):
    def place(t):
        buf = torch.empty(t.numel() + 1, dtype=t.dtype, device=DEV)
        out = buf[1:].view(t.shape)
        out.copy_(t)
        return out

    check(5, C, S, dtype, place=place)


@pytest.mark.parametrize("S", [1, 4])
def test_constant_rows_and_zero_eps_free_rows(S):
    """Rows of equal values: y = beta; their gradient is finite with eps > 0."""
    x = torch.full((3, 64, S), 2.5, device=DEV)
    gamma, beta = torch.ones(64, device=DEV), torch.arange(64.0, device=DEV)
    y, mean, rstd = mfpsn.layer_norm_forward(x, gamma, beta, 1e-5, axis=1, want_stats=True)
    assert torch.equal(y, beta.view(1, 64, 1).expand(3, 64, S))
    gx, _, _ = mfpsn.layer_norm_backward(x, gamma, mean, rstd, torch.randn_like(x), axis=1)
    assert torch.isfinite(gx).all()


@pytest.mark.parametrize("S", [1, 3])
def test_a_row_that_is_not_finite_spoils_no_other(S):
    x, gy, gamma, beta = make(6, 130, S, "f32", 3)
    good = mfpsn.layer_norm_forward(x.to(DEV), gamma.to(DEV), beta.to(DEV), axis=1)
    x[2, 5, 0] = float("nan")
    x[4, 0, 0] = float("inf")
    got = mfpsn.layer_norm_forward(x.to(DEV), gamma.to(DEV), beta.to(DEV), axis=1)
    bad = torch.zeros(6, S, dtype=torch.bool)
    bad[2, 0] = bad[4, 0] = True
    keep = ~bad[:, None, :].expand(6, 130, S).to(DEV)
    assert torch.equal(got[keep], good[keep])
    assert torch.isnan(got[2, :, 0]).all() and torch.isnan(got[4, 0, 0])


# rows of every part of a wave, whole and not, one more and one fewer than fill the blocks' parts
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("M,C", [(1, 8), (31, 24), (33, 32), (1025, 56), (65, 72), (15, 120), (17, 128), (255, 136), (7, 248), (9, 16),
                                 (2049, 9), (40000, 17), (3, 33)])
def test_short_rows(M, C, dtype):
    check(M, C, 1, dtype, seed=M + C)


def test_no_rows_of_many_channels():
    C = 30000  # (more than a block's registers hold)
    x, gamma = torch.empty((0, C), device=DEV), torch.ones(C, device=DEV)
    y, mean, rstd = mfpsn.layer_norm_forward(x, gamma, gamma, axis=1, want_stats=True)
    gx, gg, gb = mfpsn.layer_norm_backward(x, gamma, mean, rstd, y, axis=1)
    assert gx.shape == x.shape and not gg.any() and not gb.any() and gg.shape == gb.shape == (C,)


def test_empty_tensors_and_missing_weights():
    for shape in ((0, 5, 3), (4, 0, 3), (4, 5, 0)):
        x = torch.empty(shape, device=DEV)
        y, mean, rstd = mfpsn.layer_norm_forward(x, None, None, axis=1, want_stats=True)
        gx, gg, gb = mfpsn.layer_norm_backward(x, None, mean, rstd, x, axis=1)
        assert y.shape == gx.shape == x.shape
        assert not gg.any() and not gb.any() and gg.numel() == shape[1]


def test_axis_is_the_layout():
    """[T, N, C, S] by channels 2, [N, C, S, T] by channels 1: the same values."""
    x, _, gamma, beta = make(6, 20, 4, "f32", 5)
    x = x.view(2, 3, 20, 4).to(DEV)
    first = mfpsn.layer_norm_forward(x, gamma.to(DEV), beta.to(DEV), axis=2)
    last = mfpsn.layer_norm_forward(x.permute(1, 2, 3, 0).contiguous(), gamma.to(DEV), beta.to(DEV), axis=1)
    assert torch.allclose(last.permute(3, 0, 1, 2), first, rtol=0, atol=64 * E * first.abs().max().item())


def test_same_bits_on_repeats_another_stream_and_graph_replays():
    x, gy, gamma, beta = (t.to(DEV) for t in make(700, 192, 1, "bf16", 8))

    def run(stream=None):
        y, mean, rstd = mfpsn.layer_norm_forward(x, gamma, beta, axis=1, want_stats=True, stream=stream)
        return (y, *mfpsn.layer_norm_backward(x, gamma, mean, rstd, gy, axis=1, stream=stream))

    want = run()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        again = run()
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(want, again))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = run()
    for _ in range(3):
        for t in got:
            t.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(want, got))
        (x * 2).sum().item()


@pytest.mark.parametrize("axis", [1, 2])
def test_autograd(axis):
    x, gy, gamma, beta = make(12, 10, 6, "f32", 4)
    shape = (2, 6, 10, 6) if axis == 2 else (12, 10, 6)
    leaves = [t.to(DEV).requires_grad_() for t in (x.view(shape), gamma, beta)]
    y = mfpsn.LayerNormFunction.apply(*leaves, 1e-5, axis)
    y.backward(gy.view(shape).to(DEV))
    l64 = [t.double().requires_grad_() for t in (x.view(shape), gamma, beta)]
    want, _, _ = ref.layer_norm(*l64, 1e-5, axis)
    want.backward(gy.view(shape).double())
    for a, b in zip(leaves, l64):
        assert torch.allclose(a.grad.double().cpu(), b.grad, rtol=0, atol=2000 * E * b.grad.abs().max().item())
    # against differences of the kernel's own forward
    gen = torch.Generator().manual_seed(1)
    d = torch.randn(shape, generator=gen).to(DEV)
    h = 1e-2
    with torch.no_grad():
        f = [(mfpsn.LayerNormFunction.apply(leaves[0] + s * h * d, leaves[1], leaves[2], 1e-5, axis).double()
              * gy.view(shape).to(DEV)).sum().item() for s in (1, -1)]
    slope, along = (f[0] - f[1]) / (2 * h), (leaves[0].grad.double() * d).sum().item()
    # third derivatives times h^2/6, and the roundings of y (2^-24 of sum |gy y|) over h
    assert abs(slope - along) <= 1e-2 * leaves[0].grad.double().norm().item() * d.double().norm().item() ** 0.5 + 1e-2


def test_refusals():
    x = torch.zeros(2, 8, 1, device=DEV)
    w = torch.ones(8, device=DEV)
    st = torch.zeros(2, 1, device=DEV)
    for call, err in [
        (lambda: mfpsn.layer_norm_forward(x.double(), None, None, axis=1), TypeError),
        (lambda: mfpsn.layer_norm_forward(x.half(), None, None, axis=1), TypeError),
        (lambda: mfpsn.layer_norm_forward(x, w[:4], None, axis=1), ValueError),
        (lambda: mfpsn.layer_norm_forward(x, w.cpu(), None, axis=1), ValueError),
        (lambda: mfpsn.layer_norm_forward(x, w.bfloat16(), None, axis=1), TypeError),
        (lambda: mfpsn.layer_norm_forward(x.transpose(0, 1), None, None, axis=1), ValueError),
        (lambda: mfpsn.layer_norm_forward(x, None, None, axis=3), ValueError),
        (lambda: mfpsn.layer_norm_forward(x.cpu(), None, None, axis=1), ValueError),
        (lambda: mfpsn.layer_norm_backward(x, w, st[:1], st, x, axis=1), ValueError),
        (lambda: mfpsn.layer_norm_backward(x, w, st, st, x[:1], axis=1), ValueError),
        (lambda: mfpsn.layer_norm_backward(x, w, st, st, x.bfloat16(), axis=1), TypeError),
    ]:
        with pytest.raises(err):
            call()
    for eps in (-1.0, float("nan"), float("inf")):
        with pytest.raises(mfpsn.MfpsnError):
            mfpsn.layer_norm_forward(x, None, None, eps, axis=1)
    assert np.isfinite(mfpsn.mfpsn_layer_norm_workspace_size(4, 5, 6))
