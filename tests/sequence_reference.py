"""Layer norm and the gated delta rule from their definitions, in 64 bits on the CPU.

One time step after another, elementary operations only; gradients by torch.autograd of these."""
import torch


def layer_norm(x, gamma, beta, eps, axis):
    """y and the statistics of a float64 x."""
    mean = x.sum(axis, keepdim=True) / x.shape[axis]
    dev = x - mean
    rstd = ((dev * dev).sum(axis, keepdim=True) / x.shape[axis] + eps) ** -0.5
    shape = [1] * x.dim()
    shape[axis] = -1
    y = dev * rstd
    if gamma is not None:
        y = y * gamma.reshape(shape)
    if beta is not None:
        y = y + beta.reshape(shape)
    return y, mean, rstd


def delta(q, k, v, g, beta, scale, state=None, lengths=None):
    """o [T, N, Hv, Dv] and the last state of float64 inputs; steps behind a sequence's length give zeros."""
    T, N, Hv, Dv = v.shape
    group = Hv // q.shape[2]
    q, k = q.repeat_interleave(group, 2), k.repeat_interleave(group, 2)
    S = state if state is not None else torch.zeros(N, Hv, q.shape[3], Dv, dtype=torch.float64)
    out = []
    for t in range(T):
        live = torch.ones(N, dtype=torch.bool) if lengths is None else lengths > t

        def used(x, fill=0.0):  # (a step that is not read may hold anything)
            return torch.where(live.reshape(N, *[1] * (x.dim() - 1)), x, torch.full_like(x, fill))

        kt, qt, vt, gt, bt = used(k[t]), used(q[t]), used(v[t]), used(g[t]), used(beta[t])
        kept = torch.exp(gt)[..., None, None] * S
        res = vt - (kt[..., :, None] * kept).sum(-2)
        S = kept + kt[..., :, None] * (bt[..., None] * res)[..., None, :]
        out.append(scale * (qt[..., :, None] * S).sum(-2))
    o = torch.stack(out) if out else torch.zeros(0, N, Hv, Dv, dtype=torch.float64)
    return o, S


def delta_grads(q, k, v, g, beta, scale, grad_o, state=None, lengths=None, grad_state=None):
    """o, state and the gradients of q, k, v, g, beta (and the state)."""
    leaves = [x.clone().requires_grad_() for x in (q, k, v, g, beta)]
    if state is not None:
        leaves.append(state.clone().requires_grad_())
    o, S = delta(*leaves[:5], scale, leaves[5] if state is not None else None, lengths)
    total = (o * grad_o).sum() + (0 if grad_state is None else (S * grad_state).sum())
    return o.detach(), S.detach(), torch.autograd.grad(total, leaves, allow_unused=True)
