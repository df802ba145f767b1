"""The operators around a mixer in 64 bits, token by token from their definitions (CPU, torch.float64, differentiable)."""
import torch


def silu(x):
    return x * torch.sigmoid(x)


def bounds_of(lens):
    out = [0]
    for n in lens:
        out.append(out[-1] + n)
    return out


def conv(x, weight, bias, init, lens, linear=False):
    """x [rows, C]; init [n_seq, W - 1, C] -> y [rows, C], final [n_seq, W - 1, C]."""
    W = weight.shape[1]
    at, ys, finals = bounds_of(lens), [], []
    for n in range(len(lens)):
        window = [init[n, i] for i in range(W - 1)]
        for t in range(at[n], at[n + 1]):
            window.append(x[t])
            p = sum(weight[:, i] * window[len(window) - W + i] for i in range(W))
            if bias is not None:
                p = p + bias
            ys.append(p if linear else silu(p))
        finals.append(torch.stack(window[len(window) - (W - 1):]))
    return (torch.stack(ys) if ys else x * 0), torch.stack(finals)


def scan(q, k, v, dt, la, skip, init, lens):
    """q, k [rows, G, N]; v [rows, H, P]; dt, la [rows, H] (la: log decay, dt a); init [n_seq, H, N, P]."""
    per = v.shape[1] // q.shape[1]
    at, ys, finals = bounds_of(lens), [], []
    for n in range(len(lens)):
        s = init[n]
        for t in range(at[n], at[n + 1]):
            kt, qt = k[t].repeat_interleave(per, 0), q[t].repeat_interleave(per, 0)
            s = torch.exp(la[t])[:, None, None] * s + (dt[t][:, None] * kt)[:, :, None] * v[t][:, None, :]
            y = (qt[:, :, None] * s).sum(1)
            ys.append(y if skip is None else y + skip[:, None] * v[t])
        finals.append(s)
    return (torch.stack(ys) if ys else v * 0), torch.stack(finals)


def norm(x, weight, eps, residual=None, scale=None, gate=None, group=None, gate_first=False):
    """-> y, u (u: what is normed, the new residual)."""
    if residual is not None:
        x = residual + (x if scale is None else scale * x)
    u = x * silu(gate) if gate is not None and gate_first else x
    g = u.unflatten(-1, (-1, group or u.shape[-1]))
    y = (g / torch.sqrt((g * g).mean(-1, keepdim=True) + eps)).flatten(-2) * weight
    if gate is not None and not gate_first:
        y = y * silu(gate)
    return y, u


def leaf(t):
    """A float64 CPU leaf with the values of t (None for None)."""
    return None if t is None else t.detach().double().cpu().requires_grad_()


def grads(outs, d_outs, leaves):
    """Gradients of sum <out, d_out> by each leaf (None for None, zeros for one that no output depends on)."""
    loss = sum((o * d.detach().double().cpu()).sum() for o, d in zip(outs, d_outs) if d is not None)
    got = torch.autograd.grad(loss, [x for x in leaves if x is not None], allow_unused=True)
    got = iter(got)
    return [None if x is None else (lambda g: torch.zeros_like(x) if g is None else g)(next(got)) for x in leaves]


def half_step(t):
    """Largest relative error of one rounding to the dtype of t; 0 for what is stored as it is."""
    return torch.finfo(t.dtype).eps / 2


def check(got, ref, size, rel, what, rounded=True):
    """|got - ref| <= rel x size + half a step of got's dtype at ref.  `size`: sum of the magnitudes of the terms that make up each value,
    `rel`: the relative error of one such term and its place in a sum, both in the arithmetic that the kernel uses."""
    ref, size = ref.detach(), size.detach()
    g = got.detach().double().cpu().reshape(ref.shape)
    bound = rel * size.abs() + (half_step(got) * (ref.abs() + rel * size.abs()) if rounded else 0) + 1e-37
    off = (g - ref).abs()
    bad = ~(off <= bound)
    assert not bad.any(), "%s: %d of %d beyond the bound, worst %.3g of it" % (what, bad.sum(), bad.numel(), (off / bound).max())
