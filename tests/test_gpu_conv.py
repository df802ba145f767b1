"""Short causal convolution on the GPU against its definition in 64 bits.

Tolerance.  A value p is a sum of at most 5 fp32 terms: (W + 1) 2^-24 of the sum of their magnitudes.  sigmoid costs an exponential (argument
rounded: |p| 2^-23, the instruction 2^-22), a sum, a quotient (2^-22): (4 + |p|) 2^-22 of the value, and p's own error is multiplied by
|act'| <= 1.1.  The tests' |p| stay below 16, so 32 x 2^-22 = 2^-17 covers it all; a weight's gradient is a sum over the rows, in
runs of at most (rows / 8 + partials) additions: + (rows + 64) 2^-24."""
import pytest
import torch

from layer_refs import check, conv, grads, leaf
from paper_2605_08587_b200 import KLA_FLAG_CONV_LINEAR, KLA_FLAG_NONE, kla_conv_bwd, kla_conv_fwd, kla_conv_step

DEV = "cuda:0"
REL = 2.0 ** -17


def _case(lens, C, W, dtype, bias=True, state=True, seed=0, wide=0):
    """x as a slice of an array `wide` channels wider."""
    g = torch.Generator().manual_seed(seed)
    rows = sum(lens)
    x = torch.randn(1, rows, C + wide, generator=g).to(dtype).to(DEV)[..., wide:]
    w = ((2 * torch.rand(C, W, generator=g) - 1) / W ** 0.5).to(DEV)
    b = 0.1 * torch.randn(C, generator=g).to(DEV) if bias else None
    s = torch.randn(len(lens), W - 1, C, generator=g).to(dtype).to(DEV) if state else None
    dy = torch.randn(1, rows, C, generator=g).to(dtype).to(DEV)
    ds = torch.randn(len(lens), W - 1, C, generator=g).to(dtype).to(DEV) if state else None
    host = torch.tensor([0] + list(torch.tensor(lens).cumsum(0)), dtype=torch.int32)
    return x, w, b, s, dy, ds, dict(cu_seqlens=host.to(DEV), host_seqlens=host)


CASES = [([1], 8, 4, torch.bfloat16, 0), ([2, 1, 3], 64, 4, torch.bfloat16, 0), ([37, 0, 5, 64, 1], 264, 4, torch.bfloat16, 8), ([300], 96, 3, torch.bfloat16, 0),
         ([130, 70], 7, 4, torch.bfloat16, 5), ([9, 100], 40, 2, torch.float32, 4), ([65, 0, 2], 13, 3, torch.float32, 0), ([0, 0], 16, 4, torch.bfloat16, 0),
         ([1200, 333], 2304, 4, torch.bfloat16, 0)]


@pytest.mark.gpu
@pytest.mark.parametrize("flags", [KLA_FLAG_NONE, KLA_FLAG_CONV_LINEAR])
@pytest.mark.parametrize("state", [False, True])
@pytest.mark.parametrize("lens, C, W, dtype, wide", CASES)
def test_forward_and_backward(lens, C, W, dtype, wide, state, flags):
    if sum(lens) > 1000 and (flags or not state):
        pytest.skip("the long case once")
    wide = wide if dtype == torch.float32 or wide % 8 == 0 or C % 2 else 0
    if wide % (8 if dtype == torch.bfloat16 else 4):   # the first element has to lie on a 16-byte boundary
        x, w, b, s, dy, ds, seqs = _case(lens, C, W, dtype, state=state, wide=0, seed=C)
    else:
        x, w, b, s, dy, ds, seqs = _case(lens, C, W, dtype, state=state, wide=wide, seed=C)
    y, fin = kla_conv_fwd(x, w, bias=b, init_state=s, flags=flags, **seqs)
    g = kla_conv_bwd(x, w, dy, bias=b, init_state=s, d_final_state=ds, flags=flags, **seqs)
    torch.cuda.synchronize()
    zero = torch.zeros(len(lens), W - 1, C, dtype=torch.float64)
    lx, lw, lb, ls = leaf(x[0]), leaf(w), leaf(b), leaf(s if state else zero)
    ry, rf = conv(lx, lw, lb, ls, lens, linear=bool(flags))
    # magnitudes of the terms: the linear form on absolute values (|silu(p)| <= |p|, |silu'| <= 1.1)
    ax, aw, ab, as_ = (t.detach().abs().requires_grad_() for t in (lx, lw, lb, ls))
    my, mf = conv(ax, aw, ab, as_, lens, linear=True)
    check(y[0], ry, my, REL, "out")
    assert torch.equal(fin.double().cpu(), rf.detach())
    rg = grads((ry, rf), (dy[0], ds), (lx, lw, lb, ls))
    mg = grads((my, mf), (dy[0].abs(), None if ds is None else ds.abs()), (ax, aw, ab, as_))
    sums = REL + (sum(lens) + 64) * 2.0 ** -24
    for name, r, m, rel in zip(("dx", "dweight", "dbias", "dinit_state"), rg, mg, (2 * REL, 2 * REL + sums, 2 * REL + sums, 2 * REL)):
        check(g[name][0] if name == "dx" else g[name], r, 1.1 * m, rel, name)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_fixed_length_batch_is_the_same_as_packed(dtype):
    B, T, C = 3, 29, 48
    x, w, b, s, dy, ds, seqs = _case([T] * B, C, 4, dtype)
    y, fin = kla_conv_fwd(x, w, bias=b, init_state=s, **seqs)
    y2, fin2 = kla_conv_fwd(x.reshape(B, T, C), w, bias=b, init_state=s)
    assert torch.equal(y.reshape(B, T, C), y2) and torch.equal(fin, fin2)
    g = kla_conv_bwd(x, w, dy, bias=b, init_state=s, d_final_state=ds, **seqs)
    g2 = kla_conv_bwd(x.reshape(B, T, C), w, dy.reshape(B, T, C), bias=b, init_state=s, d_final_state=ds)
    for n in g:
        assert torch.equal(g[n].flatten(), g2[n].flatten()), n


@pytest.mark.gpu
@pytest.mark.parametrize("C, dtype", [(64, torch.bfloat16), (9, torch.bfloat16), (20, torch.float32)])
@pytest.mark.parametrize("W", [2, 3, 4])
def test_steps_are_the_forward(C, dtype, W):
    """The same sums in the same order: bit for bit."""
    T, B = 7, 5
    x, w, b, s, *_ = _case([T] * B, C, W, dtype, seed=W)
    x = x.reshape(B, T, C)
    y, fin = kla_conv_fwd(x, w, bias=b, init_state=s)
    state = s.clone()
    for t in range(T):
        assert torch.equal(kla_conv_step(x[:, t].contiguous(), w, state, bias=b), y[:, t])
    assert torch.equal(state, fin)
    state = s.clone()
    if C % 8 == 0:   # a slice of [B, T, C]: rows T C apart
        assert torch.equal(kla_conv_step(x[:, 0], w, state, bias=b), y[:, 0])


@pytest.mark.gpu
def test_neighbours_that_are_not_finite_stay_apart():
    lens = [5, 40, 3, 70]
    x, w, b, s, dy, ds, seqs = _case(lens, 64, 4, torch.bfloat16)
    good = [kla_conv_fwd(x, w, bias=b, init_state=s, **seqs), kla_conv_bwd(x, w, dy, bias=b, init_state=s, d_final_state=ds, **seqs)]
    x2, s2, dy2, ds2 = x.clone(), s.clone(), dy.clone(), ds.clone()
    for lo, hi in ((0, 5), (45, 48)):   # sequences 0 and 2
        x2[0, lo:hi] = float("nan")
        dy2[0, lo:hi] = float("inf")
    for n in (0, 2):
        s2[n] = float("nan")
        ds2[n] = float("nan")
    y, fin = kla_conv_fwd(x2, w, bias=b, init_state=s2, **seqs)
    g = kla_conv_bwd(x2, w, dy2, bias=b, init_state=s2, d_final_state=ds2, **seqs)
    for lo, hi in ((5, 45), (48, 118)):
        assert torch.equal(y[0, lo:hi], good[0][0][0, lo:hi]) and torch.equal(g["dx"][0, lo:hi], good[1]["dx"][0, lo:hi])
    for n in (1, 3):
        assert torch.equal(fin[n], good[0][1][n]) and torch.equal(g["dinit_state"][n], good[1]["dinit_state"][n])


@pytest.mark.gpu
def test_gradient_against_differences():
    """Central differences of the kernel's own forward in fp32, h = 2^-6: its error h^2 |f'''| / 6 + 2^-24 |f| / h, f of size 10."""
    lens = [6, 2, 9]
    x, w, b, s, dy, ds, seqs = _case(lens, 12, 4, torch.float32, seed=5)
    g = kla_conv_bwd(x, w, dy, bias=b, init_state=s, d_final_state=ds, **seqs)

    def loss(x, w, b, s):
        y, f = kla_conv_fwd(x, w, bias=b, init_state=s, **seqs)
        return float((y.double() * dy).sum() + (f.double() * ds).sum())
    args, h = [x, w, b, s], 2.0 ** -6
    gen = torch.Generator().manual_seed(1)
    for i, name in enumerate(("dx", "dweight", "dbias", "dinit_state")):
        u = torch.randn(args[i].shape, generator=gen).to(DEV)
        u /= u.norm()
        up, down = list(args), list(args)
        up[i], down[i] = (args[i] + h * u).contiguous(), (args[i] - h * u).contiguous()
        diff = (loss(*up) - loss(*down)) / (2 * h)
        assert abs(diff - float((g[name] * u).sum())) <= 2e-3 * max(1.0, float(g[name].norm())), name


@pytest.mark.gpu
@pytest.mark.parametrize("C, dtype", [(64, torch.bfloat16), (9, torch.bfloat16), (20, torch.float32)])
@pytest.mark.parametrize("lens", [[300], [40, 0, 1, 2, 90], [0, 0], [1]])
def test_states_in_place(lens, C, dtype):
    """final_state may be init_state: the same bits as apart.  The output may not be the input."""
    x, w, b, s, _, _, seqs = _case(lens, C, 4, dtype)
    y, fin = kla_conv_fwd(x, w, bias=b, init_state=s, **seqs)
    state = s.clone()
    y2, fin2 = kla_conv_fwd(x, w, bias=b, init_state=state, final_state=state, **seqs)
    assert fin2.data_ptr() == state.data_ptr() and torch.equal(y, y2) and torch.equal(state, fin)
    if sum(lens):
        with pytest.raises(ValueError, match="out"):
            kla_conv_fwd(x, w, bias=b, out=x, **seqs)
