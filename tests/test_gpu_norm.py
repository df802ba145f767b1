"""RMS norms on the GPU against their definition in 64 bits.

Tolerance.  The mean of squares is a sum of L positive fp32 terms in a tree of at most L / 32 + 40 additions: relative error (L / 32 + 40) 2^-24,
half of that in its root; a handful of products and the sigmoid (as the convolution's) follow: rel = (L / 64 + 40) 2^-24 + 2^-17 of the sum of
the magnitudes.  Sums over rows: + (rows + 64) 2^-24."""
import pytest
import torch

from layer_refs import check, grads, leaf, norm
from paper_2605_08587_b200 import KLA_FLAG_GATE_FIRST, KLA_FLAG_NONE, KlaError, kla_norm_bwd, kla_norm_fwd

DEV = "cuda:0"
EPS = 1e-6
BF, F32 = torch.bfloat16, torch.float32


def _args(rows, D, mode, dtype, res=F32, seed=0, pad=0):
    g = torch.Generator().manual_seed(seed)
    new = lambda *s, dt=dtype: torch.randn(*s, generator=g).to(dt).to(DEV)  # noqa: E731
    x = new(rows, D + pad)[:, pad:]
    a = dict(residual=None, scale=None, gate=None)
    w = 1.0 + 0.2 * new(D, dt=F32)
    if mode == "add":
        a["residual"], a["scale"] = 2 * new(rows, D, dt=res), 0.5 + new(D, dt=F32).abs()
    if mode == "add1":
        a["residual"] = new(rows, D, dt=res)
    if mode.startswith("gate"):
        a["gate"] = new(rows, D + pad)[:, pad:]
    dy = new(rows, D)
    dr = new(rows, D, dt=res) if mode.startswith("add") else None
    return x, w, a, dy, dr


SHAPES = [(1, 8, 8), (5, 64, 64), (33, 128, 128), (7, 48, 48), (9, 1024, 1024), (12, 1000, 1000), (6, 2048, 128), (5, 2304, 128), (4, 1536, 512), (3, 8192, 8192),
          (3, 48, 16), (11, 96, 32), (2, 8200, 8200), (5, 63, 63), (4, 90, 30), (3, 4608, 4608), (700, 256, 256), (2, 16, 1), (300, 77, 77), (3, 9216, 4608)]


@pytest.mark.gpu
@pytest.mark.parametrize("mode", ["plain", "add", "add1", "gate", "gate_first"])
@pytest.mark.parametrize("dtype, res", [(BF, F32), (BF, BF), (F32, F32)])
@pytest.mark.parametrize("rows, D, group", SHAPES)
def test_forward_and_backward(rows, D, group, dtype, res, mode):
    if res == BF and not mode.startswith("add"):
        pytest.skip("no residual")
    pad = 8 if D % 8 == 0 and D < 4096 else 0
    x, w, a, dy, dr = _args(rows, D, mode, dtype, res, seed=D, pad=pad)
    flags = KLA_FLAG_GATE_FIRST if mode == "gate_first" else KLA_FLAG_NONE
    y, r = kla_norm_fwd(x, w, EPS, group=group, flags=flags, **a)
    g = kla_norm_bwd(x, w, EPS, dy, d_residual_out=dr, group=group, flags=flags, **a)
    torch.cuda.synchronize()
    names = ("x", "weight", "residual", "scale", "gate")
    leaves = [leaf(t) for t in (x, w, a["residual"], a["scale"], a["gate"])]
    how = dict(group=group, gate_first=mode == "gate_first")
    ry, ru = norm(leaves[0], leaves[1], EPS, *leaves[2:], **how)
    rel = (group / 64 + 40) * 2.0 ** -24 + 2.0 ** -17
    add = mode.startswith("add")
    # u may cancel in residual + scale x: the terms' size instead of the result's
    size_u = (leaves[0].abs() * (1 if leaves[3] is None else leaves[3]) + leaves[2].abs()) if add else ru.abs()
    rms = torch.sqrt((ru.unflatten(-1, (-1, group)) ** 2).mean(-1, keepdim=True) + EPS).expand(rows, D // group, group).flatten(-2)
    act = leaves[4].abs() if mode == "gate" else torch.ones_like(ru)
    size_y = (size_u + ru.abs()) / rms * leaves[1].abs() * act
    check(y, ry, size_y, rel, "out")
    if add:
        check(r, ru, size_u, 2.0 ** -23, "residual_out")
    else:
        assert r is None
    rg = dict(zip(names, grads((ry, ru), (dy, dr), leaves)))
    # sizes of the gradients' terms: r (|g| + |y| mean |g y|), with every factor at its magnitude
    lx, lw, lr, lsc, lz = (None if t is None else t.detach() for t in leaves)
    gy = dy.double().cpu().abs() * lw.abs() * (act.detach() + (0.3 if mode == "gate" else 0))
    yy = (size_u / rms).detach()
    mean = (gy * yy).unflatten(-1, (-1, group)).mean(-1, keepdim=True).expand(rows, D // group, group).flatten(-2)
    du = (gy + yy * mean) / rms.detach() + (0 if dr is None else dr.double().cpu().abs())
    sums = (rows + 64) * 2.0 ** -24
    sizes = {"weight": (gy / lw.abs() * yy).sum(0), "x": du}
    if add:
        sizes |= {"residual": du, "x": du * (1 if lsc is None else lsc)}
        if lsc is not None:
            sizes["scale"] = (du * lx.abs()).sum(0)
    if mode == "gate":
        sizes["gate"] = dy.double().cpu().abs() * lw.abs() * yy * 1.1 + 1e-30
    if mode == "gate_first":
        sizes |= {"gate": du * lx.abs() * 1.1, "x": du * (lz.abs() + 0.3)}
    for n in names:
        if rg[n] is None:
            assert g["d" + n] is None
        else:
            check(g["d" + n], rg[n], sizes[n], 4 * rel + (sums if n in ("weight", "scale") else 0), "d" + n)


@pytest.mark.gpu
@pytest.mark.parametrize("D", [512, 65])
def test_residual_in_place_and_outputs_given(D):
    x, w, a, *_ = _args(9, D, "add", BF, F32)
    y, r = kla_norm_fwd(x, w, EPS, **a)
    res, out = a["residual"].clone(), torch.full_like(x, float("nan"))
    y2, r2 = kla_norm_fwd(x, w, EPS, residual=res, scale=a["scale"], out=out, residual_out=res)
    assert y2.data_ptr() == out.data_ptr() and r2.data_ptr() == res.data_ptr()
    assert torch.equal(y, y2) and torch.equal(r, r2)


@pytest.mark.gpu
@pytest.mark.parametrize("D", [256, 2048, 33])
def test_rows_of_zeros_and_rows_that_are_not_finite(D):
    """A row of zeros normalises to zeros (eps > 0); a row that is not finite spoils no other, nor the other rows' gradients."""
    x, w, a, dy, _ = _args(6, D, "gate", BF)
    y, _ = kla_norm_fwd(x, w, EPS, **a)
    g = kla_norm_bwd(x, w, EPS, dy, **a)
    x2, dy2, gate = x.clone(), dy.clone(), a["gate"].clone()
    x2[2], x2[4], dy2[4], gate[2] = 0, float("nan"), float("inf"), float("-inf")
    gate[2] = 0
    y2, _ = kla_norm_fwd(x2, w, EPS, gate=gate)
    g2 = kla_norm_bwd(x2, w, EPS, dy2, gate=gate)
    keep = [0, 1, 3, 5]
    assert torch.equal(y2[keep], y[keep]) and torch.equal(g2["dx"][keep], g["dx"][keep]) and torch.equal(g2["dgate"][keep], g["dgate"][keep])
    assert (y2[2] == 0).all() and (g2["dgate"][2] == 0).all() and torch.isnan(y2[4]).all()
    assert torch.isnan(g2["dweight"]).all()


@pytest.mark.gpu
def test_no_rows():
    x = torch.empty(0, 64, device=DEV, dtype=BF)
    w = torch.ones(64, device=DEV)
    y, _ = kla_norm_fwd(x, w, EPS)
    g = kla_norm_bwd(x, w, EPS, x)
    assert y.shape == (0, 64) and g["dx"].shape == (0, 64) and (g["dweight"] == 0).all()


@pytest.mark.gpu
def test_sums_over_rows_do_not_vary():
    x, w, a, dy, dr = _args(5000, 512, "add", BF, F32)
    first = kla_norm_bwd(x, w, EPS, dy, d_residual_out=dr, **a)
    for _ in range(3):
        again = kla_norm_bwd(x, w, EPS, dy, d_residual_out=dr, **a)
        assert all(torch.equal(first[n], again[n]) for n in ("dx", "dweight", "dresidual", "dscale"))


@pytest.mark.gpu
@pytest.mark.parametrize("group, error", [(-1, ValueError), (1 << 40, ValueError), (0, KlaError), (7, KlaError)])
def test_groups_that_are_refused(group, error):
    x, w = torch.ones(4, 64, dtype=BF, device=DEV), torch.ones(64, device=DEV)
    with pytest.raises(error):
        kla_norm_fwd(x, w, 1e-6, group=group)
    with pytest.raises(error):
        kla_norm_bwd(x, w, 1e-6, x, group=group)
