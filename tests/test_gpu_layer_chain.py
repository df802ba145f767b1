"""The operators around a mixer one after another, as a layer uses them: norm of the residual stream, convolution, scan (or the delta rule), gated norm."""
import pytest
import torch

import paper_2605_08587_b200 as kla
from layer_refs import conv, leaf, norm, scan
from paper_2605_08587_b200 import workloads as W

DEV, EPS = "cuda:0", 1e-6
H, G, N, P = 4, 1, 64, 64
C = H * P + 2 * G * N
BF, F32 = torch.bfloat16, torch.float32


def _layer(dtype, lens, seed=0):
    g = torch.Generator().manual_seed(seed)
    rows = sum(lens)
    r = lambda *s: torch.randn(*s, generator=g)  # noqa: E731
    p = dict(w_norm=1 + 0.1 * r(C), conv_w=0.5 * r(C, 4), conv_b=0.1 * r(C), a=-(1 + 7 * torch.rand(H, generator=g)), skip=1 + 0.1 * r(H),
             w_out=1 + 0.1 * r(H * P))
    p = {n: t.to(DEV) for n, t in p.items()}
    host = torch.tensor([0] + list(torch.tensor(lens).cumsum(0)), dtype=torch.int32)
    x = dict(x=r(1, rows, C).to(dtype).to(DEV), res=2 * r(1, rows, C).to(DEV), z=r(1, rows, H * P).to(dtype).to(DEV),
             dt=torch.exp(-5 + 2 * torch.rand(1, rows, H, generator=g)).to(DEV))
    return p, x, dict(cu_seqlens=host.to(DEV), host_seqlens=host)


def _split(u):
    return u[..., :H * P].unflatten(-1, (H, P)), u[..., H * P:H * P + G * N].unflatten(-1, (G, N)), u[..., H * P + G * N:].unflatten(-1, (G, N))


def _forward(p, x, seqs, conv_state=None, state=None):
    u, res = kla.kla_norm_fwd(x["x"], p["w_norm"], EPS, residual=x["res"])
    c, conv_fin = kla.kla_conv_fwd(u, p["conv_w"], bias=p["conv_b"], init_state=conv_state, **seqs)
    v, k, q = _split(c)   # views: rows C apart
    o, fin = kla.kla_ssm_fwd(q, k, v, x["dt"], p["a"], d_skip=p["skip"], init_state=state, **seqs)
    y, _ = kla.kla_norm_fwd(o.flatten(-2), p["w_out"], EPS, gate=x["z"], group=P)
    return dict(y=y, res=res, u=u, c=c, o=o, conv_fin=conv_fin, fin=fin)


def _reference(p, x, lens):
    lp, lx = {n: leaf(t) for n, t in p.items()}, {n: leaf(t[0]) for n, t in x.items()}
    n = len(lens)
    u, res = norm(lx["x"], lp["w_norm"], EPS, residual=lx["res"])
    c, _ = conv(u, lp["conv_w"], lp["conv_b"], torch.zeros(n, 3, C, dtype=torch.float64), lens)
    v, k, q = _split(c)
    o, fin = scan(q, k, v, lx["dt"], lx["dt"] * lp["a"], lp["skip"], torch.zeros(n, H, N, P, dtype=torch.float64), lens)
    y, _ = norm(o.flatten(-2), lp["w_out"], EPS, gate=lx["z"], group=P)
    return lp, lx, y, res, fin


def _off(got, ref):
    got, ref = got.detach().double().cpu().reshape(ref.shape), ref.detach()
    return float((got - ref).norm() / ref.norm())


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [F32, BF])
def test_forward_and_gradients_of_a_layer(dtype):
    """2-norm errors.  fp32: sums of a few hundred terms, 1e-5.  bf16: five roundings of intermediate results lie one behind the other (u, c, P and S, o, y), each
    2^-8 / sqrt(3) of its value in the 2-norm and at most doubled on its way (every operator's gain is of size 1): 5 x 2 x 2^-8 / sqrt(3) = 2.3e-2;
    the gradients pass as many again: 4.6e-2."""
    lens = [37, 130, 5]
    p, x, seqs = _layer(dtype, lens)
    f = _forward(p, x, seqs)
    g = torch.Generator().manual_seed(5)
    dy = torch.randn(f["y"].shape, generator=g).to(dtype).to(DEV)
    dres = torch.randn(f["res"].shape, generator=g).to(DEV)
    b1 = kla.kla_norm_bwd(f["o"].flatten(-2), p["w_out"], EPS, dy, gate=x["z"], group=P)
    v, k, q = _split(f["c"])
    b2 = kla.kla_ssm_bwd(q, k, v, x["dt"], p["a"], b1["dx"].unflatten(-1, (H, P)), d_skip=p["skip"], **seqs)
    dc = torch.cat([b2["dv"].flatten(-2), b2["dk"].flatten(-2), b2["dq"].flatten(-2)], -1)
    b3 = kla.kla_conv_bwd(f["u"], p["conv_w"], dc, bias=p["conv_b"], want_dinit_state=False, **seqs)
    b4 = kla.kla_norm_bwd(x["x"], p["w_norm"], EPS, b3["dx"], residual=x["res"], d_residual_out=dres)
    lp, lx, ry, rres, rfin = _reference(p, x, lens)
    tol = 1e-5 if dtype == F32 else 2.3e-2
    for got, ref in ((f["y"], ry), (f["res"], rres), (f["fin"], rfin)):
        assert _off(got, ref) <= tol
    ((ry * dy[0].double().cpu()).sum() + (rres * dres[0].double().cpu()).sum()).backward()
    pairs = [(b4["dx"], lx["x"]), (b4["dresidual"], lx["res"]), (b4["dweight"], lp["w_norm"]), (b3["dweight"], lp["conv_w"]), (b3["dbias"], lp["conv_b"]), (b2["ddt"], lx["dt"]),
             (b2["da"], lp["a"]), (b2["dd"], lp["skip"]), (b1["dweight"], lp["w_out"]), (b1["dgate"], lx["z"])]
    for got, ref in pairs:
        assert _off(got, ref.grad) <= 2 * tol


@pytest.mark.gpu
def test_a_prompt_and_then_single_tokens():
    """Prompt of T tokens and three steps against a prompt of T + 3, fp32."""
    T, n = 70, 3
    p, x, _ = _layer(F32, [T + n])
    part = lambda lo, hi: {k: t[:, lo:hi].contiguous() for k, t in x.items()}  # noqa: E731
    whole = _forward(p, x, {})
    f = _forward(p, part(0, T), {})
    cs, st = f["conv_fin"], f["fin"]
    for t in range(T, T + n):
        s = {k: v[:, t] for k, v in x.items()}
        u, _ = kla.kla_norm_fwd(s["x"], p["w_norm"], EPS, residual=s["res"].contiguous())
        v, k, q = _split(kla.kla_conv_step(u, p["conv_w"], cs, bias=p["conv_b"]))
        o = kla.kla_ssm_step(q, k, v, s["dt"].contiguous(), p["a"], st, d_skip=p["skip"])
        y, _ = kla.kla_norm_fwd(o.flatten(-2), p["w_out"], EPS, gate=s["z"], group=P)
        torch.testing.assert_close(y, whole["y"][:, t], rtol=1e-4, atol=1e-4)
    torch.testing.assert_close(st, whole["fin"], rtol=1e-4, atol=1e-4)
    assert torch.equal(cs, whole["conv_fin"])


@pytest.mark.gpu
def test_around_the_delta_rule():
    """The convolution before and the gated norm behind kla_chunk_fwd: the mixer's output enters the norm as it is, per head."""
    w = W.config3(B=1, H=2, T=200, seed=9)
    q, k, v = (t.to(DEV) for t in (w.q, w.k, w.v))
    cw, cb = 0.5 * torch.randn(256, 4, device=DEV), torch.zeros(256, device=DEV)
    mixed = [kla.kla_conv_fwd(t.flatten(-2), cw, bias=cb)[0].unflatten(-1, (2, 128)) for t in (q, k, v)]
    o, _ = kla.kla_chunk_fwd(*mixed, w.log_alpha.to(DEV), w.eta.to(DEV), w.eps)
    z = torch.randn(1, 200, 256, device=DEV).to(BF)
    y, _ = kla.kla_norm_fwd(o.flatten(-2), torch.ones(256, device=DEV), EPS, gate=z, group=128)
    ref, _ = norm(o.flatten(-2).double().cpu(), torch.ones(256, dtype=torch.float64), EPS, gate=z.double().cpu(), group=128)
    assert _off(y, ref) <= 2.0 ** -8


def _all_calls(p, x, seqs, state):
    """Every operator once, forward, backward and a token; the step's states are updated in place."""
    f = _forward(p, x, seqs)
    b1 = kla.kla_norm_bwd(f["o"].flatten(-2), p["w_out"], EPS, f["y"], gate=x["z"], group=P)
    v, k, q = _split(f["c"])
    b2 = kla.kla_ssm_bwd(q, k, v, x["dt"], p["a"], b1["dx"].unflatten(-1, (H, P)), d_skip=p["skip"], **seqs)
    b3 = kla.kla_conv_bwd(f["u"], p["conv_w"], f["c"], bias=p["conv_b"], **seqs)
    b4 = kla.kla_norm_bwd(x["x"], p["w_norm"], EPS, b3["dx"], residual=x["res"])
    o = kla.kla_ssm_step(q[:, 0], k[:, 0], v[:, 0], x["dt"][:, 0], p["a"], state, d_skip=p["skip"])
    outs = [f["y"], f["res"], f["fin"], f["conv_fin"], o, state]
    for b in (b1, b2, b3, b4):
        outs += [t for t in b.values() if t is not None]
    return outs


@pytest.mark.gpu
@pytest.mark.parametrize("dtype, T", [(BF, 300), (F32, 90), (BF, 1500)])
def test_captured_and_replayed(dtype, T):
    """One graph of all operators, replayed on other inputs; a second graph captured in between has workspaces of its own."""
    p, x, seqs = _layer(dtype, [T, 3])
    _, x2, _ = _layer(dtype, [T, 3], seed=8)
    state = torch.zeros(1, H, N, P, device=DEV)
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        for _ in range(2):
            _all_calls(p, x, seqs, state.clone())
    torch.cuda.synchronize()
    xs, st = {n: t.clone() for n, t in x.items()}, state.clone()
    graph, other = torch.cuda.CUDAGraph(), torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        outs = _all_calls(p, xs, seqs, st)
    st_b = state.clone()
    with torch.cuda.graph(other):
        outs_b = _all_calls(p, xs, seqs, st_b)
    for src in (x2, x):
        for n in xs:
            xs[n].copy_(src[n])
        st.zero_()
        st_b.zero_()
        want = [t.clone() for t in _all_calls(p, src, seqs, state.clone())]
        graph.replay()
        other.replay()
        torch.cuda.synchronize()
        kla.check()
        for got in (outs, outs_b):
            for a, b in zip(got, want):
                assert torch.equal(a, b)


@pytest.mark.gpu
def test_two_streams_at_once():
    p, x, seqs = _layer(BF, [700, 9])
    p2, x2, seqs2 = _layer(BF, [400, 333], seed=4)
    state = torch.zeros(1, H, N, P, device=DEV)
    want = [t.clone() for t in _all_calls(p, x, seqs, state.clone())], [t.clone() for t in _all_calls(p2, x2, seqs2, state.clone())]
    torch.cuda.synchronize()
    a, b = torch.cuda.Stream(), torch.cuda.Stream()
    for _ in range(3):
        with torch.cuda.stream(a):
            ga = _all_calls(p, x, seqs, state.clone())
        with torch.cuda.stream(b):
            gb = _all_calls(p2, x2, seqs2, state.clone())
        torch.cuda.synchronize()
        for got, ref in ((ga, want[0]), (gb, want[1])):
            assert all(torch.equal(s, t) for s, t in zip(got, ref))
