"""Selective state space scan on the GPU against its recurrence in 64 bits.

Tolerance.  Every result is a sum of products of the inputs and of decays; `size` is the same sum over their magnitudes.  A term's
own error: the decays' exponents (sums of up to one chunk's log decays, |l| <= 210 in these tests, rounded to 2^-24 of that, and the exponential
2^-22) and a few products: 256 x 2^-24 = 2^-16; on the tensor cores derived operands are pairs of bf16 (2^-17 each, two in a row): 2^-16; its place
in sums over T tokens and N or P channels: (T + N + P) 2^-24.  rel = 2^-15 + (T + N + P) 2^-24; twice that for gradients, whose terms
have twice the factors.  A bf16 output of bf16 inputs is formed on the tensor cores from one bf16 each of P and of the state: a term of either
kind then carries one rounding of at most half a bf16 step, 2^-8 of itself, so 2^-8 is added to rel.  So it is with the bf16 gradients dq, dk, dv,
whose terms hold one such operand each.  The last state's decay exponents are the
short sums from a token to the end."""
import pytest
import torch

from layer_refs import check, grads, leaf, scan
from paper_2605_08587_b200 import (KLA_FLAG_FORCE_SIMT, KLA_FLAG_NO_SEGMENTS, KLA_FLAG_NONE, KlaError, check as check_status, kla_ssm_bwd, kla_ssm_fwd,
                                   kla_ssm_step, launch_count)
from paper_2605_08587_b200.binding import KLA_INTERNAL_FLAG_TEST_TIMEOUT

DEV = "cuda:0"
BF, F32 = torch.bfloat16, torch.float32


def make(lens, H, G, N, P, dtype, state=True, skip=True, seed=0, strong=False):
    """q, k, v as slices of one array, as a convolution before the scan leaves them."""
    g = torch.Generator().manual_seed(seed)
    rows = sum(lens)
    z = torch.nn.functional.silu(1.5 * torch.randn(1, rows, H * P + 2 * G * N, generator=g)).to(dtype).to(DEV)
    s = dict(v=z[..., :H * P].unflatten(-1, (H, P)), k=z[..., H * P:H * P + G * N].unflatten(-1, (G, N)), q=z[..., H * P + G * N:].unflatten(-1, (G, N)))
    s["dt"] = torch.exp(-6.9 + 4.6 * torch.rand(1, rows, H, generator=g)).to(DEV)
    s["a"] = -(1 + 15 * torch.rand(H, generator=g)).to(DEV)
    if strong:
        s["dt"] *= 20
    s["d_skip"] = (1 + 0.1 * torch.randn(H, generator=g)).to(DEV) if skip else None
    s["init_state"] = torch.randn(len(lens), H, N, P, generator=g).to(DEV) if state else None
    host = torch.tensor([0] + list(torch.tensor(lens).cumsum(0)), dtype=torch.int32)
    seqs = dict(cu_seqlens=host.to(DEV), host_seqlens=host)
    dy = torch.randn(1, rows, H, P, generator=g).to(dtype).to(DEV)
    df = torch.randn(len(lens), H, N, P, generator=g).to(DEV) if state else None
    return s, seqs, dy, df


def reference(s, lens):
    """Leaves, results and sizes: la = dt a is a leaf of its own, so that both parts of ddt have their size."""
    H, N, P = s["v"].shape[2], s["q"].shape[3], s["v"].shape[3]
    init = s["init_state"] if s["init_state"] is not None else torch.zeros(len(lens), H, N, P)
    la = s["dt"][0].double().cpu() * s["a"].double().cpu()
    leaves = [leaf(s["q"][0]), leaf(s["k"][0]), leaf(s["v"][0]), leaf(s["dt"][0]), leaf(la), leaf(s["d_skip"]), leaf(init)]
    sizes = [None if t is None else (t.detach() if i == 4 else t.detach().abs()).requires_grad_() for i, t in enumerate(leaves)]
    return leaves, scan(*leaves, lens), sizes, scan(*sizes, lens)


def rel_of(lens, N, P):
    return 2.0 ** -15 + (max(lens + [0]) + N + P) * 2.0 ** -24


CASES = [([1], 1, 1, 64, 64), ([5, 0, 1, 2], 2, 1, 64, 64), ([31, 32, 33], 4, 2, 64, 64), ([127, 128, 1, 129, 0], 2, 1, 128, 64), ([260, 63], 2, 2, 128, 128), ([64, 65, 3], 4, 4, 64, 128),
         ([0, 0], 2, 1, 64, 64), ([70, 9], 2, 1, 16, 32), ([40, 41], 4, 2, 96, 80), ([21], 2, 1, 8, 8), ([35], 1, 1, 256, 256), ([50, 16], 3, 1, 32, 48), ([300], 6, 2, 128, 192)]


@pytest.mark.gpu
@pytest.mark.parametrize("flags", [KLA_FLAG_NONE, KLA_FLAG_FORCE_SIMT])
@pytest.mark.parametrize("state, skip, strong", [(True, True, False), (False, False, True)])
@pytest.mark.parametrize("dtype, out_dtype", [(BF, BF), (BF, F32), (F32, F32), (F32, BF)])
@pytest.mark.parametrize("lens, H, G, N, P", CASES)
def test_forward(lens, H, G, N, P, dtype, out_dtype, state, skip, strong, flags):
    s, seqs, _, _ = make(lens, H, G, N, P, dtype, state, skip, seed=N + P, strong=strong)
    y, fin = kla_ssm_fwd(**s, **seqs, out_dtype=out_dtype, flags=flags)
    torch.cuda.synchronize()
    _, (ry, rf), _, (my, mf) = reference(s, lens)
    rel = rel_of(lens, N, P) + (2.0 ** -8 if dtype == BF and out_dtype == BF else 0)
    assert y.dtype == out_dtype
    check(y[0], ry, my, rel, "out")
    check(fin, rf, mf, 2.0 ** -17 + (max(lens) + 64) * 2.0 ** -24, "final_state")


@pytest.mark.gpu
@pytest.mark.parametrize("flags", [KLA_FLAG_NONE, KLA_FLAG_FORCE_SIMT])
@pytest.mark.parametrize("state, skip, strong", [(True, True, False), (False, False, True)])
@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("lens, H, G, N, P", CASES)
def test_backward(lens, H, G, N, P, dtype, state, skip, strong, flags):
    s, seqs, dy, df = make(lens, H, G, N, P, dtype, state, skip, seed=N + P, strong=strong)
    g = kla_ssm_bwd(s["q"], s["k"], s["v"], s["dt"], s["a"], dy, d_skip=s["d_skip"], init_state=s["init_state"], d_final_state=df, flags=flags, **seqs)
    torch.cuda.synchronize()
    leaves, outs, sizes, mags = reference(s, lens)
    r = grads(outs, (dy[0], df), leaves)
    m = grads(mags, (dy[0].abs(), None if df is None else df.abs()), sizes)
    a, dt, rel = s["a"].double().cpu(), s["dt"][0].double().cpu(), 2 * rel_of(lens, N, P)
    ref = dict(dq=r[0], dk=r[1], dv=r[2], ddt=r[3] + a * r[4], da=(dt * r[4]).sum(0), dd=r[5], dinit_state=r[6])
    size = dict(dq=m[0], dk=m[1], dv=m[2], ddt=m[3] + a.abs() * m[4], da=(dt * m[4]).sum(0), dd=m[5], dinit_state=m[6])
    assert (g["dd"] is None) == (not skip)
    one_part = 2.0 ** -8 if dtype == BF else 0
    for n in ref:
        if ref[n] is not None:
            check(g[n][0] if n in ("dq", "dk", "dv", "ddt") else g[n], ref[n], size[n], rel + (one_part if n in ("dq", "dk", "dv") else 0), n)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype, out_dtype", [(BF, BF), (F32, BF), (BF, F32)])
@pytest.mark.parametrize("B, H, G, N, P", [(1, 2, 1, 64, 64), (5, 4, 2, 128, 64), (3, 2, 1, 128, 128), (2, 3, 3, 16, 24), (4, 2, 1, 96, 40), (2, 1, 1, 256, 256), (3, 2, 2, 8, 8)])
def test_step(B, H, G, N, P, dtype, out_dtype):
    """Three tokens, one after another."""
    T = 3
    s, _, _, _ = make([T] * B, H, G, N, P, dtype, seed=B)
    z = {n: s[n].reshape(B, T, *s[n].shape[2:]) for n in ("q", "k", "v", "dt")}
    state, ys = s["init_state"].clone(), []
    for t in range(T):
        ys.append(kla_ssm_step(z["q"][:, t], z["k"][:, t], z["v"][:, t], z["dt"][:, t].contiguous(), s["a"], state, d_skip=s["d_skip"], out_dtype=out_dtype))
    torch.cuda.synchronize()
    _, (ry, rf), _, (my, mf) = reference(s, [T] * B)
    rel = 2.0 ** -19 + (N + 16) * 2.0 ** -24
    check(torch.stack(ys, 1).reshape(B * T, H, P), ry, my, rel, "out")
    check(state, rf, mf, 2.0 ** -19, "state")


@pytest.mark.gpu
@pytest.mark.parametrize("N, P", [(128, 64), (64, 128), (32, 48)])
def test_fixed_length_batch_is_the_same_as_packed(N, P):
    B, T, H, G = 3, 150, 4, 2
    s, seqs, dy, df = make([T] * B, H, G, N, P, BF)
    z = dict(s, **{n: s[n].reshape(B, T, *s[n].shape[2:]) for n in ("q", "k", "v", "dt")})
    y, f = kla_ssm_fwd(**s, **seqs)
    y2, f2 = kla_ssm_fwd(**z)
    assert torch.equal(y.flatten(), y2.flatten()) and torch.equal(f, f2)
    names = ("q", "k", "v", "dt", "a")
    more = dict(d_skip=s["d_skip"], init_state=s["init_state"], d_final_state=df)
    g = kla_ssm_bwd(*(s[n] for n in names), dy, **more, **seqs)
    g2 = kla_ssm_bwd(*(z[n] for n in names), dy.reshape(B, T, H, P), **more)
    for n in g:
        assert torch.equal(g[n].flatten(), g2[n].flatten()), n


@pytest.mark.gpu
@pytest.mark.parametrize("N, P", [(128, 64), (64, 64), (16, 32)])
def test_neighbours_that_are_not_finite_stay_apart(N, P):
    """Packed sequences around the chunks' borders beside ones full of NaN and infinities: not one bit changes."""
    lens, H, G = [3, 130, 1, 200, 64, 5], 4, 2
    s, seqs, dy, df = make(lens, H, G, N, P, BF)
    bad = [0, 2, 4]
    at = [0, 3, 133, 134, 334, 398, 403]
    t, dy2, df2 = {n: x.clone() if torch.is_tensor(x) else x for n, x in s.items()}, dy.clone(), df.clone()
    for n in bad:
        for x in ("q", "k", "v"):
            t[x][0, at[n]:at[n + 1]] = float("nan") if n else float("inf")
        t["dt"][0, at[n]:at[n + 1]] = float("nan")
        dy2[0, at[n]:at[n + 1]] = float("nan")
        t["init_state"][n] = float("nan")
        df2[n] = float("inf")
    y, f = kla_ssm_fwd(**s, **seqs)
    y2, f2 = kla_ssm_fwd(**t, **seqs)
    args = lambda u: [u[n] for n in ("q", "k", "v", "dt", "a")]  # noqa: E731
    g = kla_ssm_bwd(*args(s), dy, d_skip=s["d_skip"], init_state=s["init_state"], d_final_state=df, **seqs)
    g2 = kla_ssm_bwd(*args(t), dy2, d_skip=s["d_skip"], init_state=t["init_state"], d_final_state=df2, **seqs)
    for n in range(len(lens)):
        if n in bad:
            continue
        rows = slice(at[n], at[n + 1])
        assert torch.equal(y[0, rows], y2[0, rows]) and torch.equal(f[n], f2[n]) and torch.equal(g["dinit_state"][n], g2["dinit_state"][n])
        for x in ("dq", "dk", "dv", "ddt"):
            assert torch.equal(g[x][0, rows], g2[x][0, rows]), x


@pytest.mark.gpu
@pytest.mark.parametrize("N, P", [(128, 64), (32, 32)])
def test_parts_of_a_sequence_hand_on_their_state(N, P):
    T, cut, H, G = 333, 150, 2, 1
    s, _, dy, df = make([T], H, G, N, P, F32, seed=3)
    part = lambda lo, hi: {n: s[n][:, lo:hi] if n in ("q", "k", "v", "dt") else s[n] for n in ("q", "k", "v", "dt", "a", "d_skip")}  # noqa: E731
    y, f = kla_ssm_fwd(**s)
    y1, f1 = kla_ssm_fwd(**part(0, cut), init_state=s["init_state"])
    y2, f2 = kla_ssm_fwd(**part(cut, T), init_state=f1)
    tol = dict(rtol=1e-4, atol=1e-4)   # two orders of the same fp32 sums of some hundred terms of size 1
    torch.testing.assert_close(torch.cat([y1, y2], 1), y, **tol)
    torch.testing.assert_close(f2, f, **tol)
    late = kla_ssm_bwd(**part(cut, T), d_out=dy[:, cut:].contiguous(), init_state=f1, d_final_state=df)
    early = kla_ssm_bwd(**part(0, cut), d_out=dy[:, :cut].contiguous(), init_state=s["init_state"], d_final_state=late["dinit_state"])
    whole = kla_ssm_bwd(**{n: s[n] for n in ("q", "k", "v", "dt", "a", "d_skip", "init_state")}, d_out=dy, d_final_state=df)
    for n in ("dq", "dk", "dv", "ddt"):
        torch.testing.assert_close(torch.cat([early[n], late[n]], 1), whole[n], rtol=1e-3, atol=1e-3 * float(whole[n].abs().max()))
    torch.testing.assert_close(early["dinit_state"], whole["dinit_state"], **tol)
    torch.testing.assert_close(early["da"] + late["da"], whole["da"], rtol=1e-3, atol=1e-2)


@pytest.mark.gpu
@pytest.mark.parametrize("N, P", [(64, 64), (24, 16)])
def test_gradient_against_differences(N, P):
    """Central differences of the kernel's forward in fp32 along a random direction of each input."""
    lens = [20, 7]
    s, seqs, dy, df = make(lens, 2, 1, N, P, F32, seed=9)
    names = ("q", "k", "v", "dt", "a", "d_skip", "init_state")
    s = {n: s[n].contiguous() for n in names}
    g = kla_ssm_bwd(**s, d_out=dy, d_final_state=df, **seqs)

    def loss(u):
        y, f = kla_ssm_fwd(**u, **seqs)
        return float((y.double() * dy).sum() + (f.double() * df).sum())
    gen = torch.Generator().manual_seed(2)
    for n, d in zip(names, ("dq", "dk", "dv", "ddt", "da", "dd", "dinit_state")):
        u = torch.randn(s[n].shape, generator=gen).to(DEV)
        h = 2.0 ** -5 if n != "dt" else 2.0 ** -9
        u /= u.norm()
        diff = (loss(dict(s, **{n: s[n] + h * u})) - loss(dict(s, **{n: s[n] - h * u}))) / (2 * h)
        assert abs(diff - float((g[d] * u).sum())) <= 4e-3 * max(1.0, float(g[d].norm())), n


@pytest.mark.gpu
@pytest.mark.parametrize("lens, H, N, P", [([2000], 1, 128, 64), ([1500, 0, 7], 2, 64, 64), ([0, 1800, 129], 1, 128, 128), ([0, 0, 1300], 1, 64, 64)])
@pytest.mark.parametrize("state", [False, True])
def test_long_sequences_in_parts(lens, H, N, P, state):
    """Cut into parts that run side by side, against the recurrence and against the uncut launch."""
    s, seqs, dy, df = make(lens, H, 1, N, P, BF, state=state, seed=7)
    y, f = kla_ssm_fwd(**s, **seqs, out_dtype=F32)
    y1, f1 = kla_ssm_fwd(**s, **seqs, out_dtype=F32, flags=KLA_FLAG_NO_SEGMENTS)
    n0 = launch_count()
    kla_ssm_fwd(**s, **seqs)
    assert launch_count() - n0 == 3      # what the parts add, their starts, the scan
    _, (ry, rf), _, (my, mf) = reference(s, lens)
    rel = rel_of(lens, N, P)
    for got in (y, y1):
        check(got[0], ry, my, rel, "out")
    for got in (f, f1):
        check(got, rf, mf, 2.0 ** -17 + (max(lens) + 64) * 2.0 ** -24, "final_state")


@pytest.mark.gpu
def test_results_do_not_vary():
    s, seqs, dy, df = make([500, 77, 900], 4, 1, 128, 64, BF)
    args = [s[n] for n in ("q", "k", "v", "dt", "a")]
    more = dict(d_skip=s["d_skip"], init_state=s["init_state"], **seqs)
    y, f = kla_ssm_fwd(*args, **more)
    g = kla_ssm_bwd(*args, dy, d_final_state=df, **more)
    for _ in range(3):
        y2, f2 = kla_ssm_fwd(*args, **more)
        g2 = kla_ssm_bwd(*args, dy, d_final_state=df, **more)
        assert torch.equal(y, y2) and torch.equal(f, f2) and all(torch.equal(g[n], g2[n]) for n in g)


@pytest.mark.gpu
@pytest.mark.parametrize("lens, H, G, N, P", [([2000], 1, 1, 128, 64), ([0, 1700, 129], 2, 1, 64, 64), ([1300, 0], 1, 1, 64, 128)])
def test_backward_of_long_sequences_in_parts(lens, H, G, N, P):
    """Against the fp32 kernels on CUDA cores (each bf16 gradient has one rounding of its own and one of its operands; fp32 sums over T, N and P)."""
    s, seqs, dy, df = make(lens, H, G, N, P, BF, seed=11)
    args = [s[n] for n in ("q", "k", "v", "dt", "a")]
    more = dict(d_skip=s["d_skip"], init_state=s["init_state"], d_final_state=df, **seqs)
    g, r = kla_ssm_bwd(*args, dy, **more), kla_ssm_bwd(*args, dy, flags=KLA_FLAG_FORCE_SIMT, **more)
    whole = kla_ssm_bwd(*args, dy, flags=KLA_FLAG_NO_SEGMENTS, **more)
    for n in r:
        for got in (g[n], whole[n]):
            off = float((got.double() - r[n].double()).norm() / r[n].double().norm())
            assert off <= (2.0 ** -7 if n in ("dq", "dk", "dv") else 2.0 ** -15), (n, off)


@pytest.mark.gpu
@pytest.mark.parametrize("N, P", [(128, 64), (64, 128)])
def test_a_wait_that_runs_out_is_reported(N, P):
    """A completion that is withheld: the block gives up after about a second, says so, and the context stays usable."""
    s, seqs, dy, _ = make([200], 1, 1, N, P, BF)
    args = [s[n] for n in ("q", "k", "v", "dt", "a")]
    word = torch.zeros(1, dtype=torch.int32, device=DEV)
    kla_ssm_fwd(*args, flags=KLA_INTERNAL_FLAG_TEST_TIMEOUT, status_word=word, **seqs)
    assert int(word) == -10
    word.zero_()
    kla_ssm_bwd(*args, dy, flags=KLA_INTERNAL_FLAG_TEST_TIMEOUT, status_word=word, **seqs)
    assert int(word) == -10
    kla_ssm_fwd(*args, flags=KLA_INTERNAL_FLAG_TEST_TIMEOUT, **seqs)   # the binding's own word
    with pytest.raises(KlaError):
        check_status()
    check_status()
    y, _ = kla_ssm_fwd(*args, **seqs)
    y1, _ = kla_ssm_fwd(*args, flags=KLA_FLAG_FORCE_SIMT, **seqs)
    assert float((y.double() - y1.double()).norm() / y1.double().norm()) <= 2.0 ** -8


@pytest.mark.gpu
@pytest.mark.parametrize("flags", [KLA_FLAG_NONE, KLA_FLAG_FORCE_SIMT])
@pytest.mark.parametrize("N, P", [(64, 64), (128, 64)])
def test_tokens_that_wipe_the_state(N, P, flags):
    """Steps of 1e6 and decays of exp(-1e6 and less) among ordinary ones, at most one to 32 tokens: what follows them keeps its digits (the sums of
    log decays that count stay below those of the other tests), and the gradient of a decay that is zero is zero."""
    lens, H, G = [200, 90], 2, 1
    s, seqs, dy, df = make(lens, H, G, N, P, BF, seed=3)
    at = [5, 40, 64, 127, 128, 199, 200, 250]
    s["dt"][0, at] = 1e6
    y, fin = kla_ssm_fwd(**s, **seqs, out_dtype=F32, flags=flags)
    g = kla_ssm_bwd(s["q"], s["k"], s["v"], s["dt"], s["a"], dy, d_skip=s["d_skip"], init_state=s["init_state"], d_final_state=df, flags=flags, **seqs)
    torch.cuda.synchronize()
    leaves, (ry, rf), sizes, (my, mf) = reference(s, lens)
    rel = rel_of(lens, N, P)
    check(y[0], ry, my, rel, "out")
    check(fin, rf, mf, 2.0 ** -17 + (max(lens) + 64) * 2.0 ** -24, "final_state")
    r = grads((ry, rf), (dy[0], df), leaves)
    m = grads((my, mf), (dy[0].abs(), df.abs()), sizes)
    for i, n in enumerate(("dq", "dk", "dv")):
        check(g[n][0], r[i], m[i], 2 * rel + 2.0 ** -8, n)
    check(g["dd"], r[5], m[5], 2 * rel, "dd")
    check(g["dinit_state"], r[6], m[6], 2 * rel, "dinit_state")
    check(g["ddt"][0, at], r[3][at], m[3][at], 2 * rel, "ddt")


@pytest.mark.gpu
@pytest.mark.parametrize("lens, H, N, P", [([70, 0, 200], 2, 64, 64), ([2000], 1, 128, 64), ([33, 0, 5], 2, 24, 16)])
def test_states_in_place(lens, H, N, P):
    """final_state may be init_state: the same bits as apart, in one pass, in parts and on CUDA cores."""
    s, seqs, _, _ = make(lens, H, 1, N, P, BF, seed=1)
    y, fin = kla_ssm_fwd(**s, **seqs)
    state = s["init_state"].clone()
    y2, fin2 = kla_ssm_fwd(**dict(s, init_state=state), final_state=state, **seqs)
    assert fin2.data_ptr() == state.data_ptr() and torch.equal(y, y2) and torch.equal(state, fin)


# (At these sizes every (chunk, group) is one block's: heads are shared among blocks only where there are fewer than half as many as SMs, see
# test_gpu_ssm_shares.py.)
@pytest.mark.gpu
@pytest.mark.parametrize("H, G, N, P", [(4, 2, 64, 64), (6, 2, 128, 64)])
def test_backward_of_more_chunks_than_blocks_run_at_once(H, G, N, P):
    """Between one and two chunks (times groups) to an SM: the second round's share their heads among several blocks."""
    sms = torch.cuda.get_device_properties(0).multi_processor_count
    lens = [1 + 5 * i % 13 for i in range(sms // 2 + 12)] + [0, 300]
    s, seqs, dy, df = make(lens, H, G, N, P, BF, seed=4)
    g = kla_ssm_bwd(s["q"], s["k"], s["v"], s["dt"], s["a"], dy, d_skip=s["d_skip"], init_state=s["init_state"], d_final_state=df, **seqs)
    torch.cuda.synchronize()
    leaves, outs, sizes, mags = reference(s, lens)
    r, m = grads(outs, (dy[0], df), leaves), grads(mags, (dy[0].abs(), df.abs()), sizes)
    a, dt, rel = s["a"].double().cpu(), s["dt"][0].double().cpu(), 2 * rel_of(lens, N, P)
    for i, n in enumerate(("dq", "dk", "dv")):
        check(g[n][0], r[i], m[i], rel + 2.0 ** -8, n)
    check(g["ddt"][0], r[3] + a * r[4], m[3] + a.abs() * m[4], rel, "ddt")
    check(g["da"], (dt * r[4]).sum(0), (dt * m[4]).sum(0), rel + sum(lens) * 2.0 ** -24, "da")
    check(g["dinit_state"], r[6], m[6], rel, "dinit_state")
