"""Scan on the GPU with steps far larger than the others: what such a token writes outweighs its neighbours', and its decay may wipe the state.

Tolerance: that of test_gpu_ssm.py, `rel` times the sum of the magnitudes of the terms that make up each value.  A term of a token's ddt has to span that
token, so a large step elsewhere has no part in its size."""
import pytest
import torch

from layer_refs import check, grads
from paper_2605_08587_b200 import KLA_FLAG_FORCE_SIMT, KLA_FLAG_NONE, kla_ssm_bwd, kla_ssm_fwd
from test_gpu_ssm import BF, F32, make, reference, rel_of


def backward(s, seqs, dy, df, flags):
    g = kla_ssm_bwd(s["q"], s["k"], s["v"], s["dt"], s["a"], dy, d_skip=s["d_skip"], init_state=s["init_state"], d_final_state=df, flags=flags, **seqs)
    torch.cuda.synchronize()
    return g


def check_gradients(g, s, dy, df, lens, N, P):
    leaves, outs, sizes, mags = reference(s, lens)
    r, m = grads(outs, (dy[0], df), leaves), grads(mags, (dy[0].abs(), df.abs()), sizes)
    a, dt, rel = s["a"].double().cpu(), s["dt"][0].double().cpu(), 2 * rel_of(lens, N, P)
    one_part = 2.0 ** -8 if s["v"].dtype == BF else 0
    check(g["ddt"][0], r[3] + a * r[4], m[3] + a.abs() * m[4], rel, "ddt")
    check(g["da"], (dt * r[4]).sum(0), (dt * m[4]).sum(0), rel + sum(lens) * 2.0 ** -24, "da")
    check(g["dd"], r[5], m[5], rel, "dd")
    check(g["dinit_state"], r[6], m[6], rel, "dinit_state")
    for i, n in enumerate(("dq", "dk", "dv")):
        check(g[n][0], r[i], m[i], rel + one_part, n)


@pytest.mark.gpu
@pytest.mark.parametrize("step", [1.0, 15.0, 1e3, 1e6])
@pytest.mark.parametrize("N, P, dtype, flags", [(64, 64, BF, KLA_FLAG_NONE), (128, 64, BF, KLA_FLAG_NONE), (64, 128, BF, KLA_FLAG_NONE),
                                                (64, 64, BF, KLA_FLAG_FORCE_SIMT), (128, 64, F32, KLA_FLAG_NONE), (24, 16, F32, KLA_FLAG_NONE), (96, 40, BF, KLA_FLAG_NONE)])
def test_gradients_beside_large_steps(N, P, dtype, flags, step):
    """At most one large step to 32 tokens; every token's gradients, those before such a step among them."""
    lens, H, G = [200, 90], 4, 2
    s, seqs, dy, df = make(lens, H, G, N, P, dtype, seed=3)
    s["dt"][0, [5, 40, 64, 127, 128, 199, 200, 250]] = step
    check_gradients(backward(s, seqs, dy, df, flags), s, dy, df, lens, N, P)


@pytest.mark.gpu
@pytest.mark.parametrize("step", [8.0, 1e6, 1e30])
@pytest.mark.parametrize("N, P, dtype, flags", [(64, 64, BF, KLA_FLAG_NONE), (128, 64, BF, KLA_FLAG_NONE), (64, 64, BF, KLA_FLAG_FORCE_SIMT), (24, 16, F32, KLA_FLAG_NONE)])
def test_runs_of_tokens_that_wipe_the_state(N, P, dtype, flags, step):
    """Up to 24 of 32 tokens decay by exp(-8) and more each (and write nothing: their keys are zero); the decays between the ordinary ones behind them keep
    their digits."""
    lens, H, G = [200, 90], 4, 2
    s, seqs, dy, df = make(lens, H, G, N, P, dtype, seed=3)
    at = [*range(3, 19), 64, 65, *range(70, 94), *range(130, 140), 199, 200, 201, 250]
    s["dt"][0, at] = step
    s["k"][0, at] = 0
    y, fin = kla_ssm_fwd(**s, **seqs, out_dtype=F32, flags=flags)
    g = backward(s, seqs, dy, df, flags)
    _, (ry, rf), _, (my, mf) = reference(s, lens)
    check(y[0], ry, my, rel_of(lens, N, P), "out")
    check(fin, rf, mf, 2.0 ** -17 + (max(lens) + 64) * 2.0 ** -24, "final_state")
    check_gradients(g, s, dy, df, lens, N, P)
