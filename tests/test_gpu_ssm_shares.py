"""Scan backward on the GPU with the heads of a group shared among several blocks: fewer chunks than SMs.  Tolerance: that of test_gpu_ssm.py."""
import pytest
import torch

from paper_2605_08587_b200 import kla_ssm_bwd
from test_gpu_ssm import BF, make
from test_gpu_ssm_steps import check_gradients


@pytest.mark.gpu
@pytest.mark.parametrize("N, P", [(64, 64), (128, 128)])
@pytest.mark.parametrize("heads, G, blocks_a_group", [(5, 1, 2), (5, 2, 3), (7, 1, 3), (7, 1, 4), (3, 1, 40)])
def test_backward_with_uneven_shares(heads, G, blocks_a_group, N, P):
    """As many blocks to a group as there are SMs to a (chunk, group): 3 and 2 heads, 2 2 1, 3 3 1, 2 2 2 1, and one each."""
    sms = torch.cuda.get_device_properties(0).multi_processor_count
    lens = [130]
    while sms // ((sum(lens + [4]) // 128 + len(lens) + 1) * G) >= blocks_a_group:
        lens.append(1 + 5 * len(lens) % 7)
    s, seqs, dy, df = make(lens, heads * G, G, N, P, BF, seed=heads)
    call = lambda: kla_ssm_bwd(s["q"], s["k"], s["v"], s["dt"], s["a"], dy, d_skip=s["d_skip"], init_state=s["init_state"], d_final_state=df, **seqs)  # noqa: E731
    g = call()
    torch.cuda.synchronize()
    check_gradients(g, s, dy, df, lens, N, P)
    g2 = call()
    assert all(torch.equal(g[n], g2[n]) for n in g)
