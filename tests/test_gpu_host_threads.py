"""Calls from several host threads at once, each on a stream of its own: the same bits as alone."""
import threading

import pytest
import torch

from paper_2605_08587_b200 import kla_ssm_bwd
from test_gpu_ssm import BF, F32, make


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [F32, BF])
def test_scan_backward_at_different_widths(dtype):
    """The widest heads (214 KB of shared memory) and the narrowest (24 KB) of one kernel."""
    work = []
    for width in (256, 8):
        s, seqs, dy, df = make([40], 1, 1, width, width, dtype, seed=width)
        work.append((dict(s, d_out=dy, d_final_state=df, **seqs), torch.cuda.Stream()))
        work.append((work[-1][0], torch.cuda.Stream()))
    want = [kla_ssm_bwd(**w) for w, _ in work]
    torch.cuda.synchronize()
    wrong = []

    def loop(w, stream, ref):
        try:
            with torch.cuda.stream(stream):
                for _ in range(2000):
                    g = kla_ssm_bwd(**w)
                stream.synchronize()
                wrong.extend(n for n in g if not torch.equal(g[n], ref[n]))
        except Exception as e:   # (an assertion in a thread would be lost)
            wrong.append(e)
    threads = [threading.Thread(target=loop, args=(*w, ref)) for w, ref in zip(work, want)]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    assert not wrong
