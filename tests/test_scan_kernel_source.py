"""Rules of the scan's kernels that no run can show (see test_kernel_source.py)."""
import re

import pytest

from test_kernel_source import _block, _code


@pytest.mark.parametrize("name", ["ssm_bwd.cu", "ssm_chunk.cu", "ssm_state.cu"])
def test_a_warp_gives_up_as_one(name):
    """A wait ends in a vote of the whole warp.  The flag that another warp raises may be seen by some lanes of a warp and not by others, so no
    lane leaves by what it has read itself as long as a wait follows: the rest would vote without it, for good."""
    text = _code(name)
    functions = 0
    for m in re.finditer(r"__device__ void (\w+)\([^{;]*\)\s*\{", text):
        functions += 1
        body, _ = _block(text, m.end() - 1)
        for r in re.finditer(r"if \(([^;{}]*?)\)\s*(?:\{[^{}]*)?(?:return|break)", body):
            cond = re.sub(r"(?:bar_wait|__all_sync|__any_sync)\((?:[^()]|\([^()]*\))*\)", "", r.group(1))
            if "abort_flag" in cond:
                assert not re.search(r"\b(?:bar_)?wait\(|_sync\(", body[r.end():]), (name, m.group(1), r.group(0))
    assert functions >= 1
