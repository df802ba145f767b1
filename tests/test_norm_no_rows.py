"""Norms of no rows with a residual and its scale: an array without rows has no address."""
import pytest
import torch

from paper_2605_08587_b200 import kla_norm_bwd, kla_norm_fwd
from test_layer_refusals import FAKE, NORM, SHAPE, call, desc, lib, norm  # noqa: F401


def test_a_scale_without_rows_is_accepted(lib):  # noqa: F811
    ok = (0, -11)   # the latter: no sm_100 device is present, which is looked at last
    if not torch.cuda.is_available():   # (the arrays below are nowhere)
        assert norm(lib, desc(T=0), x=None, scale=FAKE, outs=(None, None)) in ok
        assert call(lib, "kla_norm_bwd", desc(T=0), {**NORM, "x": None, "scale": FAKE}, (None, None, None, None, FAKE, None, FAKE)) in ok
    assert norm(lib, scale=FAKE) == SHAPE


@pytest.mark.gpu
@pytest.mark.parametrize("width", [64, 65, 8200])
@pytest.mark.parametrize("res", [torch.float32, torch.bfloat16])
def test_gradients_of_no_rows_are_zero(width, res):
    x = torch.empty(0, width, device="cuda:0", dtype=torch.bfloat16)
    r, w, s = x.to(res), torch.ones(width, device="cuda:0"), torch.ones(width, device="cuda:0")
    y, u = kla_norm_fwd(x, w, 1e-6, residual=r, scale=s)
    assert y.shape == x.shape and u.shape == x.shape and u.dtype == res
    torch.full((4 * width,), float("nan"), device="cuda:0")   # (freed at once: what is not written would be found there)
    g = kla_norm_bwd(x, w, 1e-6, x, residual=r, scale=s, d_residual_out=r)
    assert g["dx"].shape == x.shape and g["dresidual"].shape == x.shape
    assert (g["dweight"] == 0).all() and (g["dscale"] == 0).all()
