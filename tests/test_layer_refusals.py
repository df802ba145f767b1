"""What the operators around a mixer refuse on the host, before anything is launched (no GPU needed)."""
import ctypes

import numpy as np
import pytest
import torch

import paper_2605_08587_b200 as kla
from paper_2605_08587_b200 import binding, build

FAKE = 0x1000   # 16-byte aligned, never dereferenced
NULL, SHAPE, DTYPE, ALIGN, SEQLENS, WORKSPACE, EPS = -1, -2, -3, -4, -6, -7, -8


@pytest.fixture(scope="module")
def lib():
    build.build()
    return binding.load()


def desc(**kw):
    base = dict(B=2, T=10, H=4, d_k=64, d_v=64, n_seq=2, cu_seqlens=None, host_seqlens=None, io_dtype=binding.KLA_BF16, out_dtype=binding.KLA_BF16,
                flags=0, workspace=FAKE, workspace_bytes=1 << 40, status_word=None, stream=None)
    base.update(kw)
    return binding.KlaDesc(**base)


def packed(lens, T, **kw):
    at = np.asarray(lens, dtype=np.int32)
    d = desc(**{**dict(B=1, T=T, n_seq=len(lens) - 1, cu_seqlens=FAKE, host_seqlens=at.ctypes.data), **kw})
    d._keep = at
    return d


CONV = dict(channels=32, taps=4, x=FAKE, x_stride=32, weight=FAKE, bias=FAKE)
NORM = dict(width=64, group=64, x=FAKE, x_stride=64, residual=None, residual_dtype=0, scale=None, gate=None, gate_stride=0, weight=FAKE, eps=1e-6)
SSM = dict(groups=2, q=FAKE, q_stride=128, k=FAKE, k_stride=128, v=FAKE, v_stride=256, dt=FAKE, a=FAKE, d_skip=FAKE)


def call(lib, name, d, args, outs):
    return getattr(lib, name)(None if d is None else ctypes.byref(d), *args.values(), *outs)


def conv(lib, d=None, outs=(None, FAKE, None), **kw):
    return call(lib, "kla_conv_fwd", d or desc(), {**CONV, **kw}, outs)


def ssm(lib, d=None, outs=(None, FAKE, None), **kw):
    return call(lib, "kla_ssm_fwd", d or desc(), {**SSM, **kw}, outs)


def norm(lib, d=None, outs=(FAKE, FAKE), **kw):
    return call(lib, "kla_norm_fwd", d or desc(), {**NORM, **kw}, outs)


def test_convolution(lib):
    assert call(lib, "kla_conv_fwd", None, CONV, (None, FAKE, None)) == NULL
    assert conv(lib, x=None) == NULL and conv(lib, weight=None) == NULL and conv(lib, outs=(None, None, None)) == NULL
    assert conv(lib, taps=1) == SHAPE and conv(lib, taps=5) == SHAPE and conv(lib, channels=0) == SHAPE and conv(lib, x_stride=31) == SHAPE
    assert conv(lib, desc(B=0)) == SHAPE and conv(lib, desc(T=-1)) == SHAPE and conv(lib, desc(n_seq=3)) == SHAPE
    assert conv(lib, desc(B=1 << 16, n_seq=1 << 16, T=1 << 16)) == SHAPE
    assert conv(lib, desc(io_dtype=5)) == DTYPE
    assert conv(lib, x=FAKE + 2) == ALIGN and conv(lib, weight=FAKE + 2) == ALIGN and conv(lib, outs=(FAKE + 8, FAKE, None)) == ALIGN and conv(lib, outs=(None, FAKE, FAKE + 4)) == ALIGN
    step = (FAKE, FAKE)
    assert call(lib, "kla_conv_step", desc(T=2), CONV, step) == SHAPE
    assert call(lib, "kla_conv_step", desc(T=1), CONV, (None, FAKE)) == NULL
    back = (None, FAKE, None, FAKE, FAKE, FAKE, None)
    assert call(lib, "kla_conv_bwd", desc(workspace=None), CONV, back) == WORKSPACE
    assert call(lib, "kla_conv_bwd", desc(workspace_bytes=64), CONV, back) == WORKSPACE
    assert call(lib, "kla_conv_bwd", desc(workspace=FAKE + 4), CONV, back) == ALIGN
    assert call(lib, "kla_conv_bwd", desc(), CONV, (None, None) + back[2:]) == NULL
    assert lib.kla_conv_bwd_workspace_bytes(ctypes.byref(desc()), 32, 9) == 0 and lib.kla_conv_bwd_workspace_bytes(None, 32, 4) == 0


@pytest.mark.parametrize("name", ["conv", "ssm"])
def test_offsets(lib, name):
    f = {"conv": conv, "ssm": ssm}[name]
    assert f(lib, packed([0, 5, 3, 10], 10)) == SEQLENS and f(lib, packed([1, 5, 10], 10)) == SEQLENS and f(lib, packed([0, 5, 9], 10)) == SEQLENS
    assert f(lib, packed([0, 5, 10], 10, B=2)) == SHAPE and f(lib, packed([0, 5, 10], 10, host_seqlens=None)) == NULL
    assert f(lib, packed([0, 5, 10], 10, cu_seqlens=FAKE + 2)) == ALIGN


def test_scan(lib):
    assert call(lib, "kla_ssm_fwd", None, SSM, (None, FAKE, None)) == NULL
    for n in ("q", "k", "v", "dt", "a"):
        assert ssm(lib, **{n: None}) == NULL and ssm(lib, **{n: FAKE + (4 if n in "qkv" else 2)}) == ALIGN
    assert ssm(lib, outs=(None, None, None)) == NULL and ssm(lib, d_skip=FAKE + 1) == ALIGN
    assert ssm(lib, groups=3) == SHAPE and ssm(lib, groups=0) == SHAPE and ssm(lib, desc(H=0)) == SHAPE
    for bad in (0, 4, 12, 264):
        assert ssm(lib, desc(d_k=bad), q_stride=8192, k_stride=8192) == SHAPE and ssm(lib, desc(d_v=bad), v_stride=8192) == SHAPE
    assert ssm(lib, q_stride=127) == SHAPE and ssm(lib, v_stride=252) == SHAPE
    assert ssm(lib, q_stride=132) == ALIGN and ssm(lib, v_stride=260) == ALIGN       # rows of bf16 that do not start on 16 bytes
    assert ssm(lib, desc(out_dtype=4)) == DTYPE and ssm(lib, desc(n_seq=1)) == SHAPE
    assert ssm(lib, desc(status_word=FAKE + 2)) == ALIGN
    assert call(lib, "kla_ssm_step", desc(T=1), SSM, (None, FAKE)) == NULL and call(lib, "kla_ssm_step", desc(T=0), SSM, (FAKE, FAKE)) == SHAPE
    back = (None, FAKE, None) + (FAKE,) * 5 + (None, None)
    assert call(lib, "kla_ssm_bwd", desc(workspace=None), SSM, back) == WORKSPACE
    assert call(lib, "kla_ssm_bwd", desc(), SSM, (None, None) + back[2:]) == NULL
    need = lib.kla_ssm_bwd_workspace_bytes(ctypes.byref(desc()), 2)
    assert need > 0 and call(lib, "kla_ssm_bwd", desc(workspace_bytes=need - 1), SSM, back) == WORKSPACE
    assert lib.kla_ssm_bwd_workspace_bytes(ctypes.byref(desc(n_seq=5)), 2) == 0 and lib.kla_ssm_bwd_workspace_bytes(None, 2) == 0


def test_norm(lib):
    assert call(lib, "kla_norm_fwd", None, NORM, (FAKE, FAKE)) == NULL
    assert norm(lib, x=None) == NULL and norm(lib, weight=None) == NULL and norm(lib, outs=(None, None)) == NULL
    assert norm(lib, residual=FAKE, outs=(FAKE, None)) == NULL
    assert norm(lib, group=48) == SHAPE and norm(lib, group=0) == SHAPE and norm(lib, width=0, group=1) == SHAPE and norm(lib, x_stride=63) == SHAPE
    assert norm(lib, gate=FAKE, gate_stride=63) == SHAPE and norm(lib, gate=FAKE, gate_stride=64, residual=FAKE) == SHAPE and norm(lib, scale=FAKE) == SHAPE
    assert norm(lib, residual=FAKE, residual_dtype=2) == DTYPE and norm(lib, desc(io_dtype=binding.KLA_F32), residual=FAKE, residual_dtype=binding.KLA_BF16) == DTYPE
    assert norm(lib, eps=-1.0) == EPS and norm(lib, eps=float("nan")) == EPS
    assert norm(lib, x=FAKE + 8) == ALIGN and norm(lib, outs=(FAKE + 2, None)) == ALIGN
    assert norm(lib, desc(B=1, T=1 << 30), group=1) == SHAPE          # more groups than a grid has blocks
    back = (FAKE, None, FAKE, None, None, None, FAKE)
    assert call(lib, "kla_norm_bwd", desc(workspace=None), NORM, back) == WORKSPACE
    assert call(lib, "kla_norm_bwd", desc(), {**NORM, "residual": FAKE}, back) == NULL
    assert call(lib, "kla_norm_bwd", desc(), {**NORM, "gate": FAKE, "gate_stride": 64}, back) == NULL


def test_no_fallback_without_sm100(lib):
    if torch.cuda.is_available() and torch.cuda.get_device_capability(0)[0] == 10:
        pytest.skip("an sm_100 device is present")
    assert conv(lib) == -11 and ssm(lib) == -11 and norm(lib) == -11


B, T, H, G, D, C = 2, 5, 4, 2, 64, 32


def _conv():
    x = torch.zeros(B, T, C, dtype=torch.bfloat16)
    return dict(x=x, weight=torch.zeros(C, 4), bias=torch.zeros(C), init_state=torch.zeros(B, 3, C, dtype=torch.bfloat16))


def _ssm():
    z = torch.zeros(B, T, G, D, dtype=torch.bfloat16)
    return dict(q=z, k=z, v=torch.zeros(B, T, H, D, dtype=torch.bfloat16), dt=torch.zeros(B, T, H), a=torch.zeros(H), d_skip=torch.zeros(H),
                init_state=torch.zeros(B, H, D, D))


def _norm():
    return dict(x=torch.zeros(B, T, C), weight=torch.zeros(C), eps=1e-6)


def test_tensors_that_are_not_on_a_gpu():
    for f, a in ((kla.kla_conv_fwd, _conv()), (kla.kla_ssm_fwd, _ssm()), (kla.kla_norm_fwd, _norm()),
                 (kla.kla_conv_bwd, dict(_conv(), d_out=torch.zeros(B, T, C, dtype=torch.bfloat16))),
                 (kla.kla_ssm_bwd, dict(_ssm(), d_out=torch.zeros(B, T, H, D, dtype=torch.bfloat16))), (kla.kla_norm_bwd, dict(_norm(), d_out=torch.zeros(B, T, C)))):
        with pytest.raises(ValueError, match="CUDA tensor"):
            f(**a)


@pytest.mark.parametrize("what, change, error", [
    ("_conv", dict(x=torch.zeros(B, C)), ValueError), ("_conv", dict(x=torch.zeros(B, T, C, dtype=torch.float16)), TypeError), ("_conv", dict(weight=torch.zeros(C + 1, 4)), ValueError),
    ("_conv", dict(x=None), ValueError), ("_conv", dict(weight=3.0), ValueError),
    ("_ssm", dict(v=torch.zeros(B, T, H, D)), TypeError), ("_ssm", dict(k=torch.zeros(B, T, G, D + 8, dtype=torch.bfloat16)), ValueError),
    ("_ssm", dict(q=torch.zeros(B, T + 1, G, D, dtype=torch.bfloat16)), ValueError), ("_ssm", dict(v=torch.zeros(B, T, H, D, dtype=torch.float16)), TypeError),
    ("_norm", dict(x=torch.zeros(B, T, C, dtype=torch.float64)), TypeError), ("_norm", dict(weight=None), ValueError), ("_norm", dict(eps="x"), TypeError)])
def test_arguments_of_another_kind(what, change, error):
    f = {"_conv": kla.kla_conv_fwd, "_ssm": kla.kla_ssm_fwd, "_norm": kla.kla_norm_fwd}[what]
    with pytest.raises(error):
        f(**dict(globals()[what](), **change))


@pytest.mark.parametrize("change, groups", [(dict(d_v=0), 2), (dict(d_v=-64), 2), (dict(d_k=0), 2), (dict(d_v=512), 2), (dict(d_k=68), 2), (dict(H=0), 2), (dict(), 3), (dict(), 0),
                                            (dict(B=0, n_seq=0), 2), (dict(T=-1), 2)])
def test_scratch_of_calls_that_are_refused(lib, change, groups):
    assert lib.kla_ssm_fwd_workspace_bytes(ctypes.byref(desc(**change)), groups) == 0
    assert lib.kla_ssm_bwd_workspace_bytes(ctypes.byref(desc(**change)), groups) == 0


def test_more_rows_than_loops_can_step_over(lib):
    for T in ((1 << 31) - (1 << 21), (1 << 31) - 1):
        d = desc(B=1, n_seq=1, T=T)
        assert conv(lib, d) == SHAPE and ssm(lib, d) == SHAPE and norm(lib, d) == SHAPE
