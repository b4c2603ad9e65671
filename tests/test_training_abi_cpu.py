"""gtr_layernorm_fwd / _bwd and gtr_ffn_fwd / _bwd on the CPU: every host-side check returns its status without
launching (pointers are fake, never dereferenced), the workspace sizes, and the binding's own refusals."""
import ctypes

import pytest
import torch

import paper_2609_26590_amd as gtr

OK, NULL, SHAPE, UNSUP, ALIAS, WS = 0, 1, 2, 3, 4, 5
STEP = 1 << 36  # between fake buffers


@pytest.fixture(scope="module")
def lib():
    return gtr.load()


def at(k, off=0):
    return (1 << 44) + k * STEP + off


def ln_fwd(**kw):
    a = gtr.LayernormFwdArgs(x=at(0), w=at(1), b=at(2), y=at(3), mean=at(4), rstd=at(5), dtype=gtr.F16, d=384, M=100,
                             eps=1e-6)
    for k, v in kw.items():
        setattr(a, k, v)
    return a


def ln_bwd(**kw):
    a = gtr.LayernormBwdArgs(dy=at(0), x=at(1), mean=at(2), rstd=at(3), w=at(4), dres=at(5), dx=at(6), dw=at(7),
                             db=at(8), dtype=gtr.F16, d=384, M=10000, accumulate=0)
    a.workspace, a.workspace_bytes = at(9), 1 << 30
    for k, v in kw.items():
        setattr(a, k, v)
    return a


def ffn_fwd(**kw):
    a = gtr.FfnFwdArgs(x=at(0), w_gate=at(1), w_value=at(2), w_out=at(3), residual=at(4), y=at(5), gate=at(6),
                       value=at(7), dtype=gtr.BF16, act=0, M=100, d=384, hidden=1536)
    a.workspace, a.workspace_bytes = at(8), 1 << 30
    for k, v in kw.items():
        setattr(a, k, v)
    return a


def ffn_bwd(**kw):
    a = gtr.FfnBwdArgs(dy=at(0), x=at(1), w_gate=at(2), w_value=at(3), w_out=at(4), gate=at(5), value=at(6), dx=at(7),
                       dw_gate=at(8), dw_value=at(9), dw_out=at(10), dtype=gtr.BF16, dw_dtype=gtr.F32, act=1,
                       accumulate=0, M=100, d=384, hidden=1536)
    a.workspace, a.workspace_bytes = at(11), 1 << 30
    for k, v in kw.items():
        setattr(a, k, v)
    return a


@pytest.mark.parametrize("change,status", [
    ({"M": 0}, SHAPE), ({"M": -3}, SHAPE), ({"d": 0}, SHAPE), ({"M": 1 << 31}, SHAPE), ({"d": 16385}, UNSUP),
    ({"dtype": 3}, UNSUP), ({"eps": -1e-6}, UNSUP), ({"eps": float("nan")}, UNSUP), ({"eps": float("inf")}, UNSUP),
    ({"x": None}, NULL), ({"y": None}, NULL), ({"x": at(0, 1)}, UNSUP), ({"w": at(1, 2)}, UNSUP),
    ({"mean": at(4, 2)}, UNSUP), ({"y": at(0, 2)}, ALIAS), ({"y": at(1)}, ALIAS), ({"mean": at(0)}, ALIAS),
    ({"rstd": at(4)}, ALIAS), ({"mean": at(3, 100 * 384 * 2 - 4)}, ALIAS)])
def test_layernorm_fwd_refuses(lib, change, status):
    assert lib.gtr_layernorm_fwd(ctypes.byref(ln_fwd(**change)), None) == status


@pytest.mark.parametrize("change,status", [
    ({"M": 0}, SHAPE), ({"d": -1}, SHAPE), ({"d": 20000}, UNSUP), ({"dtype": 7}, UNSUP), ({"dy": None}, NULL),
    ({"x": None}, NULL), ({"mean": None}, NULL), ({"rstd": None}, NULL), ({"dx": None, "dw": None, "db": None}, NULL),
    ({"dres": at(5, 1)}, UNSUP), ({"db": at(8, 2)}, UNSUP), ({"workspace": None}, WS), ({"workspace_bytes": 255}, WS),
    ({"workspace": at(9, 16)}, WS), ({"dx": at(0, 2)}, ALIAS), ({"dx": at(2)}, ALIAS), ({"dw": at(4)}, ALIAS),
    ({"db": at(7)}, ALIAS), ({"dw": at(6, 4)}, ALIAS), ({"workspace": at(1)}, ALIAS)])
def test_layernorm_bwd_refuses(lib, change, status):
    assert lib.gtr_layernorm_bwd(ctypes.byref(ln_bwd(**change)), None) == status


@pytest.mark.parametrize("change,status", [
    ({"M": 0}, SHAPE), ({"hidden": 0}, SHAPE), ({"d": -8}, SHAPE), ({"M": 1 << 31}, SHAPE), ({"M": 1 << 30}, SHAPE),
    ({"d": 380}, UNSUP), ({"hidden": 1540}, UNSUP), ({"d": (1 << 20) + 8}, UNSUP), ({"dtype": gtr.F32}, UNSUP),
    ({"act": 2}, UNSUP), ({"act": -1}, UNSUP), ({"x": None}, NULL), ({"w_value": None}, NULL), ({"w_out": None}, NULL),
    ({"y": None}, NULL), ({"x": at(0, 8)}, UNSUP), ({"gate": at(6, 2)}, UNSUP), ({"workspace": None}, WS),
    ({"workspace_bytes": 1}, WS), ({"workspace": at(8, 64)}, WS), ({"y": at(0)}, ALIAS), ({"y": at(4, 16)}, ALIAS),
    ({"gate": at(7)}, ALIAS), ({"value": at(1)}, ALIAS), ({"workspace": at(5)}, ALIAS), ({"gate": at(5, 16)}, ALIAS)])
def test_ffn_fwd_refuses(lib, change, status):
    assert lib.gtr_ffn_fwd(ctypes.byref(ffn_fwd(**change)), None) == status


@pytest.mark.parametrize("change,status", [
    ({"M": 0}, SHAPE), ({"hidden": -8}, SHAPE), ({"d": 12}, UNSUP), ({"dtype": gtr.F32}, UNSUP),
    ({"dw_dtype": gtr.F16}, UNSUP), ({"act": 9}, UNSUP), ({"dy": None}, NULL), ({"gate": None}, NULL),
    ({"value": None}, NULL), ({"dx": None, "dw_gate": None, "dw_value": None, "dw_out": None}, NULL),
    ({"dw_out": at(10, 4)}, UNSUP), ({"workspace": None}, WS), ({"workspace_bytes": 1000}, WS), ({"dx": at(0)}, ALIAS),
    ({"dx": at(1)}, ALIAS), ({"dw_gate": at(2)}, ALIAS), ({"dw_value": at(8)}, ALIAS), ({"workspace": at(6)}, ALIAS)])
def test_ffn_bwd_refuses(lib, change, status):
    assert lib.gtr_ffn_bwd(ctypes.byref(ffn_bwd(**change)), None) == status


def test_null_arguments(lib):
    for name in ("gtr_layernorm_fwd", "gtr_layernorm_bwd", "gtr_ffn_fwd", "gtr_ffn_bwd"):
        assert getattr(lib, name)(None, None) == NULL
    for name in ("gtr_layernorm_bwd", "gtr_ffn_fwd", "gtr_ffn_bwd"):
        assert getattr(lib, name + "_workspace_size")(None) == 0


def test_workspace_sizes(lib):
    size = lambda fn, a: getattr(lib, fn + "_workspace_size")(ctypes.byref(a))
    assert size("gtr_layernorm_bwd", ln_bwd(d=0)) == 0
    assert size("gtr_ffn_fwd", ffn_fwd(act=5)) == 0 and size("gtr_ffn_bwd", ffn_bwd(d=9)) == 0
    # the partial sums of at most 1024 work-groups; a short batch has none
    assert size("gtr_layernorm_bwd", ln_bwd(M=1)) == 0
    assert 0 < size("gtr_layernorm_bwd", ln_bwd(M=1 << 20)) <= 1024 * 2 * 384 * 4
    for M in (1, 7, 100, 1600, 40000):
        h = (M * 1536 * 2 + 255) // 256 * 256
        assert h <= size("gtr_ffn_fwd", ffn_fwd(M=M)) <= h + 32 * M * 384 * 4
        assert 3 * h <= size("gtr_ffn_bwd", ffn_bwd(M=M)) <= 3 * h + 32 * max(3 * 384 * 1536, M * 384) * 4
    # products large enough to fill the chip are not cut
    assert size("gtr_ffn_fwd", ffn_fwd(M=100000, d=4096, hidden=8192)) == 100000 * 8192 * 2
    # without dw_out the gated activations are not formed again
    assert size("gtr_ffn_bwd", ffn_bwd(M=100000, d=4096, hidden=8192, dw_out=None)) == 2 * 100000 * 8192 * 2


def test_the_binding_refuses_host_tensors():
    x = torch.zeros(4, 64, dtype=torch.float16)
    w = torch.zeros(64, 64, dtype=torch.float16)
    m = torch.zeros(4)
    for call in (lambda: gtr.gtr_layernorm_fwd(x), lambda: gtr.gtr_layernorm_bwd(x, x, m, m),
                 lambda: gtr.gtr_ffn_fwd(x, w, w, w), lambda: gtr.gtr_ffn_bwd(x, x, w, w, w, x, x)):
        with pytest.raises(ValueError):
            call()
