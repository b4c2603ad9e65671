"""gtr_recurrence_fwd / _bwd on the CPU: every host-side check returns its status without launching (pointers are fake,
never dereferenced), and the workspace sizes."""
import ctypes

import pytest
import torch

import paper_2609_26590_amd as gtr

OK, NULL, SHAPE, UNSUP, ALIAS, WS = 0, 1, 2, 3, 4, 5
STEP = 1 << 36  # between fake buffers
B, H, W, D = 2, 40, 40, 384
N = B * H * W * D


@pytest.fixture(scope="module")
def lib():
    return gtr.load()


def at(k, off=0):
    return (1 << 44) + k * STEP + off


def fwd(**kw):
    a = gtr.RecurrenceFwdArgs(x=at(0), g=at(1), h=at(2), h0=at(3), h_final=at(4), dtype=gtr.F16, g_dtype=gtr.F16, g_kind=1,
                              gate_tau=16.0, complement=1, B=B, H=H, W=W, d=D, scan=1)
    a.workspace, a.workspace_bytes = at(5), 1 << 30
    for k, v in kw.items():
        setattr(a, k, v)
    return a


def bwd(**kw):
    a = gtr.RecurrenceBwdArgs(dh=at(0), g=at(1), h=at(2), x=at(3), h0=at(4), dh_final=at(5), dx=at(6), dg=at(7), dh0=at(8),
                              dtype=gtr.F16, g_dtype=gtr.F32, g_kind=1, gate_tau=16.0, complement=1, B=B, H=H, W=W, d=D)
    a.workspace, a.workspace_bytes = at(9), 1 << 30
    for k, v in kw.items():
        setattr(a, k, v)
    return a


@pytest.mark.parametrize("change,status", [
    ({"B": 0}, SHAPE), ({"H": -1}, SHAPE), ({"W": 0}, SHAPE), ({"d": 0}, SHAPE), ({"H": 65536, "W": 32768}, SHAPE),
    ({"x_ld": 383}, SHAPE), ({"g_ld": -384}, SHAPE), ({"x_ld": 1 << 62}, SHAPE), ({"d": 1 << 30, "H": 1 << 15}, SHAPE),
    ({"dtype": 3}, UNSUP), ({"g_dtype": 2}, UNSUP), ({"dtype": 0}, UNSUP), ({"scan": 4}, UNSUP), ({"scan": -1}, UNSUP),
    ({"g_kind": 2}, UNSUP), ({"gate_tau": 0.0}, UNSUP), ({"gate_tau": float("nan")}, UNSUP),
    ({"gate_tau": float("inf")}, UNSUP), ({"gate_tau": 1e-40}, UNSUP), ({"x": None}, NULL), ({"g": None}, NULL),
    ({"h": None}, NULL), ({"x": at(0, 1)}, UNSUP), ({"h": at(2, 1)}, UNSUP), ({"h0": at(3, 2)}, UNSUP),
    ({"h_final": at(4, 1)}, UNSUP), ({"workspace": None}, WS), ({"workspace": at(5, 64)}, WS), ({"workspace_bytes": 256}, WS),
    ({"h": at(1)}, ALIAS), ({"h": at(0, 2)}, ALIAS), ({"h": at(0), "x_ld": 400}, ALIAS), ({"h": at(3)}, ALIAS),
    ({"h_final": at(0, 4)}, ALIAS), ({"h_final": at(3, 4)}, ALIAS), ({"h_final": at(2, N * 2 - 4)}, ALIAS),
    ({"workspace": at(0)}, ALIAS), ({"workspace": at(4)}, ALIAS)])
def test_forward_refuses(lib, change, status):
    assert lib.gtr_recurrence_fwd(ctypes.byref(fwd(**change)), None) == status


@pytest.mark.parametrize("change,status", [
    ({"B": -1}, SHAPE), ({"d": 0}, SHAPE), ({"dx_ld": 1}, SHAPE), ({"dg_ld": 100}, SHAPE), ({"dtype": 9}, UNSUP),
    ({"g_dtype": 2}, UNSUP), ({"scan": 9}, UNSUP), ({"g_kind": -1}, UNSUP), ({"gate_tau": -1.0}, UNSUP), ({"dh": None}, NULL),
    ({"g": None}, NULL), ({"h": None}, NULL), ({"x": None}, NULL), ({"dx": None, "dg": None, "dh0": None}, NULL),
    ({"dg": at(7, 2)}, UNSUP), ({"dx": at(6, 1)}, UNSUP), ({"dh0": at(8, 3)}, UNSUP), ({"workspace": None}, WS),
    ({"workspace_bytes": 0}, WS), ({"dx": at(2)}, ALIAS), ({"dg": at(0)}, ALIAS), ({"dx": at(1)}, ALIAS),
    ({"dx": at(0, 2)}, ALIAS), ({"dx": at(7)}, ALIAS), ({"dh0": at(4)}, ALIAS), ({"dh0": at(6, 4)}, ALIAS),
    ({"workspace": at(2)}, ALIAS), ({"dx": at(0), "dx_ld": 385}, ALIAS),
    # columns of one matrix that share a byte, and rows that run past the next ones' start
    ({"g_dtype": 1, "dx": at(6), "dx_ld": 800, "dg": at(6, 383 * 2), "dg_ld": 800}, ALIAS),
    ({"g_dtype": 1, "dx": at(6), "dx_ld": 760, "dg": at(6, 384 * 2), "dg_ld": 760}, ALIAS)])
def test_backward_refuses(lib, change, status):
    assert lib.gtr_recurrence_bwd(ctypes.byref(bwd(**change)), None) == status


def test_null_arguments(lib):
    for name in ("gtr_recurrence_fwd", "gtr_recurrence_bwd"):
        assert getattr(lib, name)(None, None) == NULL
        assert getattr(lib, name + "_workspace_size")(None) == 0


def test_workspace_sizes(lib):
    size = lambda fn, a: getattr(lib, fn + "_workspace_size")(ctypes.byref(a))
    for name, make in (("gtr_recurrence_fwd", fwd), ("gtr_recurrence_bwd", bwd)):
        assert size(name, make(d=0)) == 0 and size(name, make(g_kind=7)) == 0
        # a short sequence is one work-group's per block of channels
        assert size(name, make(H=1, W=1)) == 0 and size(name, make(H=1, W=64)) == 0
        # two words of 8 bytes per channel and tile at most, of a tile of 64 tokens or more
        for L in (200, 1600, 1 << 20):
            tiles = -(-L // 64)
            assert 0 <= size(name, make(H=1, W=L)) <= 256 + 2 * B * tiles * D * 8
        assert size(name, make(H=1, W=1 << 20)) > 0


def test_the_binding_refuses_host_tensors():
    x = torch.zeros(2, 12, 40)
    for call in (lambda: gtr.gtr_recurrence_fwd(x, x, H=3, W=4), lambda: gtr.gtr_recurrence_bwd(x, x, x, H=3, W=4)):
        with pytest.raises(ValueError):
            call()


@pytest.mark.parametrize("size", [{"d": (1 << 29) + 1}, {"d": (1 << 31) - 1}, {"B": 1 << 30, "d": 1 << 20},
                                  {"B": (1 << 31) - 1, "d": 1 << 29}, {"B": (1 << 31) - 1, "H": 1 << 20, "W": 2047},
                                  {"B": 1 << 26, "d": 128}, {"B": (1 << 31) - 1, "H": 46340, "W": 46340, "d": 1 << 29}])
def test_sizes_beyond_a_launch(lib, size):
    """Numbers whose products pass 32 or 64 bits on the way."""
    size = {"H": 1, "W": 1, **size}
    for name, make in (("gtr_recurrence_fwd", fwd), ("gtr_recurrence_bwd", bwd)):
        assert getattr(lib, name)(ctypes.byref(make(**size)), None) == SHAPE
        assert getattr(lib, name + "_workspace_size")(ctypes.byref(make(**size))) == 0


@pytest.mark.parametrize("size,most", [({"d": 128}, (1 << 26) - 1), ({"d": 3}, (1 << 26) - 1), ({"d": 129}, (1 << 25) - 1),
                                       ({"W": 4, "d": 1}, (1 << 26) - 1), ({"W": 16, "d": 256}, (1 << 23) - 1),
                                       ({"W": 32768, "d": 128}, (1 << 15) - 1)])
def test_the_largest_batch(lib, size, most):
    """Up to 2^32 - 1 threads: waves of 64 for 1, 4 (here up to 16 tokens) or 16 (forward) tokens of 128 channels."""
    size = {"H": 1, "W": 1, **size}
    for name, make in (("gtr_recurrence_fwd", fwd), ("gtr_recurrence_bwd", bwd)):
        if size["W"] > 32 and make is bwd:
            continue
        assert getattr(lib, name)(ctypes.byref(make(B=most, g=None, **size)), None) == NULL
        assert getattr(lib, name)(ctypes.byref(make(B=most + 1, g=None, **size)), None) == SHAPE
