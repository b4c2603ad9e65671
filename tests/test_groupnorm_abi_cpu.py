"""gtr_groupnorm_fwd / _bwd on the CPU: every host-side check returns its status without launching (pointers are fake,
never dereferenced), and the workspace sizes."""
import ctypes

import pytest
import torch

import paper_2609_26590_amd as gtr

OK, NULL, SHAPE, UNSUP, ALIAS, WS = 0, 1, 2, 3, 4, 5
STEP = 1 << 36  # between fake buffers
B, L, C, G = 2, 6400, 384, 32
N = B * L * C


@pytest.fixture(scope="module")
def lib():
    return gtr.load()


def at(k, off=0):
    return (1 << 44) + k * STEP + off


def fwd(**kw):
    a = gtr.GroupnormFwdArgs(x=at(0), w=at(1), b=at(2), y=at(3), mean=at(4), rstd=at(5), dtype=gtr.F16, act=0, L=L, B=B, C=C,
                             groups=G, eps=1e-5)
    a.workspace, a.workspace_bytes = at(6), 1 << 30
    for k, v in kw.items():
        setattr(a, k, v)
    return a


def bwd(**kw):
    a = gtr.GroupnormBwdArgs(dy=at(0), x=at(1), mean=at(2), rstd=at(3), w=at(4), b=at(5), dres=at(6), dx=at(7), dw=at(8),
                             db=at(9), dtype=gtr.F16, act=1, L=L, B=B, C=C, groups=G, accumulate=0)
    a.workspace, a.workspace_bytes = at(10), 1 << 30
    for k, v in kw.items():
        setattr(a, k, v)
    return a


@pytest.mark.parametrize("change,status", [
    ({"B": 0}, SHAPE), ({"L": 0}, SHAPE), ({"L": 1 << 31}, SHAPE), ({"C": -384}, SHAPE), ({"groups": 0}, SHAPE),
    ({"groups": 5}, SHAPE), ({"groups": 768}, SHAPE), ({"C": 16416}, UNSUP), ({"dtype": 3}, UNSUP), ({"act": 3}, UNSUP),
    ({"act": -1}, UNSUP), ({"eps": -1e-6}, UNSUP), ({"eps": float("nan")}, UNSUP), ({"eps": float("inf")}, UNSUP),
    ({"B": 1 << 30, "L": 1 << 12}, SHAPE), ({"x": None}, NULL), ({"y": None}, NULL), ({"x": at(0, 1)}, UNSUP),
    ({"w": at(1, 2)}, UNSUP), ({"mean": at(4, 1)}, UNSUP), ({"workspace": None}, WS), ({"workspace": at(6, 8)}, WS),
    ({"workspace_bytes": 64}, WS), ({"y": at(0, 2)}, ALIAS), ({"y": at(2)}, ALIAS), ({"mean": at(0)}, ALIAS),
    ({"rstd": at(4)}, ALIAS), ({"mean": at(3, N * 2 - 4)}, ALIAS), ({"workspace": at(0)}, ALIAS), ({"workspace": at(3)}, ALIAS)])
def test_forward_refuses(lib, change, status):
    assert lib.gtr_groupnorm_fwd(ctypes.byref(fwd(**change)), None) == status


@pytest.mark.parametrize("change,status", [
    ({"B": -2}, SHAPE), ({"L": -1}, SHAPE), ({"groups": 7}, SHAPE), ({"C": 32768}, UNSUP), ({"dtype": 9}, UNSUP),
    ({"act": 7}, UNSUP), ({"dy": None}, NULL), ({"x": None}, NULL), ({"mean": None}, NULL), ({"rstd": None}, NULL),
    ({"dx": None, "dw": None, "db": None}, NULL), ({"dres": at(6, 1)}, UNSUP), ({"db": at(9, 2)}, UNSUP),
    ({"workspace": None}, WS), ({"workspace_bytes": 1000}, WS), ({"dx": at(0, 2)}, ALIAS), ({"dx": at(2)}, ALIAS),
    ({"dw": at(4)}, ALIAS), ({"db": at(8)}, ALIAS), ({"dw": at(7, 4)}, ALIAS), ({"workspace": at(1)}, ALIAS),
    ({"workspace": at(9)}, ALIAS)])
def test_backward_refuses(lib, change, status):
    assert lib.gtr_groupnorm_bwd(ctypes.byref(bwd(**change)), None) == status


def test_null_arguments(lib):
    for name in ("gtr_groupnorm_fwd", "gtr_groupnorm_bwd"):
        assert getattr(lib, name)(None, None) == NULL
        assert getattr(lib, name + "_workspace_size")(None) == 0


def test_workspace_sizes(lib):
    size = lambda fn, a: getattr(lib, fn + "_workspace_size")(ctypes.byref(a))
    assert size("gtr_groupnorm_fwd", fwd(groups=5)) == 0 and size("gtr_groupnorm_bwd", bwd(act=5)) == 0
    # an image's block that fits a work-group needs none (one image: no sums over images either)
    assert size("gtr_groupnorm_fwd", fwd(L=100)) == 0
    assert size("gtr_groupnorm_bwd", bwd(L=100, B=1)) == 0
    assert 0 < size("gtr_groupnorm_bwd", bwd(L=100)) <= B * 2 * C * 4 + 256
    for n in (6400, 1 << 20):
        assert 0 < size("gtr_groupnorm_fwd", fwd(L=n)) <= B * 256 * G * 8 + 256
        whole = size("gtr_groupnorm_bwd", bwd(L=n))
        assert 0 < whole <= B * 256 * (G + C) * 8 + 512
        assert whole == size("gtr_groupnorm_bwd", bwd(L=n, dx=None)) + size("gtr_groupnorm_bwd", bwd(L=n, dw=None, db=None))


def test_the_binding_refuses_host_tensors():
    x, m = torch.zeros(2, 12, 40), torch.zeros(2, 4)
    for call in (lambda: gtr.gtr_groupnorm_fwd(x, 4), lambda: gtr.gtr_groupnorm_bwd(x, x, m, m)):
        with pytest.raises(ValueError):
            call()
