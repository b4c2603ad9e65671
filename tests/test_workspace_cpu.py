"""Workspace on the CPU: which of its buffers a call is given, and how long a captured one lives (its memory is host
memory here, and streams are stand-ins)."""
import contextlib
import gc
import weakref

import pytest
import torch

import paper_2609_26590_amd as gtr


@pytest.fixture
def host(monkeypatch):
    """A Workspace of host memory; state["capturing"] says whether its stream is being captured."""
    state = {"capturing": False, "zeroed": []}
    monkeypatch.setattr(torch.cuda, "stream", lambda s: contextlib.nullcontext())
    monkeypatch.setattr(torch.cuda, "current_stream", lambda device=None: object())
    monkeypatch.setattr(torch._C, "_cuda_isCurrentStreamCapturing", lambda: state["capturing"])
    monkeypatch.setattr(gtr, "gtr_gla_workspace_init", lambda buf, stream=None: state["zeroed"].append(buf.zero_().numel()))
    state["ws"] = gtr.Workspace("cpu")
    return state


def test_other_calls_leave_the_zeroed_buffer_alone(host):
    """gtr_gla_fwd's synchronisation words stay zeroed whatever other calls were given the same Workspace."""
    ws = host["ws"]
    words = ws.get(4096)
    for need in (256, 4096, 100_000):
        got = gtr._scratch(need, torch.device("cpu"), ws)
        assert got.numel() >= need and got.untyped_storage().data_ptr() != words.untyped_storage().data_ptr()
        got.fill_(0xFF)
    assert ws.get(4096) is words and not words.any()
    assert len(host["zeroed"]) == 1  # the other calls' memory is not filled


def test_growth(host):
    ws = host["ws"]
    small = ws.scratch(1000)
    assert small.numel() == 1024 and ws.scratch(500) is small and ws.scratch(1025) is not small
    assert ws.scratch(0).numel() >= 256
    first = ws.get(300)
    assert ws.get(10) is first and ws.get(600).numel() == 768


@pytest.mark.parametrize("kind", ["get", "scratch"])
def test_a_captured_buffer_outlives_its_replacement(host, kind):
    """A graph's replays use the memory that its capture was given; others' is released when it is replaced."""
    ws, take = host["ws"], getattr(host["ws"], kind)
    before = weakref.ref(take(256))
    kept = weakref.ref(take(1000))
    gc.collect()
    assert before() is None
    host["capturing"] = True
    assert take(1000) is kept()
    host["capturing"] = False
    last = take(5000)
    gc.collect()
    assert kept() is not None and kept() is not last and kept().numel() == 1024
    del ws, take, last
    host.pop("ws")
    gc.collect()
    assert kept() is None
