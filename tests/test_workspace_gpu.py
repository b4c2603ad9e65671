"""One Workspace for calls of every kind, in turn: each result as with memory of the call's own."""
import pytest
import torch

pytestmark = pytest.mark.gpu


def inputs(dtype, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    n = lambda *s, std=1.0: (torch.randn(s, generator=g, device="cuda") * std).to(dtype)
    H = W = 20
    q, k, v = (n(2, 3, H * W, 64, std=0.3) for _ in range(3))
    decay = torch.nn.functional.logsigmoid(n(2, 3, H * W, 64).float() + 3).to(dtype)
    x, wg, wv, wo = n(2, H * W, 192), n(768, 192, std=0.07), n(768, 192, std=0.07), n(192, 768, std=0.04)
    conv = torch.randn(768, 3, 3, generator=g, device="cuda") * 0.3
    return (q, k, v, decay, H, W), (x, wg, wv, wo), conv, n(2, H * W, 192), n(3000, 384), n(3000, 384)


def calls(gtr, data, ws):
    (q, k, v, g, H, W), (x, *w), conv, dy, x2, dy2 = data
    scan = lambda: gtr.gtr_gla_fwd(q, k, v, g, H=H, W=W, scan="col", want_final=True, workspace=ws)
    out = [*scan()]
    y, gate, value = gtr.gtr_ffn_fwd(x, *w, save=True, workspace=ws)
    out += [y, *scan()]
    out += [*gtr.gtr_ffn_bwd(dy, x, *w, gate, value, workspace=ws), *scan()]
    _, mean, rstd = gtr.gtr_layernorm_fwd(x2)
    out += [*gtr.gtr_layernorm_bwd(dy2, x2, mean, rstd, workspace=ws), *scan()]
    out += [gtr.gtr_spatial_swiglu(x, *w, conv, H=H, W=W, workspace=ws), *scan()]
    return out


@pytest.mark.parametrize("dtype", [torch.float16, torch.bfloat16])
def test_one_workspace_for_every_call(gtr, dtype):
    data = inputs(dtype, 1)
    want = calls(gtr, data, None)
    ws = gtr.Workspace()
    for _ in range(2):  # (the second time with buffers that have their size)
        got = calls(gtr, data, ws)
        assert gtr.gtr_gla_workspace_fault(ws.buf) == 0
        assert all(torch.equal(a, b) for a, b in zip(got, want))


def test_a_graph_outlives_its_workspaces_growth(gtr):
    """Calls recorded with a Workspace that larger eager calls make grow afterwards: the replays keep their memory."""
    small, ws = inputs(torch.float16, 2), gtr.Workspace()
    want = calls(gtr, small, None)
    calls(gtr, small, ws)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        held = calls(gtr, small, ws)
    for k in range(3):
        sizes = ws.buf.numel(), ws.plain.numel()
        x, wg, wo = (torch.randn(s, device="cuda").half() for s in ((3000 + 1000 * k, 384), (1536, 384), (384, 1536)))
        gtr.gtr_ffn_fwd(x, wg, wg, wo, workspace=ws)
        q = torch.randn(2 + k, 6, 400, 64, device="cuda").half()
        gtr.gtr_gla_fwd(q, q, q, -q.abs(), H=20, W=20, workspace=ws)
        assert ws.buf.numel() > sizes[0] and ws.plain.numel() > sizes[1]
        others = [torch.full((n,), 0x5A, dtype=torch.uint8, device="cuda") for n in sizes for _ in range(4)]
        graph.replay()
        torch.cuda.synchronize()
        assert all((t == 0x5A).all() for t in others)
        assert all(torch.equal(a, b) for a, b in zip(held, want))
