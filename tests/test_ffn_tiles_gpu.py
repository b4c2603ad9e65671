"""gtr_ffn_fwd and gtr_ffn_bwd at sizes whose plans reach what smaller ones do not: every product in 256 x 256 tiles
with several K steps and broken edges, and weights' gradients cut along K, alone and beside a cut dx. (That they do is
held on the CPU, tests/test_ffn_plan_cpu.py.) Tolerances and checks are tests/test_ffn_gpu.py's."""
import pytest
import torch

from test_ffn_gpu import check_backward, check_forward, inputs

pytestmark = pytest.mark.gpu

LARGE = [(3000, 1544, 4104), (5000, 2568, 2568)]
CUT = [(16384, 64, 96), (12800, 384, 1536), (3000, 512, 2048)]


@pytest.mark.parametrize("dtype", [torch.float16, torch.bfloat16])
@pytest.mark.parametrize("act", ["silu", "gelu"])
@pytest.mark.parametrize("M,d,hidden", LARGE)
def test_large_tiles(gtr, M, d, hidden, act, dtype):
    s = inputs(M, d, hidden, dtype, 21)
    w = (s["wg"], s["wv"], s["wo"])
    got = gtr.gtr_ffn_fwd(s["x"], *w, act=act, residual=s["res"], save=True)
    check_forward(got, s, act)
    back = gtr.gtr_ffn_bwd(s["dy"], s["x"], *w, got[1], got[2], act=act)
    check_backward(back, s, got[1], got[2], act)


@pytest.mark.parametrize("dtype,act", [(torch.float16, "gelu"), (torch.bfloat16, "silu")])
@pytest.mark.parametrize("f32", [False, True])
@pytest.mark.parametrize("M,d,hidden", CUT)
def test_cut_weights_gradients(gtr, M, d, hidden, f32, dtype, act):
    """Fresh, added to what is there, and without dx, whose launch has other slices."""
    s = inputs(M, d, hidden, dtype, 22)
    w = (s["wg"], s["wv"], s["wo"])
    wt = torch.float32 if f32 else dtype
    _, gate, value = gtr.gtr_ffn_fwd(s["x"], *w, act=act, save=True)
    for want_dx in (True, False):
        back = gtr.gtr_ffn_bwd(s["dy"], s["x"], *w, gate, value, act=act, want_dx=want_dx, dw_dtype=wt)
        check_backward(back, s, gate, value, act, wt)
        sums = [torch.randn_like(t) for t in back[1:]]
        before = [t.clone() for t in sums]
        added = gtr.gtr_ffn_bwd(s["dy"], s["x"], *w, gate, value, act=act, want_dx=want_dx, dw_gate=sums[0],
                                dw_value=sums[1], dw_out=sums[2], accumulate=True)
        assert added[3] is sums[2]
        check_backward(added, s, gate, value, act, wt, before)
        again = gtr.gtr_ffn_bwd(s["dy"], s["x"], *w, gate, value, act=act, want_dx=want_dx, dw_dtype=wt)
        assert all(a is b or torch.equal(a, b) for a, b in zip(again, back))
