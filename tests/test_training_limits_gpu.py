"""Sizes past the 32-bit integers of the ABI are refused, not cut to their lower bits."""
import pytest
import torch

pytestmark = pytest.mark.gpu

WIDE = (1 << 32) + 8  # lower 32 bits: 8, a size that the calls take


@pytest.fixture
def wide():
    """64 GiB of weights, never written, as [8, WIDE] or [WIDE, 8]."""
    yield torch.empty(8 * WIDE, dtype=torch.float16, device="cuda")
    torch.cuda.empty_cache()


def test_wide_rows_are_refused(gtr, wide):
    x, dy, out = wide[:WIDE], wide[WIDE:2 * WIDE], wide[2 * WIDE:3 * WIDE]
    one = torch.ones((), device="cuda")
    with pytest.raises(gtr.GtrError):
        gtr.gtr_layernorm_fwd(x, out=out)
    with pytest.raises(gtr.GtrError):
        gtr.gtr_layernorm_bwd(dy, x, one, one, out=out, want_dw=False)


@pytest.mark.parametrize("d,hidden", [(8, WIDE), (WIDE, 8)])
def test_wide_weights_are_refused(gtr, wide, d, hidden):
    up, down = wide.view(hidden, d), wide.view(d, hidden)
    x = torch.zeros(1, d, dtype=torch.float16, device="cuda")
    kept = torch.zeros(1, hidden, dtype=torch.float16, device="cuda")
    with pytest.raises(gtr.GtrError):
        gtr.gtr_ffn_fwd(x, up, up, down)
    with pytest.raises(gtr.GtrError):
        gtr.gtr_ffn_bwd(x, x, up, up, down, kept, kept, want_dw=False)
