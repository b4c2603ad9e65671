"""The channel mixer's half of a block without its convolution, for training and
serving: y = x + FFN(LN(x)) (pre-norm layer normalisation, the gated feed-forward
[act(n W_gate^T) * (n W_value^T)] W_out^T, a residual around both) as a sequence of
libgtr calls, and its gradients:

    n, mean, rstd = LN(x)              gtr_layernorm_fwd
    y = x + FFN(n)                     gtr_ffn_fwd with the residual in its epilogue, both projections kept
    dn, dW_gate, dW_value, dW_out      gtr_ffn_bwd from the projections kept
    dx = dy + LN'(dn), dw, db          gtr_layernorm_bwd with the residual's gradient in its epilogue

``p`` holds ln_w, ln_b ([d] float32), w_gate, w_value ([hidden, d]) and w_out ([d,
hidden], all in x's type). The calls allocate what they return and may be recorded
into a HIP graph. Gradients come from ``backward`` alone: nothing is recorded for
torch's automatic differentiation, also where x or p require a gradient.
"""
from __future__ import annotations

from typing import Optional

import torch

from . import gtr_ffn_bwd, gtr_ffn_fwd, gtr_layernorm_bwd, gtr_layernorm_fwd

GRADS = ("ln_w", "ln_b", "w_gate", "w_value", "w_out")


def forward(x: torch.Tensor, p: dict, *, act: str = "silu", ln_eps: float = 1e-6, train: bool = False, stream=None):
    """x [..., d] (fp16 or bf16, one token upwards) -> y, or with ``train`` (y, what ``backward`` needs)."""
    n, mean, rstd = gtr_layernorm_fwd(x, p["ln_w"], p["ln_b"], eps=ln_eps, stream=stream)
    y, gate, value = gtr_ffn_fwd(n, p["w_gate"], p["w_value"], p["w_out"], act=act, residual=x, save=train, stream=stream)
    return (y, (x, n, mean, rstd, gate, value)) if train else y


def backward(dy: torch.Tensor, kept: tuple, p: dict, *, act: str = "silu", dw_dtype: Optional[torch.dtype] = None,
             grads: Optional[dict] = None, stream=None) -> tuple:
    """(dx, gradients by the names of GRADS). The matrices' gradients are in ``dw_dtype`` (x's type or float32), the
    layer norm's in float32. ``grads``: an earlier call's gradients, which this call's are added to (micro-batches)."""
    x, n, mean, rstd, gate, value = kept
    into = {} if grads is None else {"accumulate": True}
    g = grads or dict.fromkeys(GRADS)
    dn, dwg, dwv, dwo = gtr_ffn_bwd(dy, n, p["w_gate"], p["w_value"], p["w_out"], gate, value, act=act, dw_dtype=dw_dtype,
                                    dw_gate=g["w_gate"], dw_value=g["w_value"], dw_out=g["w_out"], stream=stream, **into)
    dx, dw, db = gtr_layernorm_bwd(dn, x, mean, rstd, p["ln_w"], dres=dy, dw=g["ln_w"], db=g["ln_b"], stream=stream,
                                   **into)
    return dx, dict(zip(GRADS, (dw, db, dwg, dwv, dwo)))
