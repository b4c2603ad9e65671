"""A token mixer's half of a block with a diagonal state, for training and serving:
y = x + REC(act(GN(x)); z) (group normalisation over the token grid with an activation,
the gated linear recurrence along one of the scan orders, a residual around both) as a
sequence of libgtr calls, and its gradients:

    n, mean, rstd = act(GN(x))         gtr_groupnorm_fwd
    h, last = REC(n; z)                gtr_recurrence_fwd, its input weighed by 1 - a
    y = x + h                          gtr_add
    dn, dz, dh0 = REC'(dy)             gtr_recurrence_bwd from the states kept
    dx = dy + GN'(dn), dw, db          gtr_groupnorm_bwd with the residual's gradient in its epilogue

x [B, H*W, d] (fp16 or bf16, spatial order, a multiple of 8 elements: gtr_add's) and z, the gate logits of the same shape (a
projection of the caller's); ``p`` holds gn_w and gn_b ([d] float32). The calls allocate
what they return and may be recorded into a HIP graph. Gradients come from ``backward``
alone: nothing is recorded for torch's automatic differentiation. The statistics are an
image's, over all of its tokens: ``forward`` is no causal model's, and ``step`` does not go on
where it stopped. A server that goes on token by token normalises its tokens itself and calls
``step``.
"""
from __future__ import annotations

from typing import Optional

import torch

from . import gtr_add, gtr_groupnorm_bwd, gtr_groupnorm_fwd, gtr_recurrence_bwd, gtr_recurrence_fwd

GRADS = ("gn_w", "gn_b")


def forward(x: torch.Tensor, z: torch.Tensor, p: dict, *, H: int, W: int, groups: int, scan: str = "row", tau: float = 16.0,
            act: Optional[str] = "silu", eps: float = 1e-5, h0: Optional[torch.Tensor] = None, train: bool = False,
            stream=None):
    """(y, the state after the last token [B, d] float32), or with ``train`` (y, that state, what ``backward`` needs)."""
    n, mean, rstd = gtr_groupnorm_fwd(x, groups, p["gn_w"], p["gn_b"], act=act, eps=eps, stream=stream)
    h, last = gtr_recurrence_fwd(n, z, H=H, W=W, scan=scan, gate_tau=tau, complement=True, h0=h0, want_final=True,
                                 stream=stream)
    y = gtr_add(x, h, stream=stream)
    return (y, last, (x, n, mean, rstd, z, h, h0)) if train else (y, last)


def backward(dy: torch.Tensor, kept: tuple, p: dict, *, H: int, W: int, scan: str = "row", tau: float = 16.0,
             act: Optional[str] = "silu", dlast: Optional[torch.Tensor] = None, grads: Optional[dict] = None,
             stream=None) -> tuple:
    """(dx, dz, the first state's gradient or None, gradients by the names of GRADS). ``dlast``: the last state's
    gradient. ``grads``: an earlier call's, which this call's are added to (micro-batches)."""
    x, n, mean, rstd, z, h, h0 = kept
    dn, dz, dh0 = gtr_recurrence_bwd(dy, z, h, n, H=H, W=W, scan=scan, gate_tau=tau, complement=True, h0=h0, dh_final=dlast,
                                     want_dh0=h0 is not None, stream=stream)
    into = {} if grads is None else {"accumulate": True, "dw": grads["gn_w"], "db": grads["gn_b"]}
    dx, dw, db = gtr_groupnorm_bwd(dn, x, mean, rstd, p["gn_w"], p["gn_b"], act=act, dres=dy, out=dn, stream=stream, **into)
    return dx, dz, dh0, dict(zip(GRADS, (dw, db)))


def step(n: torch.Tensor, z: torch.Tensor, state: torch.Tensor, *, tau: float = 16.0,
         out: Optional[torch.Tensor] = None, stream=None) -> torch.Tensor:
    """One token further: n and z [B, d], ``state`` [B, d] float32 updated in place. Returns h [B, d]."""
    B, d = n.shape
    h, _ = gtr_recurrence_fwd(n.reshape(B, 1, d), z.reshape(B, 1, d), H=1, W=1, gate_tau=tau, complement=True, h0=state,
                              h_final=state, out=None if out is None else out.reshape(B, 1, d), stream=stream)
    return h.reshape(B, d)
