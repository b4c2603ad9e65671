"""The training operators of the channel mixer's half of a block, as cases that can be timed.

Four operators, each through the package's public entry points and, beside it, in
elementary torch operations:

* ``ln_fwd``: ``gtr_layernorm_fwd``, layer normalisation that also returns the rows' statistics;
* ``ln_bwd``: ``gtr_layernorm_bwd``, its gradients: of the input (plus the gradient that the residual
  path brings along) and, reduced over the rows, of weight and bias;
* ``ffn_fwd``: ``gtr_ffn_fwd``, the gated feed-forward [act(x W_g^T) * (x W_v^T)] W_o^T plus a residual,
  which may keep both projections for the backward pass;
* ``ffn_bwd``: ``gtr_ffn_bwd``, its gradients: of the input and of the three weights.

Widths are those of GTR-S (192) and GTR-L (384) with their expansion of 4, and generic wider ones. Token
counts are images at patch stride 16 (640 x 640 pixels are 1600 tokens), one token, and generic batches.
Weights and gradients are in the inputs' type, affine weights, statistics and their gradients in float32.
"""
import math

import torch

own = False

DTYPES = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
LN_EPS = 1e-6


def ln(name, kind, M, d, dtype, res):
    case = {"kind": kind, "M": M, "d": d, "dtype": dtype, "res": res}
    return dict(case, name=name) if name else case


def ffn(name, kind, M, d, hidden, dtype, act, keep):
    case = {"kind": kind, "M": M, "d": d, "hidden": hidden, "dtype": dtype, "act": act, "keep": keep}
    return dict(case, name=name) if name else case


def listed():
    return [
        # one token at the GTR-L width: the latency of a call
        ln("ln_fwd_one_token", "ln_fwd", 1, 384, "f16", False),
        # GTR-L training, a batch of 8 images of 640 x 640 pixels
        ln("ln_fwd_l_batch8", "ln_fwd", 12800, 384, "f16", False),
        # a wide model's long batch: larger than every cache
        ln("ln_fwd_wide", "ln_fwd", 32768, 4096, "bf16", False),
        # GTR-L training, one image; the residual's gradient joins
        ln("ln_bwd_l_640", "ln_bwd", 1600, 384, "f16", True),
        # float32 rows of odd width (gradient checks), no row aligned to a vector
        ln("ln_bwd_f32_odd", "ln_bwd", 777, 1001, "f32", False),
        # a wide model's batch
        ln("ln_bwd_wide", "ln_bwd", 16384, 4096, "bf16", True),
        # serving one token: the weights' bytes are the work
        ffn("ffn_fwd_one_token", "ffn_fwd", 1, 1024, 2816, "bf16", "silu", False),
        # GTR-L training, a batch of 8 images, both projections kept
        ffn("ffn_fwd_l_batch8", "ffn_fwd", 12800, 384, 1536, "f16", "silu", True),
        # a wide model's training batch, both projections kept
        ffn("ffn_fwd_wide", "ffn_fwd", 8192, 4096, 11008, "bf16", "silu", True),
        # GTR-S training, one image
        ffn("ffn_bwd_s_640", "ffn_bwd", 1600, 192, 768, "f16", "silu", True),
        # sizes that no tile divides
        ffn("ffn_bwd_ragged", "ffn_bwd", 1027, 1000, 2728, "f16", "gelu", True),
        # a wide model's training batch
        ffn("ffn_bwd_wide", "ffn_bwd", 8192, 4096, 11008, "bf16", "silu", True),
    ]


def _log(rng, lo, hi):
    return math.exp(rng.uniform(math.log(lo), math.log(hi)))


def draw(rng):
    kind = rng.choice(("ln_fwd", "ln_bwd", "ffn_fwd", "ffn_bwd"))
    if kind in ("ln_fwd", "ln_bwd"):
        d = int(_log(rng, 64, 8192.99))
        if rng.random() < 0.6:  # widths of most models
            d = max(64, d // 32 * 32)
        M = int(_log(rng, 1, min(32768, 2 ** 26 // d) + 0.99))
        return ln(None, kind, M, d, rng.choice(("f16", "bf16", "f32")), kind == "ln_bwd" and rng.random() < 0.5)
    d = 8 * round(_log(rng, 64, 4096) / 8)
    hidden = 8 * round(d * _log(rng, 1.5, 4.5) / 8)
    if rng.random() < 0.5:
        d, hidden = max(64, d // 64 * 64), max(64, hidden // 64 * 64)
    most = 8192 * 4096 * 11008 // (d * hidden)
    M = int(_log(rng, 1, min(16384, most) + 0.99))
    return ffn(None, kind, M, d, hidden, rng.choice(("f16", "bf16")), rng.choice(("silu", "gelu")),
               kind == "ffn_bwd" or rng.random() < 0.5)


# ---------------------------------------------------------------------------
# inputs
# ---------------------------------------------------------------------------
def prepare(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(int(seed) * 7919 + 17)
    dt, M, d = DTYPES[case["dtype"]], case["M"], case["d"]

    def n(*shape, std=1.0, mu=0.0, to=dt):
        return torch.randn(shape, generator=gen, device="cuda").mul_(std).add_(mu).to(to)

    f32 = torch.float32
    s = {"case": case, "x": n(M, d)}
    if case["kind"] in ("ln_fwd", "ln_bwd"):
        s["x"] += n(M, 1)  # rows of a residual stream are not centred
        s["w"], s["b"] = n(d, std=0.1, mu=1.0, to=f32), n(d, std=0.1, to=f32)
        s["out"] = torch.empty(M, d, dtype=dt, device="cuda")
        if case["kind"] == "ln_fwd":
            s["mean"], s["rstd"] = torch.empty(M, device="cuda"), torch.empty(M, device="cuda")
            return s
        s["dy"] = n(M, d, std=0.5)
        s["dres"] = n(M, d, std=0.5) if case["res"] else None
        x = s["x"].double()  # what the forward pass left
        mean = x.mean(-1, keepdim=True)
        s["rstd"] = (x - mean).square().mean(-1).add(LN_EPS).rsqrt().float()
        s["mean"] = mean[:, 0].float()
        s["dw"], s["db"] = torch.empty(d, device="cuda"), torch.empty(d, device="cuda")
        return s
    h = case["hidden"]
    s["wg"], s["wv"], s["wo"] = n(h, d, std=d ** -0.5), n(h, d, std=d ** -0.5), n(d, h, std=h ** -0.5)
    s["out"] = torch.empty(M, d, dtype=dt, device="cuda")
    if case["kind"] == "ffn_fwd":
        s["res"] = n(M, d)
        s["gate"] = torch.empty(M, h, dtype=dt, device="cuda") if case["keep"] else None
        s["value"] = torch.empty(M, h, dtype=dt, device="cuda") if case["keep"] else None
        return s
    s["dy"] = n(M, d, std=0.5)
    s["gate"] = (s["x"].float() @ s["wg"].float().t()).to(dt)  # what the forward pass kept
    s["value"] = (s["x"].float() @ s["wv"].float().t()).to(dt)
    s["dwg"], s["dwv"], s["dwo"] = (torch.empty_like(s[k]) for k in ("wg", "wv", "wo"))
    return s


# ---------------------------------------------------------------------------
# one pass
# ---------------------------------------------------------------------------
def run(s):
    if own:
        return RUN_OWN[s["case"]["kind"]](s)
    return RUN_PLAIN[s["case"]["kind"]](s)


def _own_ln_fwd(s):
    import paper_2609_26590_amd as gtr
    return gtr.gtr_layernorm_fwd(s["x"], s["w"], s["b"], eps=LN_EPS, out=s["out"], mean=s["mean"], rstd=s["rstd"])


def _own_ln_bwd(s):
    import paper_2609_26590_amd as gtr
    return gtr.gtr_layernorm_bwd(s["dy"], s["x"], s["mean"], s["rstd"], s["w"], dres=s["dres"], out=s["out"],
                                 dw=s["dw"], db=s["db"])


def _own_ffn_fwd(s):
    import paper_2609_26590_amd as gtr
    return gtr.gtr_ffn_fwd(s["x"], s["wg"], s["wv"], s["wo"], act=s["case"]["act"], residual=s["res"], out=s["out"],
                           gate=s["gate"], value=s["value"])


def _own_ffn_bwd(s):
    import paper_2609_26590_amd as gtr
    return gtr.gtr_ffn_bwd(s["dy"], s["x"], s["wg"], s["wv"], s["wo"], s["gate"], s["value"], act=s["case"]["act"],
                           out=s["out"], dw_gate=s["dwg"], dw_value=s["dwv"], dw_out=s["dwo"])


def _plain_ln_fwd(s):
    x = s["x"].float()
    mean = x.mean(-1, keepdim=True)
    c = x - mean
    rstd = (c.square().mean(-1, keepdim=True) + LN_EPS).rsqrt()
    return (c * rstd * s["w"] + s["b"]).to(s["x"].dtype), mean[:, 0], rstd[:, 0]


def _plain_ln_bwd(s):
    dy, rstd = s["dy"].float(), s["rstd"][:, None]
    xh = (s["x"].float() - s["mean"][:, None]) * rstd
    t = dy * s["w"]
    dx = rstd * (t - t.mean(-1, keepdim=True) - xh * (t * xh).mean(-1, keepdim=True))
    if s["dres"] is not None:
        dx = dx + s["dres"].float()
    return dx.to(s["x"].dtype), (dy * xh).sum(0), dy.sum(0)


def _act(g, kind):
    """act(g) and its derivative."""
    if kind == "silu":
        p = 1 / (1 + torch.exp(-g))
        return g * p, p * (1 + g * (1 - p))
    p = 0.5 * (1 + torch.erf(g * 0.5 ** 0.5))
    return g * p, p + g * torch.exp(-0.5 * g * g) * (2 * math.pi) ** -0.5


def _plain_ffn_fwd(s):
    dt, x = s["x"].dtype, s["x"].float()
    g, v = x @ s["wg"].float().t(), x @ s["wv"].float().t()
    y = (_act(g, s["case"]["act"])[0] * v) @ s["wo"].float().t() + s["res"].float()
    keep = s["case"]["keep"]
    return y.to(dt), g.to(dt) if keep else None, v.to(dt) if keep else None


def _plain_ffn_bwd(s):
    dt, dy, x = s["x"].dtype, s["dy"].float(), s["x"].float()
    a, da = _act(s["gate"].float(), s["case"]["act"])
    v = s["value"].float()
    dh = dy @ s["wo"].float()
    dg, dv = dh * v * da, dh * a
    dx = dg @ s["wg"].float() + dv @ s["wv"].float()
    return dx.to(dt), (dg.t() @ x).to(dt), (dv.t() @ x).to(dt), (dy.t() @ (a * v)).to(dt)


RUN_OWN = {"ln_fwd": _own_ln_fwd, "ln_bwd": _own_ln_bwd, "ffn_fwd": _own_ffn_fwd, "ffn_bwd": _own_ffn_bwd}
RUN_PLAIN = {"ln_fwd": _plain_ln_fwd, "ln_bwd": _plain_ln_bwd, "ffn_fwd": _plain_ffn_fwd, "ffn_bwd": _plain_ffn_bwd}


# ---------------------------------------------------------------------------
# what a pass cannot do without; the result in 64 bits
# ---------------------------------------------------------------------------
def work(case):
    M, d, kind = case["M"], case["d"], case["kind"]
    e = 4 if case["dtype"] == "f32" else 2
    if kind == "ln_fwd":  # x, w, b in; y, mean, rstd out
        return {"bytes": 2 * M * d * e + 8 * M + 8 * d, "flops": 8 * M * d}
    if kind == "ln_bwd":  # dy, x, (dres,) mean, rstd, w in; dx, dw, db out
        return {"bytes": (3 + case["res"]) * M * d * e + 8 * M + 12 * d, "flops": 16 * M * d}
    h = case["hidden"]
    if kind == "ffn_fwd":  # x, residual, weights in; y and, where kept, both projections out
        return {"bytes": (3 * M * d + 3 * d * h + (2 * M * h if case["keep"] else 0)) * e, "flops": 6 * M * d * h}
    # dy, x, both projections, weights in; dx and the weights' gradients out
    return {"bytes": (3 * M * d + 2 * M * h + 6 * d * h) * e, "flops": 12 * M * d * h}


def exact(case, seed):
    s = prepare(case, seed)
    x = s["x"].double().requires_grad_()
    if case["kind"] in ("ln_fwd", "ln_bwd"):
        w, b = s["w"].double().requires_grad_(), s["b"].double().requires_grad_()
        var, mean = torch.var_mean(x, -1, keepdim=True, correction=0)
        sd = (var + LN_EPS).sqrt()
        if case["kind"] == "ln_fwd":
            with torch.no_grad():
                return torch.addcmul(b, (x - mean).div_(sd), w), mean[:, 0], 1 / sd[:, 0]
        dx, dw, db = torch.autograd.grad(torch.addcmul(b, (x - mean) / sd, w), (x, w, b), s["dy"].double())
        return dx if s["dres"] is None else dx + s["dres"].double(), dw, db
    wg, wv, wo = (s[k].double() for k in ("wg", "wv", "wo"))

    def act(g):
        return g / (1 + torch.exp(-g)) if case["act"] == "silu" else g * torch.special.ndtr(g)

    if case["kind"] == "ffn_fwd":
        with torch.no_grad():
            g, v = x @ wg.t(), x @ wv.t()
            y = torch.addmm(s["res"].double(), act(g) * v, wo.t())
        return y, g if case["keep"] else None, v if case["keep"] else None
    g, v = s["gate"].double().requires_grad_(), s["value"].double().requires_grad_()
    wo.requires_grad_()
    dg, dv, dwo = torch.autograd.grad((act(g) * v) @ wo.t(), (g, v, wo), s["dy"].double())
    x = x.detach()
    return dg @ wg + dv @ wv, dg.t() @ x, dv.t() @ x, dwo
