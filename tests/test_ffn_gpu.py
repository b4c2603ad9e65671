"""gtr_ffn_fwd and gtr_ffn_bwd on the GPU against the formulas in 64 bits.

Tolerances (u: half a step of the 16-bit type, 2^-8 for bfloat16, 2^-11 for float16):
* per element, the bound of the arithmetic: every 16-bit intermediate (act(g) v, dg, dv) is off by at most u of
  itself, so a product of it with B by at most u (|intermediate| |B|) summed over K, and the result by u of itself
  more; float32 accumulation adds under (K + 64) 2^-24 of that sum of absolute values, the activation 2^-18 of its
  terms. In fp16 an intermediate below the normal range is off by half the smallest step, 2^-25, instead.
* over a whole output, relative to its 2-norm: the intermediates' and the result's roundings are independent and
  each at most u, so a root mean square of u / sqrt(3): sqrt(2 / 3) u together, held to u. Of outputs with fewer
  than 1000 elements, to 1.5 u.
"""
import math

import pytest
import torch

pytestmark = pytest.mark.gpu

E = 2.0 ** -24
U = {torch.float32: 2.0 ** -24, torch.float16: 2.0 ** -11, torch.bfloat16: 2.0 ** -8}
TINY = {torch.float16: 2.0 ** -25, torch.bfloat16: 0.0}

# M, d, hidden: one token upwards; the three tile sizes, whole and broken tiles on each axis, K axes cut and not,
# one 64-deep step and a part of one
SHAPES = [(1, 64, 64), (1, 8, 8), (1, 1024, 2816), (2, 72, 40), (5, 192, 768), (16, 128, 520), (17, 520, 136),
          (33, 384, 1536), (64, 64, 64), (65, 136, 200), (100, 1000, 264), (128, 256, 512), (129, 264, 520),
          (256, 512, 512), (257, 72, 1032), (300, 1032, 72), (700, 320, 2728), (1027, 1000, 2728), (1600, 192, 768),
          (1600, 384, 1536), (2050, 2056, 2048), (4150, 384, 1536)]


def inputs(M, d, hidden, dtype, seed=1):
    g = torch.Generator(device="cuda").manual_seed(1000 * seed + 13 * M + 7 * d + hidden)
    n = lambda *s, std=1.0: (torch.randn(s, generator=g, device="cuda") * std).to(dtype)
    return {"x": n(M, d), "wg": n(hidden, d, std=d ** -0.5), "wv": n(hidden, d, std=d ** -0.5),
            "wo": n(d, hidden, std=hidden ** -0.5), "res": n(M, d), "dy": n(M, d, std=0.5)}


def act64(g, act):
    if act == "silu":
        p = torch.sigmoid(g)
        return g * p, p * (1 + g * (1 - p))
    p = 0.5 * torch.special.erfc(-g / math.sqrt(2))
    return g * p, p + g * torch.exp(-g * g / 2) / math.sqrt(2 * math.pi)


def near(got, want, bound, dtype, roundings=True):
    """bound: the error per element that intermediates and accumulation may make."""
    got, diff = got.double(), (got.double() - want).abs()
    assert torch.isfinite(got).all()
    assert (diff <= bound + U[dtype] * want.abs() + TINY.get(dtype, 0.0)).all()
    if roundings and want.norm() > 0:
        limit = max(U[dtype], U.get(roundings, 0.0)) * (1.0 if want.numel() >= 1000 else 1.5)
        assert diff.norm() <= limit * want.norm(), (float(diff.norm() / want.norm()), limit)


def check_forward(got, s, act, residual=True):
    y, gate, value = got
    dt = s["x"].dtype
    x, wg, wv, wo = (s[k].double() for k in ("x", "wg", "wv", "wo"))
    g, v = x @ wg.t(), x @ wv.t()
    k = (x.shape[-1] + 64) * E
    eg, ev = k * (x.abs() @ wg.abs().t()), k * (x.abs() @ wv.abs().t())
    if gate is not None:
        near(gate, g, eg, dt, dt)
    if value is not None:
        near(value, v, ev, dt, dt)
    a, da = act64(g, act)
    h = a * v
    eh = (eg * 1.2 + 2.0 ** -18 * a.abs() + E) * v.abs() + ev * a.abs() + eg * ev  # |act'| < 1.2
    eh = eh + U[dt] * (h.abs() + eh) + TINY[dt]
    want = h @ wo.t()
    bound = eh @ wo.abs().t() + (wo.shape[1] + 64) * E * (h.abs() @ wo.abs().t())
    if residual:
        want = want + s["res"].double()
    near(y, want, bound, dt, dt)


def check_backward(got, s, gate, value, act, dw_dtype=None, before=None):
    dx, dwg, dwv, dwo = got
    dt = s["x"].dtype
    x, wg, wv, wo, dy = (s[k].double() for k in ("x", "wg", "wv", "wo", "dy"))
    g, v = gate.double(), value.double()
    a, da = act64(g, act)
    dh = dy @ wo
    edh = (wo.shape[0] + 64) * E * (dy.abs() @ wo.abs())
    rnd = lambda t, e: e + U[dt] * (t.abs() + e) + TINY[dt]
    slope = 2.0 ** -18 * (1 + g.abs())  # of the slope and of the activation
    dg, dv, h = dh * v * da, dh * a, a * v
    edg = rnd(dg, edh * (v * da).abs() + dh.abs() * v.abs() * slope)
    edv = rnd(dv, edh * a.abs() + dh.abs() * slope)
    eh = rnd(h, v.abs() * slope)
    M, hid = g.shape
    if dx is not None:
        acc = (2 * hid + 64) * E
        near(dx, dg @ wg + dv @ wv, edg @ wg.abs() + edv @ wv.abs() + acc * (dg.abs() @ wg.abs() + dv.abs() @ wv.abs()),
             dt, dt)
    wt, acc = dw_dtype or dt, (M + 64) * E
    for i, (t, p, ep, q) in enumerate(((dwg, dg, edg, x), (dwv, dv, edv, x), (dwo, h, eh, dy))):
        if t is None:
            continue
        want, err = p.t() @ q, ep.t() @ q.abs() + acc * (p.abs().t() @ q.abs())
        if i == 2:
            want, err = want.t(), err.t()
        if before is not None:
            want = want + before[i].double()
        near(t, want, err, wt, dt)


@pytest.mark.parametrize("dtype,act", [(torch.float16, "silu"), (torch.bfloat16, "gelu"), (torch.bfloat16, "silu")])
@pytest.mark.parametrize("M,d,hidden", SHAPES)
def test_both_passes(gtr, M, d, hidden, dtype, act):
    s = inputs(M, d, hidden, dtype)
    got = gtr.gtr_ffn_fwd(s["x"], s["wg"], s["wv"], s["wo"], act=act, residual=s["res"], save=True)
    check_forward(got, s, act)
    back = gtr.gtr_ffn_bwd(s["dy"], s["x"], s["wg"], s["wv"], s["wo"], got[1], got[2], act=act)
    check_backward(back, s, got[1], got[2], act)


@pytest.mark.parametrize("M,d,hidden", [(1, 64, 128), (50, 136, 264), (1100, 256, 520)])
def test_options(gtr, M, d, hidden):
    """No residual, nothing kept, parts not wanted, float32 gradients, gradients added to, leading dimensions."""
    dt = torch.bfloat16
    s = inputs(M, d, hidden, dt, 2)
    w = (s["wg"], s["wv"], s["wo"])
    got = gtr.gtr_ffn_fwd(s["x"], *w)
    assert got[1] is None and got[2] is None
    check_forward(got, s, "silu", residual=False)
    x3 = s["x"].reshape(1, M, 1, d)
    y3, g3, v3 = gtr.gtr_ffn_fwd(x3, *w, save=True)
    assert y3.shape == x3.shape and g3.shape == (1, M, 1, hidden) and torch.equal(y3.reshape(M, d), got[0])
    one = torch.empty(M, hidden, dtype=dt, device="cuda")
    r = s["res"].clone()
    y, g, v = gtr.gtr_ffn_fwd(s["x"], *w, residual=r, out=r, value=one)  # in place, one projection kept
    assert g is None and torch.equal(one, v3.reshape(M, hidden)) and y is r
    check_forward((y, None, None), s, "silu")
    g, v = g3.reshape(M, hidden), v3.reshape(M, hidden)
    full = gtr.gtr_ffn_bwd(s["dy"], s["x"], *w, g, v)
    only = gtr.gtr_ffn_bwd(s["dy"], s["x"], *w, g, v, want_dw=False)
    assert only[1:] == (None, None, None) and torch.equal(only[0], full[0])
    only = gtr.gtr_ffn_bwd(s["dy"], s["x"], *w, g, v, want_dx=False)
    assert only[0] is None and all(torch.equal(a, b) for a, b in zip(only[1:], full[1:]))
    for wt in (torch.float32, dt):
        f32 = gtr.gtr_ffn_bwd(s["dy"], s["x"], *w, g, v, dw_dtype=wt)
        assert all(t.dtype == wt for t in f32[1:])
        check_backward(f32, s, g, v, "silu", wt)
        sums = [torch.randn_like(t) for t in f32[1:]]
        before = [t.clone() for t in sums]
        added = gtr.gtr_ffn_bwd(s["dy"], s["x"], *w, g, v, dw_gate=sums[0], dw_value=sums[1], dw_out=sums[2],
                                accumulate=True)
        assert added[1] is sums[0]
        check_backward(added, s, g, v, "silu", wt, before)


def test_rows_do_not_meet(gtr):
    """A token's output depends on that token alone: NaN and infinity in one, and in no other."""
    M, d, hidden = 130, 200, 328
    s = inputs(M, d, hidden, torch.float16, 3)
    w = (s["wg"], s["wv"], s["wo"])
    want = gtr.gtr_ffn_fwd(s["x"], *w, residual=s["res"], save=True)
    x = s["x"].clone()
    x[7, 199], x[64, 0] = float("nan"), float("inf")
    got = gtr.gtr_ffn_fwd(x, *w, residual=s["res"], save=True)
    keep = [i for i in range(M) if i not in (7, 64)]
    for a, b in zip(got, want):
        assert torch.equal(a[keep], b[keep]) and not torch.isfinite(a[7]).any()
    dy = s["dy"].clone()
    dy[9, 3] = float("nan")
    back = gtr.gtr_ffn_bwd(dy, s["x"], *w, want[1], want[2], want_dw=False)[0]
    ref = gtr.gtr_ffn_bwd(s["dy"], s["x"], *w, want[1], want[2], want_dw=False)[0]
    keep = [i for i in range(M) if i != 9]
    assert torch.equal(back[keep], ref[keep]) and back[9].isnan().all()


def test_memory_around_the_outputs_stays(gtr):
    """Tiles reach past the last row and the last column; nothing is written there."""
    M, d, hidden = 67, 136, 72
    s = inputs(M, d, hidden, torch.bfloat16, 4)

    def framed(rows, cols):
        t = torch.full((rows + 2, cols), 5.0, dtype=torch.bfloat16, device="cuda")
        return t, t[1:-1]

    (y, y_), (g, g_), (v, v_), (dx, dx_) = framed(M, d), framed(M, hidden), framed(M, hidden), framed(M, d)
    (a, a_), (b, b_), (c, c_) = framed(hidden, d), framed(hidden, d), framed(d, hidden)
    w = (s["wg"], s["wv"], s["wo"])
    gtr.gtr_ffn_fwd(s["x"], *w, out=y_, gate=g_, value=v_)
    gtr.gtr_ffn_bwd(s["dy"], s["x"], *w, g_, v_, out=dx_, dw_gate=a_, dw_value=b_, dw_out=c_)
    for t in (y, g, v, dx, a, b, c):
        assert (t[0] == 5).all() and (t[-1] == 5).all()
    check_forward((y_, g_, v_), s, "silu", residual=False)
    check_backward((dx_, a_, b_, c_), s, g_, v_, "silu")


def test_extreme_projections(gtr):
    """Activations far out on both sides: act and its slope go to 0 and to the identity, without NaN."""
    for act in ("silu", "gelu"):
        s = inputs(64, 64, 64, torch.bfloat16, 5)
        gate = torch.linspace(-300, 300, 64 * 64, device="cuda").reshape(64, 64).bfloat16()
        value = torch.randn(64, 64, device="cuda").bfloat16()
        back = gtr.gtr_ffn_bwd(s["dy"], s["x"], s["wg"], s["wv"], s["wo"], gate, value, act=act)
        check_backward(back, s, gate, value, act)


def test_gradients_against_differences(gtr):
    """The loss sum r y of the formula in 64 bits, differenced along random directions of x and the weights. The
    gradients are off by at most u of their 2-norm (above), along a direction of independent normal entries by u
    times a normal number: under 5 u of the 2-norm; and the projections kept are off by u, which moves the gradients
    by under 2 u more. The quotient's own error (step 1e-4) is under 1e-6."""
    M, d, hidden, h = 40, 72, 136, 1e-4
    for act in ("silu", "gelu"):
        s = inputs(M, d, hidden, torch.float16, 6)
        p = (s["x"], s["wg"], s["wv"], s["wo"])
        _, g, v = gtr.gtr_ffn_fwd(*p, act=act, save=True)
        grads = gtr.gtr_ffn_bwd(s["dy"], *p, g, v, act=act)

        def loss(q):
            return (act64(q[0] @ q[1].t(), act)[0] * (q[0] @ q[2].t()) @ q[3].t() * s["dy"].double()).sum()

        for k in range(4):
            step = torch.randn(p[k].shape, device="cuda", dtype=torch.float64)
            at = lambda e: [t.double() + (e * h * step if i == k else 0) for i, t in enumerate(p)]
            quotient = (loss(at(1)) - loss(at(-1))) / (2 * h)
            along = (grads[k].double() * step).sum()
            assert (quotient - along).abs() <= 7 * 2.0 ** -11 * grads[k].double().norm() + 1e-6


@pytest.mark.parametrize("M,d,hidden", [(3, 64, 136), (600, 384, 1536), (1500, 1024, 1032)])
def test_repeatable_streams_and_graph(gtr, M, d, hidden):
    """The same call again, on another stream, and replayed from a graph between eager calls: bit for bit."""
    dt = torch.bfloat16
    s = inputs(M, d, hidden, dt, 7)

    def run(t, **kw):
        f = gtr.gtr_ffn_fwd(t["x"], t["wg"], t["wv"], t["wo"], residual=t["res"], save=True, **kw)
        return (*f, *gtr.gtr_ffn_bwd(t["dy"], t["x"], t["wg"], t["wv"], t["wo"], f[1], f[2], **kw))

    want = run(s)
    assert all(torch.equal(a, b) for a, b in zip(run(s), want))
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    got = run(s, stream=side)
    side.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(got, want))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        held = run(s)
    for seed in (8, 9, 10):
        new = inputs(M, d, hidden, dt, seed)
        for k in s:
            s[k].copy_(new[k])
        graph.replay()
        torch.cuda.synchronize()
        eager = run(new)
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(held, eager))


def test_two_streams_at_once(gtr):
    """Two calls in flight on two streams, without a workspace of the caller's: each has scratch memory of its own."""
    sets = [inputs(1200, 512, 1024, torch.float16, k) for k in (11, 12)]
    call = lambda s, st=None: gtr.gtr_ffn_fwd(s["x"], s["wg"], s["wv"], s["wo"], residual=s["res"], stream=st)[0]
    want = [call(s) for s in sets]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    for _ in range(5):
        got = [call(s, st) for s, st in zip(sets, streams)]
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(got, want))


def test_offsets_past_32_bits(gtr):
    """Rows that end past 2^31 elements and 2^32 bytes: the last ones as on their own (products of the same tiles:
    the sums of one tile size are in one order)."""
    M, d, hidden = 1_100_000, 64, 2048
    dt = torch.float16
    s = inputs(1024, d, hidden, dt, 13)
    x = torch.randn(1024, d, device="cuda").to(dt).repeat(M // 1024 + 1, 1)[:M].contiguous()
    y, g, v = gtr.gtr_ffn_fwd(x, s["wg"], s["wv"], s["wo"], save=True)
    at = (M - 2048) // 1024 * 1024
    assert torch.equal(y[:1024], y[at:at + 1024]) and torch.equal(g[:1024], g[at:at + 1024])
    assert torch.equal(y[at + 1024:], y[:M - at - 1024])
    part = {**s, "x": x[:512]}
    check_forward((y[:512], g[:512], v[:512]), part, "silu", residual=False)
    dx = gtr.gtr_ffn_bwd(x, x, s["wg"], s["wv"], s["wo"], g, v, want_dw=False)[0]
    assert torch.equal(dx[:1024], dx[at:at + 1024]) and torch.equal(dx[at + 1024:], dx[:M - at - 1024])
    dw = gtr.gtr_ffn_bwd(x, x, s["wg"], s["wv"], s["wo"], g, v, want_dx=False, dw_dtype=torch.float32)[1:]
    # whole repeats of 1024 rows, and a rest: M / 1024 times one's gradient and the rest's
    rows = M // 1024
    one = gtr.gtr_ffn_bwd(x[:1024], x[:1024], s["wg"], s["wv"], s["wo"], g[:1024], v[:1024], want_dx=False,
                          dw_dtype=torch.float32)[1:]
    rest = M - rows * 1024
    left = gtr.gtr_ffn_bwd(x[:rest], x[:rest], s["wg"], s["wv"], s["wo"], g[:rest], v[:rest], want_dx=False,
                           dw_dtype=torch.float32)[1:]
    for a, b, c in zip(dw, one, left):
        want = b.double() * rows + c.double()
        # float32 sums of 1.1 million terms: at most M 2^-24 of the sum of absolute values, far less in the 2-norm
        assert (a.double() - want).norm() <= 2e-4 * want.norm()


def test_the_binding_refuses(gtr):
    """Shapes, types, layouts and devices that the operators do not take raise before anything runs."""
    s = inputs(24, 64, 128, torch.float16, 14)
    w = (s["wg"], s["wv"], s["wo"])
    x, dy = s["x"], s["dy"]
    _, g, v = gtr.gtr_ffn_fwd(x, *w, save=True)
    m = torch.zeros(24, device="cuda")
    fwd = lambda *a, **k: (lambda: gtr.gtr_ffn_fwd(*a, **k))
    bwd = lambda *a, **k: (lambda: gtr.gtr_ffn_bwd(*a, **k))
    lnf = lambda *a, **k: (lambda: gtr.gtr_layernorm_fwd(*a, **k))
    lnb = lambda *a, **k: (lambda: gtr.gtr_layernorm_bwd(*a, **k))
    for call in (
            fwd(x.float(), *w), fwd(x, s["wg"].bfloat16(), *w[1:]), fwd(x, s["wg"], s["wv"][:64], s["wo"]),
            fwd(x, s["wg"], s["wv"], s["wo"].t()), fwd(x[:, :32], *w), fwd(x.t(), *w), fwd(x, *w, act="relu"),
            fwd(x, *w, residual=x[:12]), fwd(x, *w, gate=g[:, :64]), fwd(x, *w, out=dy.float()), fwd(x.cpu(), *w),
            fwd(x, s["wg"].cpu(), *w[1:]), fwd(x, s["wg"][0, 0], *w[1:]),
            bwd(dy[:12], x, *w, g, v), bwd(dy, x, *w, g.t(), v), bwd(dy, x, *w, g, v[:12]),
            bwd(dy, x, *w, g, v, dw_dtype=torch.bfloat16), bwd(dy, x, *w, g, v, accumulate=True),
            bwd(dy, x, *w, g, v, dw_gate=torch.zeros_like(s["wo"])), bwd(dy, x, *w, g, v, act="none"),
            lnf(x.double()), lnf(x.t()), lnf(x, m), lnf(x, torch.ones(64, device="cuda").half()), lnf(x, mean=m[:3]),
            lnb(dy, x.float(), m, m), lnb(dy, x, m[:5], m), lnb(dy, x, m, m, dres=dy.float()),
            lnb(dy, x, m, m, accumulate=True), lnb(dy, x, m, m, dw=torch.zeros(65, device="cuda"))):
        with pytest.raises(ValueError):
            call()
    for call in (fwd(x[:0], *w), lnf(x[:0]), fwd(x, *w, out=x), bwd(dy, x, *w, g, v, out=dy), fwd(x, *w, gate=g, value=g),
                 lnf(x, eps=-1.0), fwd(torch.zeros(4, 12, device="cuda").half(), torch.zeros(8, 12, device="cuda").half(),
                                       torch.zeros(8, 12, device="cuda").half(), torch.zeros(12, 8, device="cuda").half()),
                 lnf(torch.zeros(2, 16385, device="cuda"))):
        with pytest.raises(gtr.GtrError):
            call()
