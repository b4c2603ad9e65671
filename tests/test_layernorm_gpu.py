"""gtr_layernorm_fwd and gtr_layernorm_bwd on the GPU against the formulas in 64 bits.

Tolerances, per element, from the kernels' arithmetic (e = 2^-24, the rounding of a float32 operation; u, half a
step of the output type; S = 64 + rows / 64, more than the additions that any one sum goes through one after the
other: at most 32 elements per lane and 10 steps across lanes, and in the row sums one addition per row that a
work-group takes):
* mean: 64 e times mean |x|, and through it x_hat: 64 e (|x_hat| + rstd mean |x|) = E;
* y: E |w| + 64 e |b| + u |y|;
* dx: 64 e rstd (|t| + mean |t| + |x_hat| mean |t x_hat|) plus what E makes of it, plus u |dx|;
* dw: S e sum |dy x_hat| + sum |dy| E, db: S e sum |dy|.
"""
import pytest
import torch

pytestmark = pytest.mark.gpu

E = 2.0 ** -24
U = {torch.float32: 2.0 ** -24, torch.float16: 2.0 ** -11, torch.bfloat16: 2.0 ** -8}
EPS = 1e-6

# every way of sharing a row (part of a wave, a wave, a work-group of 256 and of 1024), one vector to four, whole and
# broken vectors; rows that fill a work-group's slots or not
SHAPES = [(1, 1), (3, 7), (5, 64), (1, 128), (17, 129), (33, 192), (64, 255), (1600, 384), (9, 512), (300, 513),
          (7, 1001), (12, 1024), (21, 1536), (2049, 1025), (5, 2047), (3, 2048), (130, 2056), (2, 4096), (259, 4097),
          (4, 8192), (2, 8200), (3, 12293), (2, 16384), (4100, 200)]


def inputs(M, d, dtype, seed, shift=1.0):
    g = torch.Generator(device="cuda").manual_seed(1000 * seed + 7 * M + d)
    n = lambda *s: torch.randn(s, generator=g, device="cuda")
    x = (n(M, d) + shift * n(M, 1)).to(dtype)
    return x, 1 + 0.1 * n(d), 0.1 * n(d), (0.5 * n(M, d)).to(dtype), (0.5 * n(M, d)).to(dtype)


def forward64(x, w, b, eps=EPS):
    x = x.double()
    mean = x.mean(-1, keepdim=True)
    rstd = ((x - mean).square().mean(-1, keepdim=True) + eps).rsqrt()
    h = (x - mean) * rstd
    w = torch.ones(x.shape[-1], device=x.device).double() if w is None else w.double()
    b = torch.zeros(x.shape[-1], device=x.device).double() if b is None else b.double()
    err = 64 * E * (h.abs() + rstd * x.abs().mean(-1, keepdim=True))
    return h * w + b, mean[..., 0], rstd[..., 0], h, err, w, b


def check_forward(got, x, w, b, eps=EPS):
    y, mean, rstd = got
    ry, rm, rr, h, err, w, b = forward64(x, w, b, eps)
    assert ((y.double() - ry).abs() <= err * w.abs() + 64 * E * b.abs() + U[x.dtype] * ry.abs()).all()
    assert ((mean.double() - rm).abs() <= 64 * E * x.double().abs().mean(-1)).all()
    # 1 / rstd^2 = var + eps: its error is at most 64 e of it plus the square of the mean's
    assert ((rstd.double() - rr).abs() <= rr * (64 * E + (rr * 64 * E * x.double().abs().mean(-1)) ** 2)).all()


def check_backward(got, dy, x, w, dres, before=None):
    dx, dw, db = got
    M, d = x.reshape(-1, x.shape[-1]).shape
    _, _, rstd, h, err, w, _ = forward64(x, w, None)
    rstd, y = rstd[..., None], dy.double()
    t = y * w
    mean = lambda v: v.mean(-1, keepdim=True)
    m1, m2 = mean(t), mean(t * h)
    rdx = rstd * (t - m1 - h * m2)
    if dres is not None:
        rdx = rdx + dres.double()
    if dx is not None:
        tol = 64 * E * rstd * (t.abs() + mean(t.abs()) + h.abs() * mean((t * h).abs()))
        tol = tol + rstd * (err * m2.abs() + h.abs() * mean(t.abs() * err)) + 64 * E * rdx.abs()
        if dres is not None:
            tol = tol + 2 * E * dres.double().abs()
        assert ((dx.double() - rdx).abs() <= tol + U[x.dtype] * rdx.abs()).all()
    if dw is not None:
        S = 64 + M / 64
        flat = lambda v: v.reshape(M, d)
        add = (0, 0) if before is None else tuple(v.double() for v in before)
        rdw, rdb = flat(y * h).sum(0) + add[0], flat(y).sum(0) + add[1]
        assert ((dw.double() - rdw).abs() <= S * E * flat((y * h).abs()).sum(0) + flat(y.abs() * err).sum(0) +
                2 * E * rdw.abs()).all()
        assert ((db.double() - rdb).abs() <= S * E * flat(y.abs()).sum(0) + 2 * E * rdb.abs()).all()


@pytest.mark.parametrize("dtype", [torch.float32, torch.float16, torch.bfloat16])
@pytest.mark.parametrize("M,d", SHAPES)
def test_both_passes(gtr, M, d, dtype):
    x, w, b, dy, dres = inputs(M, d, dtype, 1)
    got = gtr.gtr_layernorm_fwd(x, w, b, eps=EPS)
    check_forward(got, x, w, b)
    back = gtr.gtr_layernorm_bwd(dy, x, got[1], got[2], w, dres=dres)
    check_backward(back, dy, x, w, dres)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_options(gtr, dtype):
    """No affine weights, parts that are not wanted, sums that are added to, leading dimensions."""
    x, w, b, dy, dres = inputs(3 * 11, 200, dtype, 2)
    x, dy, dres = (t.reshape(3, 11, 200) for t in (x, dy, dres))
    got = gtr.gtr_layernorm_fwd(x)
    assert got[0].shape == x.shape and got[1].shape == (3, 11)
    check_forward(got, x, None, None)
    check_backward(gtr.gtr_layernorm_bwd(dy, x, got[1], got[2]), dy, x, None, None)
    only = gtr.gtr_layernorm_bwd(dy, x, got[1], got[2], w, want_dw=False, dres=dres)
    assert only[1] is None and only[2] is None
    check_backward(only, dy, x, w, dres)
    only = gtr.gtr_layernorm_bwd(dy, x, got[1], got[2], w, want_dx=False)
    assert only[0] is None
    check_backward(only, dy, x, w, None)
    dw, db = torch.randn(200, device="cuda"), torch.randn(200, device="cuda")
    before = dw.clone(), db.clone()
    back = gtr.gtr_layernorm_bwd(dy, x, got[1], got[2], w, dw=dw, db=db, accumulate=True)
    assert back[1] is dw
    check_backward(back, dy, x, w, None, before)


@pytest.mark.parametrize("M,d", [(40, 384), (6, 3001), (3, 12293)])
@pytest.mark.parametrize("dtype", [torch.float32, torch.float16])
def test_in_place_and_repeatable(gtr, M, d, dtype):
    """The output over each input that it may be, bit for bit as beside them (the weights' gradients, which are summed
    another way where dx overwrites what they are formed from, within their bounds); the same call again, bit for bit."""
    x, w, b, dy, dres = inputs(M, d, dtype, 3)
    y, mean, rstd = gtr.gtr_layernorm_fwd(x, w, b)
    assert torch.equal(gtr.gtr_layernorm_fwd(z := x.clone(), w, b, out=z)[0], y)
    want = gtr.gtr_layernorm_bwd(dy, x, mean, rstd, w, dres=dres)
    for k in range(3):
        t = [dy.clone(), x.clone(), dres.clone()]
        got = gtr.gtr_layernorm_bwd(t[0], t[1], mean, rstd, w, dres=t[2], out=t[k])
        assert torch.equal(got[0], want[0])
        check_backward(got, dy, x, w, dres)
    again = gtr.gtr_layernorm_bwd(dy, x, mean, rstd, w, dres=dres)
    assert all(torch.equal(a, b) for a, b in zip(again, want))


@pytest.mark.parametrize("shift", [100.0, 3000.0])
def test_far_from_zero(gtr, shift):
    """Rows whose mean is large next to their spread."""
    x, w, b, dy, _ = inputs(50, 768, torch.float32, 4, shift)
    got = gtr.gtr_layernorm_fwd(x, w, b)
    check_forward(got, x, w, b)


def test_constant_rows_and_rows_beyond(gtr):
    """Rows of equal values give the bias and no gradient through the statistics; memory around the rows stays."""
    M, d = 5, 101
    big = torch.full((M + 2, d), 7.0, dtype=torch.float16, device="cuda")
    out = torch.full((M + 2, d), -3.0, dtype=torch.float16, device="cuda")
    w, b = torch.randn(d, device="cuda"), torch.randn(d, device="cuda")
    y, mean, rstd = gtr.gtr_layernorm_fwd(big[1:-1], w, b, out=out[1:-1])  # rows at odd element offsets
    assert torch.equal(out[1:-1], b.half().expand(M, d)) and (out[0] == -3).all() and (out[-1] == -3).all()
    assert (mean == 7).all() and torch.allclose(rstd, torch.full_like(rstd, 1e3), rtol=1e-6, atol=0)
    dx = torch.full((M + 2, d), 9.0, dtype=torch.float16, device="cuda")
    gtr.gtr_layernorm_bwd(torch.zeros_like(y), big[1:-1], mean, rstd, w, out=dx[1:-1])
    assert (dx[1:-1] == 0).all() and (dx[0] == 9).all() and (dx[-1] == 9).all()


def test_a_row_with_nan_or_infinity_stays_alone(gtr):
    x, w, b, dy, _ = inputs(9, 640, torch.float32, 5)
    clean = gtr.gtr_layernorm_fwd(x, w, b)
    bad = x.clone()
    bad[2, 17], bad[6, 639] = float("nan"), float("inf")
    got = gtr.gtr_layernorm_fwd(bad, w, b)
    keep = [i for i in range(9) if i not in (2, 6)]
    assert torch.equal(got[0][keep], clean[0][keep]) and got[0][2].isnan().all() and got[0][6].isnan().any()
    dx, dw, db = gtr.gtr_layernorm_bwd(dy, bad, got[1], got[2], w)
    want = gtr.gtr_layernorm_bwd(dy, x, clean[1], clean[2], w)
    assert torch.equal(dx[keep], want[0][keep]) and dw.isnan().any() and torch.equal(db, want[2])


def test_gradient_against_differences(gtr):
    """The loss sum r y of the formula in 64 bits, differenced along random directions of x, w and b: with float32
    inputs the analytic gradient differs from the difference quotient by its own error (checked above, under 1e-4 of
    it) and the quotient's, h^2 / 6 times a third derivative of the loss (h 1e-4: under 1e-6)."""
    M, d, h = 6, 150, 1e-4
    x, w, b, r, _ = inputs(M, d, torch.float32, 6)
    _, mean, rstd = gtr.gtr_layernorm_fwd(x, w, b)
    grads = gtr.gtr_layernorm_bwd(r, x, mean, rstd, w)
    loss = lambda p: (forward64(*p)[0] * r.double()).sum()
    for k in range(3):
        step = torch.randn_like((x, w, b)[k]).double()
        at = lambda s: [t.double() + (s * h * step if i == k else 0) for i, t in enumerate((x, w, b))]
        quotient = (loss(at(1)) - loss(at(-1))) / (2 * h)
        along = (grads[k].double() * step).sum()
        assert (quotient - along).abs() <= 1e-4 * grads[k].double().norm() * 5


def test_streams_and_graph(gtr):
    """On a stream given, and recorded into a graph that is replayed between eager calls."""
    x, w, b, dy, dres = inputs(700, 1000, torch.bfloat16, 7)
    want_f = gtr.gtr_layernorm_fwd(x, w, b)
    want_b = gtr.gtr_layernorm_bwd(dy, x, want_f[1], want_f[2], w, dres=dres)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    got_f = gtr.gtr_layernorm_fwd(x, w, b, stream=side)
    got_b = gtr.gtr_layernorm_bwd(dy, x, got_f[1], got_f[2], w, dres=dres, stream=side)
    side.synchronize()
    assert all(torch.equal(a, b) for a, b in zip((*got_f, *got_b), (*want_f, *want_b)))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        f = gtr.gtr_layernorm_fwd(x, w, b)
        g = gtr.gtr_layernorm_bwd(dy, x, f[1], f[2], w, dres=dres)
    for seed in (8, 9, 10):
        new = inputs(700, 1000, torch.bfloat16, seed)
        for t, s in zip((x, w, b, dy, dres), new):
            t.copy_(s)
        graph.replay()
        torch.cuda.synchronize()
        ef = gtr.gtr_layernorm_fwd(*new[:3])
        eb = gtr.gtr_layernorm_bwd(new[3], new[0], ef[1], ef[2], new[1], dres=new[4])
        torch.cuda.synchronize()
        assert all(torch.equal(p, q) for p, q in zip((*f, *g), (*ef, *eb)))


def test_more_than_2_31_elements(gtr):
    """Offsets past 32 bits: 140,000 rows of 16384 (2.3e9 elements); the last rows as on their own."""
    M, d = 140000, 16384
    x = torch.empty(M, d, dtype=torch.float16, device="cuda")
    x[:] = torch.randn(d, device="cuda").half()
    x[-40:] = torch.randn(40, d, device="cuda").half()
    y, mean, rstd = gtr.gtr_layernorm_fwd(x)
    tail = gtr.gtr_layernorm_fwd(x[-40:].clone())
    assert torch.equal(y[-40:], tail[0]) and torch.equal(mean[-40:], tail[1]) and torch.equal(y[0], y[M - 41])
    dx = gtr.gtr_layernorm_bwd(y, x, mean, rstd, want_dw=False)[0]
    assert torch.equal(dx[-40:], gtr.gtr_layernorm_bwd(tail[0], x[-40:].clone(), tail[1], tail[2], want_dw=False)[0])
