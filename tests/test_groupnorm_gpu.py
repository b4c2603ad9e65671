"""gtr_groupnorm_fwd and gtr_groupnorm_bwd on the GPU against the formulas in 64 bits.

Tolerances, per element, from the kernels' arithmetic (e = 2^-24, the rounding of a float32 operation; u, half a step of
the output type). No sum goes through more than S = 330 + L / 256 additions one after the other (a lane's rows, at most
n = 16 + L / 256 at these sizes; 16 waves, 8 channels of a team's thread and 6 steps across its threads; at most 256
tiles). D is the largest |x - mean| of a group, A its largest |x|:
* mean: S e (2 D + mean |x|) + 2 e A (sums about one of the values, which is at most 2 D from any);
* var, relative: (S + 2 n^2) e (a lane's sum of squares about one of its n values is at most 2 (n + 1) times that about
  their mean) + 8 (e A + 2 n e D) rstd (the lanes' means against the group's) + (mean's error rstd)^2; rstd: half of it
  and 4 e;
* xh: rstd (mean's error + 2 e |x|) + |xh| (rstd's + 3 e) = Ex; xh w + b: Ex |w| + 2 e (|xh w| + |b|) = Eu;
* act: 1.13 Eu (its steepest slope) and its own error, of |y|: SiLU (|u| + 6) e; GELU 10^-6 + (1.25 u^2 + 4) e; both 0
  where the exponential leaves float32's range (10^-35);
* its slope: 0.8 Eu (the largest second derivative) + (4 |u| + 10) e + 2 10^-6 for GELU; du: |dy| times that = Ed;
* dw: sum of Ed |xh| + |du| Ex, and (S + 300) e sum |du xh|; db likewise;
* dx: what Ed, Ex and the means' errors make of rstd (t - m1 - xh m2), and 8 e of its terms.
"""
import pytest
import torch

pytestmark = pytest.mark.gpu

E = 2.0 ** -24
U = {torch.float32: 2.0 ** -24, torch.float16: 2.0 ** -11, torch.bfloat16: 2.0 ** -8}
TINY = {torch.float32: 2.0 ** -149, torch.float16: 2.0 ** -25, torch.bfloat16: 2.0 ** -133}
EPS = 1e-5
ACTS = (None, "silu", "gelu")

# images, tokens, channels, groups: one token, one channel, fewer channels than a vector; groups that vectors cut, in
# blocks of several and blocks that the last one breaks; groups wider than a block; images in one work-group's
# registers (one vector per thread to all) and in tiles, whole and broken
SHAPES = [(1, 1, 1, 1), (2, 1, 64, 4), (3, 5, 3, 1), (1, 70, 6, 3), (2, 9, 8, 8), (1, 256, 192, 32), (2, 49, 100, 5),
          (1, 1600, 192, 32), (3, 851, 330, 6), (2, 300, 33, 33), (1, 4099, 40, 4), (2, 64, 1024, 2), (1, 33, 4100, 2),
          (1, 7000, 16, 1), (2, 17, 2600, 650), (5, 130, 72, 9), (1, 2, 16384, 1), (40, 36, 96, 8), (2, 2500, 513, 1),
          (1, 1, 3001, 3001), (2, 513, 993, 993)]


def inputs(B, L, C, dtype, seed, shift=1.0):
    g = torch.Generator(device="cuda").manual_seed(100003 * seed + 17 * L + C)
    n = lambda *s, std=1.0, mu=0.0: torch.randn(s, generator=g, device="cuda") * std + mu
    return dict(x=(n(B, L, C) + shift * n(B, 1, C)).to(dtype), w=n(C, std=0.1, mu=1.0), b=n(C, std=0.1),
                dy=n(B, L, C, std=0.5).to(dtype), dres=n(B, L, C, std=0.5).to(dtype))


class Exact:
    def __init__(self, x, w, b, groups, act, eps=EPS):
        B, L, C = x.shape
        x = x.double()
        self.split = lambda v: v.reshape(B, L, groups, C // groups)
        self.join = lambda v: v.reshape(B, L, C)
        self.over = lambda v, f: f(self.split(v), (1, 3))
        self.wide = lambda v: v.repeat_interleave(C // groups, 1)[:, None]
        self.S, n = 330 + L / 256, 16 + L / 256
        mean = self.over(x, torch.mean)
        c = x - self.wide(mean)
        var = self.over(c * c, torch.mean)
        rstd = (var + eps).rsqrt()
        D, A = self.over(c.abs(), torch.amax), self.over(x.abs(), torch.amax)
        self.emean = self.S * E * (2 * D + self.over(x.abs(), torch.mean)) + 2 * E * A
        evar = (self.S + 2 * n * n) * E + 8 * (E * A + 2 * n * E * D) * rstd + (self.emean * rstd) ** 2
        self.erstd = rstd * (0.5 * evar + 4 * E)
        self.mean, self.rstd = mean, rstd
        self.w = torch.ones(C, device=x.device).double() if w is None else w.double()
        self.b = torch.zeros(C, device=x.device).double() if b is None else b.double()
        r = self.wide(rstd)
        self.xh = c * r
        self.ex = r * (self.wide(self.emean) + 2 * E * x.abs()) + self.xh.abs() * (self.wide(self.erstd) / r + 3 * E)
        u = self.u = self.xh * self.w + self.b
        self.eu = self.ex * self.w.abs() + 2 * E * ((self.xh * self.w).abs() + self.b.abs())
        s, P = torch.sigmoid(u), torch.special.ndtr(u)
        if act is None:
            self.y, self.slope, own, eslope = u, torch.ones_like(u), 0.0, 0.0
        elif act == "silu":
            self.y, self.slope = u * s, s * (1 + u * (1 - s))
            own, eslope = (u.abs() + 6) * E, (4 * u.abs() + 10) * E
        else:
            self.y, self.slope = u * P, P + u * torch.exp(-0.5 * u * u) * 0.3989422804014327
            own, eslope = 1e-6 + (1.25 * u * u + 4) * E, (4 * u.abs() + 10) * E + 2e-6
        self.ey = 1.13 * self.eu + own * self.y.abs() + (1e-35 if act else 0.0)
        self.eslope = 0.8 * self.eu + eslope if act else torch.zeros_like(u)


def close(got, want, err, u, tiny=0.0):
    bad = ~((got.double() - want).abs() <= err + u * (want.abs() + err) + tiny)
    assert not bad.any(), (int(bad.sum()), float(((got.double() - want).abs() / (err + u * want.abs() + tiny)).max()))


def check_forward(got, i, groups, act, w=True, eps=EPS):
    y, mean, rstd = got
    k = Exact(i["x"], i["w"] if w else None, i["b"] if w else None, groups, act, eps)
    assert mean.shape == rstd.shape == (i["x"].shape[0], groups) and mean.dtype == rstd.dtype == torch.float32
    close(mean, k.mean, k.emean, 0.0)
    close(rstd, k.rstd, k.erstd, 0.0)
    close(y, k.y, k.ey, U[y.dtype], TINY[y.dtype])


def check_backward(got, i, groups, act, res=True, w=True, before=None):
    dx, dw, db = got
    k = Exact(i["x"], i["w"] if w else None, i["b"] if w else None, groups, act)
    dy = i["dy"].double()
    du, ed = dy * k.slope, dy.abs() * (k.eslope + 2 * E * k.slope.abs())
    t, et = du * k.w, ed * k.w.abs() + E * (du * k.w).abs()
    mean = lambda v: k.wide(k.over(v, torch.mean))
    m1, m2 = mean(t), mean(t * k.xh)
    em1 = mean(et) + k.S * E * mean(t.abs())
    em2 = mean(et * k.xh.abs() + t.abs() * k.ex) + k.S * E * mean((t * k.xh).abs())
    r = k.wide(k.rstd)
    want = r * (t - m1 - k.xh * m2)
    err = r * (et + em1 + k.xh.abs() * em2 + k.ex * m2.abs()) + k.wide(k.erstd) / r * want.abs()
    err = err + 8 * E * r * (t.abs() + m1.abs() + (k.xh * m2).abs())
    if res:
        want = want + i["dres"].double()
        err = err + 2 * E * i["dres"].double().abs()
    if dx is not None:
        close(dx, want, err, U[dx.dtype], TINY[dx.dtype])
    if dw is not None:
        S = k.S + 300
        add = (0.0, 0.0) if before is None else tuple(v.double() for v in before)
        rdw, rdb = (du * k.xh).sum((0, 1)) + add[0], du.sum((0, 1)) + add[1]
        close(dw, rdw, S * E * (du * k.xh).abs().sum((0, 1)) + (ed * k.xh.abs() + du.abs() * k.ex).sum((0, 1)), 2 * E)
        close(db, rdb, S * E * du.abs().sum((0, 1)) + ed.sum((0, 1)), 2 * E)


@pytest.mark.parametrize("dtype", [torch.float32, torch.float16, torch.bfloat16])
@pytest.mark.parametrize("n,shape", list(enumerate(SHAPES)))
def test_both_passes(gtr, n, shape, dtype):
    B, L, C, G = shape
    i = inputs(B, L, C, dtype, 1)
    for act in (ACTS[n % 3], ACTS[(n + 1) % 3]):
        got = gtr.gtr_groupnorm_fwd(i["x"], G, i["w"], i["b"], act=act, eps=EPS)
        check_forward(got, i, G, act)
        res = i["dres"] if n % 2 else None
        back = gtr.gtr_groupnorm_bwd(i["dy"], i["x"], got[1], got[2], i["w"], i["b"], act=act, dres=res)
        check_backward(back, i, G, act, res is not None)


@pytest.mark.parametrize("dtype", [torch.float32, torch.float16])
@pytest.mark.parametrize("B,L,C,G", [(4096, 4, 384, 32), (3000, 1, 40, 4), (700, 16, 96, 8)])
def test_many_images_of_a_few_tokens(gtr, B, L, C, G, dtype):
    """dw and db from an image's sums each: 8 threads per column add B / 8 of them, so that no sum goes through more than
    B / 8 + 100 additions one after the other (fewer than the 630 of the bounds)."""
    i = inputs(B, L, C, dtype, 18)
    got = gtr.gtr_groupnorm_fwd(i["x"], G, i["w"], i["b"], act="silu", eps=EPS)
    check_forward(got, i, G, "silu")
    back = gtr.gtr_groupnorm_bwd(i["dy"], i["x"], got[1], got[2], i["w"], i["b"], act="silu", dres=i["dres"])
    check_backward(back, i, G, "silu")


@pytest.mark.parametrize("B,L,C,G", [(3, 100, 48, 6), (2, 5000, 72, 8)])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_options(gtr, B, L, C, G, dtype):
    """No affine weights, parts that are not wanted, sums that are added to, a grid of two dimensions."""
    i = inputs(B, L, C, dtype, 2)
    grid = {k: i[k].reshape(B, L // 10, 10, C) for k in ("x", "dy", "dres")}
    got = gtr.gtr_groupnorm_fwd(grid["x"], G, act="silu")
    assert got[0].shape == grid["x"].shape
    check_forward((got[0].reshape(B, L, C), *got[1:]), i, G, "silu", w=False)
    back = gtr.gtr_groupnorm_bwd(grid["dy"], grid["x"], got[1], got[2], act="silu")
    check_backward((back[0].reshape(B, L, C), *back[1:]), i, G, "silu", res=False, w=False)
    got = gtr.gtr_groupnorm_fwd(i["x"], G, i["w"], i["b"], act="gelu")
    args = (i["dy"], i["x"], got[1], got[2], i["w"], i["b"])
    want = gtr.gtr_groupnorm_bwd(*args, act="gelu", dres=i["dres"])
    check_backward(want, i, G, "gelu")
    only = gtr.gtr_groupnorm_bwd(*args, act="gelu", want_dw=False, dres=i["dres"])
    assert only[1] is None and only[2] is None and torch.equal(only[0], want[0])
    only = gtr.gtr_groupnorm_bwd(*args, act="gelu", want_dx=False)
    assert only[0] is None and torch.equal(only[1], want[1]) and torch.equal(only[2], want[2])
    for n in (1, B):  # one image, whose sums need no second launch, and more
        j = {k: (v[:n].contiguous() if v.dim() == 3 else v) for k, v in i.items()}
        dw, db = torch.randn(C, device="cuda"), torch.randn(C, device="cuda")
        before = dw.clone(), db.clone()
        back = gtr.gtr_groupnorm_bwd(j["dy"], j["x"], got[1][:n].contiguous(), got[2][:n].contiguous(), i["w"], i["b"],
                                     act="gelu", dw=dw, db=db, accumulate=True)
        assert back[1] is dw and back[2] is db
        check_backward(back, j, G, "gelu", res=False, before=before)


@pytest.mark.parametrize("B,L,C,G", [(2, 40, 100, 5), (1, 4500, 70, 7), (2, 9, 5, 5)])
@pytest.mark.parametrize("dtype", [torch.float32, torch.float16])
def test_in_place_repeatable_and_nothing_beyond(gtr, B, L, C, G, dtype):
    """The output over each input that it may be, bit for bit as beside them; the same call again; memory around stays."""
    i = inputs(B, L, C, dtype, 3)
    fwd = lambda x, **kw: gtr.gtr_groupnorm_fwd(x, G, i["w"], i["b"], act="silu", **kw)
    y, mean, rstd = fwd(i["x"])
    assert all(torch.equal(a, b) for a, b in zip(fwd(i["x"]), (y, mean, rstd)))
    assert torch.equal(fwd(z := i["x"].clone(), out=z)[0], y)
    room = torch.full((B + 2, L, C), 3.0, dtype=dtype, device="cuda")
    room[1:-1] = i["x"]
    out = torch.full_like(room, 5.0)
    fwd(room[1:-1], out=out[1:-1])
    assert torch.equal(out[1:-1], y) and (out[0] == 5).all() and (out[-1] == 5).all()
    bwd = lambda dy, x, dres, **kw: gtr.gtr_groupnorm_bwd(dy, x, mean, rstd, i["w"], i["b"], act="silu", dres=dres, **kw)
    want = bwd(i["dy"], i["x"], i["dres"])
    assert all(torch.equal(a, b) for a, b in zip(bwd(i["dy"], i["x"], i["dres"]), want))
    for k in range(3):
        t = [i["dy"].clone(), i["x"].clone(), i["dres"].clone()]
        assert all(torch.equal(a, b) for a, b in zip(bwd(*t, out=t[k]), want))
    bwd(i["dy"], i["x"], i["dres"], out=out[1:-1])
    assert torch.equal(out[1:-1], want[0]) and (out[0] == 5).all() and (out[-1] == 5).all()


@pytest.mark.parametrize("shift", [100.0, 3000.0])
@pytest.mark.parametrize("L", [200, 6000])
def test_far_from_zero(gtr, shift, L):
    """Groups whose mean is large next to their spread, and channels far from each other."""
    i = inputs(2, L, 96, torch.float32, 4, 1.0)
    i["x"] += shift
    check_forward(gtr.gtr_groupnorm_fwd(i["x"], 8, i["w"], i["b"], act="silu"), i, 8, "silu")
    i = inputs(2, L, 96, torch.float32, 5, shift)
    check_forward(gtr.gtr_groupnorm_fwd(i["x"], 8, i["w"], i["b"]), i, 8, None)


@pytest.mark.parametrize("L", [50, 9000])
def test_an_outlier_first(gtr, L):
    """The value that a lane's sums are taken about is far from all others."""
    i = inputs(1, L, 64, torch.float32, 6)
    i["x"][0, 0] = 3e4
    check_forward(gtr.gtr_groupnorm_fwd(i["x"], 4, i["w"], i["b"], act="silu"), i, 4, "silu")


@pytest.mark.parametrize("L,C,G,dtype,spread", [(5000, 16, 4, torch.float32, 3e16), (64, 3, 1, torch.float32, 6e17),
                                                (64, 4, 2, torch.bfloat16, 6e17)])
def test_a_mean_whose_square_is_past_float32(gtr, L, C, G, dtype, spread):
    """Means of 3e19, of which the square is no float32, and sums of squares about them that are (at most 2e37)."""
    i = inputs(2, L, C, dtype, 17)
    i["x"] = (3e19 + spread * i["x"].float()).to(dtype)
    check_forward(gtr.gtr_groupnorm_fwd(i["x"], G, i["w"], i["b"]), i, G, None)


@pytest.mark.parametrize("dtype,rows", [(torch.float32, 2048), (torch.bfloat16, 1500), (torch.float32, 403)])
def test_many_equal_values_behind_others(gtr, dtype, rows):
    """The first row of each lane is 0 and its `rows` others c (an image below a border): mean c (1 - p) and variance
    c^2 p (1 - p), p = 1 / (rows + 1). A lane's sums are taken about values that leave at most 4 times its n = rows + 1
    values' sum of squares about their mean, of which the sum of the deviations, squared over n, takes off at most 3:
    n + 2 roundings of each, so (4 + 2 * 3) (n + 2) e, and 60 e for the moves from value to value (10 at each of 6). The
    lanes' means are the group's; sums over them go through S = 330 additions, S e more, and the mean is off by
    (S + 8) e c: relative to the deviation that squared is the variance's. rstd: half of all that and 4 e."""
    C, G, S = 64, 8, 330
    lanes = 256 // (C // (4 if dtype == torch.float32 else 8)) * 256  # of one channel: a work-group's rows, 256 tiles
    n = rows + 1
    c = torch.linspace(0.7, 2.1, G, device="cuda").to(dtype)
    x = c.repeat_interleave(C // G).expand(1, lanes * n, C).contiguous()
    x[:, :lanes] = 0
    _, mean, rstd = gtr.gtr_groupnorm_fwd(x, G, eps=0.0)
    c, p = c.double(), 1.0 / n
    std = c * (p * (1 - p)) ** 0.5
    emean = (S + 8) * E * c
    close(mean[0], c * (1 - p), emean, 0.0)
    close(rstd[0], 1 / std, (0.5 * ((10 * (n + 2) + 60 + S) * E + (emean / std) ** 2) + 4 * E) / std, 0.0)


@pytest.mark.parametrize("L", [21, 5001])
def test_equal_values(gtr, L):
    """A group of equal values gives act(b) and no gradient through the statistics."""
    C, G = 60, 5
    x = torch.full((2, L, C), 7.0, dtype=torch.float16, device="cuda")
    w, b = torch.randn(C, device="cuda"), torch.randn(C, device="cuda")
    y, mean, rstd = gtr.gtr_groupnorm_fwd(x, G, w, b)
    assert torch.equal(y, b.half().expand(2, L, C)) and (mean == 7).all()
    assert torch.allclose(rstd, torch.full_like(rstd, 1e5 ** 0.5), rtol=1e-6, atol=0)
    dx, dw, db = gtr.gtr_groupnorm_bwd(torch.zeros_like(x), x, mean, rstd, w, b)
    assert (dx == 0).all() and (dw == 0).all() and (db == 0).all()


@pytest.mark.parametrize("L", [30, 5000])
def test_nan_and_infinity_stay_in_their_group(gtr, L):
    i = inputs(3, L, 40, torch.float32, 7)
    args = (4, i["w"], i["b"])
    clean = gtr.gtr_groupnorm_fwd(i["x"], *args, act="silu")
    for bad in (float("nan"), float("inf"), float("-inf")):
        x = i["x"].clone()
        x[1, L // 2, 13] = bad
        got = gtr.gtr_groupnorm_fwd(x, *args, act="silu")
        assert got[0][1, :, 10:20].isnan().any(0).all() and got[2][1, 1].isnan()
        got[0][1, :, 10:20] = clean[0][1, :, 10:20]
        assert torch.equal(got[0], clean[0])
        dx, dw, db = gtr.gtr_groupnorm_bwd(i["dy"], x, got[1], got[2], i["w"], i["b"], act="silu")
        want = gtr.gtr_groupnorm_bwd(i["dy"], i["x"], clean[1], clean[2], i["w"], i["b"], act="silu")
        assert dw[10:20].isnan().all()
        dx[1, :, 10:20], dw[10:20], db[10:20] = want[0][1, :, 10:20], want[1][10:20], want[2][10:20]
        assert all(torch.equal(a, b) for a, b in zip((dx, dw, db), want))


@pytest.mark.parametrize("B,L,C,G", [(2, 12, 30, 5), (1, 4200, 14, 2)])
@pytest.mark.parametrize("act", ACTS)
def test_gradient_against_differences(gtr, B, L, C, G, act):
    """The loss sum r y of the formula in 64 bits, differenced along random directions of x, w and b: with float32
    inputs the gradient differs from the difference quotient by its own error (checked above, under 1e-4 of it) and
    the quotient's, h^2 / 6 times a third derivative of the loss (h 1e-4: under 1e-6)."""
    i, h = inputs(B, L, C, torch.float32, 8), 1e-4
    _, mean, rstd = gtr.gtr_groupnorm_fwd(i["x"], G, i["w"], i["b"], act=act)
    grads = gtr.gtr_groupnorm_bwd(i["dy"], i["x"], mean, rstd, i["w"], i["b"], act=act)
    for name, grad in zip(("x", "w", "b"), grads):
        step = torch.randn_like(i[name]).double()
        at = lambda s: (Exact(*(i[n].double() + (s * h * step if n == name else 0) for n in ("x", "w", "b")), G, act).y *
                        i["dy"].double()).sum()
        quotient = (at(1) - at(-1)) / (2 * h)
        assert (quotient - (grad.double() * step).sum()).abs() <= 1e-4 * grad.double().norm() * 5


def test_streams_and_graph(gtr):
    """On a stream given, and recorded into a graph that is replayed between eager calls."""
    for B, L, C, G in ((2, 4000, 96, 8), (3, 100, 64, 4)):
        make = lambda seed: inputs(B, L, C, torch.bfloat16, seed)

        def run(i, **kw):
            f = gtr.gtr_groupnorm_fwd(i["x"], G, i["w"], i["b"], act="silu", **kw)
            return (*f, *gtr.gtr_groupnorm_bwd(i["dy"], i["x"], f[1], f[2], i["w"], i["b"], act="silu", dres=i["dres"], **kw))

        i = make(9)
        want = run(i)
        torch.cuda.synchronize()
        side = torch.cuda.Stream()
        got = run(i, stream=side)
        side.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(got, want))
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            held = run(i)
        for seed in (10, 11, 12, 9):
            new = make(seed)
            for k in i:
                i[k].copy_(new[k])
            graph.replay()
            torch.cuda.synchronize()
            eager = run(new)
            torch.cuda.synchronize()
            assert all(torch.equal(a, b) for a, b in zip(held, eager))
        assert all(torch.equal(a, b) for a, b in zip(held, want))


def test_calls_side_by_side(gtr):
    """Two graphs on two streams and an eager call on a third with a Workspace, at once, many times."""
    sets = [inputs(2, 6000, 128, torch.float16, s) for s in (13, 14, 15)]
    run = lambda i, **kw: gtr.gtr_groupnorm_fwd(i["x"], 16, i["w"], i["b"], act="gelu", **kw)[0]
    want = [run(i) for i in sets]
    torch.cuda.synchronize()
    graphs, outs = [], []
    for i in sets[:2]:
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            outs.append(run(i))
        graphs.append(graph)
    streams = [torch.cuda.Stream() for _ in range(3)]
    ws = gtr.Workspace(stream=streams[2])
    for _ in range(10):
        for graph, st in zip(graphs, streams):
            with torch.cuda.stream(st):
                graph.replay()
        third = run(sets[2], workspace=ws, stream=streams[2])
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip((*outs, third), want))


def test_more_than_2_31_elements(gtr):
    """Offsets past 32 bits: 2.3e9 elements in two images; the second's values as with the first left out."""
    L, C, G = 1_150_000, 1000, 5
    x = torch.empty(2, L, C, dtype=torch.float16, device="cuda")
    x[:] = torch.randn(C, device="cuda").half()
    x[1, ::3] += 1
    y, mean, rstd = gtr.gtr_groupnorm_fwd(x, G, act="silu")
    one = gtr.gtr_groupnorm_fwd(x[1:].clone(), G, act="silu")
    rel = lambda a, b: float(((a - b).abs() / b.abs()).max())
    assert rel(rstd[1:], one[2]) <= 1e-3 and (mean[1:] - one[1]).abs().max() <= 1e-3
    assert (y[1, -3000:].float() - one[0][0, -3000:].float()).abs().max() <= 0.02
    del one
    dx = gtr.gtr_groupnorm_bwd(x, x, mean, rstd, act="silu", want_dw=False)[0]
    single = gtr.gtr_groupnorm_bwd(x[1:].clone(), x[1:].clone(), mean[1:].clone(), rstd[1:].clone(), act="silu", want_dw=False)[0]
    assert (dx[1, -3000:].float() - single[0, -3000:].float()).abs().max() <= 0.02


def test_more_than_2_31_elements_bit_for_bit(gtr):
    """The second of two images, 1.15e9 elements each, has the bits of a call of its own: both calls have 256 tiles per
    image, the most there are. Its last group against 64 bits: a lane's n rows are summed about values that leave at most
    4 times their sum of squares about their mean, of which their sum takes off 3, with n + 2 roundings of each (10 (n + 2)
    e); its mean is off by 2 n e D + 3 e A (D the largest deviation from the group's mean, A the largest value), which
    with a deviation makes twice as much, over the spread, of the variance; sums over lanes and tiles S = 330 e more."""
    L, C, G, S = 1_150_000, 1000, 5, 330
    n = L // 1024 + 2  # 4 rows of 64 lanes at a time, in 256 tiles
    gen = torch.Generator(device="cuda").manual_seed(19)
    x = torch.empty(2, L, C, dtype=torch.float16, device="cuda")
    for k in range(2):
        for at in range(0, L, 50_000):
            x[k, at:at + 50_000] = torch.randn(50_000, C, generator=gen, device="cuda").half()
    x[1, ::3] += 1
    y, mean, rstd = gtr.gtr_groupnorm_fwd(x, G, act="silu")
    own = x[1:].clone()
    one = gtr.gtr_groupnorm_fwd(own, G, act="silu")
    assert torch.equal(y[1], one[0][0]) and torch.equal(mean[1:], one[1]) and torch.equal(rstd[1:], one[2])
    del one
    dx = gtr.gtr_groupnorm_bwd(x, x, mean, rstd, act="silu", want_dw=False)[0]
    single = gtr.gtr_groupnorm_bwd(own, own, mean[1:].clone(), rstd[1:].clone(), act="silu", want_dw=False)[0]
    assert torch.equal(dx[1], single[0])
    del dx, single, own
    last = x[1, :, 800:].double()
    m = last.mean()
    dev = last - m
    var = dev.square().mean()
    D, A, std = float(dev.abs().max()), float(last.abs().max()), float(var.sqrt())
    emean = S * E * (2 * D + A) + 2 * n * E * D + 3 * E * A
    erstd = 0.5 * ((10 * (n + 2) + 60 + S) * E + 2 * (2 * n * E * D + 3 * E * A) / std + (emean / std) ** 2) + 4 * E
    r = 1 / (var + EPS).sqrt()
    assert (mean[1, 4].double() - m).abs() <= emean and (rstd[1, 4].double() * (var + EPS).sqrt() - 1).abs() <= erstd
    u = dev[-3000:] * r
    eu = r * (emean + 2 * E * A) + u.abs() * (erstd + 3 * E)
    want = u * torch.sigmoid(u)
    close(y[1, -3000:, 800:], want, 1.13 * eu + (u.abs() + 6) * E * want.abs(), U[torch.float16], TINY[torch.float16])


def test_the_binding_refuses(gtr):
    i = inputs(2, 12, 40, torch.float16, 16)
    x, w = i["x"], i["w"]
    f = gtr.gtr_groupnorm_fwd
    _, mean, rstd = f(x, 4)
    b = lambda *a, **kw: gtr.gtr_groupnorm_bwd(i["dy"], x, *(a or (mean, rstd)), **kw)
    for call in (lambda: f(x, 3), lambda: f(x, 0), lambda: f(x, -4), lambda: f(x, 80), lambda: f(x, 4, w.half()),
                 lambda: f(x, 4, w[:20]), lambda: f(x, 4, act="relu"), lambda: f(x[:, ::2], 4), lambda: f(x[0, 0], 4),
                 lambda: f(x.double(), 4), lambda: f(x, 4, out=x.float()), lambda: f(x, 4, mean=rstd[:1]),
                 lambda: f(x, 4, bias=i["b"].cpu()), lambda: b(mean, rstd[:, :2]), lambda: b(mean[0], rstd[0]),
                 lambda: b(act="tanh"), lambda: b(accumulate=True), lambda: b(dres=x.float()), lambda: b(dw=w.half())):
        with pytest.raises(ValueError):
            call()
    for call in (lambda: f(x, 4, eps=-1.0), lambda: f(x[:0], 4), lambda: f(x, 4, out=x[:, :, :].view(2, 12, 40), mean=mean, rstd=mean),
                 lambda: f(torch.zeros(1, 1, 20000, device="cuda"), 4), lambda: b(dw=w, db=w)):
        with pytest.raises(gtr.GtrError):
            call()
