"""gtr_recurrence_fwd and gtr_recurrence_bwd on the GPU against the recurrence in 64 bits, token by token.

Tolerances, per element, from the kernels' arithmetic (e = 2^-24, the rounding of a float32 operation; u, half a step of
the output type). Relative errors of what is formed from a gate, r that of log a: none for log decays; for logits the
exponential's argument (1.5 |g| e), and under 16 e of exponential, logarithm (2 e each), reciprocal and products;
* a: |log a| (r + 2 e) + 2 e (exponent and exponential); an a below 2^-126, the least normal number, is 0, as the
  machine's exponential gives it: an error of a itself, and of at most 2^-126;
* 1 - a: r + 20 e (8 series steps near a = 1; elsewhere a / (1 - a) < 1.6 times that of a, and |log a| a < 0.4);
* sigmoid(-g): 1.5 |g| e + 8 e.
A scan forms each state from products and sums of these, in some association: with hb_t = a_t hb_{t-1} + |b_t|, which
bounds every partial sum, a step adds its gate's error and at most 4 e to what it multiplies and 4 e to what it adds,
and 2 e of hb_t (its own rounding, and that of the maps composed at the ends of waves and tiles, of which there are
fewer than steps): err_t = a_t err_{t-1} + (ea + 4 e) a_t hb_{t-1} + (eb + 4 e) |b_t| + 2 e hb_t. The backward pass is
the same recurrence from the end.
"""
import pytest
import torch

pytestmark = pytest.mark.gpu

E = 2.0 ** -24
U = {torch.float32: 2.0 ** -24, torch.float16: 2.0 ** -11, torch.bfloat16: 2.0 ** -8}
TINY = {torch.float32: 2.0 ** -149, torch.float16: 2.0 ** -25, torch.bfloat16: 2.0 ** -133}  # half the least step or more
SCANS = ("row", "col", "row_rev", "col_rev")
TAU = 16.0

# one token; parts of a wave's steps, all of them, one more; parts of a work-group's, all, one more; many tiles (with
# and without a broken last one) and several groups of them; a channel, an odd last one, several blocks
SHAPES = [(1, 1, 1, 1), (5, 1, 1, 200), (2, 1, 2, 5), (3, 2, 4, 64), (1, 3, 3, 129), (1, 1, 16, 128), (2, 17, 1, 31),
          (2, 5, 7, 333), (1, 8, 16, 127), (2, 1, 129, 2), (1, 16, 16, 192), (1, 1, 257, 257), (2, 40, 40, 130),
          (3, 37, 23, 33), (1, 1, 5003, 66), (2, 1, 2048, 1), (1, 64, 100, 3)]


def visits(H, W, scan):
    order = torch.arange(H * W).reshape(H, W)
    order = (order.t() if scan.startswith("col") else order).reshape(-1)
    return (order.flip(0) if scan.endswith("rev") else order).cuda()


def inputs(B, L, d, dtype, logits, seed, g32=False):
    gen = torch.Generator(device="cuda").manual_seed(100003 * seed + 31 * L + 7 * d + B)
    n = lambda *s, std=1.0, mu=0.0: torch.randn(s, generator=gen, device="cuda") * std + mu
    g = n(B, L, d, std=2.0, mu=2.0 if logits else 0.0)
    if not logits:
        g = -torch.exp(g - 3)  # from hardly any memory to thousands of tokens
    return dict(x=n(B, L, d).to(dtype), g=g.float() if g32 else g.to(dtype), h0=n(B, d), dh=n(B, L, d, std=0.5).to(dtype),
                dh_final=n(B, d, std=0.5))


class Gates:
    """log a, a, 1 - a, d log a / d g of g in 64 bits, and the bounds of the kernels' relative errors."""

    def __init__(self, g, tau):
        g = g.double()
        if tau is None:
            self.la, self.slope, self.eslope, r = g, torch.ones_like(g), 0.0, 0.0
        else:
            self.la = torch.nn.functional.logsigmoid(g) / tau
            self.slope, self.eslope = torch.sigmoid(-g) / tau, (1.5 * g.abs() + 8) * E
            r = (1.5 * g.abs() + 16) * E
        self.a, self.keep = torch.exp(self.la), -torch.expm1(self.la)
        far = self.la.abs().nan_to_num(posinf=0.0)  # (a = 0 there, exactly)
        small = torch.where(self.a < 2.0 ** -125, (2.0 ** -126 / self.a).clamp(max=1.0), 0.0)
        self.ea, self.ekeep = far * (r + 2 * E) + 2 * E + small, r + 20 * E


def scan64(a, b, ea, eb, first):
    """States, bounds of the partial sums and of the errors, [steps, B, d] each, and what is before each step."""
    h = first.double()
    bar, err = h.abs(), torch.zeros_like(h)
    out = []
    for t in range(a.shape[0]):
        before = (h, bar, err)
        err = a[t] * err + (ea[t] + 4 * E) * a[t] * bar + (eb[t] + 4 * E) * b[t].abs()
        h, bar = a[t] * h + b[t], a[t] * bar + b[t].abs()
        err = err + 2 * E * bar
        out.append((h, bar, err))
    return [torch.stack(v) for v in zip(*out)]


def steps(t, order):
    """[B, L, d] -> [L, B, d] in the scan's order, in 64 bits."""
    return t.double().transpose(0, 1)[order]


def close(got, want, err, u, tiny=0.0):
    bad = (got.double() - want).abs() > err + u * (want.abs() + err) + tiny
    assert not bad.any(), (int(bad.sum()), float(((got.double() - want).abs() / (err + u * want.abs() + tiny)).max()))


def check_forward(got, i, H, W, scan, tau, complement, h0):
    h, last = got
    order = visits(H, W, scan)
    k = Gates(steps(i["g"], order), tau)
    x = steps(i["x"], order)
    zero = torch.zeros_like(k.a)
    b, eb = (k.keep * x, zero + k.ekeep) if complement else (x, zero)
    first = h0 if h0 is not None else torch.zeros_like(i["h0"])
    want, _, err = scan64(k.a, b, k.ea, eb, first)
    close(steps(h, order), want, err, U[h.dtype], TINY[h.dtype])
    if last is not None:
        assert last.dtype == torch.float32
        close(last, want[-1], err[-1], 0.0, TINY[torch.float32])


def check_backward(got, i, h, H, W, scan, tau, complement, h0, dh_final):
    dx, dg, dh0 = got
    order = visits(H, W, scan)
    back = order.flip(0)
    k = Gates(steps(i["g"], back), tau)
    dh, x, hb = steps(i["dh"], back), steps(i["x"], back), steps(h, back)
    first = dh_final if dh_final is not None else torch.zeros_like(i["dh_final"])
    # Y -> a (dh + Y): the scan of a and a dh; D = dh + Y behind it
    y, ybar, yerr = scan64(k.a, k.a * dh, k.ea, k.ea + 2 * E, first)
    lead = lambda v, s: torch.cat([s.double()[None], v[:-1]])
    D = dh + lead(y, first)
    Derr = lead(yerr, torch.zeros_like(first)) + 2 * E * (dh.abs() + lead(ybar, first.abs()))
    start = (h0 if h0 is not None else torch.zeros_like(i["h0"])).double()
    before = torch.cat([hb[1:], start[None]])
    size = before.abs()
    if complement:
        before, size = before - x, size + x.abs()
    if dx is not None:
        want, err = (k.keep * D, k.keep * (Derr + (k.ekeep + 2 * E) * D.abs())) if complement else (D, Derr)
        close(steps(dx, back), want, err, U[dx.dtype], TINY[dx.dtype])
    if dg is not None:
        want = y * before * k.slope
        err = k.slope * (yerr * size + 4 * E * y.abs() * size + (k.eslope + 2 * E) * (y * before).abs())
        close(steps(dg, back), want, err, U[dg.dtype], TINY[dg.dtype])
    if dh0 is not None:
        close(dh0, y[-1], yerr[-1], 0.0, TINY[torch.float32])


def both(gtr, B, H, W, d, dtype, scan, logits, complement, state, g32=False, seed=1):
    i = inputs(B, H * W, d, dtype, logits, seed, g32)
    kind = dict(H=H, W=W, scan=scan, gate_tau=TAU if logits else None, complement=complement)
    h0, dlast = (i["h0"], i["dh_final"]) if state else (None, None)
    got = gtr.gtr_recurrence_fwd(i["x"], i["g"], h0=h0, want_final=state, **kind)
    assert got[0].dtype == dtype and (got[1] is not None) == state
    check_forward(got, i, H, W, scan, kind["gate_tau"], complement, h0)
    back = gtr.gtr_recurrence_bwd(i["dh"], i["g"], got[0], i["x"], h0=h0, dh_final=dlast, want_dh0=state, **kind)
    assert back[0].dtype == dtype and back[1].dtype == i["g"].dtype
    check_backward(back, i, got[0], H, W, scan, kind["gate_tau"], complement, h0, dlast)


@pytest.mark.parametrize("dtype", [torch.float32, torch.float16, torch.bfloat16])
@pytest.mark.parametrize("n,shape", list(enumerate(SHAPES)))
def test_both_passes(gtr, n, shape, dtype):
    k = n + {torch.float32: 0, torch.float16: 1, torch.bfloat16: 2}[dtype]
    both(gtr, *shape, dtype, SCANS[k % 4], k % 2 == 0, k % 3 != 0, k % 5 != 0)


@pytest.mark.parametrize("dtype", [torch.float16, torch.bfloat16])
@pytest.mark.parametrize("complement", [False, True])
@pytest.mark.parametrize("n,shape", list(enumerate([(5, 19, 79, 333), (9, 40, 40, 256), (20, 1, 1000, 1), (1, 1, 33000, 70),
                                                    (300, 1, 131, 64), (257, 3, 7, 24)])))
def test_more_tiles_than_cus(gtr, n, shape, complement, dtype):
    """Where a backward pass in 16 bits has other tiles."""
    both(gtr, *shape, dtype, SCANS[(n + complement) % 4], (n + (dtype == torch.float16)) % 2 == 0, complement, n % 2 == 0,
         n in (1, 4), seed=20 + n)


@pytest.mark.parametrize("dtype", [torch.float32, torch.float16, torch.bfloat16])
@pytest.mark.parametrize("n,shape", list(enumerate([(3, 1, 2, 130), (40, 1, 5, 65), (5, 4, 4, 333), (300, 1, 17, 24), (7, 8, 4, 200),
                                                    (2, 11, 3, 64), (9, 2, 8, 1), (6, 1, 32, 1)])))
def test_short_sequences(gtr, n, shape, dtype):
    """From two tokens on, about the lengths at which a wave takes other numbers of steps."""
    for complement in (False, True):
        both(gtr, *shape, dtype, SCANS[n % 4], (n + complement) % 2 == 0, complement, n % 2 == 0, seed=40 + n)


def test_more_tiles_than_cus_in_parts(gtr):
    """Broken steps, one gradient alone, and gradients in place have the same bits as whole steps."""
    B, L, d = 6, 1111, 258
    i = inputs(B, L, d, torch.bfloat16, True, 31)
    for complement in (False, True):
        kind = dict(H=1, W=L, gate_tau=TAU, complement=complement, h0=i["h0"], dh_final=i["dh_final"])
        h = gtr.gtr_recurrence_fwd(i["x"], i["g"], H=1, W=L, gate_tau=TAU, complement=complement, h0=i["h0"])[0]
        want = gtr.gtr_recurrence_bwd(i["dh"], i["g"], h, i["x"], want_dh0=True, **kind)
        one = gtr.gtr_recurrence_bwd(i["dh"], i["g"], h, i["x"], want_dx=False, **kind)
        assert torch.equal(one[1], want[1])
        one = gtr.gtr_recurrence_bwd(i["dh"], i["g"], h, i["x"], want_dg=False, **kind)
        assert torch.equal(one[0], want[0])
        t = {k: v.clone() for k, v in i.items()}
        got = gtr.gtr_recurrence_bwd(t["dh"], t["g"], h, t["x"], out=t["dh"], dg=t["g"], want_dh0=True, **kind)
        assert all(torch.equal(a, b) for a, b in zip(got, want))


@pytest.mark.parametrize("scan", SCANS)
@pytest.mark.parametrize("logits,complement,g32", [(False, False, False), (False, True, True), (True, False, True),
                                                   (True, True, False)])
def test_kinds(gtr, scan, logits, complement, g32):
    both(gtr, 2, 24, 19, 70, torch.float16, scan, logits, complement, True, g32, 2)
    both(gtr, 1, 24, 19, 65, torch.bfloat16, scan, logits, complement, False, g32, 3)


@pytest.mark.parametrize("dtype", [torch.float32, torch.float16, torch.bfloat16])
@pytest.mark.parametrize("n,shape", list(enumerate([(35, 1, 600, 70), (16, 20, 30, 330), (11, 40, 40, 384), (67, 1, 1100, 5),
                                                    (13, 1, 300, 600)])))
def test_several_sequences_per_counter(gtr, n, shape, dtype):
    """35, 48, 33, 67 and 65 sequences of several tiles: counters that number the tiles of 2 or 3 of them each, the last
    one with numbers that belong to none where these do not divide the sequences."""
    for complement in (False, True):
        both(gtr, *shape, dtype, SCANS[(n + complement) % 4], (n + complement) % 2 == 0, complement, n % 2 == 0, seed=60 + n)


@pytest.mark.parametrize("tau", [1.0, 3.0, 0.7, 0.01, 1000.0])
@pytest.mark.parametrize("dtype", [torch.float32, torch.float16])
def test_other_taus(gtr, tau, dtype):
    """1 / tau rounded, and products by it that round: two of the 16 roundings of log a and of the 8 of its slope."""
    B, H, W, d = 2, 24, 19, 70
    i = inputs(B, H * W, d, dtype, True, 70)
    for complement in (False, True):
        kind = dict(H=H, W=W, scan="col", gate_tau=tau, complement=complement)
        got = gtr.gtr_recurrence_fwd(i["x"], i["g"], h0=i["h0"], want_final=True, **kind)
        check_forward(got, i, H, W, "col", tau, complement, i["h0"])
        back = gtr.gtr_recurrence_bwd(i["dh"], i["g"], got[0], i["x"], h0=i["h0"], dh_final=i["dh_final"], want_dh0=True,
                                      **kind)
        check_backward(back, i, got[0], H, W, "col", tau, complement, i["h0"], i["dh_final"])


def test_several_groups_of_tiles(gtr):
    """More tokens than two groups of tiles take, and a group and a tile that the end breaks."""
    both(gtr, 1, 1, 20011, 20, torch.float16, "row", True, True, True, seed=4)


def test_gates_at_their_limits(gtr):
    """Gates that keep all, forget all, and logits past every range; -inf starts a sequence anew."""
    B, L, d = 2, 700, 40
    for logits in (False, True):
        i = inputs(B, L, d, torch.float32, logits, 5)
        i["g"][:, 100:120] = 1e4 if logits else 0.0
        i["g"][:, 300] = float("-inf")
        i["g"][:, 333, ::2] = float("-inf")
        i["g"][:, 500:510] = -1e4
        if logits:
            i["g"][:, 600] = float("inf")
            i["g"][:, 610] = -60.0
            i["g"][:, 611] = 60.0
        for complement in (False, True):
            kind = dict(H=1, W=L, gate_tau=TAU if logits else None, complement=complement)
            h, last = gtr.gtr_recurrence_fwd(i["x"], i["g"], h0=i["h0"], want_final=True, **kind)
            j = dict(i, g=i["g"].clamp(-1e30, 1e30))  # (0 times infinity in the bounds' own formulas)
            check_forward((h, last), j, 1, L, "row", kind["gate_tau"], complement, i["h0"])
            back = gtr.gtr_recurrence_bwd(i["dh"], i["g"], h, i["x"], h0=i["h0"], dh_final=i["dh_final"], want_dh0=True,
                                          **kind)
            check_backward(back, j, h, 1, L, "row", kind["gate_tau"], complement, i["h0"], i["dh_final"])
            assert torch.equal(h[:, 300], i["x"][:, 300])  # a = 0: what came before is gone
            assert (back[1][:, 300] == 0).all()


def test_nan_and_infinity_stay_where_they_are(gtr):
    """In one channel, from their token on (forward) and up to it (backward)."""
    B, L, d = 2, 900, 70
    i = inputs(B, L, d, torch.float16, True, 6)
    kind = dict(H=1, W=L, gate_tau=TAU, complement=True)
    clean = gtr.gtr_recurrence_fwd(i["x"], i["g"], h0=i["h0"], want_final=True, **kind)
    for bad in (float("nan"), float("inf")):
        x = i["x"].clone()
        x[1, 400, 33] = bad
        got = gtr.gtr_recurrence_fwd(x, i["g"], h0=i["h0"], want_final=True, **kind)
        assert not got[0][1, 400:, 33].isfinite().any() and not got[1][1, 33].isfinite()
        got[0][1, 400:, 33], got[1][1, 33] = clean[0][1, 400:, 33], clean[1][1, 33]
        assert torch.equal(got[0], clean[0]) and torch.equal(got[1], clean[1])
        want = gtr.gtr_recurrence_bwd(i["dh"], i["g"], clean[0], i["x"], h0=i["h0"], want_dh0=True, **kind)
        dh = i["dh"].clone()
        dh[0, 500, 69] = bad
        back = gtr.gtr_recurrence_bwd(dh, i["g"], clean[0], i["x"], h0=i["h0"], want_dh0=True, **kind)
        assert not back[0][0, :501, 69].isfinite().any() and not back[2][0, 69].isfinite()
        for t, w in zip(back[:2], want):
            t[0, :501, 69] = w[0, :501, 69]
        back[2][0, 69] = want[2][0, 69]
        assert all(torch.equal(a, b) for a, b in zip(back, want))


@pytest.mark.parametrize("B,H,W,d", [(3, 1, 1, 77), (2, 20, 31, 130), (1, 1, 700, 65)])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_rows_of_a_projection(gtr, B, H, W, d, dtype):
    """x and g as the two halves of one matrix, their gradients into the halves of another: bit for bit as on their own,
    and nothing else written."""
    i = inputs(B, H * W, d, dtype, True, 7)
    kind = dict(H=H, W=W, scan="col", gate_tau=TAU, complement=True, h0=i["h0"])
    want = gtr.gtr_recurrence_fwd(i["x"], i["g"], want_final=True, **kind)
    back = gtr.gtr_recurrence_bwd(i["dh"], i["g"], want[0], i["x"], **kind)
    both_in = torch.full((B, H * W, 2 * d + 3), 5.0, dtype=dtype, device="cuda")
    x, g = both_in[..., :d], both_in[..., d + 1:2 * d + 1]
    x.copy_(i["x"])
    g.copy_(i["g"])
    got = gtr.gtr_recurrence_fwd(x, g, want_final=True, **kind)
    assert all(torch.equal(a, b) for a, b in zip(got, want))
    both_out = torch.full((B, H * W, 2 * d + 3), 5.0, dtype=dtype, device="cuda")
    dx, dg = both_out[..., :d], both_out[..., d + 1:2 * d + 1]
    gb = gtr.gtr_recurrence_bwd(i["dh"], g, got[0], x, out=dx, dg=dg, **kind)
    assert gb[0] is dx and torch.equal(dx, back[0]) and torch.equal(dg, back[1])
    assert (both_out[..., d] == 5).all() and (both_out[..., 2 * d + 1:] == 5).all()
    # over the halves themselves
    gtr.gtr_recurrence_bwd(i["dh"], g, got[0], x, out=x, dg=g, **kind)
    assert torch.equal(x, back[0]) and torch.equal(g, back[1])


@pytest.mark.parametrize("B,L,d", [(4, 1, 129), (2, 700, 33), (1, 9, 64)])
@pytest.mark.parametrize("dtype", [torch.float32, torch.float16])
def test_in_place_repeatable_and_nothing_beyond(gtr, B, L, d, dtype):
    i = inputs(B, L, d, dtype, False, 8)
    kind = dict(H=1, W=L, scan="row_rev", complement=True)
    h, last = gtr.gtr_recurrence_fwd(i["x"], i["g"], h0=i["h0"], want_final=True, **kind)
    again = gtr.gtr_recurrence_fwd(i["x"], i["g"], h0=i["h0"], want_final=True, **kind)
    assert torch.equal(again[0], h) and torch.equal(again[1], last)
    x, state = i["x"].clone(), i["h0"].clone()
    got = gtr.gtr_recurrence_fwd(x, i["g"], h0=state, out=x, h_final=state, **kind)
    assert got[0] is x and got[1] is state and torch.equal(x, h) and torch.equal(state, last)
    room = torch.full((B + 2, L, d), 3.0, dtype=dtype, device="cuda")
    gtr.gtr_recurrence_fwd(i["x"], i["g"], h0=i["h0"], out=room[1:-1], **kind)
    assert torch.equal(room[1:-1], h) and (room[0] == 3).all() and (room[-1] == 3).all()
    args = dict(h0=i["h0"], dh_final=i["dh_final"], want_dh0=True, **kind)
    want = gtr.gtr_recurrence_bwd(i["dh"], i["g"], h, i["x"], **args)
    for over_x in (False, True):
        t = {k: v.clone() for k, v in i.items()}
        args = dict(h0=i["h0"], dh_final=t["dh_final"], dh0=t["dh_final"], **kind)
        got = gtr.gtr_recurrence_bwd(t["dh"], t["g"], h, t["x"], out=t["x"] if over_x else t["dh"], dg=t["g"], **args)
        assert all(torch.equal(a, b) for a, b in zip(got, want))
    only = gtr.gtr_recurrence_bwd(i["dh"], i["g"], h, i["x"], want_dx=False, h0=i["h0"], dh_final=i["dh_final"], **kind)
    assert only[0] is None and only[2] is None and torch.equal(only[1], want[1])
    only = gtr.gtr_recurrence_bwd(i["dh"], i["g"], h, i["x"], want_dg=False, h0=i["h0"], dh_final=i["dh_final"], **kind)
    assert only[1] is None and torch.equal(only[0], want[0])


def test_a_server_in_steps(gtr):
    """A prompt in one call and then token by token, the state in place, against the whole sequence."""
    B, L, d = 3, 400, 96
    i = inputs(B, L, d, torch.bfloat16, True, 9)
    kind = dict(gate_tau=TAU, complement=True)
    state = i["h0"].clone()
    h = torch.empty_like(i["x"])
    cut = 377
    for t0, t1 in [(0, 300), (300, cut)] + [(t, t + 1) for t in range(cut, L)]:
        part = lambda t: t[:, t0:t1].contiguous()
        h[:, t0:t1] = gtr.gtr_recurrence_fwd(part(i["x"]), part(i["g"]), H=1, W=t1 - t0, h0=state, h_final=state, **kind)[0]
    check_forward((h, state), i, 1, L, "row", TAU, True, i["h0"])


def test_gradient_against_differences(gtr):
    """The loss sum r h + sum s h_last of the recurrence in 64 bits, differenced along random directions (step 1e-4:
    the quotient is off by 1e-8 times a third derivative): the float32 gradients' own errors, bounded above, are under
    1e-4 of their norm; h enters the gates' gradients as the kernel rounded it (2^-24)."""
    B, H, W, d, step = 2, 9, 13, 21, 1e-4
    for logits in (False, True):
        for complement in (False, True):
            i = inputs(B, H * W, d, torch.float32, logits, 10)
            tau = TAU if logits else None
            kind = dict(H=H, W=W, scan="col", gate_tau=tau, complement=complement, h0=i["h0"])
            h, _ = gtr.gtr_recurrence_fwd(i["x"], i["g"], **kind)
            grads = gtr.gtr_recurrence_bwd(i["dh"], i["g"], h, i["x"], dh_final=i["dh_final"], want_dh0=True, **kind)
            order = visits(H, W, "col")
            names = ("x", "g", "h0")

            def loss(p):
                k = Gates(steps(p["g"], order), tau)
                b = k.keep * steps(p["x"], order) if complement else steps(p["x"], order)
                s, out = p["h0"].double(), 0.0
                dh = steps(i["dh"], order)
                for t in range(H * W):
                    s = k.a[t] * s + b[t]
                    out = out + (s * dh[t]).sum()
                return out + (s * i["dh_final"].double()).sum()

            for name, grad in zip(names, grads):
                way = torch.randn_like(i[name]).double()
                at = lambda sign: loss({n: i[n].double() + (sign * step * way if n == name else 0) for n in names})
                quotient = (at(1) - at(-1)) / (2 * step)
                assert (quotient - (grad.double() * way).sum()).abs() <= 1e-4 * grad.double().norm() * 5


def test_streams_and_graph(gtr):
    """On a stream given, and recorded into a graph that is replayed between eager calls of other data."""
    B, L, d = 2, 3000, 192
    make = lambda seed: inputs(B, L, d, torch.bfloat16, True, seed)
    kind = dict(H=1, W=L, gate_tau=TAU, complement=True)

    def run(i, **kw):
        h, last = gtr.gtr_recurrence_fwd(i["x"], i["g"], h0=i["h0"], want_final=True, **kind, **kw)
        return (h, last, *gtr.gtr_recurrence_bwd(i["dh"], i["g"], h, i["x"], h0=i["h0"], dh_final=i["dh_final"],
                                                 want_dh0=True, **kind, **kw))

    i = make(11)
    want = run(i)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    got = run(i, stream=side)
    side.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(got, want))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        held = run(i)
    for seed in (12, 13, 14, 11):
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
    """Two graphs on two streams and an eager call on a third, at once, many times; one Workspace for all calls of a
    stream."""
    sets = [inputs(4, 2500, 256, torch.float16, True, s) for s in (15, 16, 17)]
    kind = dict(H=50, W=50, scan="col_rev", gate_tau=TAU)
    want = [gtr.gtr_recurrence_fwd(i["x"], i["g"], **kind)[0] for i in sets]
    torch.cuda.synchronize()
    graphs, outs = [], []
    for i in sets[:2]:
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            outs.append(gtr.gtr_recurrence_fwd(i["x"], i["g"], **kind)[0])
        graphs.append(graph)
    streams = [torch.cuda.Stream() for _ in range(3)]
    ws = gtr.Workspace(stream=streams[2])
    for _ in range(10):
        for graph, st in zip(graphs, streams):
            with torch.cuda.stream(st):
                graph.replay()
        third = gtr.gtr_recurrence_fwd(sets[2]["x"], sets[2]["g"], workspace=ws, stream=streams[2], **kind)[0]
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip((*outs, third), want))


def test_a_wait_that_runs_out_gives_nan(gtr):
    """With one poll per wait every state is right or NaN, and the call ends."""
    i = inputs(2, 6000, 200, torch.float32, True, 18)
    kind = dict(H=1, W=6000, gate_tau=TAU)
    want = gtr.gtr_recurrence_fwd(i["x"], i["g"], **kind)[0]
    got = gtr.gtr_recurrence_fwd(i["x"], i["g"], spin_limit=1, **kind)[0]
    assert (got.isnan() | (got == want)).all() and not got[:, :64].isnan().any()


def test_more_than_2_31_elements(gtr):
    """Offsets past 32 bits: 2.3e9 elements in one sequence; its end as from the state before it."""
    L, d, cut = 1_100_000, 2100, 1_099_000
    x = torch.empty(1, L, d, dtype=torch.float16, device="cuda")
    x[:] = torch.randn(d, device="cuda").half()
    g = torch.full((1, L, d), 2.0, dtype=torch.float16, device="cuda")
    x[:, cut - 500:] = torch.randn(1, L - cut + 500, d, device="cuda").half()
    kind = dict(gate_tau=TAU, complement=True)
    state = torch.empty(1, d, device="cuda")
    h, last = gtr.gtr_recurrence_fwd(x, g, H=1, W=L, want_final=True, **kind)
    gtr.gtr_recurrence_fwd(x[:, :cut].contiguous(), g[:, :cut].contiguous(), H=1, W=cut, h_final=state, **kind)
    i = dict(x=x[:, cut:].contiguous(), g=g[:, cut:].contiguous(), h0=state)
    check_forward((h[:, cut:].contiguous(), last), i, 1, L - cut, "row", TAU, True, state)
    del x
    dx, dg, _ = gtr.gtr_recurrence_bwd(h, g, h, H=1, W=L, gate_tau=TAU, want_dg=False)
    tail = gtr.gtr_recurrence_bwd(h[:, cut:].contiguous(), i["g"], h[:, cut:].contiguous(), H=1, W=L - cut, gate_tau=TAU,
                                  want_dg=False)[0]
    assert (dx[:, cut:].float() - tail.float()).abs().max() <= 2 * U[torch.float16] * tail.float().abs().max()
    head = gtr.gtr_recurrence_bwd(h[:, :9000].contiguous(), g[:, :9000].contiguous(), h[:, :9000].contiguous(), H=1, W=9000,
                                  gate_tau=TAU, want_dg=False)[0]  # (8000 tokens on: a^8000 is 0)
    assert (dx[:, :1000].float() - head[:, :1000].float()).abs().max() <= 2 * U[torch.float16] * head.float().abs().max()


def test_the_binding_refuses(gtr):
    i = inputs(2, 12, 40, torch.float16, True, 19)
    x, g, f = i["x"], i["g"], gtr.gtr_recurrence_fwd
    b = lambda **kw: gtr.gtr_recurrence_bwd(i["dh"], g, x, **{**dict(H=3, W=4), **kw})
    for call in (lambda: f(x, g, H=3, W=5), lambda: f(x[0], g, H=3, W=4), lambda: f(x, g.cpu(), H=3, W=4),
                 lambda: f(x, g[..., :20], H=3, W=4), lambda: f(x, g.bfloat16(), H=3, W=4), lambda: f(x, g, H=3, W=4, scan="up"),
                 lambda: f(x, g, H=3, W=4, gate_tau=0.0), lambda: f(x, g, H=3, W=4, gate_tau=float("nan")),
                 lambda: f(x[..., ::2], g[..., :20], H=3, W=4), lambda: f(x, g, H=3, W=4, h0=i["h0"].half()),
                 lambda: f(x, g, H=3, W=4, h0=i["h0"][:1]), lambda: f(x, g, H=3, W=4, out=x.float()),
                 lambda: f(x[:, :1].expand(2, 12, 40), g, H=3, W=4), lambda: f(x.double(), g.double(), H=3, W=4),
                 lambda: b(complement=True), lambda: b(out=x.float()), lambda: b(dg=g.float()), lambda: b(dh0=i["h0"].half()),
                 lambda: b(dh_final=i["h0"][:, :3])):
        with pytest.raises(ValueError):
            call()
    for call in (lambda: f(x, g, H=3, W=4, out=g), lambda: f(x, g, H=-3, W=-4), lambda: b(out=x),
                 lambda: f(x[:0], g[:0], H=3, W=4)):
        with pytest.raises(gtr.GtrError):
            call()
