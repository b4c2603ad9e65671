"""The channel mixer's half block (paper_2609_26590_amd/mixer.py): its calls together, as a training step and a server
make them, against the formula in 64 bits with its gradients by torch's differentiation.

Tolerances, relative to 2-norms (u: half a step of the 16-bit type; each rounding is at most u, its root mean square
u / sqrt(3), and the roundings are independent):
* forward, against f = FFN(LN(x)) and y: n is rounded (both factors of act(g) v move with it: twice), then act(g) v,
  then y: under 2 u of |f| and u of |y|;
* gradients: each is a product of at most the rounded n, act(g) v or the projections kept (n's and their own
  rounding, through two factors), dg or dv, and is rounded itself; dx passes the layer norm's backward pass besides:
  eight roundings, under sqrt(8 / 3) u < 2 u of the gradient. Held to 3 u, which leaves room for terms that a
  cancellation in dx makes larger than their sum.
"""
import pytest
import torch

from paper_2609_26590_amd import mixer

pytestmark = pytest.mark.gpu

U = {torch.float16: 2.0 ** -11, torch.bfloat16: 2.0 ** -8}


def setup(M, d, hidden, dtype, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    n = lambda *s, std=1.0, mu=0.0: torch.randn(s, generator=g, device="cuda") * std + mu
    p = {"ln_w": n(d, std=0.1, mu=1.0), "ln_b": n(d, std=0.1), "w_gate": n(hidden, d, std=d ** -0.5).to(dtype),
         "w_value": n(hidden, d, std=d ** -0.5).to(dtype), "w_out": n(d, hidden, std=hidden ** -0.5).to(dtype)}
    return n(M, d).to(dtype), p, n(M, d, std=0.5).to(dtype)


def reference(x, p, dy, act):
    t = {k: v.double().requires_grad_() for k, v in {"x": x, **p}.items()}
    mean = t["x"].mean(-1, keepdim=True)
    var = (t["x"] - mean).square().mean(-1, keepdim=True)
    n = (t["x"] - mean) * (var + 1e-6).rsqrt() * t["ln_w"] + t["ln_b"]
    g, v = n @ t["w_gate"].t(), n @ t["w_value"].t()
    a = g * torch.sigmoid(g) if act == "silu" else g * torch.special.ndtr(g)
    f = (a * v) @ t["w_out"].t()
    y = t["x"] + f
    y.backward(dy.double())
    return y.detach(), f.detach(), {k: v.grad for k, v in t.items()}


def close(got, want, u, times):
    assert torch.isfinite(got).all()
    assert (got.double() - want).norm() <= times * u * want.norm(), float((got.double() - want).norm() / want.norm() / u)


@pytest.mark.parametrize("M,d,hidden", [(1600, 192, 768), (1600, 384, 1536), (333, 1000, 2728), (9, 64, 256)])
@pytest.mark.parametrize("dtype,act", [(torch.float16, "silu"), (torch.bfloat16, "gelu")])
def test_training_step(gtr, M, d, hidden, dtype, act):
    x, p, dy = setup(M, d, hidden, dtype, 1)
    u = U[dtype]
    y, kept = mixer.forward(x, p, act=act, train=True)
    dx, grads = mixer.backward(dy, kept, p, act=act)
    ry, rf, rg = reference(x, p, dy, act)
    assert (y.double() - ry).norm() <= 2 * u * rf.norm() + u * ry.norm()
    close(dx, rg["x"], u, 3)
    for k in mixer.GRADS:
        close(grads[k], rg[k], u, 3)
    assert torch.equal(mixer.forward(x, p, act=act), y)


def test_micro_batches(gtr):
    """Two micro-batches' gradients, accumulated in float32, are the whole batch's."""
    x, p, dy = setup(1200, 192, 768, torch.bfloat16, 2)
    *_, want = reference(x, p, dy, "silu")
    grads = None
    for part in (slice(0, 500), slice(500, 1200)):
        _, kept = mixer.forward(x[part], p, train=True)
        _, grads = mixer.backward(dy[part], kept, p, dw_dtype=torch.float32, grads=grads)
    for k in mixer.GRADS:
        assert grads[k].dtype == torch.float32
        close(grads[k], want[k], U[torch.bfloat16], 3)


def test_one_token_at_a_time(gtr):
    """A server's single tokens against the batch's rows: two results of one formula, each within the forward bound."""
    x, p, _ = setup(20, 384, 1536, torch.bfloat16, 3)
    batch = mixer.forward(x, p).double()
    rows = torch.cat([mixer.forward(x[i:i + 1], p) for i in range(20)]).double()
    f = batch - x.double()
    assert (rows - batch).norm() <= 2 * U[torch.bfloat16] * (2 * f.norm() + batch.norm())


def test_stack_in_a_graph(gtr):
    """Two layers forward and backward recorded once and replayed on other data, between eager steps of the same
    weights whose results live on: bit for bit."""
    data = [setup(700, 192, 768, torch.float16, s) for s in (4, 5, 6, 7)]
    layers = [data[0][1], data[1][1]]
    x, dy = data[0][0].clone(), data[0][2].clone()

    def step(x, dy):
        y1, k1 = mixer.forward(x, layers[0], train=True)
        y2, k2 = mixer.forward(y1, layers[1], train=True)
        d1, g2 = mixer.backward(dy, k2, layers[1])
        d0, g1 = mixer.backward(d1, k1, layers[0])
        return [y2, d0, *g1.values(), *g2.values()]

    alive = step(x, dy)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        held = step(x, dy)
    for nx, _, ndy in data[1:] + data[:1]:
        x.copy_(nx)
        dy.copy_(ndy)
        graph.replay()
        torch.cuda.synchronize()
        eager = step(nx, ndy)
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(held, eager))
    assert all(torch.equal(a, b) for a, b in zip(alive, eager))


def test_two_graphs_replayed_side_by_side(gtr):
    """Two recordings on the default settings share no scratch memory: replayed on two streams at once, many times."""
    sets = [setup(900, 384, 1536, torch.bfloat16, s) for s in (8, 9)]
    graphs, outs, want = [], [], []
    for x, p, dy in sets:
        y, kept = mixer.forward(x, p, train=True)
        want.append((y, *mixer.backward(dy, kept, p)[1].values()))
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            y, kept = mixer.forward(x, p, train=True)
            outs.append((y, *mixer.backward(dy, kept, p)[1].values()))
        graphs.append(graph)
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    for _ in range(10):
        for graph, st in zip(graphs, streams):
            with torch.cuda.stream(st):
                graph.replay()
    torch.cuda.synchronize()
    for got, ref in zip(outs, want):
        assert all(torch.equal(a, b) for a, b in zip(got, ref))
