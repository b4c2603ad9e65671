"""What a feed-forward call plans, on the CPU: sizes up to the largest that the calls take."""
import pytest

import ffn_plans as plans
from test_ffn_gpu import SHAPES
from test_ffn_tiles_gpu import CUT, LARGE

SHAPE, UNSUP = 2, 3
MOST_ROWS, MOST_WIDTH, MOST_ACTIVATIONS, MOST_WEIGHTS = 1 << 30, 1 << 20, 1 << 37, 1 << 36  # (gtr.h)
WIDTHS = (8, 16, 24, 32, 56, 64, 72, 120, 128, 136, 200, 264, 520, 1032, 4104, 65544, 1 << 20)


def largest(d, hidden):
    return min(MOST_ROWS, MOST_ACTIVATIONS // max(d, hidden))


@pytest.mark.parametrize("d", WIDTHS)
def test_every_launch_holds_its_threads(d):
    """A launch takes less than 2^32 threads, a product's sum over its K slices too: what the calls accept, they can
    launch."""
    for hidden in WIDTHS:
        if d * hidden > MOST_WEIGHTS:
            continue
        most = largest(d, hidden)
        for M in {most, most - 1, most - 63, most - 64, most - 255, most // 2 + 1, most // 3, 100_000, 9, 1}:
            up, down = plans.forward(M, d, hidden)
            assert up["ksplit"] == 1
            launches = [up, down]
            sums = [M * d * (down["ksplit"] > 1)]
            for want in (15, 1, 14, 8, 2):
                dh, dx, dw = plans.backward(M, d, hidden, want=want)
                assert dh["ksplit"] == 1
                n = [p["tiles"] * p["ksplit"] for p in (dx, dw)]
                launches += [dh, {"tiles": sum(n) + 7, "ksplit": 1, "threads": dw["threads"]}]
                products = bin(want & 14).count("1")
                sums.append(M * d * (dx["ksplit"] > 1) + products * d * hidden * (dw["ksplit"] > 1))
            for p in launches:
                assert 0 < p["tiles"] * p["ksplit"] * p["threads"] < 1 << 32, (M, d, hidden, p)
            assert all(s / 8 + 256 < 1 << 32 for s in sums), (M, d, hidden)


def test_sizes_past_the_limits_are_refused():
    assert plans.forward(MOST_ROWS, 8, 8) != SHAPE and plans.forward(MOST_ROWS + 1, 8, 8) == SHAPE
    assert plans.forward(1 << 20, 1 << 17, 8) != SHAPE and plans.forward((1 << 20) + 1, 1 << 17, 8) == SHAPE
    assert plans.backward(1 << 20, 8, 1 << 17) != SHAPE and plans.backward((1 << 20) + 1, 8, 1 << 17) == SHAPE
    assert plans.forward(64, 1 << 20, 1 << 16) != SHAPE and plans.forward(64, 1 << 20, (1 << 16) + 8) == SHAPE
    assert plans.backward(64, 1 << 18, 1 << 18) != SHAPE and plans.backward(64, (1 << 18) + 8, 1 << 18) == SHAPE
    assert plans.forward(1, MOST_WIDTH + 8, 8) == UNSUP and plans.forward(1, 8, MOST_WIDTH) != UNSUP


def test_the_gpu_tests_reach_every_tile_and_cut():
    """The shapes that the GPU tests check values at, by what they plan: each product in each tile size, with K steps
    behind the first, and cut along K and not."""
    for shape in LARGE:
        up, down = plans.forward(*shape)
        dh, dx, dw = plans.backward(*shape)
        assert {p["tile"] for p in (up, down, dh, dx, dw)} == {256}, shape
        M, d, hidden = shape
        assert M % 256 and d % 256 and hidden % 256 and d > 4 * 64 and hidden > 4 * 64
    cuts = [plans.backward(*shape)[1:] for shape in CUT]
    assert all(dw["ksplit"] > 1 for _, dw in cuts)
    assert any(dx["ksplit"] > 1 for dx, _ in cuts) and any(dx["ksplit"] == 1 for dx, _ in cuts)
    alone = [plans.backward(*shape, want=14)[2] for shape in CUT]
    assert {dw["tile"] for _, dw in cuts} | {dw["tile"] for dw in alone if dw["ksplit"] > 1} == {256, 128, 64}
    seen = [set(), set(), set(), set(), set()]  # tile and whether it is cut, of each product
    for shape in SHAPES + LARGE + CUT:
        for s, p in zip(seen, plans.forward(*shape) + plans.backward(*shape)):
            s.add((p["tile"], p["ksplit"] > 1))
    assert seen[0] == seen[2] == {(256, False), (128, False), (64, False)}
    for s in (seen[1], seen[3], seen[4]):
        assert {t for t, _ in s} == {256, 128, 64} and {c for _, c in s} == {False, True}, seen
