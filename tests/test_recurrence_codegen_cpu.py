"""The compiled listing of the recurrence kernels (recurrence.hip) on the CPU: every address that they form, against the
buffers that they are given and their LDS, in the wave emulator, every outcome of a wait included."""
import struct

import pytest

from test_training_codegen_cpu import Buffers, check_kernel, emu, kernel_named, listing

WAVES, TILE_WAVES, STEPS = 16, 8, (16, 8)  # of a sequence in one tile, of a tile; steps of a wave forward and backward


def _brev(w, i):
    v, o, d = w.s32(i.ops[1], i)
    w.s32set(i.ops[0], int(f"{v & 0xffffffff:032b}"[::-1], 2), emu.M32 if o else 0, d)


def _sign_extend(w, i):  # the lower 32 bits of a pair
    assert i.ops[2] == "0x200000", i.raw
    at = int(i.ops[1][2:].split(":")[0])
    v, o, d = w.s32(f"s{at}", i)
    w.s64set(i.ops[0], v | (0xffffffff00000000 if v >> 31 else 0), (1 << 64) - 1 if o else 0, d)
    emu.set_scc(w, v != 0, bool(o), d)


emu.HANDLERS.update({"s_brev_b32": _brev, "s_bfe_i64": _sign_extend})
for _c in ("ngt", "nlt", "gt", "lt"):  # (of loaded values: every outcome)
    for _e in ("e32", "sdwa"):
        emu.HANDLERS.setdefault(f"v_cmp_{_c}_f16_{_e}", emu.vcmp(lambda a, b: a < a, "u32"))


def tiles_of(L, T):
    T = 1 if L == 1 else T
    waves = -(-L // T)
    most = waves if waves <= WAVES else TILE_WAVES
    return T, most, -(-waves // most)


def tiles(new, seqs, n, V, group, blocks):
    groups = -(-n // group)
    maps, states = (new(k, seqs * m * 64 * V * 8, "rw") if n > 1 else 0 for k, m in (("maps", n), ("states", groups)))
    # no counters: a work-group's tile is its index, which the emulator knows
    return struct.pack("<QQQiiiiIII4x", maps, states, 0, n, group, groups, blocks, seqs, 1, 1)


# one token; a wave's steps, broken; several waves; several tiles, groups of them, a broken last one; a grid by columns
CASES = [(3, 1, 1, 130), (1, 1, 1, 1), (2, 1, 7, 65), (1, 4, 5, 129), (1, 1, 2000, 64), (2, 9, 300, 131), (1, 1, 259, 1)]
# types of rows and gates, logits, complement, scan


@pytest.mark.parametrize("dt,gt,logits,complement,scan", [(1, 1, 1, 1, 0), (2, 0, 0, 1, 1), (0, 0, 1, 0, 2), (2, 2, 0, 0, 3)])
@pytest.mark.parametrize("B,H,W,d", CASES)
def test_addresses(B, H, W, d, dt, gt, logits, complement, scan):
    addresses(B, H, W, d, dt, gt, logits, complement, scan, ((True, STEPS[0]), (False, STEPS[1])))


# the backward steps of calls of many tiles in 16-bit types
@pytest.mark.parametrize("dt,gt,logits,complement,scan,steps", [(1, 1, 1, 0, 0, 12), (2, 0, 0, 0, 1, 12), (1, 0, 1, 1, 2, 10),
                                                                (2, 2, 0, 1, 3, 10)])
@pytest.mark.parametrize("B,H,W,d", [(2, 1, 7, 65), (1, 4, 5, 129), (1, 1, 2000, 64), (2, 9, 300, 131),
                                     (1, 1, 259, 1)])
def test_addresses_of_more_steps(B, H, W, d, dt, gt, logits, complement, scan, steps):
    addresses(B, H, W, d, dt, gt, logits, complement, scan, ((False, steps),))


# short sequences
@pytest.mark.parametrize("dt,gt,logits,complement,scan", [(1, 1, 1, 1, 0), (2, 0, 0, 1, 1), (0, 0, 1, 0, 2), (2, 2, 0, 0, 3)])
@pytest.mark.parametrize("B,H,W,d", [(3, 1, 2, 130), (2, 1, 7, 65), (1, 8, 4, 129), (1, 5, 3, 1), (2, 4, 4, 64)])
def test_addresses_of_few_steps(B, H, W, d, dt, gt, logits, complement, scan):
    addresses(B, H, W, d, dt, gt, logits, complement, scan, ((True, 4), (False, 4)))


def addresses(B, H, W, d, dt, gt, logits, complement, scan, passes):
    text, L, V = listing("recurrence.hip"), H * W, 1 if d == 1 else 2
    es, gs = (4 if dt == 0 else 2), (4 if gt == 0 else 2)
    ld = d + 3  # x and g as parts of wider rows
    blocks = -(-d // (64 * V))
    seqs = B * blocks
    for forward, steps in passes:
        T, waves, n = tiles_of(L, steps)
        new = Buffers()
        t = tiles(new, seqs, n, V, 4, blocks)
        span = ((B * L - 1) * ld + d)
        x, g = new("x", span * es, "r"), new("g", span * gs, "r")
        h, h0, last = new("h", B * L * d * es, "w" if forward else "r"), new("h0", B * d * 4, "r"), new("last", B * d * 4, "rw")
        if forward:
            kern = t + struct.pack("<QQQQQqqqiiiiIf", x, g, h, h0, last, ld * es, ld * gs, L, H, W, d, scan, seqs, 1 / 16)
        else:
            dh, dh0 = new("dh", B * L * d * es, "r"), new("dh0", B * d * 4, "w")
            dx, dg = new("dx", B * L * d * es, "w"), new("dg", B * L * d * gs, "w")
            kern = t + struct.pack("<QQQQQQQQQqqqqqiiiiIf", dh, g, h, x if complement else 0, h0, last, dx, dg, dh0, ld * es,
                                   ld * gs, d * es, d * gs, L, H, W, d, scan, seqs, 1 / 16)
        kern += struct.pack("<IIIHHH", seqs * n, 1, 1, 64 * waves, 1, 1)
        kern += bytes(1024 - len(kern))
        name = kernel_named(text, f"rec_{'fwd' if forward else 'bwd'}_kernelILi{dt}ELi{gt}ELi{V}ELi{T}ELb{logits}ELb{complement}E")
        groups = {0, seqs - 1, seqs * (n - 1), seqs * n - 1, seqs * min(n - 1, 3), seqs * min(n - 1, 6)}
        few = sorted({0, 1, waves // 2, waves - 2, waves - 1} & set(range(waves)))
        check_waves(text, name, kern, new.regions, [(k, 0, 0) for k in sorted(groups)], few)


def check_waves(text, name, kern, regions, groups, waves):
    prog, labels, desc = emu.parse_kernel(text, name)
    rep = emu.Report()
    for wg in groups:
        for wave in waves:
            emu.run_wave(prog, labels, desc, kern, regions, desc["amdhsa_group_segment_fixed_size"], wg, wave, rep)
    bad = {k: sorted(v)[:4] for k, v in rep.items.items() if k.startswith(("ERR", "WARN", "NOTIMPL"))}
    assert not bad, f"{name}: {bad}"
    assert "INFO-PATHLIMIT" not in rep.counts
