"""The compiled listing of the group norm kernels (groupnorm.hip) on the CPU: every address that they form, against the
buffers that they are given and their LDS, in the wave emulator."""
import struct

import pytest

from test_recurrence_codegen_cpu import check_waves
from test_training_codegen_cpu import Buffers, kernel_named, listing

up = lambda a, b: -(-a // b)


def blocks(G, Cg, kg, VE):
    kg = up(G, up(G, kg))
    while kg < G and (G - (up(G, kg) - 1) * kg) * Cg < VE:
        kg += 1
    return kg, 1, Cg, up(G, kg)


def team(width, kg, threads):
    t = 1
    while t < 64 and t < width and t * 2 * kg <= threads:
        t *= 2
    return t


def tiles_plan(B, L, C, G, dt, tiles):
    """Two launches: as groupnorm.hip lays out its blocks, with the tiles given."""
    VE, Cg, CB = (4 if dt == 0 else 8), C // G, 64 * (4 if dt == 0 else 8)
    if Cg <= CB:
        kg, pieces, pw, nb = blocks(G, Cg, min(256, CB // Cg), VE)
    else:
        kg, pieces = 1, up(Cg, CB)
        pw, nb = up(Cg, pieces), G * pieces
    rp = 256 // up(kg * Cg if pieces == 1 else pw, VE)
    R = up(up(L, tiles), rp) * rp
    return dict(kg=kg, pieces=pieces, pw=pw, blocks=nb, tiles=up(L, R), R=R, team=team(Cg if pieces == 1 else pw, kg, 256),
                threads=256, NV=0)


def slab_plan(B, L, C, G, dt, row_bytes, most):
    VE, ES, Cg = (4, 4, C // G) if dt == 0 else (8, 2, C // G)
    kg, pieces, pw, nb = blocks(G, Cg, up(row_bytes, Cg * ES), VE)
    nl = up(kg * Cg, VE)
    threads = min(1024, max(up(L * nl, 64), up(kg, 64)) * 64)
    nv = up(L, threads // nl)
    assert nv <= most
    return dict(kg=kg, pieces=pieces, pw=pw, blocks=nb, tiles=1, R=0, team=team(Cg, kg, threads), threads=threads,
                NV=next(v for v in (1, 2, 4, 8, 16) if v >= nv))


def shape(B, L, C, G, p):
    return struct.pack("<qiiiiiiiiiii4x", L, B, C, G, C // G, p["kg"], p["pieces"], p["pw"], p["blocks"], p["tiles"], p["R"],
                       p["team"])


def run(text, name, kern, new, grid, threads):
    kern = kern + struct.pack("<IIIHHH", grid, 1, 1, threads, 1, 1)
    waves = threads // 64
    check_waves(text, name, kern + bytes(1024 - len(kern)), new.regions,
                [(k, 0, 0) for k in sorted({0, 1 % grid, grid // 2, grid - 1})], sorted({0, waves // 2, waves - 1}))


# rows shorter than a vector; broken vectors and groups that they cut; blocks of several groups, a broken last one;
# groups in pieces; tiles that the end breaks
TILED = [(2, 70, 3, 1, 1, 3), (1, 1, 1, 1, 0, 1), (2, 130, 100, 5, 2, 3), (1, 300, 993, 993, 1, 2), (1, 41, 4100, 2, 1, 2),
         (3, 97, 600, 2, 0, 4)]


@pytest.mark.parametrize("B,L,C,G,dt,tiles", TILED)
@pytest.mark.parametrize("act", [0, 2])
def test_tiles(B, L, C, G, dt, tiles, act):
    text, es = listing("groupnorm.hip"), (4 if dt == 0 else 2)
    p = tiles_plan(B, L, C, G, dt, tiles)
    tiny, grid, n = int(C < 16 // es), B * p["tiles"] * p["blocks"], B * L * C * es
    new = Buffers()
    x, w, b, y = new("x", n, "r"), new("w", C * 4, "r"), new("b", C * 4, "r"), new("y", n, "w")
    mean, rstd = new("mean", B * G * 4, "rw"), new("rstd", B * G * 4, "rw")
    part = new("part", B * p["tiles"] * p["pieces"] * G * 8, "rw")
    kern = shape(B, L, C, G, p) + struct.pack("<QQQQQQQfi", x, w, b, y, mean, rstd, part, 1e-5, act)
    for which in ("sums", "rows"):
        run(text, kernel_named(text, f"gn_fwd_{which}_kernelILi{dt}ELb{tiny}E"), kern, new, grid, 256)
    dy, dres, dx = new("dy", n, "r"), new("dres", n, "r"), new("dx", n, "w")
    wpart = new("wpart", B * p["tiles"] * 2 * C * 4, "rw")
    dw, db = new("dw", C * 4, "rw"), new("db", C * 4, "rw")
    kern = shape(B, L, C, G, p) + struct.pack("<QQQQQQQQQQQQii", dy, x, mean, rstd, w, b, dres, dx, part, wpart, dw, db, 1, act)
    run(text, kernel_named(text, f"gn_bwd_sums_kernelILi{dt}ELb{tiny}E"), kern, new, grid, 256)
    run(text, kernel_named(text, f"gn_bwd_rows_kernelILi{dt}ELb{tiny}E"), kern, new, grid + up(2 * C, 32), 256)
    run(text, kernel_named(text, "gn_reduce_kernel"), kern + struct.pack("<q", B * p["tiles"]), new, up(2 * C, 32), 256)


# one token; all of a wave's, a work-group's threads; one to all vectors per thread; broken vectors and groups
SLABS = [(2, 1, 64, 4, 1, 64, 8), (1, 49, 100, 5, 2, 64, 8), (2, 300, 33, 33, 0, 64, 8), (1, 1600, 40, 5, 1, 64, 16),
         (1, 700, 192, 32, 1, 128, 8)]


@pytest.mark.parametrize("B,L,C,G,dt,row_bytes,most", SLABS)
def test_slabs(B, L, C, G, dt, row_bytes, most):
    text, es = listing("groupnorm.hip"), (4 if dt == 0 else 2)
    p = slab_plan(B, L, C, G, dt, row_bytes, most)
    grid, n = B * p["blocks"], B * L * C * es
    new = Buffers()
    x, w, b, y = new("x", n, "r"), new("w", C * 4, "r"), new("b", C * 4, "r"), new("y", n, "w")
    mean, rstd = new("mean", B * G * 4, "rw"), new("rstd", B * G * 4, "rw")
    kern = shape(B, L, C, G, p) + struct.pack("<QQQQQQQfi", x, w, b, y, mean, rstd, 0, 1e-5, 0)
    run(text, kernel_named(text, f"gn_fwd_slab_kernelILi{dt}ELi{p['NV']}E"), kern, new, grid, p["threads"])
    if p["NV"] > 8:
        return
    dy, dres, dx = new("dy", n, "r"), new("dres", n, "r"), new("dx", n, "w")
    wpart = new("wpart", B * 2 * C * 4, "rw")
    dw, db = new("dw", C * 4, "rw"), new("db", C * 4, "rw")
    kern = shape(B, L, C, G, p) + struct.pack("<QQQQQQQQQQQQii", dy, x, mean, rstd, w, b, dres, dx, 0, wpart if B > 1 else 0,
                                              dw, db, 1, 1)
    run(text, kernel_named(text, f"gn_bwd_slab_kernelILi{dt}ELi{p['NV']}E"), kern, new, grid, p["threads"])
