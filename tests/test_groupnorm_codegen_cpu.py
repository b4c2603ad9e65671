"""The compiled listing of the group norm kernels (groupnorm.hip) on the CPU: every address that they form, against the
buffers that they are given and their LDS, in the wave emulator."""
import struct

import pytest

import test_training_codegen_cpu as training
from test_recurrence_codegen_cpu import check_waves
from test_training_codegen_cpu import Buffers, emu, kernel_named, listing

emu.HANDLERS["v_permlane32_swap_b32_e32"] = training._swap

up = lambda a, b: -(-a // b)


def pow2(n):
    p = 1
    while p < n:
        p *= 2
    return p


def blocks(G, Cg, kg, VE):
    kg = up(G, up(G, kg))
    while kg < G and (G - (up(G, kg) - 1) * kg) * Cg < VE:
        kg += 1
    return kg, 1, Cg, up(G, kg)


def lanes(p, threads, VE):
    width = p["pw"]
    p["nl"] = pow2(up(p["kg"] * width, VE))
    p["team"] = 1
    while p["team"] < 64 and p["team"] < width and p["team"] * 2 * p["kg"] <= threads:
        p["team"] *= 2
    return threads // p["nl"]


def tiles_plan(B, L, C, G, dt, tiles):
    """Two launches: as groupnorm.hip lays out its blocks, with the tiles given."""
    VE, Cg, CB = (4 if dt == 0 else 8), C // G, 64 * (4 if dt == 0 else 8)
    p = {}
    if Cg <= CB:
        p["kg"], p["pieces"], p["pw"], p["blocks"] = blocks(G, Cg, min(256, CB // Cg), VE)
    else:
        p["kg"], p["pieces"] = 1, up(Cg, CB)
        p["pw"], p["blocks"] = up(Cg, p["pieces"]), G * p["pieces"]
    lanes(p, 256, VE)
    p["tiles"] = tiles
    return p


def image_plan(L, C, G, dt, row_bytes):
    """An image's block in the registers of a work-group."""
    VE, ES, Cg, p = (4 if dt == 0 else 8), (4 if dt == 0 else 2), C // G, {}
    p["kg"], p["pieces"], p["pw"], p["blocks"] = blocks(G, Cg, up(row_bytes, Cg * ES), VE)
    lanes(p, 1024, VE)
    p["threads"] = 1024 if L * p["nl"] >= 1024 else up(L * p["nl"], 64) * 64
    p["NV"] = pow2(up(L, lanes(p, p["threads"], VE)))
    p["tiles"] = 1
    return p


def shape(B, L, C, G, p):
    return struct.pack("<qiiiiiiiiiiiiiff4x", L, B, C, G, C // G, p["kg"], p["pieces"], p["pw"], p["blocks"], p["nl"],
                       p["nl"].bit_length() - 1, p["tiles"], p["team"], p["team"].bit_length() - 1, 1 / p["pw"],
                       1 / p["pieces"])


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
    kern = shape(B, L, C, G, p) + struct.pack("<QQQQQQQQQQQQiiq", dy, x, mean, rstd, w, b, dres, dx, part, wpart, dw, db, 1,
                                              act, B * p["tiles"])
    run(text, kernel_named(text, f"gn_bwd_sums_kernelILi{dt}ELb{tiny}E"), kern, new, grid, 256)
    run(text, kernel_named(text, f"gn_bwd_rows_kernelILi{dt}ELb{tiny}E"), kern, new, grid + up(2 * C, 32), 256)
    run(text, kernel_named(text, "gn_reduce_kernel"), kern, new, up(2 * C, 32), 256)


# images, tokens, channels, groups, type, bytes per row: one token; part of a wave's, all of a work-group's threads; one
# to all vectors per thread; broken vectors and groups
IMAGES = [(2, 1, 64, 4, 1, 32), (1, 49, 100, 5, 2, 32), (2, 300, 33, 33, 0, 32), (1, 700, 40, 5, 1, 32),
          (1, 1950, 192, 12, 1, 32), (2, 333, 72, 9, 0, 128)]


@pytest.mark.parametrize("B,L,C,G,dt,row_bytes", IMAGES)
def test_images(B, L, C, G, dt, row_bytes):
    text, es = listing("groupnorm.hip"), (4 if dt == 0 else 2)
    p = image_plan(L, C, G, dt, row_bytes)
    grid, n = B * p["blocks"], B * L * C * es
    new = Buffers()
    x, w, b, y = new("x", n, "r"), new("w", C * 4, "r"), new("b", C * 4, "r"), new("y", n, "w")
    mean, rstd = new("mean", B * G * 4, "rw"), new("rstd", B * G * 4, "rw")
    kern = shape(B, L, C, G, p) + struct.pack("<QQQQQQQfi", x, w, b, y, mean, rstd, 0, 1e-5, 0)
    run(text, kernel_named(text, f"gn_fwd_image_kernelILi{dt}ELi{p['NV']}E"), kern, new, grid, p["threads"])
    if p["NV"] > 2:
        return
    dy, dres, dx = new("dy", n, "r"), new("dres", n, "r"), new("dx", n, "w")
    wpart = new("wpart", B * 2 * C * 4, "rw")
    dw, db = new("dw", C * 4, "rw"), new("db", C * 4, "rw")
    kern = shape(B, L, C, G, p) + struct.pack("<QQQQQQQQQQQQiiq", dy, x, mean, rstd, w, b, dres, dx, 0, wpart if B > 1 else 0,
                                              dw, db, 1, 1, B)
    run(text, kernel_named(text, f"gn_bwd_image_kernelILi{dt}ELi{p['NV']}E"), kern, new, grid, p["threads"])
