"""The compiled listings of the training kernels (norm.hip, ffn.hip) on the CPU: every address that they form, against
the buffers that they are given and their LDS, in the wave emulator; that nothing but the feed-forward's transfers to
LDS uses M0; and that its tiles keep their registers."""
import hashlib
import os
import re
import struct
import subprocess
import sys

import numpy as np
import pytest

sys.path.insert(0, os.path.dirname(os.path.abspath(__file__)))
import gfx950_wave as emu  # noqa: E402

from test_codegen_cpu import BUILD, CSRC, ROOT, check_kernel  # noqa: E402


# ---------------------------------------------------------------------------
# instructions that these kernels have besides: results that only matter as data, and the loads through a descriptor
# that go straight to LDS
# ---------------------------------------------------------------------------
def _swap(w, i):
    for tok, other in ((i.ops[0], i.ops[1]), (i.ops[1], i.ops[0])):
        r = emu.vres(np.zeros(emu.NL, np.uint32), w.v32(tok, i), w.v32(other, i))
        r.o = np.ones(emu.NL, bool)
        w.vwrite(tok, r)


_plain_buffer_load = emu.HANDLERS["buffer_load_dwordx4"]


def _buffer_load(w, i):
    if "lds" not in i.mods:
        return _plain_buffer_load(w, i)
    base, stride, nrec, rd, ro = emu.rsrc(w, i, i.ops[1])
    v, lanes = w.v32(i.ops[0], i), w.active()
    assert stride == 0 and i.ops[2] == "0" and "offen" in i.mods, i.raw
    if not rd or (~v.d & lanes).any():
        w.rep.add("ERR-UNDEF-ADDR", i)
    if ro or (v.o & lanes).any():
        w.rep.add("WARN-DATA-ADDR", i)
    off = emu.u64(v.v)
    inr = lanes & (off + np.uint64(16) <= np.uint64(nrec))
    w.check_addr(i, np.uint64(base) + off, v.d, v.o, 16, "r", inr)
    m0, mo, md = w.s32("m0", i)
    at = (np.uint32(m0) + np.arange(emu.NL, dtype=np.uint32) * np.uint32(16)).astype(np.uint32)
    emu.lds_check(w, i, emu.VVal(at, np.full(emu.NL, bool(md)), np.full(emu.NL, bool(mo))), [0], 16, lanes)


_plain_sub = emu.HANDLERS["v_sub_u32_e64"]
_clamped_sub = emu.valu(lambda a, b: np.where(a > b, a - b, np.uint32(0)).astype(np.uint32), 2)


def _sub(w, i):
    return (_clamped_sub if "clamp" in i.mods else _plain_sub)(w, i)


def _bfrev(a):
    return np.array([int(f"{int(x):032b}"[::-1], 2) for x in a], np.uint32)


emu.HANDLERS.update({"v_permlane16_swap_b32_e32": _swap, "buffer_load_dwordx4": _buffer_load,
                     "v_cvt_f16_f32_sdwa": emu.dataop(1), "v_cvt_pk_bf16_f32": emu.dataop(2),
                     "v_bfrev_b32_e32": emu.valu(_bfrev, 1), "v_sub_u32_e64": _sub,
                     "v_cmp_gt_f16_e32": emu.vcmp(lambda a, b: np.zeros(a.shape, bool), "u32"),
                     "v_cmp_lt_f16_sdwa": emu.vcmp(lambda a, b: np.zeros(a.shape, bool), "u32")})


def listing(name: str) -> str:
    from paper_2609_26590_amd import build as b
    h = hashlib.sha256()
    for f in sorted(os.listdir(CSRC)):
        if f == name or f.endswith(".h"):
            with open(os.path.join(CSRC, f), "rb") as fh:
                h.update(fh.read())
    with open(os.path.join(ROOT, "include", "gtr.h"), "rb") as fh:
        h.update(fh.read())
    h.update(" ".join(b.HIPCC_FLAGS).encode())
    os.makedirs(BUILD, exist_ok=True)
    path = os.path.join(BUILD, f"{name[:-4]}.gfx950.{h.hexdigest()[:16]}.s")
    if not os.path.exists(path):
        tmp = path + f".tmp{os.getpid()}"
        r = subprocess.run([b._hipcc(), *b.HIPCC_FLAGS, "-S", "--cuda-device-only", os.path.join(CSRC, name), "-o", tmp],
                           capture_output=True, text=True)
        assert r.returncode == 0, r.stderr[-2000:]
        os.replace(tmp, path)
    with open(path) as fh:
        return fh.read()


def kernel_named(text, sub):
    return [n for n in emu.kernel_names(text) if sub in n][0]


def shape(d, dt):
    """How a row is shared (T, threads, vectors per lane, tiny), as norm.hip chooses."""
    ve = 4 if dt == 0 else 8
    n = -(-d // ve)
    for t in (16, 32, 64):
        if n <= t:
            return t, 256, 1, int(d < ve)
    if n <= 128:
        return 64, 256, 2, 0
    nv = -(-n // 1024)
    return 0, -(-(-(-n // nv)) // 64) * 64, nv, 0


# every way of sharing a row; a broken last vector; rows at odd addresses; more rows than a launch takes at a time
SHAPES = [(5, 3, 1), (40, 128, 1), (9, 129, 2), (33, 384, 1), (7, 1001, 2), (5, 1001, 0), (3, 4097, 1), (2, 8192, 2),
          (2, 16384, 2), (2, 16383, 0), (2, 9000, 0)]


@pytest.mark.parametrize("M,d,dt", SHAPES)
def test_layernorm_forward_addresses(M, d, dt):
    text = listing("norm.hip")
    T, threads, nv, tiny = shape(d, dt)
    es, R = (4 if dt == 0 else 2), (256 // T if T else 1)
    X, W, B, Y, MU, RS = (0x1000_0000_0000 + i * 0x10_0000_0000 for i in range(6))
    regions = [emu.Region("x", X, M * d * es, "r"), emu.Region("w", W, d * 4, "r"), emu.Region("b", B, d * 4, "r"),
               emu.Region("y", Y, M * d * es, "w"), emu.Region("mean", MU, M * 4, "w"),
               emu.Region("rstd", RS, M * 4, "w"), emu.Region("kernarg", emu.KERNARG_BASE, 256, "r")]
    groups = max(1, -(-M // R) // 2)  # half the rows' work-groups: the loop runs twice
    kern = struct.pack("<QQQQQQqif", X, W, B, Y, MU, RS, M, d, 1e-6) + struct.pack("<IIIHHH", groups, 1, 1, threads, 1, 1)
    kern += bytes(256 - len(kern))
    name = kernel_named(text, f"ln_fwd_kernelILi{dt}ELi{T}ELi{nv}ELb{tiny}E")
    check_kernel(text, name, kern, regions, sorted({(0, 0, 0), (groups - 1, 0, 0)}), threads // 64)


@pytest.mark.parametrize("by_columns", [False, True])
@pytest.mark.parametrize("M,d,dt", SHAPES)
def test_layernorm_backward_addresses(M, d, dt, by_columns):
    text = listing("norm.hip")
    T, threads, nv, tiny = shape(d, dt)
    ve, es, R = (4 if dt == 0 else 8), (4 if dt == 0 else 2), (256 // T if T else 1)
    DY, X, MU, RS, W, DR, DX, P, DW, DB = (0x1000_0000_0000 + i * 0x10_0000_0000 for i in range(10))
    rows = max(1, -(-M // R) // 2)
    pairs = -(-d // (2 * ve))
    grid = rows + (pairs if by_columns else 0)
    regions = [emu.Region("dy", DY, M * d * es, "r"), emu.Region("x", X, M * d * es, "r"),
               emu.Region("mean", MU, M * 4, "r"), emu.Region("rstd", RS, M * 4, "r"), emu.Region("w", W, d * 4, "r"),
               emu.Region("dres", DR, M * d * es, "r"), emu.Region("dx", DX, M * d * es, "w"),
               emu.Region("part", P, rows * 2 * d * 4, "w"), emu.Region("dw", DW, d * 4, "rw"),
               emu.Region("db", DB, d * 4, "rw"), emu.Region("kernarg", emu.KERNARG_BASE, 256, "r")]
    kern = struct.pack("<QQQQQQQQqiiQQi4x", DY, X, MU, RS, W, DR, DX, 0 if by_columns else P, M, d,
                       rows if by_columns else 0, DW, DB, 1)
    kern += struct.pack("<IIIHHH", grid, 1, 1, threads, 1, 1)
    kern += bytes(256 - len(kern))
    name = kernel_named(text, f"ln_bwd_kernelILi{dt}ELi{T}ELi{nv}ELb{tiny}E")
    groups = {(0, 0, 0), (rows - 1, 0, 0), (grid - 1, 0, 0)} | ({(rows, 0, 0)} if by_columns else set())
    check_kernel(text, name, kern, regions, sorted(groups), threads // 64)


@pytest.mark.parametrize("G,d", [(1, 3), (256, 384), (40, 1001)])
def test_layernorm_reduce_addresses(G, d):
    text = listing("norm.hip")
    P, DW, DB = (0x1000_0000_0000 + i * 0x10_0000_0000 for i in range(3))
    regions = [emu.Region("part", P, G * 2 * d * 4, "r"), emu.Region("dw", DW, d * 4, "rw"),
               emu.Region("db", DB, d * 4, "rw"), emu.Region("kernarg", emu.KERNARG_BASE, 256, "r")]
    kern = struct.pack("<QiiQQi4x", P, G, d, DW, DB, 1)
    blocks = (2 * d + 31) // 32
    kern += struct.pack("<IIIHHH", blocks, 1, 1, 1024, 1, 1)
    kern += bytes(256 - len(kern))
    check_kernel(text, kernel_named(text, "ln_reduce_kernel"), kern, regions, sorted({(0, 0, 0), (blocks - 1, 0, 0)}), 16)


# ---------------------------------------------------------------------------
# the feed-forward's products
# ---------------------------------------------------------------------------
TILE = {256: (256, 2, 4), 128: (128, 2, 2), 64: (64, 2, 2)}  # columns, waves


def prod(a, b, c, res, lda, ldb, ldc, M, N, K, nseg, gx, gy, part_off=0):
    return struct.pack("<QQQQQQqqqiiiiiiq", *a, *b, c, res, lda, ldb, ldc, M, N, K, nseg, gx, gy, part_off)


def gemm(prods, ksplit, cdt, part, part_slice, act, gates=(0, 0, 0, 0)):
    out = b"".join(prods) + bytes(104 * (3 - len(prods)))
    return out + struct.pack("<iii4xQqi4xQQQQ", len(prods), ksplit, cdt, part, part_slice, act, *gates)


class Buffers:
    def __init__(self):
        self.regions, self.at = [emu.Region("kernarg", emu.KERNARG_BASE, 1024, "r")], 0x1000_0000_0000

    def __call__(self, name, size, mode):
        self.at += 0x10_0000_0000
        self.regions.append(emu.Region(name, self.at, size, mode))
        return self.at


# tile, M, d, hidden, gates kept, dtype: whole and broken tiles on each axis, one step and broken ones
@pytest.mark.parametrize("bm,M,d,hidden,kept,dt", [(256, 300, 136, 264, True, 1), (128, 129, 72, 520, False, 2),
                                                   (64, 1, 8, 40, True, 1), (64, 130, 192, 64, True, 2)])
def test_ffn_gate_addresses(bm, M, d, hidden, kept, dt):
    text, new = listing("ffn.hip"), Buffers()
    x, wg, wv = new("x", M * d * 2, "r"), new("w_gate", hidden * d * 2, "r"), new("w_value", hidden * d * 2, "r")
    h, g, v = (new(n, M * hidden * 2, "w") for n in ("h", "gate", "value"))
    bn, wm, wn = TILE[bm]
    gx, gy = -(-M // bm), -(-hidden // (bn // 2))
    kern = gemm([prod((x, x), (wg, wv), h, 0, d, d, hidden, M, hidden, d, 1, gx, gy)], 1, dt, 0, 0, 0,
                (g, v, 0, 0) if kept else (0, 0, 0, 0))
    kern += struct.pack("<III", gx * gy, 1, 1) + bytes(100)
    name = kernel_named(text, f"ffn_gemm_kernelILi{dt}ELi0ELi0ELi1ELi{bm}E")
    check_kernel(text, name, kern, new.regions, sorted({(0, 0, 0), (gx * gy - 1, 0, 0)}), wm * wn)


@pytest.mark.parametrize("bm,M,d,hidden,dt", [(256, 260, 72, 264, 2), (128, 257, 200, 136, 1), (64, 65, 64, 72, 2)])
def test_ffn_gate_gradient_addresses(bm, M, d, hidden, dt):
    text, new = listing("ffn.hip"), Buffers()
    dy, wo = new("dy", M * d * 2, "r"), new("w_out", d * hidden * 2, "r")
    g, v = (new(n, M * hidden * 2, "r") for n in ("gate", "value"))
    h, dg, dv = (new(n, M * hidden * 2, "w") for n in ("h", "dgate", "dvalue"))
    bn, wm, wn = TILE[bm]
    gx, gy = -(-M // bm), -(-hidden // bn)
    kern = gemm([prod((dy, dy), (wo, wo), h, 0, d, hidden, hidden, M, hidden, d, 1, gx, gy)], 1, dt, 0, 0, 0, (g, v, dg, dv))
    kern += struct.pack("<III", gx * gy, 1, 1) + bytes(100)
    name = kernel_named(text, f"ffn_gemm_kernelILi{dt}ELi0ELi1ELi2ELi{bm}E")
    check_kernel(text, name, kern, new.regions, sorted({(0, 0, 0), (gx * gy - 1, 0, 0)}), wm * wn)


@pytest.mark.parametrize("bm,M,d,hidden,ks,res,dt", [(256, 300, 264, 72, 1, True, 1), (128, 100, 136, 520, 3, True, 2),
                                                     (64, 70, 72, 136, 1, False, 1), (64, 9, 72, 328, 2, True, 2)])
def test_ffn_down_addresses(bm, M, d, hidden, ks, res, dt):
    text, new = listing("ffn.hip"), Buffers()
    h, wo, y = new("h", M * hidden * 2, "r"), new("w_out", d * hidden * 2, "r"), new("y", M * d * 2, "w")
    r = new("residual", M * d * 2, "r") if res else 0
    part = new("part", ks * M * d * 4, "rw")
    bn, wm, wn = TILE[bm]
    gx, gy = -(-M // bm), -(-d // bn)
    kern = gemm([prod((h, h), (wo, wo), y, r, hidden, hidden, d, M, d, hidden, 1, gx, gy)], ks, dt, part, M * d, 0)
    T = gx * gy * ks
    name = kernel_named(text, f"ffn_gemm_kernelILi{dt}ELi0ELi0ELi0ELi{bm}E")
    check_kernel(text, name, kern + struct.pack("<III", T, 1, 1) + bytes(100), new.regions,
                 sorted({(0, 0, 0), (T - 1, 0, 0)}), wm * wn)
    if ks > 1:
        blocks = (M * d // 8 + 255) // 256
        none = gemm([], 0, 0, 0, 0, 0)
        check_kernel(text, kernel_named(text, "ffn_reduce_kernel"), kern + none + bytes(100), new.regions,
                     [(0, 0, 0), (blocks - 1, 0, 0)])


@pytest.mark.parametrize("bm,M,d,hidden,kx,kw,cdt,add,dt", [(256, 70, 264, 136, 1, 1, 2, False, 2),
                                                           (128, 200, 72, 136, 2, 2, 0, True, 1),
                                                           (64, 100, 72, 64, 1, 1, 1, True, 1)])
def test_ffn_gradient_addresses(bm, M, d, hidden, kx, kw, cdt, add, dt):
    """The gradients of input and weights in one launch, in either order."""
    text, new = listing("ffn.hip"), Buffers()
    es = 4 if cdt == 0 else 2
    dg, dv, h = (new(n, M * hidden * 2, "r") for n in ("dgate", "dvalue", "h"))
    x, dy = new("x", M * d * 2, "r"), new("dy", M * d * 2, "r")
    wg, wv = new("w_gate", hidden * d * 2, "r"), new("w_value", hidden * d * 2, "r")
    dx = new("dx", M * d * 2, "w")
    dws = [new(f"dw{k}", hidden * d * es, "rw") for k in range(3)]
    px, pw = new("part x", kx * M * d * 4, "rw"), new("part w", kw * 3 * d * hidden * 4, "rw")
    bn, wm, wn = TILE[bm]
    t = lambda m, n: (-(-m // bm), -(-n // bn))
    gx = gemm([prod((dg, dv), (wg, wv), dx, 0, hidden, d, d, M, d, hidden, 2, *t(M, d))], kx, dt, px, M * d, 0)
    prods = [prod((a, a), (b, b), c, c if add else 0, lda, ldb, n, m, n, M, 1, *t(m, n), k * d * hidden)
             for k, (a, b, c, lda, ldb, m, n) in enumerate(((dg, x, dws[0], hidden, d, hidden, d),
                                                            (dv, x, dws[1], hidden, d, hidden, d),
                                                            (dy, h, dws[2], d, hidden, d, hidden)))]
    gw = gemm(prods, kw, cdt, pw, 3 * d * hidden, 0)
    count = lambda m, n: t(m, n)[0] * t(m, n)[1]
    nx, nw = count(M, d) * kx, (2 * count(hidden, d) + count(d, hidden)) * kw
    name = kernel_named(text, f"ffn_grad_kernelILi{dt}ELi{bm}E")
    for first in (0, 1):
        n0, n1 = (nx, nw) if first else (nw, nx)
        r0 = (n0 + 7) // 8 * 8
        kern = gx + gw + struct.pack("<iii4x", nx, nw, first) + struct.pack("<III", r0 + n1, 1, 1) + bytes(100)
        groups = {(0, 0, 0), (n0 - 1, 0, 0), (r0 - 1, 0, 0), (r0, 0, 0), (r0 + n1 - 1, 0, 0)}
        check_kernel(text, name, kern, new.regions, sorted(groups), wm * wn)


@pytest.mark.parametrize("M,K,N,two,dt", [(1, 200, 40, True, 1), (8, 1032, 72, True, 2), (3, 2056, 24, False, 1)])
def test_ffn_few_addresses(M, K, N, two, dt):
    text, new = listing("ffn.hip"), Buffers()
    x, w0, w1 = new("x", M * K * 2, "r"), new("w0", N * K * 2, "r"), new("w1", N * K * 2, "r")
    c, r, g, v = new("c", M * N * 2, "w"), new("res", M * N * 2, "r"), new("gate", M * N * 2, "w"), new("value", M * N * 2, "w")
    kern = struct.pack("<QQQQQQQiiii", x, w0, w1 if two else 0, c, 0 if two else r, g if two else 0, v if two else 0, M, N,
                       K, 1) + bytes(100)
    blocks = -(-N // 8)
    check_kernel(text, kernel_named(text, f"ffn_few_kernelILi{dt}ELi{2 if two else 1}E"), kern, new.regions,
                 sorted({(0, 0, 0), (blocks - 1, 0, 0)}), 4 if two else 8)


def bodies(text, sub):
    for name in emu.kernel_names(text):
        if sub in name:
            body = text[text.index(f"\n{name}:"):]
            yield name, body[:body.index(".Lfunc_end")]


def test_nothing_but_the_transfers_uses_m0():
    """The feed-forward's transfers set M0 without the compiler's knowledge: it appears only as their LDS address, one
    instruction (the wait state it needs) before each, and nothing reads it implicitly."""
    found = 0
    for name, body in bodies(listing("ffn.hip"), "ffn_"):
        lines = [x for x in (ln.split(";")[0].strip() for ln in body.split("\n")) if x and not x.startswith(".")]
        moves = [i for i, ln in enumerate(lines) if re.match(r"buffer_load_dwordx4 v\d+, s\[\d+:\d+\], 0 offen lds$", ln)]
        assert not [ln for ln in lines if " lds" in ln and "buffer_load_dwordx4" not in ln], name
        found += bool(moves)
        for i in moves:
            assert re.match(r"s_mov_b32 m0, s\d+$", lines[i - 2]) and lines[i - 1].startswith("s_add_u32 s"), lines[i - 2:i + 1]
        if moves:
            assert sum(bool(re.search(r"\bm0\b", ln)) for ln in lines) == len(moves), name
            implicit = re.compile(r"(v_movrel|s_movrel|v_interp|s_sendmsg|ds_gws|ds_\w*addtid|ds_ordered|global_load_lds)")
            assert not [ln for ln in lines if implicit.match(ln)], name
    assert found == 24  # both types: the three tiles of three products and of the gradients' launch


def test_tiles_spill_nothing():
    found = 0
    text = listing("ffn.hip")
    for m in re.finditer(r"\.amdhsa_kernel (\S*ffn_(?:gemm|grad)_kernel\S*)\n(.*?)\.end_amdhsa_kernel", text, re.S):
        found += 1
        assert re.search(r"\.amdhsa_private_segment_fixed_size 0\b", m.group(2)), m.group(1)
    assert found == 24
