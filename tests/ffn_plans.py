"""The feed-forward's plans (csrc/ffn_plan.h) on the CPU, from a small library built around the header."""
import ctypes
import functools
import hashlib
import os
import subprocess

from paper_2609_26590_amd import build as b

TILE, THREADS = (256, 128, 64), (512, 256, 256)  # rows and columns of a tile, threads of its work-group
SOURCE = r"""
#include "ffn_plan.h"
using namespace gtr;
static void put(const FfnPlan& p, int64_t* o) { o[0] = p.tile, o[1] = p.ksplit, o[2] = p.tiles; }
extern "C" int fwd(int64_t M, int d, int hidden, int dtype, int64_t* o) {
  gtr_ffn_fwd_args a = {};
  a.M = M, a.d = d, a.hidden = hidden, a.dtype = (gtr_dtype)dtype;
  const gtr_status st = ffn_sizes(M, d, hidden, dtype, 0);
  if (st != GTR_OK) return st;
  FfnFwdPlan f;
  ffn_fwd_plan(&a, &f);
  put(f.pu, o), put(f.pd, o + 3);
  return GTR_OK;
}
// want: 1 dx, 2 dw_gate, 4 dw_value, 8 dw_out
extern "C" int bwd(int64_t M, int d, int hidden, int dtype, int dw_dtype, int want, int64_t* o) {
  gtr_ffn_bwd_args a = {};
  char* p = reinterpret_cast<char*>(4096);
  a.M = M, a.d = d, a.hidden = hidden, a.dtype = (gtr_dtype)dtype, a.dw_dtype = (gtr_dtype)dw_dtype;
  a.dx = want & 1 ? p : nullptr, a.dw_gate = want & 2 ? p : nullptr, a.dw_value = want & 4 ? p : nullptr;
  a.dw_out = want & 8 ? p : nullptr;
  const gtr_status st = ffn_bwd_sizes(&a);
  if (st != GTR_OK) return st;
  FfnBwdPlan f;
  ffn_bwd_plan(&a, &f);
  put(f.ph, o), put(f.px, o + 3), put(f.pw, o + 6);
  return GTR_OK;
}
"""


@functools.lru_cache(maxsize=None)
def _lib():
    h = hashlib.sha256(SOURCE.encode())
    for f in (os.path.join(b.CSRC, "ffn_plan.h"), os.path.join(b.INCLUDE, "gtr.h")):
        with open(f, "rb") as fh:
            h.update(fh.read())
    os.makedirs(b.BUILD, exist_ok=True)
    so = os.path.join(b.BUILD, f"ffn_plans.{h.hexdigest()[:16]}.so")
    if not os.path.exists(so):
        src = so[:-3] + ".cpp"
        with open(src, "w") as fh:
            fh.write(SOURCE)
        tmp = so + f".tmp{os.getpid()}"
        r = subprocess.run([b._hipcc(), "-O1", "-std=c++17", "-fPIC", "-shared", "-I", b.INCLUDE, "-I", b.CSRC, src, "-o", tmp],
                           capture_output=True, text=True)
        assert r.returncode == 0, r.stderr[-2000:]
        os.replace(tmp, so)
    return ctypes.CDLL(so)


def _plans(o, n):
    return [{"tile": TILE[o[3 * i]], "ksplit": o[3 * i + 1], "tiles": o[3 * i + 2], "threads": THREADS[o[3 * i]]}
            for i in range(n)]


def forward(M, d, hidden, dtype=1):
    """Plans of the gated product and of the output product, or the status that refuses the sizes."""
    o = (ctypes.c_int64 * 6)()
    st = _lib().fwd(ctypes.c_int64(M), d, hidden, dtype, o)
    return st if st else _plans(o, 2)


def backward(M, d, hidden, dtype=1, dw_dtype=1, want=15):
    """Plans of the projections' gradients, of dx and of the weights' gradients, or the status."""
    o = (ctypes.c_int64 * 9)()
    st = _lib().bwd(ctypes.c_int64(M), d, hidden, dtype, dw_dtype, want, o)
    return st if st else _plans(o, 3)
