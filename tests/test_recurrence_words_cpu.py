"""The words in which the recurrence's tiles hand on their maps, and the wait for them (csrc/rec_words.h), on the CPU:
the header's own functions around a poll that the test answers."""
import ctypes
import hashlib
import os
import subprocess

import numpy as np
import pytest

from paper_2609_26590_amd import build as b

SOURCE = r"""
#include <stdint.h>
#define __device__
#define __forceinline__ inline
static unsigned long long poll(const unsigned long long* p);
static bool vote(bool all);
#define __hip_atomic_load(p, order, scope) poll(p)
#define __all(x) vote(x)
#define __builtin_amdgcn_s_sleep(n) (void)0
#include "rec_words.h"
static const unsigned long long* base;
static uint64_t loads, votes, ready, others;  // a word is there once `ready` polls were voted on, another lane's after `others`
static unsigned long long poll(const unsigned long long* p) {
  ++loads;
  return p == base + 5 && votes < ready ? 0 : *p;
}
static bool vote(bool all) { return votes++ >= others && all; }
extern "C" uint64_t word(float p, float e) { return gtr::rec_word(p, e); }
extern "C" void map(uint64_t w, float* o) { o[0] = gtr::rec_map(w), o[1] = gtr::rec_add(w); }
// 4 words of 2 channels; polls in *n
extern "C" void wait(const uint64_t* words, uint64_t after, uint64_t lanes, unsigned spin, uint64_t* out, uint64_t* n) {
  base = reinterpret_cast<const unsigned long long*>(words);
  loads = votes = 0, ready = after, others = lanes;
  unsigned long long w[4][2];
  const unsigned long long* at[4] = {base, base + 2, base + 4, base + 6};
  gtr::rec_wait<2, 4>(w, at, spin);
  for (int i = 0; i < 8; ++i) out[i] = w[i / 2][i % 2];
  n[0] = votes, n[1] = loads;
}
"""


@pytest.fixture(scope="module")
def lib():
    h = hashlib.sha256(SOURCE.encode())
    with open(os.path.join(b.CSRC, "rec_words.h"), "rb") as fh:
        h.update(fh.read())
    os.makedirs(b.BUILD, exist_ok=True)
    so = os.path.join(b.BUILD, f"rec_words.{h.hexdigest()[:16]}.so")
    if not os.path.exists(so):
        src = so[:-3] + ".cpp"
        with open(src, "w") as fh:
            fh.write(SOURCE)
        tmp = so + f".tmp{os.getpid()}"
        r = subprocess.run([b._hipcc(), "-O1", "-std=c++17", "-fPIC", "-shared", "-I", b.CSRC, src, "-o", tmp],
                           capture_output=True, text=True)
        assert r.returncode == 0, r.stderr[-2000:]
        os.replace(tmp, so)
    lib = ctypes.CDLL(so)
    lib.word.argtypes, lib.word.restype = [ctypes.c_float, ctypes.c_float], ctypes.c_uint64
    lib.map.argtypes = [ctypes.c_uint64, ctypes.c_void_p]
    lib.wait.argtypes = [ctypes.c_void_p, ctypes.c_uint64, ctypes.c_uint64, ctypes.c_uint, ctypes.c_void_p, ctypes.c_void_p]
    return lib


def maps(lib, words):
    out = np.zeros((len(words), 2), np.float32)
    for w, o in zip(words, out):
        lib.map(int(w), o.ctypes.data)
    return out


def test_every_map_is_a_word_that_is_not_zero(lib):
    bits = np.array([0, 1, 1 << 31, 0x3f800000, 0x007fffff, 0x7f800000, 0xff800000, 0x7fc00000, 0xffc00000, 0x7fffffff,
                     0xffffffff], np.uint32)
    values = bits.view(np.float32)
    for P in values:
        words = np.array([lib.word(float(P), float(E)) for E in values], np.uint64)
        assert ((words & np.uint64(0xffffffff)) != 0).all()
        got = maps(lib, words)
        assert np.array_equal(got[:, 0], np.full(len(values), P), equal_nan=True)
        assert np.array_equal(got[:, 1], values, equal_nan=True)


def wait(lib, after, lanes, spin):
    words = np.array([lib.word(0.5 + i, -1.0 * i) for i in range(8)], np.uint64)
    out, n = np.zeros(8, np.uint64), np.zeros(2, np.uint64)
    lib.wait(words.ctypes.data, after, lanes, spin, out.ctypes.data, n.ctypes.data)
    assert n[1] == 8 * n[0]
    return words, out, int(n[0])


@pytest.mark.parametrize("after,lanes", [(0, 0), (1, 0), (0, 3), (7, 2), (9, 9)])
def test_words_that_come_in_time(lib, after, lanes):
    words, out, polls = wait(lib, after, lanes, 9)
    assert np.array_equal(out, words) and polls == max(after, lanes) + 1


@pytest.mark.parametrize("after,lanes", [(1 << 40, 0), (0, 1 << 40), (11, 0)])
@pytest.mark.parametrize("spin", [1, 10])
def test_a_wait_that_runs_out_ends_with_nan_maps(lib, after, lanes, spin):
    """One word that never comes, of this lane or of another one, makes all of them NaN, also those that are there."""
    _, out, polls = wait(lib, after, lanes, spin)
    assert polls == spin + 1 and np.isnan(maps(lib, out)).all()
    assert ((out & np.uint64(0xffffffff)) != 0).all()
