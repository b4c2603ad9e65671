"""GELU's tail as the feed-forward kernels compute it, on the CPU: the coefficients of csrc/ffn_gemm.h in the same
sequence of float32 operations (the exponential and the reciprocal correctly rounded, which the machine's are to one
unit in the last place), against the normal distribution function in 64 bits."""
import os
import re

import numpy as np
import torch

import paper_2609_26590_amd as gtr

E = 2.0 ** -24
HEADER = os.path.join(os.path.dirname(gtr.__file__), "csrc", "ffn_gemm.h")


def coefficients():
    with open(HEADER) as fh:
        text = fh.read()
    body = text[text.index("float ffn_act("):]
    body = body[:body.index("const float q =")]
    first = re.search(r"float r = (-?[\d.]+)f;", body).group(1)
    rest = re.findall(r"r = fmaf\(r, t, (-?[\d.]+)f\);", body)
    assert len(rest) == 8 and "fmaf(fabsf(g), 0.375f, 1.f)" in body and "__expf(-0.5f * g * g)" in body
    return [np.float32(c) for c in (first, *rest)]


def tail64(x):
    """Q(x) and Q(x) exp(x^2 / 2), from erfc and the scaled erfcx in 64 bits."""
    x = torch.from_numpy(x.astype(np.float64))
    scaled = 0.5 * torch.special.erfcx(x / 2 ** 0.5)
    return (scaled * torch.exp(-x * x / 2)).numpy(), scaled.numpy()


def fma(a, b, c):
    return (a.astype(np.float64) * b.astype(np.float64) + np.float64(c)).astype(np.float32)


def horner(t, c):
    r = np.full_like(t, c[0])
    for k in c[1:]:
        r = fma(r, t, k)
    return r


X = np.concatenate([np.linspace(0, 13, 400_001), np.geomspace(1e-6, 13, 20_001)]).astype(np.float32)


def test_polynomial():
    """t R(t) against Q(x) exp(x^2 / 2), both in 64 bits, from 0 to where Q leaves float32's range and far beyond."""
    x = np.concatenate([X.astype(np.float64), np.geomspace(13, 1e6, 10_000)])
    t = 1 / (1 + 0.375 * x)
    r = np.polyval(np.array(coefficients(), np.float64), t)
    assert np.abs(t * r / tail64(x)[1] - 1).max() <= 2.6e-7


def test_float32():
    """The bound that the kernel's comment states: 10^-6 and 1.25 x^2 half units, relative. The exponent's argument x^2 /
    2 is rounded twice (and log2 e once), which moves the exponential by that times its absolute value: at most 2.5
    roundings of x^2 / 2. The rest: 2.6e-7 of the polynomial, and roundings of t (through t R(t): at most 3 times), of
    the exponential, of eight steps of which the last count, and of two products, under 12 of 2^-24."""
    one, l2e = np.float32(1), np.float32(1.4426950408889634)
    t = (one.astype(np.float64) / fma(X, np.full_like(X, 0.375), 1)).astype(np.float32)
    arg = ((np.float32(-0.5) * X) * X).astype(np.float32)
    e = np.exp2((arg * l2e).astype(np.float32).astype(np.float64)).astype(np.float32)
    q = (e * t * horner(t, coefficients())).astype(np.float64)
    want = tail64(X)[0]
    err = np.abs(q / want - 1)
    x = X.astype(np.float64)
    assert (err <= 1e-6 + 1.25 * x * x * E).all()
