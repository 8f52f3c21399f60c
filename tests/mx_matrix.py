"""Shared pieces of the tests of linear layers, residual norms and clipping:
MX matrices with their fp64 values, and the error bounds.

Bounds.  A rounding to a type is off by at most half a step, HALF[dtype]
relative (bf16 2^-8, fp32 2^-24: half of torch.finfo(t).eps).  A product
of length K is a chain of at most K / 16 matrix instructions whose
operands' products are exact; each rounds the running sum, at most S = sum
|a b| in magnitude, at most twice by 2^-24, and at most 32 more additions join
waves and splits: |error| <= (K / 16 + 32) 2^-23 S.  SiLU uses the hardware's
exp2 and reciprocal (2^-23 relative each); the rounding of exp2's argument
adds |z| 2^-23 relative, a product and a sum 2^-24 each.

Test infrastructure only.
"""
import numpy as np
import torch

import oracle

HALF = {torch.float32: 2.0 ** -24, torch.bfloat16: 2.0 ** -8}
U = 2.0 ** -24
FORMATS = {"e4m3": (0, 0), "e2m1": (1, 1), "e2m3": (2, 2), "e2m1_e3m2": (1, 3)}


def matrix(mx, rows, cols, fmt, seed, std=1.0, dev="cuda:0"):
    """A seeded normal matrix quantized on the GPU, and its fp64 values."""
    g = torch.Generator()
    g.manual_seed(seed)
    m = torch.randn((rows, cols), generator=g) * std
    q = mx.quantize_matrix(m.to(dev), fmt)
    return q, values(q)


def values(q):
    """The fp64 values of an MX matrix, by the oracle's decoder."""
    r, c, _, _ = q.shape
    codes = q.codes.cpu().numpy()[:oracle.codes_bytes(oracle.WEIGHT, q.fmt, r, c, 1, 1)]
    v = oracle.dequant(codes, q.scales.cpu().numpy(), oracle.WEIGHT, q.fmt, r, c, 1, 1)
    return np.asarray(v, dtype=np.float64).reshape(r, c)


def product_tol(a, b):
    """The bound on a product a b^T (a [m][K], b [n][K])."""
    return (a.shape[1] / 16 + 32) * 2.0 ** -23 * (np.abs(a) @ np.abs(b).T)


def act(z, fn):
    return z if fn == 0 else np.maximum(z, 0) if fn == 1 else z / (1 + np.exp(-z))


def act_grad(z, fn):
    if fn == 0:
        return np.ones_like(z)
    if fn == 1:
        return (z > 0).astype(np.float64)
    s = 1 / (1 + np.exp(-z))
    return s * (1 + z * (1 - s))


def check(got, ref, tol, dtype, what=""):
    """|got - ref| <= tol + half a step of the result's type, elementwise."""
    g = got.detach().cpu().to(torch.float64).numpy()
    assert g.shape == ref.shape, (what, g.shape, ref.shape)
    bound = tol + HALF[dtype] * (np.abs(ref) + tol) + 2.0 ** -133
    bad = ~(np.abs(g - ref) <= bound)
    assert not bad.any(), (what, int(bad.sum()), float(np.max(np.abs(g - ref) / bound)),
                           np.argwhere(bad)[:4].tolist())
