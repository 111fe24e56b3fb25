"""Plumbing of the linear layers' and norms' tests: pruned matrices, the definitions in 64 bits, and how far a result may be off."""
from __future__ import annotations

import math

import numpy as np

HALF = {0: 2.0 ** -24, 1: 2.0 ** -11, 2: 2.0 ** -8}       # half a step of a type, relative
TINY = {0: 2.0 ** -149, 1: 2.0 ** -25, 2: 2.0 ** -133}    # and absolute, where it ends
F32 = 2.0 ** -24
NAMES = {0: "f32", 1: "f16", 2: "bf16"}
BIAS, RELU, RESIDUAL, SILU, GELU, GELU_TANH = 1, 2, 4, 8, 16, 32
_erf = np.vectorize(math.erfc, otypes=[np.float64])


def torch_type(type):
    import torch
    return (torch.float32, torch.float16, torch.bfloat16)[type]


def rounded(a, type):
    """float64 copies of the values rounded to a type, by way of fp32 as a checkpoint's are."""
    import torch
    return torch.from_numpy(np.asarray(a, dtype=np.float32)).to(torch_type(type)).double().numpy()


def pruned(rows, K, sparsity, seed, type, scale=None):
    """A pruned matrix whose values are the type's (float64), and its CSR with ascending columns."""
    rng = np.random.default_rng(seed)
    w = rng.standard_normal((rows, K)) * (scale or 1.0 / math.sqrt(max(1.0, K * (1 - sparsity))))
    w = rounded(np.where(rng.random((rows, K)) >= sparsity, w, 0.0), type)
    return w, to_csr(w)


def to_csr(w):
    r, c = np.nonzero(w)
    rowptr = np.zeros(w.shape[0] + 1, dtype=np.int32)
    np.cumsum(np.bincount(r, minlength=w.shape[0]), out=rowptr[1:])
    return rowptr, c.astype(np.int32), w[r, c].astype(np.float32)


def act64(z, flags):
    if flags & RELU:
        return np.where(z > 0, z, 0.0)
    with np.errstate(over="ignore"):
        if flags & SILU:
            return z / (1 + np.exp(-z))
        if flags & GELU:
            return 0.5 * z * _erf(-z / math.sqrt(2.0))
        if flags & GELU_TANH:
            return z / (1 + np.exp(-2 * math.sqrt(2 / math.pi) * (z + 0.044715 * z ** 3)))
    return z


def linear64(x, w, type, flags, gated, bias=None, residual=None):
    """The layer in 64 bits and how far off a result may be.  Sums: each of up to n products passes through fewer than n + 16
    additions (the waves' sums among them) that round or truncate to fp32, each off by no more than a step (2^-23) of sum|w x|,
    and fp32 products by half a step; the bias is one more.  Activations have a slope of at most 1.13 and are
    computed to 16 half steps of |z| (an exponential, or erfc whose argument is rounded, a quotient, a product; the exponent of the
    tanh form is off by six half steps of itself, which its slope turns into no more than 10 of |z|).  The gate's
    product and the residual's sum are each rounded once in fp32, the result once to the type."""
    z = x @ w.T
    n = np.count_nonzero(w, axis=1)[None, :] + 16
    dz = (n * 2 + 1) * F32 * (np.abs(x) @ np.abs(w).T)
    if bias is not None:
        z = z + bias
        dz = dz + F32 * 2 * (np.abs(z) + np.abs(bias))
    M = w.shape[0] // 2 if gated else w.shape[0]
    a = act64(z[:, :M], flags)
    da = 1.13 * dz[:, :M] + (16 * F32 * np.abs(z[:, :M]) if flags & (SILU | GELU | GELU_TANH) else 0)
    if gated:
        u, du = z[:, M:], dz[:, M:]
        da = da * (np.abs(u) + du) + np.abs(a) * du + F32 * np.abs(a * u)
        a = a * u
    if residual is not None:
        a = a + residual
        da = da + F32 * np.abs(a)
    return a, da + HALF[type] * (np.abs(a) + da) + TINY[type] + 2.0 ** -140


def norm64(v, dv, kind, weight, bias, eps, offset):
    """A norm of v (off by dv) in 64 bits, and how far off: every value passes through at most D / 64 + 32 additions."""
    if kind == 0:
        return v, dv
    D = v.shape[1]
    chain = (D / 64 + 32) * F32
    mean, dmean = 0.0, 0.0
    if kind == 2:
        mean = v.mean(1, keepdims=True)
        dmean = chain * np.abs(v).mean(1, keepdims=True) + dv.mean(1, keepdims=True)
    c = v - mean
    dc = dv + dmean + F32 * np.abs(c)
    ms = (c * c).mean(1, keepdims=True) + eps
    # a norm's change: no more than the changes' own norm
    rel = chain + np.sqrt((dc * dc).mean(1, keepdims=True) / ms)
    n = c / np.sqrt(ms)
    dn = dc / np.sqrt(ms) + np.abs(n) * (rel + 4 * F32)
    if weight is not None:
        dn = dn * np.abs(weight + offset) + 2 * F32 * np.abs(n * (weight + offset)) + F32 * np.abs(n) * (np.abs(weight) + abs(offset))
        n = n * (weight + offset)
    if bias is not None:
        n = n + bias
        dn = dn + F32 * (np.abs(n) + np.abs(bias))
    return n, dn


def block64(x, y, gate, type, post, pre, eps, alpha, beta, offset, pw, pb, nw, nb):
    """h and n of the norm between two blocks, and how far off each may be."""
    h, dh = alpha * x, F32 * np.abs(alpha * x)
    if y is not None:
        b, db = norm64(y, np.zeros_like(y), post, pw, pb, eps, offset)
        g = beta * (1.0 if gate is None else gate)
        h = h + g * b
        dh = dh + np.abs(g) * db + 3 * F32 * np.abs(g * b) + F32 * np.abs(h)
    n, dn = norm64(h, dh, pre, nw, nb, eps, offset)
    last = lambda v, d: d * (1 + HALF[type]) + HALF[type] * np.abs(v) + TINY[type] + 2.0 ** -140
    return (h, last(h, dh)), (n, last(n, dn))


def to_dev(a, type):
    import torch
    return None if a is None else torch.from_numpy(np.asarray(a, dtype=np.float32)).to("cuda").to(torch_type(type))


def within(got, ref, limit, what=""):
    got = got.double().cpu().numpy() if hasattr(got, "cpu") else np.asarray(got, dtype=np.float64)
    assert got.shape == ref.shape, (what, got.shape, ref.shape)
    err = np.abs(got - ref)
    bad = ~(err <= limit)
    if bad.any():
        i = np.unravel_index(np.argmax(np.where(bad, np.nan_to_num(err / limit, nan=np.inf), 0)), err.shape)
        raise AssertionError(f"{what}: {bad.sum()} of {bad.size} off; at {i}: got {got[i]!r}, wanted {ref[i]!r} within {limit[i]!r}")
