"""Blocks of 32 elements in 4 bits, pages of them and attention over what they stand
for, in 64 bits with numpy, and how far a correctly rounded implementation may be off."""
from __future__ import annotations

import numpy as np

HALF = {"bf16": 2.0 ** -8, "f32": 2.0 ** -24}   # half a step, relative to the value
U = 2.0 ** -24                                  # half a step of fp32
LEVELS = np.array([0, 0.5, 1, 1.5, 2, 3, 4, 6])


def encode(x):
    """(codes [..., d], exponents [..., d / 32]) of x [..., d], element by element from the
    distances to the eight magnitudes."""
    b = np.asarray(x, dtype=np.float64).reshape(*x.shape[:-1], x.shape[-1] // 32, 32)
    with np.errstate(invalid="ignore"):
        top = np.abs(b).max(-1)
        f = np.floor(np.log2(np.where((top > 0) & np.isfinite(top), top, 1)))
        f += (np.exp2(f + 1) <= top) * 1.0 - (np.exp2(f) > top) * 1.0   # (log2 may round up or down)
        e = np.where(top > 0, 127 + f - 2 + (top >= 1.75 * np.exp2(f)), 2)
    e = np.where(np.isfinite(top), np.clip(e, 2, 252), 255).astype(np.int64)
    t = np.abs(np.where(np.isfinite(b), b, 0)) / np.exp2(np.where(e == 255, 127, e) - 127.0)[..., None]
    away = np.abs(t[..., None] - LEVELS)
    near = away == away.min(-1, keepdims=True)
    first, last = near.argmax(-1), 7 - near[..., ::-1].argmax(-1)
    code = np.where(first % 2 == 0, first, last)                        # of two, the even one
    code = np.where(t > 6, 7, code) + 8 * np.signbit(b)
    return code.reshape(x.shape).astype(np.uint8), e.astype(np.uint8)


def decode(code, e):
    v = LEVELS[code & 7] * np.where(code & 8, -1.0, 1.0)
    scale = np.where(e == 255, np.nan, np.exp2(e.astype(np.float64) - 127))
    return (v.reshape(*v.shape[:-1], v.shape[-1] // 32, 32) * scale[..., None]).reshape(v.shape)


def rounded(x):
    return decode(*encode(x))


def block_bytes(P, d):
    return P * d // 2 + P * d // 32


def key_index(P, d):
    """Nibble of element (token, i), byte of the exponent of (token, block), in a key page."""
    t, i, j = np.arange(P)[:, None], np.arange(d), np.arange(d // 32)
    return t * d + i, P * d // 2 + t * (d // 32) + j


def value_index(P, d):
    t, i, j = np.arange(P)[:, None], np.arange(d), np.arange(d // 32)
    part = d // 16
    return ((t // 4 * 16 + i // part) * 4 + t % 4) * part + i % part, P * d // 2 + (t // 4 * (d // 32) + j) * 4 + t % 4


def put(pages, index, code, e):
    """Writes codes and exponents [pages..., P, ...] to pages [..., bytes]."""
    nib, ex = index
    out = np.zeros((*code.shape[:-2], nib.size), np.uint8)
    out[..., nib] = code
    pages[..., :nib.size // 2] = out[..., 0::2] | out[..., 1::2] << 4
    pages[..., ex] = e


def get(pages, index):
    """What pages [..., bytes] stand for, [..., P, d]."""
    nib, ex = index
    raw = pages[..., nib // 2]
    return decode(np.where(nib % 2, raw >> 4, raw & 15), pages[..., ex])


def softmax_rows(q, k, v, seen, scale, dtype, split):
    """(out, tolerance, lse, tolerance) of q [rows][d] over k, v [L][d] where seen [rows][L].

    k and v are exact in the matrix cores' type.  A score is a sum of d products (of 3 d for
    fp32 rows, which are taken apart into three terms) in fp32, scaled; its error moves a
    weight by the same relative amount, to which the subtraction of the maximum, the scale's product and the exponential add 4 U
    and the exponent's own rounding 2 U of its size (less than 150).  The sums over the keys and the rescalings on the way
    round at most once per key and term and twice per 32 keys, the joins a few times.  A weight of a bf16 row is
    rounded to bf16 (2^-8) or, as two halves, left 2^-16 of it short.  A weight under 2^-126 of the largest may come out as zero,
    which takes at most so much times its value."""
    d, L = q.shape[1], k.shape[0]
    terms = 1 if dtype == "bf16" else 3
    some = seen.any(1)
    q, k, v = (np.where(np.isfinite(x), x, 0) if x is not q else x for x in (q, k, v))
    s = np.where(seen, q @ k.T * scale, -np.inf)
    ds = np.where(seen, (terms * d + 3) * U * scale * (np.abs(q) @ np.abs(k).T), 0).max(1, initial=0)
    m = np.where(some, s.max(1, initial=-np.inf), 0)
    p = np.exp(s - m[:, None])
    total = np.where(some, p.sum(1), 1)
    out = p @ v / total[:, None]
    lse = np.where(some, m + np.log(total), -np.inf)
    size = p @ np.abs(v) / total[:, None]
    sums = terms + 1 if dtype == "f32" else 2
    w = 2 * ds + (sums * L + L / 16 + 24 + 300) * U
    weight = (2.0 ** -16 if split else 2.0 ** -8) if dtype == "bf16" else 0.0
    lost = 2.0 ** -126 * np.abs(v).sum(0)
    return out, (2 * w + weight)[:, None] * size + lost, lse, w + 4 * U * np.abs(np.where(some, lse, 0))
