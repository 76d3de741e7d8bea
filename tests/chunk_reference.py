"""Norm and rotation, the paged cache's rows and causal attention over them, in 64
bits with numpy, and how far a correctly rounded implementation may be off."""
from __future__ import annotations

import numpy as np

HALF = {"bf16": 2.0 ** -8, "f32": 2.0 ** -24}   # half a step, relative to the value
U = 2.0 ** -24                                  # half a step of fp32


def table(positions, rot, base):
    """[positions][rot / 2][2] cosine and sine, rounded to fp32."""
    freq = base ** (-np.arange(0, rot, 2) / max(rot, 1))
    a = np.arange(positions)[:, None] * freq
    return np.stack([np.cos(a), np.sin(a)], axis=-1).astype(np.float32)


def turn(x, weight, tab, positions, rot, interleaved, eps, dtype):
    """(y, tolerance) of x [rows][heads][d] at positions [rows].

    The sum of squares has at most 13 roundings, the mean, eps, root, quotient and
    three products one each, the rotation three: below 32 U on each of the two
    terms; then one rounding to the type."""
    x = x.astype(np.float64)
    if weight is not None:
        x = x / np.sqrt((x * x).mean(-1, keepdims=True) + eps) * weight.astype(np.float64)
    y, size = x.copy(), np.abs(x)
    if rot:
        cs = tab[positions].astype(np.float64)[:, None]
        c, s = cs[..., 0], cs[..., 1]
        i = np.arange(rot // 2)
        a, b = (2 * i, 2 * i + 1) if interleaved else (i, i + rot // 2)
        y[..., a] = x[..., a] * c - x[..., b] * s
        y[..., b] = x[..., b] * c + x[..., a] * s
        size[..., a] = size[..., b] = size[..., a] + size[..., b]
    return y, HALF[dtype] * np.abs(y) + 32 * U * size


def attend(q, k, v, positions, stored, scale, dtype):
    """(out, tolerance, lse, tolerance) of q [n][hq][d] at positions [n] over k, v
    [len][hk][d], where stored [len] says which tokens count.

    A score is a sum of d products in fp32, scaled; its error moves a weight by
    the same relative amount, to which the exponential adds 4 U.  The sums over
    the keys and the rescalings on the way round at most once per key and twice
    per 32 keys, and the two ways' join a few times.  A bf16 weight is rounded
    once for its product, and the result once."""
    n, hq, d = q.shape
    L, hk = k.shape[0], k.shape[1]
    out, lse = np.zeros((n, hq, d)), np.full((n, hq), -np.inf)
    t_out, t_lse = np.zeros((n, hq, d)), np.zeros((n, hq))
    q, k, v = (x.astype(np.float64) for x in (q, k, v))
    seen = (np.arange(L) <= positions[:, None]) & stored
    some = seen.any(1)
    if not some.any():
        return out, t_out, lse, t_lse
    for h in range(hq):
        kh, vh = k[:, h // (hq // hk)], np.where(stored[:, None], v[:, h // (hq // hk)], 0)
        kh = np.where(stored[:, None], kh, 0)
        s = np.where(seen, q[:, h] @ kh.T * scale, -np.inf)
        ds = (d + 3) * U * scale * (np.abs(q[:, h]) @ np.abs(kh).T)
        ds = np.where(seen, ds, 0).max(1)
        m = np.where(some, s.max(1, initial=-np.inf), 0)
        p = np.exp(s - m[:, None])
        total = np.where(some, p.sum(1), 1)
        out[:, h] = p @ vh / total[:, None]
        lse[some, h] = (m + np.log(total))[some]
        size = p @ np.abs(vh) / total[:, None]
        w = 2 * ds + (L + L / 16 + 24) * U
        weight = HALF[dtype] if dtype == "bf16" else 0.0
        t_out[:, h] = (2 * w + weight)[:, None] * size + HALF[dtype] * np.abs(out[:, h])
        t_lse[:, h] = w + 4 * U * np.abs(np.where(some, lse[:, h], 0))
    return out, t_out, lse, t_lse
