"""NaN keys and queries that are not finite over a cache in 4 bits: rows that use them are NaN, with
their log-normalisers, through every way that a window's or a chunk's results take; the
other rows are what they are without them."""
import math

import numpy as np
import pytest
import torch

import mx4_reference as M
from test_gpu_mx4_attend import Chunk, Window, _f64

pytestmark = pytest.mark.gpu


def _plan(w, splits):
    got = w.B.retro_attend_plan(w.d_, False)
    print("[plan]", got, flush=True)
    assert (got[1] > 1) == (splits > 1)


# one split, whose workgroups write the results, with one and two tiles of rows; several
WINDOWS = [("bf16", 8, 4, 8, 16, 64, 1), ("bf16", 16, 4, 11, 16, 8, 1), ("bf16", 2, 4, 16, 1, 128, 2), ("f32", 8, 4, 8, 16, 16, 1),
           ("f32", 2, 4, 16, 1, 128, 2)]


@pytest.mark.parametrize("what", ["key", "query", "infinite"])
@pytest.mark.parametrize("P,d", [(16, 128), (32, 64)])
@pytest.mark.parametrize("dtype,hk,G,W,batch,pages,splits", WINDOWS)
def test_window(dtype, hk, G, W, batch, pages, splits, P, d, what):
    budget = pages * 16
    w = Window(dtype, hk, G, d, P, [budget - 7 * b for b in range(batch)], W, budget, seed=3)
    _plan(w, splits)
    rows = torch.zeros(batch, W + 1, hk * G, dtype=torch.bool)
    if what == "key":
        # one of the stored keys of sequence 0, KV head 1: rows that use its page
        h, token = 1, 37
        page = token // P
        at = np.flatnonzero(w.sel_np[0, h, :w.num_np[0, h]] == page)
        assert at.size == 1
        ex = M.key_index(P, d)[1]
        w.kc[w.pt[0, page].long(), h, int(ex[token % P, 1])] = 255
        tau = w.step - W + np.arange(W + 1)
        uses = (w.mask_np[0, h, at[0]] < tau) | (np.arange(W + 1) == W)
        rows[0, :, h * G:(h + 1) * G] = torch.from_numpy(uses)[:, None]
        w.k[0][token, h] = 0.0       # (no row that the reference is compared for sees it)
    else:
        for b, r, j in ((0, W, 0), (batch - 1, 1, hk * G - 1)):
            w.q[b, r, j, d - 3] = math.nan if what == "query" else math.inf
            # (a row without a page has no score: it stays (0, -inf))
            known = w.mask_np[b, j // G, :w.num_np[b, j // G]]
            rows[b, r, j] = r == W or bool((known < w.step - W + r).any())
    w.run()
    assert torch.isnan(w.o.cpu()[rows]).all() and torch.isnan(w.z.cpu()[rows]).all()
    assert torch.isfinite(w.o.cpu()[~rows]).all()
    _check_others(w, rows)


def _check_others(w, rows):
    """w.check() of every row outside `rows`."""
    G, W, P = w.G, w.W, w.P
    out, lse, qq = _f64(w.o), _f64(w.z), _f64(torch.where(torch.isfinite(w.q), w.q, torch.zeros_like(w.q)))
    tau, rows = w.step - W + np.arange(W + 1), rows.numpy()
    for b, n in enumerate(w.lens):
        for h in range(w.hk):
            m = w.num_np[b, h]
            pages, known = w.sel_np[b, h, :m], w.mask_np[b, h, :m]
            tok = (pages[:, None] * P + np.arange(P)).reshape(-1)
            known = np.repeat(known, P)
            keep = tok < n
            tok, known = tok[keep], known[keep]
            seen = (tau >= 0)[:, None] & ((known < tau[:, None]) | (np.arange(W + 1) == W)[:, None])
            for j in range(h * G, (h + 1) * G):
                want, to, zz, tz = M.softmax_rows(qq[b, :, j], w.k[b][tok, h], w.v[b][tok, h], seen, w.scale, w.dtype, True)
                to += 4 * M.U * np.abs(want)
                ok, some = ~rows[b, :, j], np.isfinite(zz)
                assert (np.abs(out[b, :, j] - want) <= to)[ok].all(), (b, j)
                assert (lse[b, :, j][ok & ~some] == -np.inf).all()
                ok &= some
                assert (np.abs(lse[b, :, j][ok] - zz[ok]) <= tz[ok]).all(), (b, j)


# batch, KV heads, G, W, pages: partial results of one split, and of several
STEPS = [(1, 2, 4, 3, 16), (16, 8, 4, 8, 16), (2, 1, 8, 0, 16), (1, 2, 4, 16, 128)]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("path", ["step", "split"])
@pytest.mark.parametrize("b,hk,G,W,pages", STEPS)
def test_steps(b, hk, G, W, pages, path, dtype):
    """A stored NaN key: rows that use its page are NaN in the step and stay so in the output cache, the
    others stay finite and near a step without it."""
    from paper_2508_09001_amd.layer import RetroLayer
    P, d, t = 16, 128, 200
    got = []
    for nan in (False, True):
        lay = RetroLayer(batch=b, num_kv_heads=hk, group=G, head_dim=d, page_size=P, budget=pages * P, window=W,
                         max_pages=pages, dtype=dtype, kv="mx4")
        g = torch.Generator().manual_seed(W + hk)
        n = pages * P - 3
        k, v = torch.randn(b, n, hk, d, generator=g), torch.randn(b, n, hk, d, generator=g)
        if nan:
            k[:, 5 * P + 3, :, 7] = math.nan
        for s in range(b):
            lay.prefill(s, k[s], v[s])
        lay.last_loaded[:, :, 5] = t - W // 2 - 1        # half of the past rows may use it
        lay.o_cache.copy_(torch.randn(lay.o_cache.shape, generator=g))
        lay.lse_cache.copy_(torch.randn(lay.lse_cache.shape, generator=g))
        outs = []
        for i in range(2):
            q = torch.randn(b, W + 1, hk * G, d, generator=g)
            kv = torch.randn(b, hk, d, generator=g)
            print(f"[nonfinite] {b, hk, G, W, pages} {path} {dtype} {nan} {i}", flush=True)
            if path == "step":
                lay.step(t + i, q, kv, kv)
            else:
                lay.append(t + i, kv, kv)
                lay.select(t + i, q[:, W])
                lay.attend(t + i, q)
                lay.merge(t + i)
            torch.cuda.synchronize()
            assert lay.num_selected.eq(pages).all()
            outs.append((lay.o_out.cpu(), lay.lse_out.cpu()))
        got.append(outs)
    # first step: rows whose query is newer than the page's last use; the page is then loaded
    # by every head, so that the second one's past rows use it no more, but their cached outputs are NaN
    uses = [r == W or t - W + r > t - W // 2 - 1 for r in range(W + 1)]
    later = [r == W or uses[r + 1] for r in range(W + 1)]
    for i, bad in enumerate((uses, later)):
        (o0, z0), (o, z) = got[0][i], got[1][i]
        assert torch.isfinite(o0).all() and torch.isfinite(z0).all()
        for r, u in enumerate(bad):
            if u:
                assert torch.isnan(o[:, r]).all() and torch.isnan(z[:, r]).all(), (i, r)
            else:
                assert torch.isfinite(o[:, r]).all() and torch.isfinite(z[:, r]).all(), (i, r)
                # the same values in sums that may be rescaled elsewhere: 2e-3 (bf16), 1e-5 of each
                tol = 2 * (2e-3 if dtype == "bf16" else 1e-5)
                assert (o[:, r] - o0[:, r]).abs().max() <= tol and (z[:, r] - z0[:, r]).abs().max() <= tol


@pytest.mark.parametrize("P,d", [(16, 128), (32, 128), (16, 64), (32, 64)])
@pytest.mark.parametrize("token", [3, 707, 1599])
def test_chunk_of_many_rows(P, d, token):
    """A NaN key in front of, inside and at the end of tiles of 256 rows: rows that see it are NaN, those in
    front of it are not, whether or not the stage that holds it is converted for them."""
    seqs, h = [(1500, 100), (600, 900)], 1
    c = Chunk("bf16", 8, 1, d, P, seqs, seed=P + d)
    ex = M.key_index(P, d)[1]
    c.kc[c.pt[0, token // P].long(), h, int(ex[token % P, 0])] = 255
    c.k[0][token, h] = 0.0
    c.run()
    rows = torch.zeros(c.total, c.hk, dtype=torch.bool)
    first = c.front + max(token - 100, 0)
    rows[first:c.starts[1], h] = True
    rows = rows.cuda()
    assert torch.isnan(c.out[rows]).all() and torch.isnan(c.lse[rows]).all()
    assert torch.isfinite(c.out[~rows]).all() and torch.isfinite(c.lse[~rows]).all()
    out, lse, q = _f64(c.out), _f64(c.lse), _f64(c.q).reshape(c.total, 8, d)
    for b, (n, ctx) in enumerate(seqs):
        seen = np.arange(n + ctx) <= ctx + np.arange(n)[:, None]
        sl = slice(c.starts[b], c.starts[b + 1])
        for j in range(8):
            o, to, z, tz = M.softmax_rows(q[sl, j], c.k[b][:, j], c.v[b][:, j], seen, c.scale, "bf16", False)
            ok = ~rows[sl, j].cpu().numpy()
            assert (np.abs(out[sl, j] - o) <= to + M.HALF["bf16"] * np.abs(o))[ok].all(), (b, j)
            assert (np.abs(lse[sl, j] - z) <= tz)[ok].all(), (b, j)
