"""The paged cache in 4 bits: rows stored (with norms and rotation on the way) and read
back, bit for bit against codes made in 64 bits with numpy, and rows of caches in dtype
read back."""
import numpy as np
import pytest
import torch

import chunk_reference as R
import mx4_reference as M

pytestmark = pytest.mark.gpu
TD = {"bf16": torch.bfloat16, "f32": torch.float32}
STEP = 5


def _f64(x):
    return x.detach().cpu().double().numpy()


class Cache:
    """A pool of pages with whatever bytes in them, tables over a part of it."""

    def __init__(self, dtype, hk, G, d, P, ctx, pages, seed=0, mx4=True, unmapped=()):
        from paper_2508_09001_amd import binding as B
        self.B, self.dtype, self.hk, self.G, self.d, self.P, self.mx4 = B, dtype, hk, G, d, P, mx4
        g = torch.Generator().manual_seed(seed)
        batch, mp = len(ctx), pages
        self.pool = batch * mp + 3
        self.ctx = list(ctx)
        pt = torch.randperm(self.pool, generator=g)[:batch * mp].view(batch, mp).int()
        for b, p in unmapped:
            pt[b, p] = -1 if p % 2 else self.pool
        self.pt = pt.cuda()
        size = M.block_bytes(P, d) if mx4 else P * d * (2 if dtype == "bf16" else 4)
        self.kc, self.vc = (torch.randint(0, 255, (self.pool, hk, size), generator=g, dtype=torch.uint8).cuda()
                            for _ in range(2))
        self.lens = torch.tensor(ctx, dtype=torch.int32).cuda()
        self.digest = torch.full((batch, hk, mp, 2, d), 77.0, dtype=TD[dtype]).cuda()
        self.loaded = torch.full((batch, hk, mp), -9, dtype=torch.int32).cuda()
        self.dims = B.Dims(batch, hk, G, d, P, P, 0, mp, self.pool, B.RETRO_BF16 if dtype == "bf16" else B.RETRO_F32,
                           0.0, 0, B.RETRO_FLAG_KV_MX4 if mx4 else 0)
        self.cache = B.KVCache(*(x.data_ptr() for x in (self.kc, self.vc, self.digest, self.pt, self.lens,
                                                        self.loaded)))

    def chunk(self, n, start=None, front=0, behind=0):
        at = np.cumsum([front] + list(n))
        self._rs = torch.tensor(at, dtype=torch.int32).cuda()
        self._sp = torch.tensor(self.ctx if start is None else start, dtype=torch.int32).cuda()
        return self.B.Chunk(self._rs.data_ptr(), self._sp.data_ptr(), int(at[-1]) + behind, 0)

    def append(self, n, k, v, rotary=None, q=None, q_out=None, start=None, front=0, behind=0, step=STEP):
        r = rotary or self.B.Rotary(None, 0, 0, 0, 0.0, None, None)
        ch = self.chunk(n, start, front, behind)
        print(f"[mx4 store] {self.dtype} hk={self.hk} d={self.d} P={self.P} mx4={self.mx4} n={list(n)[:8]} "
              f"ctx={self.ctx[:8]}", flush=True)
        self.B.retro_append_kv_rotary(self.dims, step, self.cache, ch, r, q, 0 if q is None else q.stride(0), k,
                                      k.stride(0), v, v.stride(0), q_out)
        torch.cuda.synchronize()

    def read(self, n, start, keys=True, vals=True, front=0, behind=0):
        ch = self.chunk(n, start, front, behind)
        out = [torch.full((ch.n_rows, self.hk, self.d), 3.0, dtype=TD[self.dtype]).cuda() if x else None
               for x in (keys, vals)]
        print(f"[mx4 read] {self.dtype} d={self.d} P={self.P} mx4={self.mx4} n={list(n)[:8]}", flush=True)
        self.B.retro_read_kv(self.dims, self.cache, ch, *out)
        torch.cuda.synchronize()
        return out


def _rows(dtype, n, hk, d, seed, loud=True):
    g = torch.Generator().manual_seed(seed)
    x = torch.randn(n, hk, d, generator=g) * torch.exp2(torch.randint(-3, 4, (n, hk, 1), generator=g).float())
    if loud:
        x[:, :, 5] *= 8
    # elements on the borders between codes, and just beside them
    at = torch.tensor([0, .25, .5, .75, 1, 1.25, 1.5, 1.75, 2, 2.5, 3, 3.5, 4, 5, 6, 7, 7.5])
    m = torch.randint(0, 17, (n, hk, 32), generator=g)
    edge = at[m] * torch.where(torch.rand(n, hk, 32, generator=g) < .5, -1.0, 1.0)
    edge *= 1 + torch.randint(-1, 2, edge.shape, generator=g) * (2.0 ** -7 if dtype == "bf16" else 2.0 ** -23)
    x[:, :, d - 32:] = edge
    return x.to(TD[dtype])


def _check_pages(c, n, k, v, before):
    """Pages, digests, lengths and last_loaded after an append of k, v (as they would be
    stored in dtype) at the sequences' ends."""
    kb, vb, pt = (_x.cpu().numpy() for _x in (before[0], before[1], c.pt))
    ki, vi = M.key_index(c.P, c.d), M.value_index(c.P, c.d)
    at, dig = 0, _f64(before[2])
    loaded = before[3].cpu().numpy()
    for b, m in enumerate(n):
        end = c.ctx[b] + m
        for lp in range(c.ctx[b] // c.P, -(-end // c.P) if m else 0):
            ph = pt[b, lp]
            s0, s1 = max(c.ctx[b] - lp * c.P, 0), min(end - lp * c.P, c.P)
            rows = slice(at + lp * c.P + s0 - c.ctx[b], at + lp * c.P + s1 - c.ctx[b])
            for h in range(c.hk):
                for cache, idx, x in ((kb, ki, k), (vb, vi, v)):
                    code, e = M.encode(x[rows, h])
                    page, nib, ex = cache[ph, h], idx[0][s0:s1], idx[1][s0:s1]
                    full = np.stack([page[:c.P * c.d // 2] & 15, page[:c.P * c.d // 2] >> 4], -1).reshape(-1)
                    full[nib] = code
                    page[:c.P * c.d // 2] = full[0::2] | full[1::2] << 4
                    page[ex] = e
                held = M.get(kb[ph, h], ki)[s0:s1]
                lo, hi = held.min(0), held.max(0)
                if s0:
                    lo, hi = np.minimum(lo, dig[b, h, lp, 0]), np.maximum(hi, dig[b, h, lp, 1])
                dig[b, h, lp] = lo, hi
                loaded[b, h, lp] = STEP - 1
        at += m
    assert np.array_equal(c.kc.cpu().numpy(), kb), "keys"
    assert np.array_equal(c.vc.cpu().numpy(), vb), "values"
    assert np.array_equal(_f64(c.digest), dig), "digests"
    assert np.array_equal(c.loaded.cpu().numpy(), loaded)


def _before(c):
    return [x.clone() for x in (c.kc, c.vc, c.digest, c.loaded)]


SHAPES = [("bf16", 16, 128, 2), ("bf16", 32, 128, 1), ("bf16", 16, 64, 3), ("bf16", 32, 64, 2),
          ("f32", 16, 128, 1), ("f32", 32, 128, 2), ("f32", 16, 64, 2), ("f32", 32, 64, 1)]


@pytest.mark.parametrize("dtype,P,d,hk", SHAPES)
@pytest.mark.parametrize("n,ctx", [([1], [0]), ([1] * 70, list(range(70))), ([3, 0, 40, 17, 1], [0, 5, 15, 33, 64]),
                                   ([257], [31])], ids=["first", "tokens", "ragged", "long"])
def test_append_and_read(dtype, P, d, hk, n, ctx):
    c = Cache(dtype, hk, 2, d, P, ctx, max(-(-(a + b) // P) for a, b in zip(n, ctx)) + 1, seed=P + d)
    rows = sum(n)
    k, v = (_rows(dtype, rows, hk, d, seed) for seed in (1, 2))
    before = _before(c)
    c.append(n, k.cuda(), v.cuda())
    assert c.lens.tolist() == [a + b for a, b in zip(n, ctx)]
    _check_pages(c, n, _f64(k), _f64(v), before)
    ko, vo = c.read(n, ctx)
    assert np.array_equal(_f64(ko), M.rounded(_f64(k))) and np.array_equal(_f64(vo), M.rounded(_f64(v)))


@pytest.mark.parametrize("dtype,P,d,hk", SHAPES[:2] + SHAPES[4:7])
@pytest.mark.parametrize("rot,interleaved,norm", [(64, False, True), (32, True, False)])
def test_append_rotated(dtype, P, d, hk, rot, interleaved, norm):
    """Keys as the cache in dtype holds them, then in 4 bits; queries as there; strided inputs."""
    from paper_2508_09001_amd import binding as B
    n, ctx, G, mp = [33, 1, 20], [7, 48, 0], 2, 6
    plain, c = (Cache(dtype, hk, G, d, P, ctx, mp, seed=3, mx4=x) for x in (False, True))
    rows, hq = sum(n), hk * G
    tab = torch.from_numpy(R.table(mp * P, rot, 1e4)).cuda()
    w = [(1 + 0.1 * torch.randn(d)).to(TD[dtype]).cuda() if norm else None for _ in range(2)]
    rotary = B.Rotary(tab.data_ptr(), mp * P, rot, int(interleaved), 1e-5, *(None if x is None else x.data_ptr()
                                                                            for x in w))
    wide = torch.randn(rows + 3, (hq + 2 * hk) * d + 16).to(TD[dtype]).cuda()
    q, k, v = (x.unflatten(1, (-1, d)) for x in wide[:, 16:].split([hq * d, hk * d, hk * d], 1))
    outs = []
    before = _before(c)
    for cache in (plain, c):
        qo = torch.full((rows + 3, hq, d), 9.0, dtype=TD[dtype]).cuda()
        cache.append(n, k, v, rotary, q, qo, front=1, behind=2)
        outs.append(qo)
    assert torch.equal(*outs) and (outs[0][0] == 9).all() and (outs[0][-2:] == 9).all()
    ko, vo = plain.read(n, ctx)
    assert torch.equal(vo, v[1:-2])
    _check_pages(c, n, _f64(ko), _f64(vo), before)


def test_special_blocks():
    """NaN and infinities make their block NaN, and no other; zeros, the smallest and the largest."""
    for dtype in ("bf16", "f32"):
        c = Cache(dtype, 1, 1, 128, 16, [0], 2, seed=1)
        x = torch.zeros(9, 1, 128)
        x[0, 0, 3], x[1, 0, 40], x[2, 0, 70] = float("nan"), float("inf"), -float("inf")
        x[3, 0] = 2.0 ** -126 * torch.linspace(-1, 1, 128)
        x[4, 0] = torch.finfo(TD[dtype]).max * torch.linspace(-1, 1, 128)
        x[5, 0, ::2] = -0.0
        x[6, 0] = 2.0 ** -124 * torch.linspace(-3, 3, 128)
        x[7, 0] = torch.finfo(TD[dtype]).smallest_normal / 2
        x[8] = _rows(dtype, 1, 1, 128, 4).float()
        x[0, 0, 32:], x[1, 0, :32] = 1.5, -3
        x = x.to(TD[dtype]).cuda()
        c.append([9], x, x)
        want = M.rounded(_f64(x))
        for got in c.read([9], [0]):
            assert np.array_equal(_f64(got), want, equal_nan=True)
        assert np.isnan(want[:3]).sum() == 96 and np.isfinite(want[3:]).all()


@pytest.mark.parametrize("mx4", [True, False])
@pytest.mark.parametrize("dtype,P,d,hk", SHAPES)
def test_read_edges(dtype, P, d, hk, mx4):
    """Rows past the lengths and of pages that are not mapped are zeros, those of no sequence stay;
    keys or values alone; sequences without rows or with a negative start."""
    ctx = [3 * P + 5, 2 * P, 0, 9, 4]
    c = Cache(dtype, hk, 1, d, P, [0] * 5, 4, seed=2, mx4=mx4)
    rows = sum(ctx)
    k, v = (_rows(dtype, rows, hk, d, s).cuda() for s in (3, 4))
    c.append(ctx, k, v)
    c.pt[0, 1] = -1
    c.pt[1, 0] = c.pool
    n, start = [4 * P + 3, P, 2, 0, 3], [1, P - 2, 0, 0, -1]
    for keys, vals in ((True, True), (True, False), (False, True)):
        got = c.read(n, start, keys, vals, front=2, behind=3)
        at = np.cumsum([0] + ctx)
        for x, src in zip(got, (k, v)):
            if x is None:
                continue
            want = np.full((sum(n) + 5, hk, d), 3.0)
            row = 2
            for b, m in enumerate(n):
                for j in range(m):
                    p = start[b] + j
                    lost = b == 0 and p // P == 1 or b == 1 and p // P == 0
                    if start[b] >= 0:
                        want[row + j] = _f64(src[at[b] + p]) if p < ctx[b] and not lost else 0
                        if mx4 and p < ctx[b] and not lost:
                            want[row + j] = M.rounded(want[row + j])
                row += m
            assert np.array_equal(_f64(x), want)


def test_rows_without_a_page_are_dropped():
    P, d, hk = 16, 128, 2
    c = Cache("bf16", hk, 1, d, P, [10, 0, 5], 4, seed=5, unmapped=[(0, 2), (1, 0)])
    n = [40, 3, 30]
    k, v = (_rows("bf16", sum(n), hk, d, s) for s in (6, 7))
    before = _before(c)
    c.append(n, k.cuda(), v.cuda())
    assert c.lens.tolist() == [32, 0, 35]
    ko, vo = c.read([22, 3, 30], [10, 0, 5])
    assert np.array_equal(_f64(ko[:22]), M.rounded(_f64(k[:22]))) and (ko[22:25] == 0).all()
    assert np.array_equal(_f64(vo[25:]), M.rounded(_f64(v[43:])))
    lost = c.pt.long()[2, 3]   # (past the third sequence's last page: left as it was)
    assert torch.equal(c.kc[lost], before[0][lost])


def test_token_by_token_is_the_chunk():
    """One row a call, in front of and behind page ends, gives the pages of one call."""
    P, d, hk = 16, 64, 2
    one, many = (Cache("bf16", hk, 1, d, P, [13], 4, seed=8) for _ in range(2))
    for c in (one, many):
        c.digest.zero_()
    k, v = (_rows("bf16", 40, hk, d, s).cuda() for s in (9, 10))
    one.append([40], k, v)
    for i in range(40):
        many.append([1], k[i:i + 1], v[i:i + 1])
        many.ctx = [14 + i]
    for name in ("kc", "vc", "digest", "loaded", "lens"):
        assert torch.equal(getattr(one, name), getattr(many, name)), name
