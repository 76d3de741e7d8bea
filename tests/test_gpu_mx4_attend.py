"""Attention over a paged cache in 4 bits, by chunks of rows and by the retrospective
window over selected pages, against 64-bit references: lengths around every tile, pages
that are not mapped, rows that nothing is left for, and whatever lies in unused slots."""
import numpy as np
import pytest
import torch

import mx4_reference as M

pytestmark = pytest.mark.gpu
TD = {"bf16": torch.bfloat16, "f32": torch.float32}


def _f64(x):
    return x.detach().cpu().double().numpy()


class Paged:
    """Sequences of stored tokens in a pool whose unused slots hold whatever bytes, NaN exponents
    among them, behind tables whose unused entries are out of range."""

    def __init__(self, dtype, hk, G, d, P, lens, seed=0, unmapped=(), grow=1.0, spare=2):
        from paper_2508_09001_amd import binding as B
        self.B, self.dtype, self.hk, self.G, self.d, self.P, self.lens = B, dtype, hk, G, d, P, lens
        rng = np.random.default_rng(seed)
        batch = len(lens)
        self.mp = max(max(-(-n // P) for n in lens), 1) + spare
        self.pool = batch * self.mp + 5
        pt = rng.permutation(self.pool)[:batch * self.mp].reshape(batch, self.mp).astype(np.int32)
        kc, vc = (rng.integers(0, 256, (self.pool, hk, M.block_bytes(P, d)), dtype=np.uint8) for _ in range(2))
        kc[..., P * d // 2:] = vc[..., P * d // 2:] = 255
        self.k, self.v, self.stored = [], [], []
        for b, n in enumerate(lens):
            both = []
            for cache, index, size in ((kc, M.key_index(P, d), grow), (vc, M.value_index(P, d), 1.0)):
                used = -(-n // P)
                x = np.zeros((used * P, hk, d))
                x[:n] = rng.normal(size=(n, hk, d)) * size
                x[:n, :, 3] *= 4
                code, e = M.encode(x.astype(np.float32))
                e[n:] = 255
                both.append(M.decode(code, e)[:n])
                for p in range(used):
                    sl = slice(p * P, (p + 1) * P)
                    M.put(cache[pt[b, p]], index, code[sl].transpose(1, 0, 2), e[sl].transpose(1, 0, 2))
            keep = np.ones(n, bool)
            for p in range(self.mp):
                if p * P >= n:
                    pt[b, p] = -1 if p % 2 else self.pool + 7
            for bb, p in unmapped:
                if bb == b:
                    pt[b, p] = -1 if p % 2 else self.pool
                    keep[p * P:(p + 1) * P] = False
            self.k.append(both[0])
            self.v.append(both[1])
            self.stored.append(keep)
        self.kc, self.vc, self.pt = (torch.from_numpy(x).cuda() for x in (kc, vc, pt))
        self.len_t = torch.tensor(lens, dtype=torch.int32).cuda()
        self.z = torch.zeros(8, dtype=torch.int32, device="cuda")
        self.cache = B.KVCache(self.kc.data_ptr(), self.vc.data_ptr(), self.z.data_ptr(), self.pt.data_ptr(),
                               self.len_t.data_ptr(), self.z.data_ptr())

    def dims(self, budget=None, window=0, sm_scale=0.0):
        return self.B.Dims(len(self.lens), self.hk, self.G, self.d, self.P, budget or self.P, window, self.mp, self.pool,
                           self.B.RETRO_BF16 if self.dtype == "bf16" else self.B.RETRO_F32, sm_scale, 0,
                           self.B.RETRO_FLAG_KV_MX4)


class Chunk(Paged):
    """n new rows of each sequence behind ctx, all stored; rows of no sequence in front and behind."""

    def __init__(self, dtype, hk, G, d, P, seqs, seed=0, sm_scale=0.0, longest=0, **kw):
        super().__init__(dtype, hk, G, d, P, [n + c for n, c in seqs], seed, **kw)
        B, hq = self.B, hk * G
        self.seqs, self.front, self.rows = seqs, 1, sum(n for n, _ in seqs)
        self.total = self.front + self.rows + 2
        self.starts = np.concatenate([[0], np.cumsum([n for n, _ in seqs])]) + self.front
        g = torch.Generator().manual_seed(seed)
        self.wide = torch.randn(self.total, (hq + 2) * d, generator=g).to(TD[dtype]).cuda()
        self.q = self.wide[:, d:(hq + 1) * d]
        self.rs = torch.tensor(self.starts, dtype=torch.int32).cuda()
        self.sp = torch.tensor([c for _, c in seqs], dtype=torch.int32).cuda()
        self.scale = sm_scale or d ** -0.5
        self.d_ = self.dims(sm_scale=sm_scale)
        self.chunk = B.Chunk(self.rs.data_ptr(), self.sp.data_ptr(), self.total, longest)
        self.out = torch.full((self.total, hq, d), 5.0).to(TD[dtype]).cuda()
        self.lse = torch.full((self.total, hq), 5.0).cuda()
        self.ws_bytes = B.retro_chunk_workspace_size(self.d_, self.total)
        self.ws = torch.zeros(self.ws_bytes, dtype=torch.uint8, device="cuda")
        print(f"[mx4 chunk] {dtype} hk={hk} G={G} d={d} P={P} seqs={seqs[:6]} {kw}", flush=True)

    def run(self, lse=True):
        self.B.retro_chunk_attend(self.d_, self.cache, self.chunk, self.q, self.q.stride(0), self.out,
                                  self.lse if lse else None, self.ws, self.ws_bytes)
        torch.cuda.synchronize()
        return self

    def check(self, lens=None):
        out, lse, G = _f64(self.out), _f64(self.lse), self.G
        q = _f64(self.q).reshape(self.total, self.hk * G, self.d)
        for b, (n, c) in enumerate(self.seqs):
            L = n + c
            keep = self.stored[b] & (np.arange(L) < (L if lens is None else lens[b]))
            seen = (np.arange(L) <= c + np.arange(n)[:, None]) & keep
            sl = slice(self.starts[b], self.starts[b + 1])
            for h in range(self.hk * G if n else 0):
                k, v = (np.where(keep[:, None], x[b][:, h // G], 0) for x in (self.k, self.v))
                o, to, z, tz = M.softmax_rows(q[sl, h], k, v, seen, self.scale, self.dtype, n * G <= 32)
                to += M.HALF[self.dtype] * np.abs(o)
                eo, some = np.abs(out[sl, h] - o), np.isfinite(z)
                assert (eo <= to).all(), f"sequence {b}: out off by {np.nanmax(eo - to)}, {np.isnan(eo).sum()} NaN"
                assert (out[sl, h][~some] == 0).all() and (lse[sl, h][~some] == -np.inf).all()
                assert (np.abs(lse[sl, h][some] - z[some]) <= tz[some]).all(), f"sequence {b}: lse"
        for i in [*range(self.front), *range(self.front + self.rows, self.total)]:
            assert (self.out[i] == 5.0).all() and (self.lse[i] == 5.0).all()


SEQS = [
    [(1, 0)],
    [(1, c) for c in (0, 1, 15, 16, 30, 31, 32, 33, 62, 63, 64, 65, 127, 200, 255, 256, 257)],
    [(1, 4099)],
    [(2, 700), (1, 1), (8, 255), (0, 50), (0, 0), (7, 0), (3, 2000)],
    [(33, 0), (64, 31), (5, 0), (65, 64)],
    [(257, 0), (1, 900)],
    [(130, 1000), (63, 1)],
    [(0, 0), (0, 17)],
]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("P,d,hk,G", [(16, 128, 2, 4), (32, 128, 1, 3), (16, 64, 1, 16), (32, 64, 3, 1)])
@pytest.mark.parametrize("seqs", SEQS, ids=[str(i) for i in range(len(SEQS))])
def test_chunks(dtype, P, d, hk, G, seqs):
    Chunk(dtype, hk, G, d, P, seqs, seed=P + d + G).run().check()


# enough work for tiles of 256 rows (bf16), whose stages of 64 keys and parts end inside
# the sequences: at least 1024 steps of 64 keys over tiles and KV heads
LARGE = [
    ([(700, 0), (300, 2500), (64, 1000), (1, 700), (9, 130)], 8, 4),
    ([(1500, 100), (600, 900)], 8, 1),
    ([(200, 1500), (130, 3)], 4, 16),
    ([(517, 1400), (300, 333)], 9, 3),
]


@pytest.mark.parametrize("P,d", [(16, 128), (32, 128), (16, 64), (32, 64)])
@pytest.mark.parametrize("seqs,hk,G", LARGE, ids=[str(i) for i in range(len(LARGE))])
def test_large_chunks(P, d, seqs, hk, G):
    Chunk("bf16", hk, G, d, P, seqs, seed=P + d + G).run().check()


def test_large_chunks_cut_unmapped_or_short():
    Chunk("f32", 2, 4, 64, 16, [(700, 0), (300, 1500)], seed=2).run().check()
    Chunk("bf16", 2, 4, 128, 16, [(150, 9000), (1, 5000)], seed=12).run().check()
    un = [(0, 0), (0, 50), (0, 107), (1, 0), (1, 1), (2, 3), (2, 62)]
    Chunk("bf16", 8, 4, 128, 16, [(700, 1000), (300, 0), (40, 960)], seed=13, unmapped=un).run().check()
    for P, d in ((32, 64), (16, 128)):
        c = Chunk("bf16", 8, 4, d, P, [(700, 1000), (300, 800), (300, 0)], seed=14)
        lens = [1350, 500, 0]
        c.len_t.copy_(torch.tensor(lens, dtype=torch.int32))
        c.run().check(lens)


def test_large_chunks_same_results_again():
    """The same call gives the same bits, also told the longest run, on a workspace that other dims used."""
    c = Chunk("bf16", 8, 4, 128, 16, [(400, 2000), (1, 3000), (30, 100)], seed=19)
    other = Chunk("f32", 3, 1, 64, 32, [(100, 900)], seed=18)
    c.run().check()
    want, z = c.out.clone(), c.lse.clone()
    other.ws, other.ws_bytes = c.ws, c.ws_bytes
    for _ in range(3):
        other.run().check()
        c.out.fill_(5.0)
        c.run()
        assert torch.equal(c.out, want) and torch.equal(c.lse, z)
    c.chunk.longest = 400
    c.run().check()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("P,d", [(16, 128), (32, 64)])
def test_chunks_unmapped(dtype, P, d):
    c = Chunk(dtype, 2, 4, d, P, [(40, 100), (1, 77), (3, 0), (300, 40)], seed=4,
              unmapped=[(0, 1), (0, 4), (1, 0), (1, 2), (2, 0), (3, 3)])
    c.run().check()
    c.out.fill_(5.0)
    c.lse.fill_(5.0)
    c.len_t.copy_(torch.tensor([60, 0, 2, 339], dtype=torch.int32))   # fewer stored than the rows' positions
    c.run().check(lens=[60, 0, 2, 339])


def test_chunks_scores_of_any_size():
    for grow, scale in ((30.0, 0.0), (1e4, 1e-6), (1e-3, 3e4)):
        Chunk("bf16", 1, 4, 64, 16, [(1, 500), (70, 130)], seed=6, grow=grow, sm_scale=scale).run().check()
        Chunk("f32", 1, 4, 64, 16, [(1, 500), (40, 130)], seed=6, grow=grow, sm_scale=scale).run().check()


def test_chunks_many_sequences():
    """More sequences than a wavefront has lanes, and than a workgroup has threads."""
    for n in (65, 530):
        seqs = [(1 + (i % 5 == 3) * 9, (i * 37) % 90) for i in range(n)]
        Chunk("bf16", 1, 4, 64, 16, seqs, seed=n).run().check()


def test_chunks_without_lse_and_in_place():
    c = Chunk("bf16", 2, 4, 128, 16, [(5, 300), (90, 10)], seed=2).run()
    want = c.out.clone()
    c.out.fill_(5.0)
    c.run(lse=False)
    assert torch.equal(c.out, want)
    q = c.q.contiguous()
    c.B.retro_chunk_attend(c.d_, c.cache, c.chunk, q, q.stride(0), q, None, c.ws, c.ws_bytes)
    got = q.view(c.total, -1, c.d)[c.front:c.front + c.rows]
    assert torch.equal(got, want[c.front:c.front + c.rows])


def test_chunks_nan():
    """A NaN key makes the rows that see it NaN; other sequences and heads stay."""
    c = Chunk("bf16", 2, 2, 64, 16, [(4, 60), (3, 40)], seed=3)
    ex = M.key_index(16, 64)[1]
    c.kc[c.pt[0, 1].long(), 1, int(ex[2, 0])] = 255          # token 18 of sequence 0, head 1
    c.run()
    hit = torch.isnan(c.out[1:5, 2:]).all() and torch.isnan(c.lse[1:5, 2:]).all()
    assert hit and torch.isfinite(c.out[1:5, :2]).all() and torch.isfinite(c.out[5:8]).all()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_chunks_replayed(dtype):
    """Captured once, replayed for other lengths and rows, with eager calls of the same workspace between."""
    c = Chunk(dtype, 2, 4, 128, 16, [(9, 400), (1, 900), (40, 0)], seed=5)
    c.run().check()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        c.B.retro_chunk_attend(c.d_, c.cache, c.chunk, c.q, c.q.stride(0), c.out, c.lse, c.ws, c.ws_bytes)
    for lens, starts in (([409, 901, 40], [400, 900, 0]), ([300, 64, 17], [291, 63, 0]), ([9, 1, 0], [0, 0, 0])):
        c.len_t.copy_(torch.tensor(lens, dtype=torch.int32))
        c.sp.copy_(torch.tensor(starts, dtype=torch.int32))
        c.run()
        want, z = c.out.clone(), c.lse.clone()
        for _ in range(3):
            c.out.fill_(5.0)
            c.lse.fill_(5.0)
            graph.replay()
            torch.cuda.synchronize()
            assert torch.equal(c.out, want) and torch.equal(c.lse, z)


# ---- the window over selected pages ---------------------------------------------------


class Window(Paged):
    def __init__(self, dtype, hk, G, d, P, lens, W, budget, seed=0, step=40, sm_scale=0.0, counts=None, **kw):
        super().__init__(dtype, hk, G, d, P, lens, seed, **kw)
        B, hq, batch = self.B, hk * G, len(lens)
        rng = np.random.default_rng(seed + 1)
        self.W, self.step, self.scale = W, step, sm_scale or d ** -0.5
        self.d_ = self.dims(budget, W, sm_scale)
        self.k_max = B.retro_k_max(self.d_)
        sel, mask = (np.full((batch, hk, self.k_max), -1, np.int32) for _ in range(2))
        num = np.zeros((batch, hk), np.int32)
        for b, n in enumerate(lens):
            for h in range(hk):
                k = min(self.k_max, -(-n // P))
                if counts is not None:
                    k = min(k, counts[(b * hk + h) % len(counts)])
                num[b, h] = k
                sel[b, h, :k] = np.sort(rng.permutation(-(-n // P))[:k])
                mask[b, h, :k] = np.where(rng.random(k) < 0.4, step - 1, rng.integers(-1, step, k))
        self.sel_np, self.mask_np, self.num_np = sel, mask, num
        self.t = [torch.from_numpy(x).cuda() for x in (sel, mask, num)]
        self.sel = B.Selection(*(x.data_ptr() for x in self.t))
        g = torch.Generator().manual_seed(seed)
        self.q = torch.randn(batch, W + 1, hq, d, generator=g).to(TD[dtype]).cuda()
        self.o = torch.full((batch, W + 1, hq, d), 5.0, device="cuda")
        self.z = torch.full((batch, W + 1, hq), 5.0, device="cuda")
        self.ws_bytes = B.retro_workspace_size(self.d_)
        self.ws = torch.zeros(self.ws_bytes, dtype=torch.uint8, device="cuda")
        print(f"[mx4 window] {dtype} hk={hk} G={G} d={d} P={P} lens={lens[:6]} W={W} budget={budget} step={step}",
              flush=True)

    def run(self):
        self.B.retro_decode_attend(self.d_, self.step, self.q, self.cache, self.sel, self.o, self.z, self.ws,
                                   self.ws_bytes)
        torch.cuda.synchronize()
        return self

    def check(self):
        out, lse, q, G, W, P = _f64(self.o), _f64(self.z), _f64(self.q), self.G, self.W, self.P
        tau = self.step - W + np.arange(W + 1)
        for b, n in enumerate(self.lens):
            for h in range(self.hk):
                m = self.num_np[b, h]
                pages, known = self.sel_np[b, h, :m], self.mask_np[b, h, :m]
                tok = (pages[:, None] * P + np.arange(P)).reshape(-1)
                M_ = np.repeat(known, P)
                keep = tok < n
                keep[keep] &= self.stored[b][tok[keep]]
                tok, M_ = tok[keep], M_[keep]
                seen = (tau >= 0)[:, None] & ((M_ < tau[:, None]) | (np.arange(W + 1) == W)[:, None])
                for j in range(h * G, (h + 1) * G):
                    o, to, z, tz = M.softmax_rows(q[b, :, j], self.k[b][tok, h], self.v[b][tok, h], seen, self.scale,
                                                  self.dtype, True)
                    to += 4 * M.U * np.abs(o)
                    eo, some = np.abs(out[b, :, j] - o), np.isfinite(z)
                    assert (eo <= to).all(), f"sequence {b} head {j}: off by {np.nanmax(eo - to)}"
                    assert (out[b, :, j][~some] == 0).all() and (lse[b, :, j][~some] == -np.inf).all()
                    assert (np.abs(lse[b, :, j][some] - z[some]) <= tz[some]).all()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("P,d,hk,G,W", [(16, 128, 2, 4, 16), (32, 128, 1, 3, 8), (16, 64, 2, 1, 0), (32, 64, 1, 16, 5),
                                        (16, 128, 1, 8, 31), (16, 64, 1, 5, 2), (32, 128, 1, 15, 64)])
@pytest.mark.parametrize("lens,budget", [([700, 33], 320), ([1, 0, 16, 17], 64), ([3001], 2048)])
def test_window(dtype, P, d, hk, G, W, lens, budget):
    Window(dtype, hk, G, d, P, lens, W, budget, seed=P + G).run().check()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_window_ramps_up(dtype):
    """Steps whose window reaches in front of the first one; heads that keep few pages or none."""
    for step in (0, 1, 7, 16):
        Window(dtype, 2, 4, 128, 16, [400, 90], 16, 256, seed=step, step=step, counts=[5, 0, 16, 1]).run().check()


def test_window_unmapped_and_large_scores():
    Window("bf16", 2, 4, 128, 16, [500, 100], 8, 512, seed=1, unmapped=[(0, 3), (0, 8), (1, 0)]).run().check()
    for grow, scale in ((30.0, 0.0), (1e4, 1e-6), (1e-3, 3e4)):
        Window("bf16", 1, 4, 64, 16, [800], 8, 512, seed=2, grow=grow, sm_scale=scale).run().check()
        Window("f32", 1, 4, 64, 32, [800], 8, 512, seed=2, grow=grow, sm_scale=scale).run().check()


def test_window_batches():
    lens = [200 + 61 * i for i in range(24)]
    Window("bf16", 4, 4, 128, 16, lens, 8, 512, seed=3).run().check()


@pytest.mark.parametrize("P,d", [(16, 128), (32, 128), (16, 64), (32, 64)])
@pytest.mark.parametrize("dtype,hk,G,W,batch,pages,tiles,splits",
                         [("bf16", 8, 4, 8, 16, 64, 2, 1), ("bf16", 8, 4, 16, 2, 128, 1, 3), ("bf16", 16, 4, 11, 16, 8, 1, 1),
                          ("bf16", 3, 4, 7, 43, 96, 2, 1), ("bf16", 8, 2, 16, 12, 128, 2, 1),
                          ("f32", 8, 4, 8, 16, 64, 1, None)])
def test_window_tiles(P, d, dtype, hk, G, W, batch, pages, tiles, splits):
    """One or two tiles of rows a workgroup, with and without splits; the last tiles not full."""
    budget = pages * 16
    w = Window(dtype, hk, G, d, P, [budget - 7 * b for b in range(batch)], W, budget, seed=tiles or 0)
    got = w.B.retro_attend_plan(w.d_, False)
    print("[plan]", got, flush=True)
    assert tiles is None or got[0] == tiles
    assert splits is None or got[1] == splits
    w.run().check()
