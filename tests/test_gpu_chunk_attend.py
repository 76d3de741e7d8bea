"""Attention of ragged chunks over the paged cache against a 64-bit reference:
single tokens to long chunks, lengths around every tile, pages that are not
mapped, rows that nothing is left for, and whatever lies in unused slots."""
import numpy as np
import pytest
import torch

import chunk_reference as R

pytestmark = pytest.mark.gpu
TD = {"bf16": torch.bfloat16, "f32": torch.float32}


def _f64(x):
    return x.detach().cpu().double().numpy()


class Batch:
    """Sequences with ctx stored tokens in front of n new ones, in a pool whose other
    slots hold NaN; rows of no sequence in front and behind; q cut out of a wider
    buffer."""

    def __init__(self, dtype, hk, G, d, P, seqs, seed=0, unmapped=(), sm_scale=0.0, spare=2, grow=1.0):
        from paper_2508_09001_amd import binding as B
        self.B, self.dtype, self.hk, self.G, self.d, self.P, self.seqs = B, dtype, hk, G, d, P, seqs
        g = torch.Generator().manual_seed(seed)
        hq = hk * G
        batch = len(seqs)
        mp = max(max(-(-(n + c) // P) for n, c in seqs), 1) + spare
        pool = batch * mp + 5
        pt = torch.randperm(pool, generator=g)[:batch * mp].view(batch, mp).int()
        kc = torch.full((pool, hk, P, d), float("nan"))
        vc = torch.full((pool, hk, d, P), float("nan"))
        self.k, self.v, self.stored = [], [], []
        for b, (n, c) in enumerate(seqs):
            L = n + c
            k, v = (torch.randn(L, hk, d, generator=g).to(TD[dtype]).float() for _ in range(2))
            k *= grow
            k = k.to(TD[dtype]).float()
            pos = torch.arange(L)
            kc[pt[b, pos // P].long(), :, pos % P] = k
            vc[pt[b, pos // P].long(), :, :, pos % P] = v
            keep = np.ones(L, bool)
            for p in range(mp):
                if p * P >= L:
                    pt[b, p] = -1 if p % 2 else pool + 7
            for bb, p in unmapped:
                if bb == b:
                    pt[b, p] = -1 if p % 2 else pool
                    keep[p * P:(p + 1) * P] = False
            self.k.append(k.numpy())
            self.v.append(v.numpy())
            self.stored.append(keep)
        self.front, self.rows = 1, sum(n for n, _ in seqs)
        self.total = self.front + self.rows + 2
        self.starts = np.concatenate([[0], np.cumsum([n for n, _ in seqs])]) + self.front
        self.wide = torch.randn(self.total, (hq + 2) * d, generator=g).to(TD[dtype]).cuda()
        self.q = self.wide[:, d:(hq + 1) * d]
        self.kc, self.vc, self.pt = kc.to(TD[dtype]).cuda(), vc.to(TD[dtype]).cuda(), pt.cuda()
        self.lens = torch.tensor([n + c for n, c in seqs], dtype=torch.int32).cuda()
        self.rs = torch.tensor(self.starts, dtype=torch.int32).cuda()
        self.sp = torch.tensor([c for _, c in seqs], dtype=torch.int32).cuda()
        self.scale = sm_scale or d ** -0.5
        self.dims = B.Dims(batch, hk, G, d, P, P, 0, mp, pool, B.RETRO_BF16 if dtype == "bf16" else B.RETRO_F32,
                           sm_scale)
        z = torch.zeros(8, dtype=torch.int32, device="cuda")
        self._z = z
        self.cache = B.KVCache(self.kc.data_ptr(), self.vc.data_ptr(), z.data_ptr(), self.pt.data_ptr(),
                               self.lens.data_ptr(), z.data_ptr())
        self.chunk = B.Chunk(self.rs.data_ptr(), self.sp.data_ptr(), self.total)
        self.out = torch.full((self.total, hq, d), 5.0).to(TD[dtype]).cuda()
        self.lse = torch.full((self.total, hq), 5.0).cuda()
        self.ws_bytes = B.retro_chunk_workspace_size(self.dims, self.total)
        self.ws = torch.zeros(self.ws_bytes, dtype=torch.uint8, device="cuda")
        print(f"[chunk] {dtype} hk={hk} G={G} d={d} P={P} seqs={seqs[:6]} unmapped={list(unmapped)}", flush=True)

    def run(self, lse=True):
        self.B.retro_chunk_attend(self.dims, self.cache, self.chunk, self.q, self.q.stride(0), self.out,
                                  self.lse if lse else None, self.ws, self.ws_bytes)
        torch.cuda.synchronize()
        return self

    def check(self, lens=None):
        out, lse = _f64(self.out), _f64(self.lse)
        q = _f64(self.q).reshape(self.total, self.hk * self.G, self.d)
        for b, (n, c) in enumerate(self.seqs):
            sl = slice(self.starts[b], self.starts[b + 1])
            keep = self.stored[b] & (np.arange(n + c) < (n + c if lens is None else lens[b]))
            o, to, z, tz = R.attend(q[sl], self.k[b], self.v[b], c + np.arange(n), keep, self.scale, self.dtype)
            eo = np.abs(out[sl] - o)
            assert (eo <= to).all(), f"sequence {b}: out off by {np.nanmax(eo - to)}, {np.isnan(eo).sum()} NaN"
            fin = np.isfinite(z)
            assert np.array_equal(lse[sl][~fin], z[~fin]) and (out[sl][~fin] == 0).all()
            ez = np.abs(lse[sl][fin] - z[fin])
            assert (ez <= tz[fin]).all(), f"sequence {b}: lse off by {ez.max(initial=0)}"
        for i in [*range(self.front), *range(self.front + self.rows, self.total)]:
            assert (self.out[i] == 5.0).all() and (self.lse[i] == 5.0).all()


# lengths around pages, tiles of 32 and 64 keys and of 32 and 256 rows
SEQS = [
    [(1, 0)],
    [(1, c) for c in (0, 1, 15, 16, 30, 31, 32, 33, 62, 63, 64, 65, 127, 200)],
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
    Batch(dtype, hk, G, d, P, seqs, seed=P + d + G).run().check()


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
    Batch("bf16", hk, G, d, P, seqs, seed=P + d + G).run().check()


def test_large_chunk_fp32():
    Batch("f32", 2, 4, 64, 16, [(700, 0), (300, 1500)], seed=2).run().check()


def test_large_chunks_whose_keys_are_cut():
    """A long context under few tiles: every tile in parts, joined by the last."""
    Batch("bf16", 2, 4, 128, 16, [(150, 9000), (1, 5000)], seed=12).run().check()


def test_large_chunks_and_pages_that_are_not_mapped():
    un = [(0, 0), (0, 50), (0, 107), (1, 0), (1, 1), (2, 3), (2, 62)]
    Batch("bf16", 8, 4, 128, 16, [(700, 1000), (300, 0), (40, 960)], seed=13, unmapped=un).run().check()


def test_large_chunks_with_fewer_tokens_stored():
    b = Batch("bf16", 8, 4, 64, 32, [(700, 1000), (300, 800), (300, 0)], seed=14)
    lens = [1350, 500, 0]
    b.lens.copy_(torch.tensor(lens, dtype=torch.int32))
    b.run().check(lens)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_pages_that_are_not_mapped_are_left_out(dtype):
    seqs = [(1, 300), (40, 300), (90, 10), (1, 16), (20, 0)]
    # one of them leaves the first rows of its sequence, one every row of its own, without a token
    un = [(0, 0), (0, 7), (1, 3), (1, 4), (1, 21), (2, 0), (2, 1), (3, 0), (3, 1), (4, 1)]
    Batch(dtype, 2, 4, 128, 16, seqs, seed=3, unmapped=un).run().check()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_fewer_tokens_stored_than_the_rows_positions(dtype):
    """A sequence whose append was cut: rows see what is there."""
    b = Batch(dtype, 2, 2, 64, 32, [(40, 100), (5, 0), (3, 64)], seed=4)
    lens = [110, 0, 64]
    b.lens.copy_(torch.tensor(lens, dtype=torch.int32))
    b.run().check(lens)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("scale,grow", [(1.0, 1.0), (0.25, 30.0), (1e-4, 1.0)])
def test_scores_far_apart_and_nearly_equal(dtype, scale, grow):
    Batch(dtype, 1, 4, 128, 16, [(70, 500), (1, 1500)], seed=5, sm_scale=scale, grow=grow).run().check()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_many_sequences(dtype):
    rng = np.random.default_rng(6)
    seqs = [(int(rng.integers(0, 4)), int(rng.integers(0, 90))) for _ in range(150)]
    Batch(dtype, 2, 2, 64, 16, seqs, seed=6).run().check()


def test_more_sequences_than_threads():
    rng = np.random.default_rng(15)
    seqs = [(int(rng.integers(0, 3)), int(rng.integers(0, 40))) for _ in range(1100)]
    seqs[700], seqs[1050] = (90, 200), (1, 3000)
    Batch("bf16", 1, 4, 64, 16, seqs, seed=16).run().check()


def test_one_workspace_for_calls_of_other_dims():
    batches = [Batch("bf16", 2, 4, 128, 16, [(1, 3000), (40, 700)], seed=17), Batch("f32", 3, 1, 64, 32, [(100, 900)], seed=18),
               Batch("bf16", 8, 4, 64, 16, [(400, 2000)], seed=19)]
    ws = torch.zeros(max(b.ws_bytes for b in batches), dtype=torch.uint8, device="cuda")
    for b in batches * 3:
        b.ws, b.ws_bytes = ws, ws.numel()
        b.out.fill_(5.0)
        b.lse.fill_(5.0)
        b.run().check()


def test_results_in_place_of_the_queries():
    b = Batch("bf16", 8, 4, 128, 16, [(300, 2000), (1, 700)], seed=20).run()
    q = b.q.contiguous().clone()
    b.B.retro_chunk_attend(b.dims, b.cache, b.chunk, q, q.stride(0), q, None, b.ws, b.ws_bytes)
    rows = slice(b.front, b.front + b.rows)
    assert torch.equal(q.view_as(b.out)[rows], b.out[rows])
    assert torch.equal(q[: b.front], b.q[: b.front])


@pytest.mark.parametrize("hk,seqs", [(2, [(1, 3000), (100, 700)]), (8, [(1, 3000), (400, 2000)])])
def test_no_lse_and_same_results_again(hk, seqs):
    b = Batch("bf16", hk, 4, 128, 16, seqs, seed=7).run()
    first, z = b.out.clone(), b.lse.clone()
    for _ in range(10):
        b.out.fill_(5.0)
        assert torch.equal(b.run().out, first)
    b.out.fill_(5.0)
    b.lse.fill_(5.0)
    b.run(lse=False)
    assert torch.equal(b.out, first) and (b.lse == 5.0).all()
    b.run()
    assert torch.equal(b.out, first) and torch.equal(b.lse, z)


@pytest.mark.parametrize("dtype,ctx,more", [("bf16", 50, ()), ("f32", 50, ()),
                                            ("bf16", 50, [(3000, 3000)] * 4)])   # (few rows, many rows)
def test_nan_and_infinite_scores(dtype, ctx, more):
    b = Batch(dtype, 1, 2, 64, 16, [(3, 200), (40, ctx), *more], seed=8)
    b.q[1, 0] = float("nan")                       # sequence 0, its first row, query head 0
    b.kc[b.pt[1, 2].long(), 0, 5, 0] = float("inf")  # position 37 of sequence 1: +-inf with every query
    b.run()
    out, lse = b.out.float(), b.lse
    assert out[1, 0].isnan().all() and lse[1, 0].isnan()
    assert out[1, 1].isfinite().all() and out[2:4].isfinite().all()
    plus = (b.q[4:44, :].reshape(40, 2, 64)[:, :, 0] > 0)
    assert out[4:44][plus].isnan().all() and lse[4:44][plus].isnan().all()
    assert out[4:44][~plus].isfinite().all() and lse[4:44][~plus].isfinite().all()


def test_captured_and_replayed_for_other_rows():
    b = Batch("bf16", 2, 4, 128, 16, [(30, 500), (1, 900), (20, 0)], seed=9)
    b.run()                                         # (the module is loaded outside the capture)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        b.B.retro_chunk_attend(b.dims, b.cache, b.chunk, b.q, b.q.stride(0), b.out, b.lse, b.ws, b.ws_bytes)
    for ns in ((30, 1, 20), (1, 1, 1), (5, 0, 20), (30, 1, 20)):
        starts = np.concatenate([[0], np.cumsum(ns)]) + b.front
        b.rs.copy_(torch.tensor(starts, dtype=torch.int32))
        b.out.fill_(5.0)
        b.lse.fill_(5.0)
        graph.replay()
        torch.cuda.synchronize()
        o, z = b.out.clone(), b.lse.clone()
        b.out.fill_(5.0)
        b.lse.fill_(5.0)
        b.run()
        assert torch.equal(o, b.out) and torch.equal(z, b.lse)
        assert (o[starts[-1]:] == 5.0).all()
        seqs, b.seqs, old = b.seqs, [(n, c) for n, (_, c) in zip(ns, b.seqs)], (b.starts, b.rows)
        b.starts, b.rows = starts, sum(ns)
        keep = b.k, b.v, b.stored
        b.k, b.v, b.stored = ([x[:n + c] for x, (n, c) in zip(y, b.seqs)] for y in keep)
        # tokens past the chunk's rows stay stored; a causal row does not see them
        b.check()
        (b.k, b.v, b.stored), b.seqs, (b.starts, b.rows) = keep, seqs, old


@pytest.mark.parametrize("hk,seqs", [(2, [(50, 500), (1, 2000)]), (8, [(500, 1500), (1, 2000)])])
def test_another_stream(hk, seqs):
    b = Batch("bf16", hk, 4, 128, 16, seqs, seed=10).run()
    want, z = b.out.clone(), b.lse.clone()
    b.out.fill_(5.0)
    b.lse.fill_(5.0)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    b.B.retro_chunk_attend(b.dims, b.cache, b.chunk, b.q, b.q.stride(0), b.out, b.lse, b.ws, b.ws_bytes, stream=s)
    s.synchronize()
    assert torch.equal(b.out, want) and torch.equal(b.lse, z)


# chunks of many rows beside other sequences' tokens: the workgroups without a part of the
# former take longer shares of the latter, all of them or not; more sequences than a
# wavefront has lanes, and than a workgroup has threads
MIXED = [
    ([(256, 3000)], 12, 4000, 8, 4, 128, 16),
    ([(300, 900), (1, 77), (150, 400)], 80, 700, 8, 4, 64, 32),
    ([(120, 130)], 560, 60, 8, 4, 64, 16),
    ([(700, 700)], 5, 5000, 4, 8, 128, 32),
    ([(130, 2100), (70, 5)], 20, 3000, 8, 4, 128, 16),
]


@pytest.mark.parametrize("chunks,tokens,ctx,hk,G,d,P", MIXED, ids=[str(i) for i in range(len(MIXED))])
def test_chunks_beside_tokens(chunks, tokens, ctx, hk, G, d, P):
    rng = np.random.default_rng(tokens)
    seqs = [(1, int(rng.integers(0, ctx))) for _ in range(tokens)]
    seqs[3:3] = chunks
    b = Batch("bf16", hk, G, d, P, seqs, seed=tokens).run()
    b.check()
    out, z = b.out.clone(), b.lse.clone()
    for _ in range(3):
        b.out.fill_(5.0)
        b.run()
        assert torch.equal(b.out, out) and torch.equal(b.lse, z)


# one chunk in a table of slots of which the others are empty, short chunks in all of them,
# and both: the kernel goes by the longest run, the results by none
@pytest.mark.parametrize("longest", [-5, 0, 1, 7, 40, 300, 2**31 - 1])
@pytest.mark.parametrize("seqs", [[(300, 500)] + [(0, 40)] * 299, [(7, 100)] * 60, [(40, 2500), (1, 9)] + [(0, 0)] * 60],
                         ids=["slots", "short", "mixed"])
def test_results_do_not_depend_on_the_longest_run_given(seqs, longest):
    b = Batch("bf16", 2, 4, 128, 16, seqs, seed=21)
    b.chunk.longest = longest
    b.run().check()


# more tiles of 256 rows than workgroups (387, 296 and 404): those of the second round are dealt
# backwards, cut or not
@pytest.mark.parametrize("seqs,hk,G,d,P", [([(1040, 0), (500, 300)], 9, 7, 64, 32),
                                           ([(1100, 0), (60, 9000)], 8, 8, 128, 16),
                                           ([(900, 200), (700, 0), (1, 3000)], 4, 16, 128, 32)], ids=["0", "1", "2"])
def test_more_tiles_of_many_rows_than_workgroups(seqs, hk, G, d, P):
    Batch("bf16", hk, G, d, P, seqs, seed=22).run().check()


# a tile or a few of 256 rows under long contexts: some 160, 88, 26 and 59 parts each
@pytest.mark.parametrize("seqs,hk,G,d,P", [([(64, 82000)], 1, 4, 64, 16), ([(64, 44800)], 2, 4, 128, 16),
                                           ([(60, 12800)], 4, 8, 128, 32),
                                           ([(70, 6000), (64, 30000), (1, 900)], 2, 4, 64, 32)], ids=["0", "1", "2", "3"])
def test_tiles_of_many_rows_in_many_parts(seqs, hk, G, d, P):
    b = Batch("bf16", hk, G, d, P, seqs, seed=23).run()
    b.check()
    out, z = b.out.clone(), b.lse.clone()
    for _ in range(3):   # (the counts are back at zero)
        b.out.fill_(5.0)
        b.run()
        assert torch.equal(b.out, out) and torch.equal(b.lse, z)


def test_two_calls_at_once():
    """On two streams, a workspace each: neither waits for the other nor changes its result."""
    a, b = (Batch("bf16", hk, 4, 128, 16, seqs, seed=24) for hk, seqs in
            ((8, [(500, 1500), (1, 2000)]), (2, [(1, 30000), (100, 700)])))
    want = [(x.run().out.clone(), x.lse.clone()) for x in (a, b)]
    streams = [torch.cuda.Stream() for _ in range(2)]
    for x in (a, b):
        x.out.fill_(5.0)
        x.lse.fill_(5.0)
    torch.cuda.synchronize()
    for _ in range(10):
        for x, s in zip((a, b), streams):
            x.B.retro_chunk_attend(x.dims, x.cache, x.chunk, x.q, x.q.stride(0), x.out, x.lse, x.ws, x.ws_bytes, stream=s)
    torch.cuda.synchronize()
    for x, (o, z) in zip((a, b), want):
        assert torch.equal(x.out, o) and torch.equal(x.lse, z)
