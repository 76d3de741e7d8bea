"""The cache in 4 bits away from the usual call: shapes drawn at random, pools whose offsets
pass 32 bits, pages of several sequences, calls at once, queries that are not finite."""
import random

import numpy as np
import pytest
import torch

import mx4_reference as M
from test_gpu_mx4_attend import Chunk, Window, _f64

pytestmark = pytest.mark.gpu
TD = {"bf16": torch.bfloat16, "f32": torch.float32}


@pytest.mark.parametrize("seed", range(24))
def test_drawn_chunks(seed):
    r = random.Random(seed)
    dtype, P, d = r.choice(["bf16", "bf16", "f32"]), r.choice([16, 32]), r.choice([64, 128])
    hk, G = r.choice([1, 2, 3, 5, 8]), r.choice([1, 2, 3, 4, 7, 8, 16])
    budget = 3000000 if dtype == "bf16" else 1000000     # pairs of a row and a token, for the reference's time
    seqs = []
    for _ in range(r.choice([1, 1, 2, 5, 17, 70])):
        n = r.choice([0, 1, 1, 1, r.randint(2, 40), r.randint(2, 300)])
        ctx = int(2 ** r.uniform(0, 11.5)) if r.random() < 0.8 else 0
        if n * (n + ctx) * hk * G <= budget:
            seqs.append((n, ctx))
            budget -= n * (n + ctx) * hk * G
    seqs = seqs or [(1, 5)]
    longest = r.choice([0, max(n for n, _ in seqs), 1])
    un = [(b, r.randrange(0, (n + c) // P + 1)) for b, (n, c) in enumerate(seqs) if r.random() < 0.15]
    Chunk(dtype, hk, G, d, P, seqs, seed=seed, longest=longest, unmapped=un).run().check()


@pytest.mark.parametrize("seed", range(24))
def test_drawn_windows(seed):
    r = random.Random(100 + seed)
    dtype, P, d = r.choice(["bf16", "bf16", "f32"]), r.choice([16, 32]), r.choice([64, 128])
    hk, G, W = r.choice([1, 2, 3, 5]), r.choice([1, 2, 4, 7, 16]), r.choice([0, 1, 3, 8, 16, 40, 64])
    if (W + 1) * G > 1024:
        W = 40
    lens = [r.choice([0, 1, r.randint(2, 100), r.randint(100, 3000)]) for _ in range(r.choice([1, 2, 3, 9]))]
    budget = max(P, r.choice([P, 100, 257, 1000, 4096]))
    Window(dtype, hk, G, d, P, lens, W, budget, seed=seed, step=r.choice([0, 2, 90]),
           counts=r.choice([None, [0, 3, 1000]])).run().check()


def _far(dtype="bf16", hk=8, d=128, P=16, pages=600000):
    """A layer whose pool is 5 GB of keys and as much of values, its tables at the far end of it."""
    from paper_2508_09001_amd.layer import RetroLayer
    pt = torch.randperm(60, generator=torch.Generator().manual_seed(1)).view(2, 30) + pages - 60
    return RetroLayer(batch=2, num_kv_heads=hk, group=2, head_dim=d, page_size=P, budget=8 * P, window=2, max_pages=30,
                      dtype=dtype, kv="mx4", num_phys_pages=pages, page_table=pt)


def test_offsets_past_32_bits():
    """The same calls on a pool of 60 pages give the same bits."""
    from paper_2508_09001_amd.layer import RetroLayer, RetroRotary
    far = _far()
    assert far.k_cache.numel() > 1 << 32
    near = RetroLayer(batch=2, num_kv_heads=8, group=2, head_dim=128, page_size=16, budget=128, window=2, max_pages=30,
                      kv="mx4")
    g = torch.Generator().manual_seed(2)

    def rand(*shape):
        return torch.randn(*shape, generator=g).to(torch.bfloat16).cuda()

    rot = RetroRotary(480, 0)
    for rows in ((300, 64), (20, 1)):
        n = sum(rows)
        k, v, q = rand(n, 8, 128), rand(n, 8, 128), rand(n, 16, 128)
        got = []
        for lay in (far, near):
            ch = lay.chunk(rows)
            lay.append_chunk(0, ch, rot, k, v)
            got.append((*lay.attend_chunk(ch, q, lse=True), *lay.read(ch)))
        assert all(torch.equal(x, y) for x, y in zip(*got))
        assert torch.equal(got[0][2], torch.from_numpy(M.rounded(_f64(k))).to(torch.bfloat16).cuda())
    for t in range(3):
        q, k, v = rand(2, 3, 16, 128), rand(2, 8, 128), rand(2, 8, 128)
        for lay in (far, near):
            lay.step(t, q, k, v)
            lay.attend(t, q)
        assert torch.equal(far.selected, near.selected)
        assert torch.equal(far.o_out, near.o_out) and torch.equal(far.o_part, near.o_part)


def test_pages_of_two_sequences():
    """A prompt that two sequences share."""
    c = Chunk("bf16", 2, 4, 128, 16, [(3, 100), (3, 100)], seed=4)
    c.pt[1] = c.pt[0]
    c.k[1], c.v[1] = c.k[0], c.v[0]
    c.run().check()


def test_calls_at_once():
    """Two attention calls and a window on streams of their own, each with a workspace of its own."""
    a = Chunk("bf16", 4, 4, 128, 16, [(300, 2000), (1, 900)], seed=5)
    b = Chunk("f32", 2, 4, 64, 32, [(70, 900), (1, 3000)], seed=6)
    w = Window("bf16", 4, 4, 128, 16, [3000, 700], 16, 1024, seed=7)
    streams = [torch.cuda.Stream() for _ in range(3)]
    torch.cuda.synchronize()
    for _ in range(10):
        with torch.cuda.stream(streams[0]):
            a.B.retro_chunk_attend(a.d_, a.cache, a.chunk, a.q, a.q.stride(0), a.out, a.lse, a.ws, a.ws_bytes)
        with torch.cuda.stream(streams[1]):
            b.B.retro_chunk_attend(b.d_, b.cache, b.chunk, b.q, b.q.stride(0), b.out, b.lse, b.ws, b.ws_bytes)
        with torch.cuda.stream(streams[2]):
            w.B.retro_decode_attend(w.d_, w.step, w.q, w.cache, w.sel, w.o, w.z, w.ws, w.ws_bytes)
    torch.cuda.synchronize()
    a.check()
    b.check()
    w.check()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("rows", [3, 200])
def test_queries_that_are_not_finite(dtype, rows):
    """A NaN query, whatever its bits, makes its own row and head NaN and no other."""
    c = Chunk(dtype, 2, 4, 128, 16, [(rows, 600)], seed=8)
    bits = torch.int16 if dtype == "bf16" else torch.int32
    odd = 0x7f81 if dtype == "bf16" else 0x7f800001      # a NaN of the last bit
    q = c.q.view(bits).view(c.total, 8, 128)
    c.run()
    want, z = c.out.clone(), c.lse.clone()
    q[2, 3, 77] = odd
    q[3, 0, 5] = 0x7fc0 if dtype == "bf16" else 0x7fc00000
    c.out.fill_(5.0)
    c.run()
    bad = torch.zeros(c.total, 8, dtype=torch.bool, device="cuda")
    bad[2, 3] = bad[3, 0] = True
    assert torch.isnan(c.out[bad]).all() and torch.isnan(c.lse[bad]).all()
    assert torch.equal(c.out[~bad], want[~bad]) and torch.equal(c.lse[~bad], z[~bad])


def test_nothing_to_do():
    c = Chunk("bf16", 2, 4, 128, 16, [(0, 100), (0, 0)], seed=9)
    c.run()
    assert (c.out == 5.0).all() and (c.lse == 5.0).all()
    for n in (0,):
        ch = c.B.Chunk(c.rs.data_ptr(), c.sp.data_ptr(), n)
        c.B.retro_chunk_attend(c.d_, c.cache, ch, c.q, c.q.stride(0), c.out, c.lse, c.ws, c.ws_bytes)
        c.B.retro_read_kv(c.d_, c.cache, ch, None, None)
    torch.cuda.synchronize()


def test_plans():
    """The launches and splits that the host tells of are those of the call."""
    from paper_2508_09001_amd import binding as B
    for flags in (B.RETRO_FLAG_KV_MX4, B.RETRO_FLAG_KV_MX4 | B.RETRO_FLAG_SEPARATE_SCORES):
        d = B.Dims(1, 8, 4, 128, 16, 2048, 16, 2064, 2064, B.RETRO_BF16, 0.0, 0, flags)
        assert B.retro_step_launches(d) in (4, 5)
        tiles, splits = B.retro_attend_plan(d, False)
        assert 1 <= tiles <= 3 and 1 <= splits <= 32
