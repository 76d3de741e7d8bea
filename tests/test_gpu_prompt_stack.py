"""Prompts and decode steps of a stack whose queries and keys carry positions: rotated
append, chunk attention, window rotation, UpdateKV and the retrospective step
together, through RetroDecoder, against a 64-bit stack."""
import numpy as np
import pytest
import torch

import chunk_reference as R

pytestmark = pytest.mark.gpu


def _f64(x):
    return x.detach().cpu().double().numpy()


def _weights(layers, dm, hk, d, seed, norms, dtype=torch.float32):
    g = torch.Generator().manual_seed(seed)
    out = []
    for _ in range(layers):
        w = {n: (torch.randn(dm, m, generator=g) * s).to(dtype)
             for n, m, s in (("wq", dm, dm ** -0.5), ("wk", hk * d, dm ** -0.5), ("wv", hk * d, dm ** -0.5),
                             ("wo", dm, 0.5 * dm ** -0.5))}
        if norms:
            w["q_norm"], w["k_norm"] = ((1 + 0.2 * torch.randn(d, generator=g)).to(dtype) for _ in range(2))
        out.append(w)
    return out


class Stack:
    """The stack in 64 bits: every row attends all tokens up to its own."""

    def __init__(self, weights, batch, hk, G, d, tab, rot, interleaved, eps):
        self.w = [{k: _f64(v) for k, v in w.items()} for w in weights]
        self.hk, self.hq, self.d = hk, hk * G, d
        self.args = (tab, rot, interleaved, eps)
        self.kv = [[(np.zeros((0, hk, d)), np.zeros((0, hk, d))) for _ in range(batch)] for _ in weights]

    def turn(self, x, weight, pos):
        tab, rot, interleaved, eps = self.args
        return R.turn(x, weight, tab, pos, rot, interleaved, eps, "f32")[0]

    def rows(self, b, emb):
        h = emb.astype(np.float64)
        if not len(h):
            return h
        for layer, w in enumerate(self.w):
            k0, v0 = self.kv[layer][b]
            pos = len(k0) + np.arange(len(h))
            q, k, v = ((h @ w[n]).reshape(len(h), -1, self.d) for n in ("wq", "wk", "wv"))
            q, k = self.turn(q, w.get("q_norm"), pos), self.turn(k, w.get("k_norm"), pos)
            k, v = np.concatenate([k0, k]), np.concatenate([v0, v])
            self.kv[layer][b] = (k, v)
            o = R.attend(q, k, v, pos, np.ones(len(k), bool), self.d ** -0.5, "f32")[0]
            h = h + o.reshape(len(h), -1) @ w["wo"]
        return h


# fp32: per layer, products of 256 terms (four), scores of 64, up to 90 keys, each
# rounding 2^-24 of its sum's size: below 1500 U of the stream's largest per layer
TOL = 2 * 1500 * R.U


@pytest.mark.parametrize("P", [16, 32])
@pytest.mark.parametrize("rot,interleaved,norms", [(64, False, True), (32, True, False), (0, False, True)])
def test_prompts_in_chunks_then_steps(P, rot, interleaved, norms):
    from paper_2508_09001_amd.decode import RetroDecoder
    hk, G, d, batch, mp = 2, 2, 64, 3, 8
    dm = hk * G * d
    w = _weights(2, dm, hk, d, 1, norms)
    dec = RetroDecoder(w, rotary=dict(rot_dim=rot, base=1e4, interleaved=interleaved, eps=1e-5),
                       batch=batch, num_kv_heads=hk, group=G, head_dim=d, page_size=P, budget=P * mp, window=0,
                       max_pages=mp, dtype="f32")
    ref = Stack(w, batch, hk, G, d, R.table(mp * P, rot, 1e4) if rot else None, rot, interleaved, 1e-5)
    rng = np.random.default_rng(2)

    def compare(got, want, what):
        want = np.concatenate(want)
        err = np.abs(_f64(got).reshape(want.shape) - want).max()
        assert err <= TOL * np.abs(want).max(), f"{what}: {err}"

    t = 0
    for what in [(20, 7, 1), (0, 30, 15), "step", "step", (1, 1, 1), "step", (2, 0, 19), "step"]:
        n = (1,) * batch if what == "step" else what
        emb = [rng.standard_normal((m, dm)).astype(np.float32) for m in n]
        print(f"[stack] P={P} rot={rot} {what}", flush=True)
        want = [ref.rows(b, emb[b]) for b in range(batch)]
        x = torch.from_numpy(np.concatenate(emb)).cuda()
        if what == "step":   # the budget keeps every page: dense attention of the newest row
            got = dec.step(t, x.view(batch, 1, dm))
            t += 1
        else:
            got = dec.prefill_chunk(n, x)
        compare(got, want, what)
    for layer in range(2):
        assert dec.layers[layer].seq_lens.tolist() == [len(ref.kv[layer][b][0]) for b in range(batch)]


@pytest.mark.parametrize("fused", [True, False])
def test_window_rows_are_rotated_to_their_positions(fused):
    """Re-embedding with positions: every step's queries and keys are the projections
    turned to the rows' positions, and UpdateKV stores these keys."""
    from paper_2508_09001_amd.decode import RetroDecoder
    hk, G, d, batch, P, mp, W, rot = 2, 4, 128, 2, 16, 8, 3, 128
    dm = hk * G * d
    w = _weights(2, dm, hk, d, 3, True, torch.bfloat16)
    dec = RetroDecoder(w, library_projections=fused, rotary=dict(rot_dim=rot, base=1e4, eps=1e-5),
                       batch=batch, num_kv_heads=hk, group=G, head_dim=d, page_size=P, budget=P * mp, window=W,
                       max_pages=mp, dtype="bf16")
    assert dec.fused is fused
    rng = np.random.default_rng(4)
    tab = R.table(mp * P, rot, 1e4)

    def emb(*s):
        return torch.from_numpy(rng.standard_normal(s).astype(np.float32)).bfloat16().float()

    dec.prefill_chunk((13, 1), emb(14, dm).cuda())      # the second one's window begins in front of it
    at, tokens = np.array([13, 1]), torch.zeros(batch, W + 1, dm)
    for t in range(6):
        tokens = torch.cat([tokens[:, 1:], emb(batch, 1, dm)], dim=1)
        trace = []
        dec.step(t, tokens.cuda(), trace=trace)
        for layer, (tr, wl) in enumerate(zip(trace, w)):
            x = _f64(tr["x"]).reshape(batch, W + 1, dm)
            for b in range(batch):
                pos = at[b] - W + np.arange(W + 1)
                live = pos >= 0
                for name, heads, mat in (("q", hk * G, "wq"), ("k", hk, "wk")):
                    p = (x[b] @ _f64(wl[mat])).reshape(W + 1, heads, d)
                    # the projection is rounded to bf16 first: half a step of each of the
                    # two elements that a turned one comes from, and the norm's sum moves
                    # by no more than its largest element's
                    y, tol = R.turn(p[live], _f64(wl[name[0] + "_norm"]), tab, pos[live], rot, False, 1e-5, "bf16")
                    size = np.abs(y) + np.abs(np.roll(y, d // 2, axis=-1))
                    got = _f64(tr[name]).reshape(batch, W + 1, heads, d)[b][live]
                    assert (np.abs(got - y) <= tol + 4 * R.HALF["bf16"] * size + 1e-4).all(), (t, layer, name)
                    if name == "k":
                        lay = dec.layers[layer]
                        n = min(W, t) + 1               # rows stored by this step
                        sl = pos[-n:]
                        ph = lay.page_table[b].long().cpu()[torch.from_numpy(sl // P)]
                        stored = lay.k_cache.cpu()[ph, :, torch.from_numpy(sl % P)]
                        new = tr["k"].reshape(batch, W + 1, hk, d)[b, -n:].cpu()
                        assert torch.equal(stored, new), (t, layer)
        at += 1


def test_layer_calls_take_views_and_lists():
    """RetroLayer's chunk calls on parts of one projection's output, two sequences, in a
    serving pattern: prompts, then tokens, equal to the whole prompt at once."""
    from paper_2508_09001_amd.layer import RetroLayer, RetroRotary
    hk, G, d, P, mp = 2, 4, 128, 16, 16
    hq = hk * G
    lays = [RetroLayer(batch=2, num_kv_heads=hk, group=G, head_dim=d, page_size=P, budget=P, window=0, max_pages=mp)
            for _ in range(2)]
    rot = RetroRotary(mp * P, 64, base=1e4, k_norm=torch.ones(d))
    qkv = torch.randn(2, 100, (hq + 2 * hk) * d).bfloat16().cuda()

    def call(lay, frm, to):
        part = [qkv[b, frm[b]:to[b]] for b in range(2)]
        x = torch.cat(part)
        ch = lay.chunk([p.shape[0] for p in part])
        q = lay.append_chunk(0, ch, rot, x[:, hq * d:(hq + hk) * d], x[:, (hq + hk) * d:].unflatten(1, (hk, d)),
                             x[:, :hq * d])
        o, z = lay.attend_chunk(ch, q, lse=True)
        n = ch.rows[0]
        return (o[:n], z[:n]), (o[n:], z[n:])

    whole = call(lays[0], (0, 0), (100, 77))
    at = [0, 0]
    parts = [[], []]
    for n in ((60, 1), (39, 75), (1, 1)):
        to = [a + m for a, m in zip(at, n)]
        for b, r in enumerate(call(lays[1], at, to)):
            parts[b].append(r)
        at = to
    for b in range(2):
        o, z = (torch.cat(x) for x in zip(*parts[b]))
        # the same weights, rounded at other maxima: a step of bf16 at most each way
        assert ((o - whole[b][0]).abs().double() <= 2 * R.HALF["bf16"] * (whole[b][0].abs().double() + 1)).all()
        assert (z - whole[b][1]).abs().max() <= 1e-4
    for name in ("k_cache", "v_cache", "digest", "seq_lens"):
        assert torch.equal(getattr(lays[0], name), getattr(lays[1], name)), name
    # positions by themselves; refusals
    pos = torch.arange(77, dtype=torch.int32)
    q, k = lays[0].rotate(rot, pos, k=qkv[1, :77, hq * d:(hq + hk) * d])
    assert q is None
    table = lays[0].page_table[1].long()
    assert torch.equal(k, lays[0].k_cache[table[torch.arange(77) // P], :, torch.arange(77) % P])
    with pytest.raises(ValueError):
        lays[0].append_chunk(0, lays[1].chunk((1, 2)), rot, qkv[0, :4, :hk * d], qkv[0, :4, :hk * d])
    ch = lays[0].chunk((1, 0))
    lays[0].append(1, torch.zeros(2, hk, d), torch.zeros(2, hk, d))
    with pytest.raises(ValueError):   # the sequences have grown since
        lays[0].append_chunk(0, ch, rot, qkv[0, :1, :hk * d], qkv[0, :1, :hk * d])


def test_layer_calls_on_another_stream_while_the_current_one_is_busy():
    """Copies of strided inputs, new tensors and the workspace's zeros are work of the
    call's stream, not of the current one, which sleeps for some milliseconds meanwhile."""
    from paper_2508_09001_amd.layer import RetroChunk, RetroLayer, RetroRotary
    hk, G, d, P, mp, n = 2, 4, 128, 16, 96, 40
    rot = RetroRotary(mp * P, d)
    # (transposed and fp32: copied by every call)
    qkv = [torch.randn(m, heads * d, device="cuda").t().contiguous().t()
           for m in (1400, n) for heads in (hk, hk, hk * G)]
    chunks = [RetroChunk((1400,), (0,), "cuda"), RetroChunk((n,), (1400,), "cuda")]
    pos = torch.arange(n, dtype=torch.int32, device="cuda")
    lays = [RetroLayer(batch=1, num_kv_heads=hk, group=G, head_dim=d, page_size=P, budget=P, window=0, max_pages=mp)
            for _ in range(2)]
    side = torch.cuda.Stream()
    torch.cuda.synchronize()

    def calls(lay, stream):
        for ch, (k, v, q) in zip(chunks, (qkv[:3], qkv[3:])):
            q = lay.append_chunk(0, ch, rot, k, v, q, stream=stream)
            o, z = lay.attend_chunk(ch, q, lse=True, stream=stream)
        return q, o, z, lay.rotate(rot, pos, q=qkv[5], stream=stream)[0]

    want = calls(lays[0], None)
    torch.cuda.synchronize()
    torch.cuda._sleep(20_000_000)
    got = calls(lays[1], side)
    side.synchronize()
    with torch.cuda.stream(side):
        same = [bool(torch.equal(a, b)) for a, b in zip(got, want)]
    assert same == [True] * 4
    torch.cuda.synchronize()


def test_captured_layer_attention_between_eager_calls():
    """A layer's attend_chunk captured after reserve_chunks: eager calls before the first
    replay, between replays and of other shapes use the same workspace."""
    from paper_2508_09001_amd.layer import RetroChunk, RetroLayer, RetroRotary
    hk, G, d, P, mp, n = 2, 4, 128, 16, 96, 40
    lay = RetroLayer(batch=1, num_kv_heads=hk, group=G, head_dim=d, page_size=P, budget=P, window=0, max_pages=mp)
    k, v = (torch.randn(1400 + n, hk, d).bfloat16().cuda() for _ in range(2))
    lay.append_chunk(0, lay.chunk((1400 + n,)), RetroRotary(mp * P, 0), k, v)
    q = torch.randn(n, hk * G, d).bfloat16().cuda()
    ch, one = RetroChunk((n,), (1400,), "cuda"), RetroChunk((1,), (1400,), "cuda")
    fresh = RetroLayer(batch=1, num_kv_heads=hk, group=G, head_dim=d, page_size=P, budget=P, window=0, max_pages=mp)
    for name in ("k_cache", "v_cache", "digest", "seq_lens", "last_loaded"):
        getattr(fresh, name).copy_(getattr(lay, name))
    want = [x.clone() for c in (ch, one) for x in fresh.attend_chunk(c, q[:c.n_rows], lse=True)]
    lay.reserve_chunks()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        o, z = lay.attend_chunk(ch, q, lse=True)
    for _ in range(3):
        eager = [x for c in (ch, one) for x in lay.attend_chunk(c, q[:c.n_rows], lse=True)]
        assert all(torch.equal(a, b) for a, b in zip(eager, want))
        o.fill_(5.0)
        z.fill_(5.0)
        graph.replay()
        assert torch.equal(o, want[0]) and torch.equal(z, want[1])
        torch.cuda.synchronize()


def test_chunks_after_rows_that_were_dropped():
    """A page that is not mapped ends a sequence's append; once it is, the next chunk goes
    on from there, as in a layer that never had the gap."""
    from paper_2508_09001_amd.layer import RetroLayer, RetroRotary
    hk, G, d, P, mp = 2, 2, 64, 16, 4
    pt = torch.arange(2 * mp).view(2, mp)
    gap = pt.clone()
    gap[0, 1] = -1
    kw = dict(batch=2, num_kv_heads=hk, group=G, head_dim=d, page_size=P, budget=P, window=0, max_pages=mp)
    lay, ref = RetroLayer(page_table=gap, **kw), RetroLayer(page_table=pt, **kw)
    rot = RetroRotary(mp * P, d)
    k, v = (torch.randn(2, 40, hk, d).bfloat16().cuda() for _ in range(2))

    def call(la, frm, to):
        ch = la.chunk([b - a for a, b in zip(frm, to)])
        assert ch.start == list(frm)
        la.append_chunk(0, ch, rot, *(torch.cat([x[0, frm[0]:to[0]], x[1, frm[1]:to[1]]]) for x in (k, v)))

    call(lay, (0, 0), (20, 9))
    assert lay.seq_lens.tolist() == [16, 9]
    lay.page_table[0, 1] = 1
    call(lay, (16, 9), (40, 30))
    call(ref, (0, 0), (40, 30))
    for name in ("k_cache", "v_cache", "digest", "seq_lens"):
        assert torch.equal(getattr(lay, name), getattr(ref, name)), name
