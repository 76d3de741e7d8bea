"""Norm and rotation of queries and keys, by themselves and on the way into the
paged cache, against 64-bit references, at the edges of their shapes."""
import numpy as np
import pytest
import torch

import chunk_reference as R

pytestmark = pytest.mark.gpu
TD = {"bf16": torch.bfloat16, "f32": torch.float32}


def _f64(x):
    return x.detach().cpu().double().numpy()


def _dims(B, dtype, d=128, hk=2, G=3, P=16, batch=1, mp=8, pool=None):
    return B.Dims(batch, hk, G, d, P, P, 0, mp, pool or batch * mp,
                  B.RETRO_BF16 if dtype == "bf16" else B.RETRO_F32)


def _within(got, want, tol, what):
    err = np.abs(_f64(got) - want)
    bad = ~(err <= tol)
    assert not bad.any(), f"{what}: {int(bad.sum())} off, e.g. {err[bad][:3]} > {tol[bad][:3]}"


@pytest.mark.parametrize("rot,base", [(16, 1e4), (64, 5e5), (128, 1e6)])
def test_table(rot, base):
    from paper_2508_09001_amd import binding as B
    n = 140001
    t = torch.full((n + 1, rot // 2, 2), 7.0, device="cuda")
    B.retro_rotary_table(t, n, rot, base)
    got = t.cpu().numpy()
    # the reference's own angles are a few units of 2^-53 of up to 140000 off
    assert np.abs(got[:n].astype(np.float64) - R.table(n, rot, base).astype(np.float64)).max() <= R.U + 1e-9
    assert (got[n] == 7.0).all()


# rows 1 .. a few workgroups; heads that fill no group of four; part rotations of
# whole and odd numbers of pieces; one projection's output and buffers of their own
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("d,rot,interleaved", [(128, 128, 0), (128, 128, 1), (128, 48, 0), (128, 48, 1),
                                               (64, 64, 0), (64, 16, 1), (64, 32, 0), (128, 0, 0)])
@pytest.mark.parametrize("rows,hk,G,norm,fused", [(1, 1, 1, True, False), (7, 2, 3, False, True),
                                                  (77, 5, 4, True, True)])
def test_rotate_qk(dtype, d, rot, interleaved, rows, hk, G, norm, fused):
    from paper_2508_09001_amd import binding as B
    g = torch.Generator().manual_seed(rows + d + rot)
    hq, n = hk * G, 5000
    if fused:
        qkv = torch.randn(rows, (hq + 2 * hk) * d, generator=g).to(TD[dtype]).cuda()
        q, k = qkv[:, :hq * d].view(rows, hq, d), qkv[:, hq * d:(hq + hk) * d].view(rows, hk, d)
    else:
        q, k = (torch.randn(rows, h, d, generator=g).to(TD[dtype]).cuda() for h in (hq, hk))
    pos = torch.randint(0, n, (rows,), generator=g, dtype=torch.int32)
    pos[0] = n - 1
    w = [(1 + 0.2 * torch.randn(d, generator=g)).to(TD[dtype]).cuda() if norm else None for _ in range(2)]
    tab = torch.from_numpy(R.table(n, rot, 1e4)).cuda() if rot else None
    r = B.Rotary(tab.data_ptr() if rot else None, n if rot else 0, rot, interleaved, 1e-6,
                 *(x.data_ptr() if norm else None for x in w))
    qo, ko = torch.full((rows + 1, hq, d), 5.0).to(TD[dtype]).cuda(), \
        torch.full((rows + 1, hk, d), 5.0).to(TD[dtype]).cuda()
    dims = _dims(B, dtype, d, hk, G)
    print(f"[rotate] {dtype} d={d} rot={rot} il={interleaved} rows={rows} hk={hk} G={G}", flush=True)
    B.retro_rotate_qk(dims, r, pos.cuda(), rows, q, q.stride(0), k, k.stride(0), qo, ko)
    for x, o, wt, name in ((q, qo, w[0], "q"), (k, ko, w[1], "k")):
        want, tol = R.turn(_f64(x), None if wt is None else _f64(wt), R.table(n, rot, 1e4), pos.numpy(),
                           rot, interleaved, 1e-6, dtype)
        _within(o[:rows], want, tol, name)
        assert (o[rows] == 5.0).all()
    # one of the two alone, and in place
    only = k.contiguous().clone()
    B.retro_rotate_qk(dims, r, pos.cuda(), rows, None, 0, only, hk * d, None, only)
    assert torch.equal(only, ko[:rows])
    only = q.contiguous().clone()
    B.retro_rotate_qk(dims, r, pos.cuda(), rows, only, hq * d, None, 0, only, None)
    assert torch.equal(only, qo[:rows])


def test_rows_without_a_position_in_the_table():
    from paper_2508_09001_amd import binding as B
    n, hk, G, d = 32, 2, 2, 128
    tab = torch.from_numpy(R.table(n, 64, 1e4)).cuda()
    pos = torch.tensor([3, -1, n, n - 1, -2147483648, 2147483647], dtype=torch.int32)
    rows = len(pos)
    q = torch.randn(rows, hk * G, d).bfloat16().cuda()
    k = torch.randn(rows, hk, d).bfloat16().cuda()
    qo, ko = torch.full_like(q, 5.0), torch.full_like(k, 5.0)
    B.retro_rotate_qk(_dims(B, "bf16", d, hk, G), B.Rotary(tab.data_ptr(), n, 64, 0, 0.0, None, None),
                      pos.cuda(), rows, q, hk * G * d, k, hk * d, qo, ko)
    for x, o in ((q, qo), (k, ko)):
        assert (o[[1, 4]] == 5.0).all()
        assert o[[2, 5], :, :64].isnan().all() and torch.equal(o[[2, 5], :, 64:], x[[2, 5], :, 64:])
        assert o[[0, 3]].isfinite().all()


def _layer(dtype, batch, hk, G, d, P, mp, seed):
    from paper_2508_09001_amd.layer import RetroLayer
    g = torch.Generator().manual_seed(seed)
    pt = torch.randperm(batch * mp + 3, generator=g)[:batch * mp].view(batch, mp)
    lay = RetroLayer(batch=batch, num_kv_heads=hk, group=G, head_dim=d, page_size=P, budget=P, window=0,
                     max_pages=mp, dtype=dtype, page_table=pt, num_phys_pages=batch * mp + 3)
    lay.k_cache.fill_(7.0)
    lay.v_cache.fill_(9.0)
    return lay


# several calls that start and end inside pages, sequences that take no part, rows
# that belong to none
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("P,d,hk,G", [(16, 128, 2, 4), (32, 64, 3, 1), (32, 128, 1, 5), (16, 64, 2, 2)])
@pytest.mark.parametrize("rot,interleaved,norm,with_q", [(64, 0, True, True), (32, 1, False, False)])
def test_append_rotary(dtype, P, d, hk, G, rot, interleaved, norm, with_q):
    from paper_2508_09001_amd import binding as B
    batch, mp, hq = 3, 12, hk * G
    lay = _layer(dtype, batch, hk, G, d, P, mp, P + d)
    g = torch.Generator().manual_seed(P * d + rot)
    tab = R.table(mp * P, rot, 1e4)
    tab_d = torch.from_numpy(tab).cuda()
    w = [(1 + 0.2 * torch.randn(d, generator=g)).to(TD[dtype]).cuda() if norm else None for _ in range(2)]
    r = B.Rotary(tab_d.data_ptr(), mp * P, rot, interleaved, 1e-5, *(x.data_ptr() if norm else None for x in w))
    kc, vc = _f64(lay.k_cache), _f64(lay.v_cache)
    tol_k = np.zeros_like(kc)
    loaded = lay.last_loaded.cpu()
    table, at = lay.page_table.cpu().long().numpy(), [0] * batch
    for step, ns in enumerate([(1, 0, P), (P - 2, 3, 1), (3, 2 * P + 1, 0), (0, 0, 0), (1, 1, 1),
                               (4 * P + 5, P, 2 * P - 1)]):
        front, rows = 2, sum(ns)
        total = front + rows + 3                     # rows of no sequence on both sides
        qkv = torch.randn(total, (hq + 2 * hk) * d, generator=g).to(TD[dtype]).cuda()
        q = qkv[:, :hq * d]
        k, v = qkv[:, hq * d:(hq + hk) * d], qkv[:, (hq + hk) * d:]
        starts = np.concatenate([[0], np.cumsum(ns)]) + front
        rs, sp = (torch.tensor(np.array(x), dtype=torch.int32).cuda() for x in (starts, at))
        qo = torch.full((total, hq, d), 5.0).to(TD[dtype]).cuda()
        print(f"[append] {dtype} P={P} d={d} hk={hk} rows of each {ns} at {at}", flush=True)
        B.retro_append_kv_rotary(lay.dims, step, lay.cache, B.Chunk(rs.data_ptr(), sp.data_ptr(), total), r,
                                 q if with_q else None, q.stride(0), k, k.stride(0), v, v.stride(0), qo)
        torch.cuda.synchronize()
        for b in range(batch):
            pos = np.arange(at[b], at[b] + ns[b])
            sl = slice(starts[b], starts[b + 1])
            want, tol = R.turn(_f64(k[sl].reshape(-1, hk, d)), _f64(w[1]) if norm else None, tab, pos, rot,
                               interleaved, 1e-5, dtype)
            kc[table[b][pos // P], :, pos % P] = want
            tol_k[table[b][pos // P], :, pos % P] = tol
            vc[table[b][pos // P], :, :, pos % P] = _f64(v[sl]).reshape(-1, hk, d)
            if with_q:
                want, tol = R.turn(_f64(q[sl].reshape(-1, hq, d)), _f64(w[0]) if norm else None, tab, pos, rot,
                                   interleaved, 1e-5, dtype)
                _within(qo[sl], want, tol, "q")
            loaded[b, :, np.unique(pos // P)] = step - 1
            at[b] += ns[b]
        outside = [i for i in range(total) if not with_q or i < front or i >= front + rows]
        assert (qo[outside] == 5.0).all()
        _within(lay.k_cache, kc, tol_k, "keys")
        assert np.array_equal(_f64(lay.v_cache), vc)
        assert lay.seq_lens.tolist() == at
        assert torch.equal(lay.last_loaded.cpu(), loaded)
        for b in range(batch):   # digests are those of the stored keys, exactly
            for p in range(-(-at[b] // P)):
                page = lay.k_cache[table[b][p], :, :min(P, at[b] - p * P)]
                assert torch.equal(lay.digest[b, :, p, 0], page.amin(1))
                assert torch.equal(lay.digest[b, :, p, 1], page.amax(1))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_append_without_rotation_is_append_kv_tokens(dtype):
    from paper_2508_09001_amd import binding as B
    batch, hk, G, d, P, mp = 70, 2, 2, 64, 16, 4     # more sequences than lanes
    one, two = (_layer(dtype, batch, hk, G, d, P, mp, 3) for _ in range(2))
    g = torch.Generator().manual_seed(9)
    r = B.Rotary(None, 0, 0, 0, 0.0, None, None)
    at = 0
    for step, n in enumerate([5, 1, 20]):
        k, v = (torch.randn(n, batch, hk, d, generator=g).to(TD[dtype]).cuda() for _ in range(2))
        one.append_tokens(step, k, v)
        kb, vb = (x.transpose(0, 1).contiguous() for x in (k, v))
        rs = torch.arange(batch + 1, dtype=torch.int32, device="cuda") * n
        sp = torch.full((batch,), at, dtype=torch.int32, device="cuda")
        B.retro_append_kv_rotary(two.dims, step, two.cache, B.Chunk(rs.data_ptr(), sp.data_ptr(), n * batch), r,
                                 None, 0, kb, hk * d, vb, hk * d, None)
        at += n
        for name in ("k_cache", "v_cache", "digest", "seq_lens", "last_loaded"):
            assert torch.equal(getattr(one, name), getattr(two, name)), (step, name)


def test_append_drops_rows_from_the_first_page_that_is_not_mapped():
    from paper_2508_09001_amd import binding as B
    batch, hk, G, d, P, mp = 4, 2, 1, 64, 16, 4
    lay = _layer("f32", batch, hk, G, d, P, mp, 1)
    lay.page_table[0, 2] = -1
    lay.page_table[1, 0] = lay.dims.num_phys_pages
    lay.page_table[2, 3] = -5
    n, start = [50, 20, 10, 70], [0, 0, -3, 0]        # a sequence that takes no part; one past the table's end
    rows = sum(n)
    k, v = torch.randn(rows, hk, d).cuda(), torch.randn(rows, hk, d).cuda()
    rs = torch.tensor([0, 50, 70, 80, 150], dtype=torch.int32).cuda()
    sp = torch.tensor(start, dtype=torch.int32).cuda()
    B.retro_append_kv_rotary(lay.dims, 0, lay.cache, B.Chunk(rs.data_ptr(), sp.data_ptr(), rows),
                             B.Rotary(None, 0, 0, 0, 0.0, None, None), None, 0, k, hk * d, v, hk * d, None)
    assert lay.seq_lens.tolist() == [32, 0, 0, 64]
    kc, vc, pt = lay.k_cache.cpu(), lay.v_cache.cpu(), lay.page_table.cpu().long()
    for b, m in ((0, 32), (3, 64)):
        pos = torch.arange(m)
        assert torch.equal(kc[pt[b, pos // P], :, pos % P], k.cpu()[rs[b]:rs[b] + m])
        assert torch.equal(vc[pt[b, pos // P], :, :, pos % P], v.cpu()[rs[b]:rs[b] + m])
    free = set(range(lay.dims.num_phys_pages)) - set(pt[pt >= 0].tolist())
    assert (kc[sorted(free)] == 7.0).all() and (vc[sorted(free)] == 9.0).all()


def test_captured_append_replayed_for_other_rows():
    """One capture over a padded batch, replayed with other lengths in its arrays."""
    from paper_2508_09001_amd import binding as B
    batch, hk, G, d, P, mp, total = 3, 2, 2, 128, 16, 6, 40
    lay, ref = (_layer("bf16", batch, hk, G, d, P, mp, 5) for _ in range(2))
    tab = torch.from_numpy(R.table(mp * P, 128, 1e4)).cuda()
    r = B.Rotary(tab.data_ptr(), mp * P, 128, 0, 0.0, None, None)
    q, k, v = (torch.randn(total, h, d).bfloat16().cuda() for h in (hk * G, hk, hk))
    rs, sp = torch.zeros(batch + 1, dtype=torch.int32, device="cuda"), torch.zeros(batch, dtype=torch.int32, device="cuda")
    qo, qr = torch.zeros_like(q), torch.zeros_like(q)

    def call(la, out):
        B.retro_append_kv_rotary(la.dims, 2, la.cache, B.Chunk(rs.data_ptr(), sp.data_ptr(), total), r,
                                 q, hk * G * d, k, hk * d, v, hk * d, out)

    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call(lay, qo)
    at = np.zeros(batch, np.int32)
    for ns in ((1, 1, 1), (0, 30, 10), (17, 0, 5), (1, 1, 1)):
        rs.copy_(torch.tensor(np.concatenate([[0], np.cumsum(ns)]), dtype=torch.int32))
        sp.copy_(torch.from_numpy(at))
        for x in (q, k, v):
            x.normal_()
        graph.replay()
        torch.cuda.synchronize()
        call(ref, qr)
        at += np.array(ns, np.int32)
        assert lay.seq_lens.tolist() == at.tolist()
        assert torch.equal(qo[:sum(ns)], qr[:sum(ns)])
        for name in ("k_cache", "v_cache", "digest", "seq_lens", "last_loaded"):
            assert torch.equal(getattr(lay, name), getattr(ref, name)), name


# more than 16384 times 64 / (lanes of a vector) heads: five groups of heads a wavefront,
# the last of a row not full, queries and keys in one group, keys alone (of 20 places 5 or 9)
@pytest.mark.parametrize("dtype,d,rot,interleaved,rows,hk,G,which", [
    ("bf16", 128, 128, 0, 3001, 5, 4, "qk"), ("bf16", 128, 48, 1, 3001, 5, 4, "qk"),
    ("f32", 128, 128, 0, 1501, 5, 4, "qk"), ("f32", 64, 64, 1, 2601, 5, 4, "qk"),
    ("bf16", 64, 32, 0, 4501, 5, 4, "qk"), ("bf16", 128, 128, 0, 9001, 5, 4, "k"),
    ("bf16", 128, 64, 0, 6001, 1, 8, "qk"), ("bf16", 128, 128, 1, 4201, 5, 4, "q"), ("f32", 128, 0, 0, 6001, 5, 1, "k")])
def test_rotate_many_rows(dtype, d, rot, interleaved, rows, hk, G, which):
    from paper_2508_09001_amd import binding as B
    g = torch.Generator().manual_seed(rows)
    hq, n = hk * G, 700
    qkv = torch.randn(rows, (hq + 2 * hk) * d, generator=g).to(TD[dtype]).cuda()
    pos = torch.randint(0, n, (rows,), generator=g, dtype=torch.int32)
    pos[[1, rows - 1]] = -1          # not written
    pos[[2, rows - 2]] = n           # past the table
    live, past = pos >= 0, pos >= n
    w = [(1 + 0.2 * torch.randn(d, generator=g)).to(TD[dtype]) for _ in range(2)]
    wd, tab = [x.cuda() for x in w], R.table(n, rot, 1e4)
    tab_d = torch.from_numpy(tab).cuda() if rot else None
    r = B.Rotary(tab_d.data_ptr() if rot else None, n if rot else 0, rot, interleaved, 1e-6, *(x.data_ptr() for x in wd))
    dims, posd, calls = _dims(B, dtype, d, hk, G), pos.cuda(), {}
    for name, at, heads in (("q", 0, hq), ("k", hq * d, hk)):
        if name in which:
            x = qkv[:, at:at + heads * d]
            calls[name] = (x, torch.full((rows + 1, heads, d), 5.0).to(TD[dtype]).cuda(), heads)

    def call(src, stride, dst):
        def arg(f, none):
            return [f(i) if i in calls else none for i in ("q", "k")]
        (q, k), (qs, ks), (qo, ko) = arg(src, None), arg(stride, 0), arg(dst, None)
        B.retro_rotate_qk(dims, r, posd, rows, q, qs, k, ks, qo, ko)
        torch.cuda.synchronize()

    print(f"[rotate] {dtype} d={d} rot={rot} il={interleaved} rows={rows} hk={hk} G={G} {which}", flush=True)
    call(lambda i: calls[i][0], lambda i: calls[i][0].stride(0), lambda i: calls[i][1])
    own = {i: x.contiguous().clone() for i, (x, _, _) in calls.items()}
    call(lambda i: own[i], lambda i: calls[i][2] * d, lambda i: own[i])      # in place
    ok = live & ~past if rot else live
    for (name, (x, o, heads)), weight in zip(calls.items(), [w["qk".index(i)] for i in calls]):
        want, tol = R.turn(_f64(x[ok.cuda()].reshape(-1, heads, d)), _f64(weight), tab, pos[ok].numpy(), rot,
                           interleaved, 1e-6, dtype)
        _within(o[:rows][ok.cuda()], want, tol, name)
        assert (o[rows] == 5.0).all() and (o[:rows][~live.cuda()] == 5.0).all()
        if rot:
            assert o[:rows][past.cuda()][..., :rot].isnan().all()
            assert o[:rows][past.cuda()][..., rot:].isfinite().all()
        same = own[name].view(rows, heads, d)
        assert torch.equal(same[ok.cuda()], o[:rows][ok.cuda()])
        assert torch.equal(same[~live.cuda()], x.reshape(rows, heads, d)[~live.cuda()])


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_norms_alone_need_no_positions(dtype):
    from paper_2508_09001_amd import binding as B
    rows, hk, G, d = 9, 2, 3, 128
    g = torch.Generator().manual_seed(6)
    q, k = (torch.randn(rows, h, d, generator=g).to(TD[dtype]).cuda() for h in (hk * G, hk))
    w = (1 + 0.2 * torch.randn(d, generator=g)).to(TD[dtype]).cuda()
    qo, ko = torch.empty_like(q), torch.empty_like(k)
    B.retro_rotate_qk(_dims(B, dtype, d, hk, G), B.Rotary(None, 0, 0, 0, 1e-6, None, w.data_ptr()), None, rows,
                      q, hk * G * d, k, hk * d, qo, ko)
    assert torch.equal(qo, q)
    want, tol = R.turn(_f64(k), _f64(w), None, None, 0, 0, 1e-6, dtype)
    _within(ko, want, tol, "k")
