"""Arguments of the rotation, rotated-append and chunk-attention calls, checked on
the host before anything is enqueued (CPU only)."""
import ctypes as C
import os

import pytest

INVALID, UNSUPPORTED, WORKSPACE, OK = -1, -2, -4, 0


@pytest.fixture(scope="module")
def B():
    from paper_2508_09001_amd import binding
    if not os.path.exists(binding.LIB_PATH):
        import __graft_entry__
        __graft_entry__.build()
    return binding


A = 1 << 20  # an address that is 16-byte aligned and never dereferenced here


def _dims(B, **kw):
    base = dict(batch=2, num_kv_heads=8, group=4, head_dim=128, page_size=16, budget_tokens=16, window=0,
                max_pages=64, num_phys_pages=128, dtype=B.RETRO_BF16, sm_scale=0.0)
    base.update(kw)
    return B.Dims(**base)


def _rotary(B, **kw):
    base = dict(table=A, positions=1024, rot_dim=128, interleaved=0, eps=1e-5, q_norm=A, k_norm=A)
    base.update(kw)
    return B.Rotary(**base)


@pytest.mark.parametrize("kw", [dict(table=None), dict(table=A + 4), dict(positions=0), dict(positions=-1),
                                dict(rot_dim=-16), dict(rot_dim=24), dict(rot_dim=144), dict(interleaved=2),
                                dict(eps=-1.0), dict(eps=float("nan")), dict(eps=float("inf")),
                                dict(q_norm=A + 2), dict(k_norm=A + 8)])
def test_bad_rotary(B, kw):
    lib, r, d = B.load_library(), _rotary(B, **kw), _dims(B)
    assert lib.retro_rotate_qk(C.byref(d), C.byref(r), A, 1, A, 4096, A, 1024, A, A, None) == INVALID
    cache, ch = B.KVCache(*[A] * 6), B.Chunk(A + 64, A + 128, 4)
    assert lib.retro_append_kv_rotary(C.byref(d), 0, C.byref(cache), C.byref(ch), C.byref(r), A, 4096, A, 1024,
                                      A, 1024, A, None) == INVALID


def test_rotary_table(B):
    lib = B.load_library()
    for args in ((None, 8, 64, 1e4), (A + 4, 8, 64, 1e4), (A, 0, 64, 1e4), (A, 8, 0, 1e4), (A, 8, 24, 1e4),
                 (A, 8, 144, 1e4), (A, 8, 64, 0.0), (A, 8, 64, float("nan")), (A, 8, 64, float("inf"))):
        assert lib.retro_rotary_table(*args, None) == INVALID


def test_rotate_qk(B):
    lib, r, d = B.load_library(), _rotary(B), _dims(B)

    def call(dims=d, rot=r, pos=A, rows=3, q=A, qs=4096, k=A, ks=1024, qo=A, ko=A):
        return lib.retro_rotate_qk(dims and C.byref(dims), rot and C.byref(rot), pos, rows, q, qs, k, ks, qo,
                                   ko, None)

    assert call(rows=0, pos=None, q=None, k=None) == OK            # nothing to do
    for kw in (dict(dims=None), dict(rot=None), dict(pos=None), dict(rows=-1), dict(q=None, k=None),
               dict(qo=None), dict(ko=None), dict(qs=4095), dict(qs=4100), dict(ks=1016), dict(q=A + 2),
               dict(k=A + 8), dict(qo=A + 4), dict(qs=6144), dict(ks=2048)):   # (in place with a stride)
        assert call(**kw) == INVALID, kw
    assert call(dims=_dims(B, head_dim=96)) == UNSUPPORTED
    # fp32: pieces of four elements
    assert call(dims=_dims(B, dtype=B.RETRO_F32), qs=4098, qo=A + 16) == INVALID


def test_append_rotary(B):
    lib, d = B.load_library(), _dims(B)
    full = B.KVCache(*[A] * 6)

    def call(dims=d, step=0, cache=full, ch=(A + 64, A + 128, 5), rot=_rotary(B), q=A, qs=4096, k=A, ks=1024,
             v=A, vs=1024, qo=A + 4096):
        c = B.Chunk(*ch)
        return lib.retro_append_kv_rotary(C.byref(dims), step, C.byref(cache), C.byref(c), C.byref(rot), q, qs,
                                          k, ks, v, vs, qo, None)

    assert call(ch=(A, A + 64, 0), q=None, k=None, v=None) == OK
    for kw in (dict(step=-1), dict(cache=B.KVCache(A, A, None, A, A, A)), dict(ch=(None, A, 5)),
               dict(ch=(A, None, 5)), dict(ch=(A + 64, A + 128, -1)),
               dict(ch=(A + 64, A, 5)),                            # start_pos is the cache's seq_lens
               dict(rot=_rotary(B, positions=1023)),               # a table shorter than the cache
               dict(q=A + 2), dict(qs=4104 - 16), dict(qo=None), dict(k=None), dict(v=None), dict(ks=1020),
               dict(vs=8), dict(cache=B.KVCache(A + 8, A, A, A, A, A)), dict(q=A + 4096, qs=6144)):
        assert call(**kw) == INVALID, kw
    assert call(rot=_rotary(B, positions=1023), dims=_dims(B, page_size=8)) == UNSUPPORTED


def test_chunk_attend(B):
    lib, d = B.load_library(), _dims(B)
    full = B.KVCache(*[A] * 6)
    ws = B.retro_chunk_workspace_size(d, 5)

    def call(dims=d, cache=full, ch=(A + 64, A + 128, 5), q=A, qs=4096, out=A, lse=A, w=A, n=ws):
        c = B.Chunk(*ch)
        return lib.retro_chunk_attend(C.byref(dims), C.byref(cache), C.byref(c), q, qs, out, lse, w, n, None)

    assert call(ch=(A + 64, A + 128, 0), q=None, out=None, w=None, n=0) == OK
    for kw in (dict(cache=B.KVCache(A, A, A, A, None, A)), dict(ch=(None, A, 5)), dict(ch=(A, None, 5)),
               dict(ch=(A + 64, A, 5)), dict(ch=(A, A + 64, -2)), dict(q=None), dict(q=A + 2), dict(qs=4088),
               dict(qs=4097), dict(out=None), dict(out=A + 8), dict(cache=B.KVCache(A, A + 4, A, A, A, A))):
        assert call(**kw) == INVALID, kw
    assert call(w=None) == WORKSPACE and call(n=ws - 1) == WORKSPACE and call(w=A + 8) == WORKSPACE
    assert call(dims=_dims(B, group=17)) == UNSUPPORTED
    with pytest.raises(B.RetroError):
        B.retro_chunk_workspace_size(d, -1)
    assert lib.retro_chunk_workspace_size(C.byref(d), 5, None) == INVALID


def test_layer_refuses_what_its_kernels_would_misread(B):
    """Weights of another length or type, tables and chunks on the wrong device, of
    another batch or past the cache: refused before anything is read."""
    import torch
    from paper_2508_09001_amd.layer import RetroChunk, RetroLayer, RetroRotary
    lay = RetroLayer(batch=2, num_kv_heads=1, group=2, head_dim=64, page_size=16, budget=16, window=0,
                     max_pages=2, device="cpu")
    x, one = torch.zeros(2, 64), torch.ones(64)
    good = RetroRotary(32, 0, k_norm=one, device="cpu")
    lay.check_rotary(good)
    bad = [RetroRotary(32, 0, device="cpu", **kw)
           for kw in (dict(q_norm=torch.ones(32)), dict(k_norm=torch.ones(128)), dict(k_norm=one, dtype="f32"))]
    elsewhere = RetroRotary(32, 64, device="cpu", table=torch.zeros(32, 32, 2, device="meta"))
    for rot in bad + [elsewhere]:
        with pytest.raises(ValueError):
            lay.rotate(rot, torch.arange(2), k=x)
        with pytest.raises(ValueError):
            lay.append_chunk(0, lay.chunk((1, 1)), rot, x, x)
    q = torch.zeros(2, 2, 64)
    for ch in (RetroChunk((2,), (0,), "cpu"), RetroChunk((1, 1), (0, 0), "meta")):
        with pytest.raises(ValueError):
            lay.attend_chunk(ch, q)
        with pytest.raises(ValueError):
            lay.append_chunk(0, ch, good, x, x)
    with pytest.raises(ValueError):   # 65 rows, 64 tokens
        lay.attend_chunk(lay.chunk((32, 33)), torch.zeros(65, 2, 64))


def test_decoder_refuses_prompts_between_the_steps_of_a_window(B):
    import torch
    from paper_2508_09001_amd.decode import RetroDecoder
    w = dict(wq=torch.zeros(128, 128), wk=torch.zeros(128, 64), wv=torch.zeros(128, 64), wo=torch.zeros(128, 128))
    kw = dict(batch=1, num_kv_heads=1, group=2, head_dim=64, page_size=16, budget=16, max_pages=2, device="cpu",
              library_projections=False, rotary=dict(rot_dim=0))
    dec = RetroDecoder([w], window=2, **kw)
    dec.decoded = 1
    with pytest.raises(ValueError, match="window"):
        dec.prefill_chunk((1,), torch.zeros(1, 128))
    with pytest.raises(ValueError):   # a norm's weights of another length
        RetroDecoder([dict(w, q_norm=torch.ones(32))], window=0, **kw)


def _small_layer(**kw):
    from paper_2508_09001_amd.layer import RetroLayer
    args = dict(batch=2, num_kv_heads=1, group=2, head_dim=64, page_size=16, budget=16, window=0, max_pages=2,
                device="cpu")
    args.update(kw)
    return RetroLayer(**args)


def test_workspace_is_not_made_inside_a_capture(B, monkeypatch):
    """Its fill would only be recorded: an eager call before the first replay would count
    parts from whatever the memory held."""
    import torch
    lay = _small_layer()
    monkeypatch.setattr(torch.cuda, "is_current_stream_capturing", lambda: True)
    with pytest.raises(RuntimeError, match="reserve_chunks"):
        lay._chunk_workspace()
    assert lay.chunk_ws is None
    monkeypatch.setattr(torch.cuda, "is_current_stream_capturing", lambda: False)
    ws = lay._chunk_workspace()
    assert (ws == 0).all() and ws.numel() == B.retro_chunk_workspace_size(lay.dims, 64)
    monkeypatch.setattr(torch.cuda, "is_current_stream_capturing", lambda: True)
    assert lay._chunk_workspace() is ws


@pytest.mark.parametrize("held,rows", [((0, 0), (33, 0)), ((0, 0), (0, 33)), ((32, 5), (1, 3)), ((20, 0), (13, 32))])
def test_rows_that_a_sequence_has_no_room_for(B, held, rows):
    """Room for 32 tokens each: refused before a layer changes, whatever the total."""
    import torch
    from paper_2508_09001_amd.decode import RetroDecoder
    from paper_2508_09001_amd.layer import RetroRotary
    lay = _small_layer()
    lay._lens = list(held)
    x = torch.zeros(sum(rows), 64)
    with pytest.raises(ValueError, match="at most 32 tokens"):
        lay.append_chunk(0, lay.chunk(rows), RetroRotary(32, 0, device="cpu"), x, x)
    assert lay._lens == list(held)
    lay._lens = [0, 32]
    lay.check_append(lay.chunk((32, 0)))    # (up to the end, and none for a full one)
    w = dict(wq=torch.zeros(128, 128), wk=torch.zeros(128, 64), wv=torch.zeros(128, 64), wo=torch.zeros(128, 128))
    dec = RetroDecoder([w, w], batch=2, num_kv_heads=1, group=2, head_dim=64, page_size=16, budget=16, max_pages=2,
                       window=0, device="cpu", library_projections=False)
    for la in dec.layers:
        la._lens = list(held)
    with pytest.raises(ValueError, match="at most 32 tokens"):
        dec.prefill_chunk(rows, torch.zeros(sum(rows), 128))
    assert all(la._lens == list(held) for la in dec.layers)
    dec.layers[1]._lens = [7, 0]            # layers that differ: before the first one changes
    with pytest.raises(ValueError, match="where the sequences end"):
        dec.prefill_chunk((0, 0), torch.zeros(0, 128))


def test_chunks_begin_where_the_device_stopped(B):
    """Rows of pages that are not mapped are dropped on the device: the next chunk begins
    at its lengths, in every layer, not at what the calls counted."""
    import torch
    from paper_2508_09001_amd.layer import RetroChunk
    table = torch.tensor([[0, -1], [2, 3]])
    lays = [_small_layer(page_table=table), _small_layer(page_table=table), _small_layer(num_phys_pages=3),
            _small_layer(), _small_layer()]
    lays[3].page_table[0, 1] = 9
    for lay in lays:
        lay._lens = [20, 7]                           # (counted)
        lay.seq_lens.copy_(torch.tensor([16, 7]))     # (stored)
    for lay in lays[:4]:
        assert lay.chunk((0, 1)).start == [16, 7]
    lays[0]._lens = [20, 7]
    lays[0].check_append(RetroChunk((0, 1), (16, 7), "cpu"))    # another layer's chunk
    assert lays[4].chunk((0, 1)).start == [20, 7]     # every page mapped: as counted, nothing waited for
    lays[4].read_lens()
    assert lays[4].chunk((0, 1)).start == [16, 7]
    with torch.inference_mode():
        assert _small_layer().chunk((1, 1)).start == [0, 0]


def test_tensors_of_another_gpu_are_refused(B):
    """Of the same kind of device, but not the layer's: its kernels would read them there."""
    import torch
    from types import SimpleNamespace as NS
    gpu = [torch.device("cuda", i) for i in (0, 1)]

    def weights(dev):
        return NS(shape=(64,), dtype=torch.bfloat16, device=dev)

    lay = _small_layer()
    lay.device, lay.seq_lens = torch.device("cuda"), NS(device=gpu[0])
    lay.check_rotary(NS(q_norm=weights(gpu[0]), k_norm=weights(gpu[0]), table=NS(device=gpu[0])))
    for kw in (dict(q_norm=weights(gpu[1])), dict(k_norm=weights(gpu[1])), dict(table=NS(device=gpu[1]))):
        with pytest.raises(ValueError, match="cuda:0"):
            lay.check_rotary(NS(**dict(dict(q_norm=None, k_norm=None, table=None), **kw)))
    with pytest.raises(ValueError, match="cuda:0"):
        lay._check_chunk(NS(rows=[1, 1], n_rows=2, row_start=NS(device=gpu[1])))
    meta = _small_layer(device="meta")      # (a layer's own chunk: on its device, whichever is current)
    meta.device = torch.device("cpu")
    assert meta.chunk((1, 1)).row_start.device == meta.seq_lens.device


@pytest.mark.parametrize("kw", [dict(batch=512, num_kv_heads=8, group=16, head_dim=128, max_pages=8192),
                                dict(batch=1024, num_kv_heads=1, group=16, max_pages=16384),
                                dict(batch=8191, num_kv_heads=8, group=4, head_dim=128, max_pages=2048)])
def test_tables_of_more_tokens_than_a_call_has_rows(B, kw, monkeypatch):
    """The workspace is for the largest call where the tables have room for more rows."""
    import torch
    monkeypatch.setattr(torch.cuda, "is_current_stream_capturing", lambda: False)
    lay = _small_layer(device="meta", num_phys_pages=4096, **kw)
    assert lay._chunk_workspace().numel() >= B.retro_chunk_workspace_size(lay.dims, 100000)


@pytest.mark.parametrize("G", [1, 7, 16])
def test_rows_whose_numbers_pass_32_bits(B, G):
    """Numbers of a tile's rows go up to 255 past the last row, and stay below 2^31."""
    lib, n = B.load_library(), C.c_size_t(0)
    d = _dims(B, batch=1, num_kv_heads=1, group=G, head_dim=64)
    full = B.KVCache(*[A] * 6)
    most = ((1 << 31) - 257) // G
    assert lib.retro_chunk_workspace_size(C.byref(d), most, C.byref(n)) == OK
    assert most * G - 1 + 256 < 1 << 31
    for rows in (most + 1, ((1 << 31) - 1) // G):
        assert lib.retro_chunk_workspace_size(C.byref(d), rows, C.byref(n)) == UNSUPPORTED
        ch = B.Chunk(A + 64, A + 128, rows)
        assert lib.retro_chunk_attend(C.byref(d), C.byref(full), C.byref(ch), A, G * 64, A, None, A, 1 << 40,
                                      None) == UNSUPPORTED


def test_rotated_rows_whose_numbers_pass_32_bits(B):
    """A wavefront's row goes up to three past the last one, and stays below 2^31."""
    lib, r = B.load_library(), _rotary(B, rot_dim=64)
    d = _dims(B, batch=1, num_kv_heads=1, group=1, head_dim=64)
    for rows in ((1 << 31) - 4, (1 << 31) - 1):
        assert lib.retro_rotate_qk(C.byref(d), C.byref(r), A, rows, None, 0, A, 64, None, A, None) == UNSUPPORTED


@pytest.mark.parametrize("dtype", [0, 1])
def test_attention_in_place_of_strided_queries(B, dtype):
    """Outputs are contiguous: those of one row would lie in another's queries, unread yet."""
    lib, d = B.load_library(), _dims(B, dtype=dtype)
    cache, ch = B.KVCache(*[A] * 6), B.Chunk(A + 64, A + 128, 5)
    assert lib.retro_chunk_attend(C.byref(d), C.byref(cache), C.byref(ch), A, 6144, A, None, None, 0, None) == INVALID
    # (contiguous queries in place: on to the workspace)
    assert lib.retro_chunk_attend(C.byref(d), C.byref(cache), C.byref(ch), A, 4096, A, None, None, 0, None) == WORKSPACE


def test_longest_run_of_a_chunk(B):
    """What the host knows of the lengths goes along with them (it chooses the kernel)."""
    from paper_2508_09001_amd.layer import RetroChunk
    assert RetroChunk([0] * 300 + [540, 1], [0] * 302, "cpu").struct.longest == 540
    assert RetroChunk([], [], "cpu").struct.longest == 0
    assert B.Chunk(A, A, 5).longest == 0        # unknown
