"""Arguments of the calls on a cache in 4 bits, checked on the host before anything is
enqueued (CPU only)."""
import ctypes as C
import os

import pytest

INVALID, UNSUPPORTED, WORKSPACE, OK = -1, -2, -4, 0
A = 1 << 20  # an address that is 16-byte aligned and never dereferenced here


@pytest.fixture(scope="module")
def B():
    from paper_2508_09001_amd import binding
    if not os.path.exists(binding.LIB_PATH):
        import __graft_entry__
        __graft_entry__.build()
    return binding


def _dims(B, **kw):
    base = dict(batch=2, num_kv_heads=8, group=4, head_dim=128, page_size=16, budget_tokens=16, window=0,
                max_pages=64, num_phys_pages=128, dtype=B.RETRO_BF16, sm_scale=0.0, flags=B.RETRO_FLAG_KV_MX4)
    base.update(kw)
    return B.Dims(**base)


def test_read_kv(B):
    lib = B.load_library()

    def call(dims=_dims(B), cache=B.KVCache(*[A] * 6), ch=(A + 64, A + 128, 5), k=A, v=A):
        c = B.Chunk(*ch)
        return lib.retro_read_kv(dims and C.byref(dims), cache and C.byref(cache), C.byref(c), k, v, None)

    for flags in (0, B.RETRO_FLAG_KV_MX4):
        d = _dims(B, flags=flags)
        assert call(d, ch=(A + 64, A + 128, 0), k=None, v=None) == OK
        for kw in (dict(k=None, v=None), dict(k=A + 8), dict(v=A + 2), dict(ch=(None, A + 128, 5)),
                   dict(ch=(A + 64, None, 5)), dict(ch=(A + 64, A + 128, -1)), dict(ch=(A + 64, A, 5)), dict(cache=None),
                   dict(cache=B.KVCache(None, A, A, A, A, A)), dict(cache=B.KVCache(A + 8, A, A, A, A, A)),
                   dict(cache=B.KVCache(A, A + 4, A, A, A, A)), dict(cache=B.KVCache(A, A, A, None, A, A))):
            assert call(**dict(dict(dims=d), **kw)) == INVALID, kw
    assert call(None) == INVALID
    assert call(_dims(B, page_size=8)) == UNSUPPORTED and call(_dims(B, head_dim=96)) == UNSUPPORTED
    assert call(_dims(B, num_kv_heads=65535, batch=1), ch=(A + 64, A + 128, 1 << 24)) == UNSUPPORTED


def test_flag(B):
    """One bit more than before; those in between stay refused."""
    for flags in (8, 24, 32, -1):
        with pytest.raises(B.RetroError):
            B.retro_k_max(_dims(B, flags=flags))
    assert B.retro_k_max(_dims(B)) == 1
    assert B.retro_workspace_size(_dims(B)) == B.retro_workspace_size(_dims(B, flags=0))
    assert B.retro_chunk_workspace_size(_dims(B), 9) == B.retro_chunk_workspace_size(_dims(B, flags=0), 9)


def test_steps(B):
    """The calls that write pages in dtype by their own launches are refused, the others check
    what they are given."""
    lib, d, cache = B.load_library(), _dims(B, window=2), B.KVCache(*[A] * 6)
    odd = B.KVCache(A, A + 8, A, A, A, A)
    sel, oc = B.Selection(A, A, A), B.OutputCache(A, A)
    D, c, s, o = C.byref(d), C.byref(cache), C.byref(sel), C.byref(oc)
    big = 1 << 40
    assert lib.retro_project_qkv_update(D, c, A, 1024, A, 1, A, A, A, None) == UNSUPPORTED
    assert lib.retro_step_attend_partials(D, 0, A, c, s, A, big, None) == UNSUPPORTED
    for ca, x in ((c, A + 8), (c, None), (C.byref(odd), A)):
        assert lib.retro_prefill_kv(D, ca, 0, 0, 1, x, A, None) == INVALID
        assert lib.retro_prefill_kv(D, ca, 0, 0, 1, A, x, None) == INVALID
        assert lib.retro_append_kv(D, 0, ca, x, A, None) == INVALID
        assert lib.retro_append_kv_tokens(D, 0, ca, 1, A, x, None) == INVALID
        assert lib.retro_update_kv(D, ca, 1, x, A, None) == INVALID
        assert lib.retro_decode_attend_partials(D, 0, x, ca, s, A, big, None) == INVALID
        assert lib.retro_step(D, 0, A, x, A, ca, s, o, A, A, A, big, None) == INVALID
        assert lib.retro_step(D, 0, x, A, A, ca, s, o, A, A, A, big, None) == INVALID
    assert lib.retro_append_kv_tokens(D, 0, c, 0, None, None, None) == OK
    assert lib.retro_append_kv_tokens(D, 0, c, -1, A, A, None) == INVALID
    assert lib.retro_update_kv(D, c, 64 * 16 + 1, A, A, None) == INVALID
    assert lib.retro_prefill_kv(D, c, 2, 0, 1, A, A, None) == INVALID
    assert lib.retro_step(D, 0, A, A, A, c, s, o, A, A, A, 1000, None) == WORKSPACE


def test_layer(B):
    import torch
    from paper_2508_09001_amd.layer import RetroChunk, RetroLayer
    kw = dict(batch=2, num_kv_heads=3, group=2, head_dim=64, page_size=16, budget=16, window=0, max_pages=2,
              device="cpu")
    lay = RetroLayer(kv="mx4", **kw)
    assert lay.dims.flags == B.RETRO_FLAG_KV_MX4 and lay.k_cache.shape == (4, 3, 16 * 64 // 2 + 32)
    assert lay.k_cache.dtype == torch.uint8 and lay.digest.dtype == torch.bfloat16
    assert RetroLayer(**kw).dims.flags == 0 and RetroLayer(flags=1, kv="mx4", **kw).dims.flags == 17
    with pytest.raises(ValueError):
        RetroLayer(kv="fp4", **kw)
    with pytest.raises(ValueError):
        lay.read(RetroChunk((1,), (0,), "cpu"))
    assert lay.read(RetroChunk((1, 0), (0, 0), "cpu"), keys=False, values=False) == (None, None)
    x = torch.zeros(130)[1:129].to(torch.bfloat16)
    assert lay._dev(torch.zeros(129, dtype=torch.bfloat16)[1:]).data_ptr() % 16 == 0 and x.is_contiguous()


def test_attention(B):
    lib, cache = B.load_library(), B.KVCache(*[A] * 6)

    def chunk(dims=_dims(B), cache=cache, ch=(A + 64, A + 128, 5), q=A, qs=512 * 8, out=A, w=A, n=1 << 30):
        c = B.Chunk(*ch)
        return lib.retro_chunk_attend(C.byref(dims), C.byref(cache), C.byref(c), q, qs, out, None, w, n, None)

    for kw in (dict(q=None), dict(q=A + 2), dict(qs=511), dict(out=A + 8), dict(qs=6144),
               dict(cache=B.KVCache(A + 8, A, A, A, A, A)), dict(ch=(A, None, 5))):
        assert chunk(**kw) == INVALID, kw
    assert chunk(w=None) == WORKSPACE and chunk(n=100) == WORKSPACE
    assert chunk(_dims(B, group=17)) == UNSUPPORTED
    d, sel = _dims(B, window=3), B.Selection(A, A, A)

    def window(dims=d, step=3, q=A, cache=cache, sel=sel, o=A, z=A, w=A, n=1 << 40):
        return lib.retro_decode_attend(C.byref(dims), step, q, C.byref(cache), C.byref(sel), o, z, w, n, None)

    for kw in (dict(step=-1), dict(q=None), dict(q=A + 4), dict(cache=B.KVCache(A, A + 8, A, A, A, A)),
               dict(sel=B.Selection(A, None, A)), dict(o=None), dict(z=None)):
        assert window(**kw) == INVALID, kw
    assert window(w=None) == WORKSPACE and window(n=1000) == WORKSPACE


def test_append(B):
    lib, d = B.load_library(), _dims(B)
    r = B.Rotary(None, 0, 0, 0, 0.0, None, None)

    def call(k=A, ks=1024, v=A, vs=1024, cache=B.KVCache(*[A] * 6)):
        ch = B.Chunk(A + 64, A + 128, 5)
        return lib.retro_append_kv_rotary(C.byref(d), 0, C.byref(cache), C.byref(ch), C.byref(r), None, 0, k, ks, v,
                                          vs, None, None)

    for kw in (dict(k=None), dict(v=A + 8), dict(ks=1020), dict(vs=1016), dict(cache=B.KVCache(A + 8, A, A, A, A, A))):
        assert call(**kw) == INVALID, kw
