"""The paged cache held in 4 bits, as cases that can be timed and compared.

Four operators on one cache:

* ``store``: a ragged batch of rows is rounded to 4 bits on its way into the pages,
  with the pages' digests (``retro_append_kv_rotary``), and read back as the values
  that the codes stand for;
* ``read``: rows of the cache as keys and values again (``retro_read_kv``);
* ``attend``: dense causal attention of a ragged batch of rows, one token to a whole
  prompt, over everything stored (``retro_chunk_attend``);
* ``window``: the retrospective window's queries over the selected pages
  (``retro_decode_attend``).

All of them take dims with ``RETRO_FLAG_KV_MX4``.  With ``own`` false ``run`` computes
them from elementary tensor operations; with ``own`` true it makes the library's calls.

A vector of d elements is cut into blocks of 32.  A block has one exponent byte e and
32 codes of a sign, two bits of exponent and one of mantissa (0, 0.5, 1, 1.5, 2, 3, 4, 6):
an element is its code's value times 2^(e - 127).  A block whose largest magnitude m is
2^f (1 <= m / 2^f < 2) gets e = 127 + f - 2, or one more from m = 1.75 * 2^f on, within
2 .. 252; elements go to the nearest code, ties to the even one, at most 6.  A page of a
KV head is ``P d / 2`` bytes of codes, then ``P d / 32`` exponents:

  keys    codes [P][d], exponents [P][d / 32]
  values  codes [P / 4][16][4][d / 16] (four tokens, 16 parts of the vector, token, element),
          exponents [P / 4][d / 32][4]

with element 2 i in the low half of a byte and 2 i + 1 in the high one.
"""
from __future__ import annotations

import math
import random

import torch

own = False

STEP = 70          # the decode step: of the appended tokens, of the window's newest query
_TD = {"bf16": torch.bfloat16, "f32": torch.float32}
_COMMON = dict(dtype="bf16", batch=1, kv_heads=8, group=4, head_dim=128, page=16, n=1, ctx=4096,
               mix="even", fused=True, window=0, budget=0)


def _case(name=None, **kw):
    c = dict(_COMMON, **kw)
    return c if name is None else dict(name=name, **c)


def listed():
    return [
        # one token of each of 64 requests: a serving batch's decode step
        _case("store-token-b64", kind="store", batch=64, ctx=2000, mix="ragged"),
        # several prompts of mixed lengths stored at once, each from inside a page
        _case("store-prompts-b8", kind="store", batch=8, n=4096, ctx=1000, mix="ragged"),
        # the small fp32 layer, a prompt that fills no page at either end
        _case("store-1k-f32", kind="store", dtype="f32", kv_heads=2, head_dim=64, n=1021, ctx=37, fused=False),
        # the last rows of each of 16 requests: what a window's re-embedding looks back at
        _case("read-window-b16", kind="read", batch=16, n=64, ctx=8000, mix="ragged"),
        # a whole sequence, to be handed to another layout or another GPU
        _case("read-32k", kind="read", n=32768, ctx=0),
        # the small fp32 layer, a few tokens after a prompt
        _case("attend-f32", kind="attend", dtype="f32", kv_heads=2, head_dim=64, n=129, ctx=2048),
        # one user's next token at 32K: dense attention where no page may be left out
        _case("attend-token-32k", kind="attend", ctx=32767),
        # the next tokens of a serving batch of mixed lengths
        _case("attend-token-b16", kind="attend", batch=16, ctx=32767, mix="ragged"),
        # a serving batch in which one request brings a chunk of its prompt and the
        # others their next tokens
        _case("attend-serving-b8", kind="attend", batch=8, n=512, ctx=32256, mix="serving"),
        # a prompt from its first token
        _case("attend-prompt-8k", kind="attend", n=8192, ctx=0),
        # one layer of a retrospective step at 32K: 17 queries a head, 128 of 2064 pages
        _case("window-32k", kind="window", ctx=33024, window=16, budget=2048),
        # the same of a serving batch with a smaller budget
        _case("window-b16", kind="window", batch=16, ctx=32768, mix="ragged", window=8, budget=1024),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    """One more case of the listed ranges, odd lengths, groups and heads among them."""
    top = [work(c) for c in listed()]
    most = {k: max(w[k] for w in top) for k in ("bytes", "flops")}
    while True:
        kind = rng.choice(["store", "read", "attend", "attend", "window"])
        d = rng.choice([64, 128, 128])
        c = _case(kind=kind, head_dim=d, dtype=rng.choice(["bf16", "bf16", "bf16", "f32"]),
                  kv_heads=rng.choice([1, 2, 4, 5, 8, 8]), group=rng.choice([1, 2, 3, 4, 4, 7, 8, 16]),
                  page=rng.choice([16, 32]), batch=rng.choice([1, 1, 2, 3, 5, 8, 16, 33, 64]),
                  n=rng.choice([1, 1, _log(rng, 2, 64), _log(rng, 64, 8192)]), ctx=_log(rng, 1, 131072),
                  mix=rng.choice(["even", "ragged", "serving"]), fused=rng.random() < 0.7)
        if kind == "window":
            c.update(n=1, window=rng.choice([0, 1, 4, 8, 16, 32, 64]), budget=32 * _log(rng, 1, 256))
            if (c["window"] + 1) * c["group"] > 1024:
                continue
        w = work(c)
        tokens = c["batch"] * (c["n"] + c["ctx"])
        scores = c["batch"] * c["kv_heads"] * c["group"] * c["n"] * (c["n"] + c["ctx"]) * 4
        if w["bytes"] > most["bytes"] or w["flops"] > most["flops"] or tokens * c["kv_heads"] * d * 2 > 1 << 31:
            continue
        if kind == "attend" and (scores > 16 << 30 or tokens * c["kv_heads"] * d * 8 > 16 << 30):
            continue
        return c


def _lengths(c):
    """Rows of each sequence and stored tokens before them, from the case alone."""
    r, b = random.Random(c["batch"] * 7919 + c["n"] * 31 + c["ctx"]), c["batch"]
    if c["mix"] == "even":
        return [c["n"]] * b, [c["ctx"]] * b
    if c["mix"] == "ragged":
        n = [r.randint(max(1, c["n"] // 4), c["n"]) for _ in range(b)]
    else:  # the first sequence brings a chunk, the others their next token
        n = [c["n"]] + [1] * (b - 1)
    ctx = [r.randint(c["ctx"] // 4, c["ctx"]) for _ in range(b)]
    n[0], ctx[0] = c["n"], c["ctx"]
    return n, ctx


def _pages(c):
    """Pages that a window's selection keeps of each sequence, and their stored tokens."""
    kept = []
    for n, ctx in zip(*_lengths(c)):
        kept.append(min(c["budget"] // c["page"], -(-(n + ctx) // c["page"])))
    return kept


def work(case):
    c, elt = case, 4 if case["dtype"] == "f32" else 2
    n, ctx = _lengths(c)
    rows, hk, hq, d, P = sum(n), c["kv_heads"], c["kv_heads"] * c["group"], c["head_dim"], c["page"]
    held = 2 * (d // 2 + d // 32)   # bytes of a token's key and value of a KV head
    if c["kind"] == "attend":
        keys = sum(a + b for a, b in zip(n, ctx))
        pairs = sum(x * (2 * y + x + 1) // 2 for x, y in zip(n, ctx))
        return {"bytes": keys * hk * held + rows * hq * (2 * d * elt + 4), "flops": 4 * d * hq * pairs}
    if c["kind"] == "window":
        tokens, W = sum(_pages(c)) * P, c["window"]
        out = c["batch"] * (W + 1) * hq
        # (half of the pages are new to the past queries)
        return {"bytes": tokens * hk * held + out * (d * (elt + 4) + 4), "flops": 4 * d * hq * tokens * (1 + W // 2)}
    vectors = rows * hk * 2
    if c["kind"] == "read":
        return {"bytes": rows * hk * held + vectors * d * elt, "flops": vectors * d}
    pages = sum((y + x - 1) // P - y // P + 1 for x, y in zip(n, ctx))
    return {"bytes": 2 * (vectors * d * elt + rows * hk * held) + (pages + c["batch"]) * hk * 2 * d * elt,
            "flops": vectors * d * 4}


# ---- blocks of 32 in 4 bits ----------------------------------------------------------


def _to_codes(x):
    """Codes [..., d] and exponents [..., d / 32] (uint8) of x [..., d]."""
    b = x.float().unflatten(-1, (-1, 32))
    top = b.abs().amax(-1, keepdim=True)
    e = (((top.view(torch.int32) + (1 << 21)) >> 23) - 2).clamp(2, 252)
    t = b.abs() * torch.exp2(127.0 - e)
    code = (t > 0.25).to(torch.uint8)
    for at, above in ((0.75, False), (1.25, True), (1.75, False), (2.5, True), (3.5, False), (5.0, True)):
        code += (t > at) if above else (t >= at)
    code += 8 * (b < 0).to(torch.uint8)
    return code.flatten(-2), e.squeeze(-1).to(torch.uint8)


def _from_codes(packed, e):
    """Values [..., 2 n] in 32 bits of packed codes [..., n] and exponents [..., n / 16]."""
    lut = torch.tensor([0, .5, 1, 1.5, 2, 3, 4, 6, -0., -.5, -1, -1.5, -2, -3, -4, -6], device=packed.device)
    code = torch.stack([packed & 15, packed >> 4], dim=-1).flatten(-2)
    x = lut.index_select(0, code.reshape(-1).int()).view(code.shape)
    return (x.unflatten(-1, (-1, 32)) * torch.exp2(e.float() - 127.0)[..., None]).flatten(-2)


def _packed(code):
    return code[..., 0::2] | (code[..., 1::2] << 4)


def _key_parts(c, cache):
    """Views of key pages: packed codes [...][P][d / 2], exponents [...][P][d / 32]."""
    P, d = c["page"], c["head_dim"]
    return cache[..., :P * d // 2].unflatten(-1, (P, d // 2)), cache[..., P * d // 2:].unflatten(-1, (P, d // 32))


def _value_parts(c, cache):
    """Views of value pages: codes [...][P / 4][16][4][d / 32], exponents [...][P / 4][d / 32][4]."""
    P, d = c["page"], c["head_dim"]
    return (cache[..., :P * d // 2].unflatten(-1, (P // 4, 16, 4, d // 32)),
            cache[..., P * d // 2:].unflatten(-1, (P // 4, d // 32, 4)))


def _keys(c, pages):
    """Keys [...][P][d] in 32 bits of pages' bytes."""
    return _from_codes(*_key_parts(c, pages))


def _values(c, pages):
    code, e = _value_parts(c, pages)
    code = code.transpose(-3, -2).flatten(-2).flatten(-3, -2)     # [...][P][d / 2]
    return _from_codes(code, e.transpose(-2, -1).flatten(-3, -2))


# ---- inputs ------------------------------------------------------------------------


def prepare(case, seed):
    c, dev, td = case, "cuda", _TD[case["dtype"]]
    g = torch.Generator(device=dev).manual_seed(int(seed))
    n, ctx = _lengths(c)
    rows, hk, G, d, P, B = sum(n), c["kv_heads"], c["group"], c["head_dim"], c["page"], c["batch"]
    hq = hk * G
    longest = max(a + b for a, b in zip(n, ctx))
    mp = -(-longest // P)
    used = [-(-(a + b) // P) for a, b in zip(n, ctx)]
    pool = sum(used)
    s = dict(case=case, rows=rows, n_max=max(n), max_pages=mp, pool=pool)
    # a few channels of every key are much larger than the others
    loud = torch.ones(hk, 1, d, device=dev)
    loud.view(hk, d)[:, torch.randperm(d, generator=g, device=dev)[:4]] = 8.0

    def normal(*shape):
        return torch.randn(*shape, generator=g, device=dev, dtype=torch.float32).to(td)

    def ints(v):
        return torch.tensor(v, dtype=torch.int32, device=dev)

    # the pool: every sequence's pages lie anywhere in it, keys and values already in 4 bits
    size = P * d // 2 + P * d // 32
    s["k_cache"] = torch.zeros(pool, hk, size, dtype=torch.uint8, device=dev)
    s["v_cache"] = torch.zeros(pool, hk, size, dtype=torch.uint8, device=dev)
    at = max(1, (1 << 26) // (hk * P * d))
    for p in range(0, pool, at):
        m = min(at, pool - p)
        for name, parts in (("k_cache", _key_parts), ("v_cache", _value_parts)):
            x = normal(m, hk, P, d).float()
            code, e = _to_codes(x * loud if name == "k_cache" else x)
            to, to_e = parts(c, s[name][p:p + m])
            code = _packed(code)
            if name == "v_cache":
                code = code.unflatten(2, (P // 4, 4)).unflatten(-1, (16, -1)).transpose(3, 4)
                e = e.unflatten(2, (P // 4, 4)).transpose(3, 4)
            to.copy_(code)
            to_e.copy_(e)
    table = torch.full((B, mp), -1, dtype=torch.int32, device=dev)
    pages = torch.randperm(pool, generator=g, device=dev).int()
    at = 0
    for b in range(B):
        table[b, :used[b]] = pages[at:at + used[b]]
        at += used[b]
    s["page_table"] = table
    s["row_start"] = ints([sum(n[:i]) for i in range(len(n) + 1)])
    s["start_pos"] = ints(ctx)
    s["seq_lens"] = ints([y if c["kind"] == "store" else x + y for x, y in zip(n, ctx)])
    s["last_loaded"] = torch.full((B, hk, mp), -1, dtype=torch.int32, device=dev)
    s["digest"] = torch.zeros(B, hk, mp, 2, d, dtype=td, device=dev)
    if c["kind"] in ("attend", "store"):
        # queries, or keys and values, of the new tokens: views of one projection's output, or buffers of their own
        if c["fused"]:
            qkv = normal(rows, (hq + 2 * hk) * d)
            parts = qkv.split([hq * d, hk * d, hk * d], dim=1)
            s["q"], s["k"], s["v"] = (x.unflatten(1, (-1, d)) for x in parts)
        else:
            s["q"], s["k"], s["v"] = normal(rows, hq, d), normal(rows, hk, d), normal(rows, hk, d)
        s["k"].mul_(loud.view(hk, d))
    if c["kind"] in ("store", "read"):
        s["k_out"], s["v_out"] = (torch.empty(rows, hk, d, dtype=td, device=dev) for _ in range(2))
    if c["kind"] == "store":
        for b in range(B):  # the digests of the pages that are begun
            lp, slot = ctx[b] // P, ctx[b] % P
            if slot:
                keys = _keys(c, s["k_cache"][table[b, lp].long()])[:, :slot]
                s["digest"][b, :, lp] = torch.stack([keys.amin(1), keys.amax(1)], dim=1).to(td)
    if c["kind"] == "attend":
        s["out"] = torch.empty(rows, hq, d, dtype=td, device=dev)
        s["lse"] = torch.empty(rows, hq, dtype=torch.float32, device=dev)
    if c["kind"] == "window":
        # every head keeps pages of its own; half of them were kept by the last step too,
        # the others were last loaded at some step before
        W, kept = c["window"], _pages(c)
        k_max = min(c["budget"] // P, mp)
        s["q"] = normal(B, W + 1, hq, d)
        s["selected"] = torch.full((B, hk, k_max), -1, dtype=torch.int32, device=dev)
        s["mask"] = torch.full((B, hk, k_max), -1, dtype=torch.int32, device=dev)
        for b in range(B):
            at = torch.rand(hk, used[b], generator=g, device=dev).argsort(-1)[:, :kept[b]]
            s["selected"][b, :, :kept[b]] = at.sort(-1).values.int()
            old = torch.randint(-1, STEP - W, (hk, kept[b]), generator=g, device=dev, dtype=torch.int32)
            again = torch.rand(hk, kept[b], generator=g, device=dev) < 0.5
            s["mask"][b, :, :kept[b]] = torch.where(again, torch.full_like(old, STEP - 1), old)
        s["num_selected"] = ints(kept)[:, None].expand(B, hk).contiguous()
        s["o_part"] = torch.empty(B, W + 1, hq, d, dtype=torch.float32, device=dev)
        s["lse_part"] = torch.empty(B, W + 1, hq, dtype=torch.float32, device=dev)
    if own:
        _handles(s)
    return s


# ---- the library's calls -------------------------------------------------------------


def _handles(s):
    from paper_2508_09001_amd import binding as B

    c = s["case"]
    s["B"] = B
    s["dims"] = B.Dims(c["batch"], c["kv_heads"], c["group"], c["head_dim"], c["page"], max(c["budget"], c["page"]),
                       c["window"], s["max_pages"], s["pool"],
                       B.RETRO_F32 if c["dtype"] == "f32" else B.RETRO_BF16, 0.0, 0, B.RETRO_FLAG_KV_MX4)
    s["cache"] = B.KVCache(*(s[k].data_ptr() for k in ("k_cache", "v_cache", "digest", "page_table", "seq_lens",
                                                        "last_loaded")))
    s["chunk"] = B.Chunk(s["row_start"].data_ptr(), s["start_pos"].data_ptr(), s["rows"], s["n_max"])
    if c["kind"] == "store":
        s["rotary"] = B.Rotary(None, 0, 0, 0, 0.0, None, None)   # keys come rotated
    if c["kind"] == "attend":
        s["ws_bytes"] = B.retro_chunk_workspace_size(s["dims"], s["rows"])
    if c["kind"] == "window":
        s["ws_bytes"] = B.retro_workspace_size(s["dims"])
        s["sel"] = B.Selection(*(s[k].data_ptr() for k in ("selected", "mask", "num_selected")))
    if "ws_bytes" in s:
        s["workspace"] = torch.zeros(s["ws_bytes"], dtype=torch.uint8, device="cuda")


def _call(s):
    B, kind = s["B"], s["case"]["kind"]
    if kind == "store":
        k, v = s["k"], s["v"]
        B.retro_append_kv_rotary(s["dims"], STEP, s["cache"], s["chunk"], s["rotary"], None, 0, k, k.stride(0),
                                 v, v.stride(0), None)
    if kind in ("store", "read"):
        B.retro_read_kv(s["dims"], s["cache"], s["chunk"], s["k_out"], s["v_out"])
        return _rows(s)
    q = s["q"]
    if kind == "attend":
        B.retro_chunk_attend(s["dims"], s["cache"], s["chunk"], q, q.stride(0), s["out"], s["lse"], s["workspace"],
                             s["ws_bytes"])
        return [s["out"], s["lse"]]
    B.retro_decode_attend(s["dims"], STEP, q, s["cache"], s["sel"], s["o_part"], s["lse_part"], s["workspace"],
                          s["ws_bytes"])
    return [s["o_part"], s["lse_part"]]


def _rows(s):
    names = ["k_out", "v_out"] + (["digest", "seq_lens", "last_loaded"] if s["case"]["kind"] == "store" else [])
    return {k: s[k] for k in names}


# ---- the plain forms -------------------------------------------------------------------


def _places(s):
    """Physical page and slot of every row."""
    row_start, start = s["row_start"].long(), s["start_pos"].long()
    rows = torch.arange(s["rows"], device="cuda")
    b = torch.searchsorted(row_start[1:].contiguous(), rows, right=True)
    pos = start[b] + rows - row_start[b]
    return s["page_table"][b, pos // s["case"]["page"]].long(), pos % s["case"]["page"]


def _plain_read(s, phys, slot):
    c = s["case"]
    code, e = _key_parts(c, s["k_cache"])
    s["k_out"].copy_(_from_codes(code[phys, :, slot], e[phys, :, slot]))
    code, e = _value_parts(c, s["v_cache"])
    code, e = code[phys, :, slot // 4, :, slot % 4], e[phys, :, slot // 4, :, slot % 4]
    s["v_out"].copy_(_from_codes(code.flatten(-2), e))
    return _rows(s)


def _plain_store(s):
    c, P = s["case"], s["case"]["page"]
    phys, slot = _places(s)
    code, e = _to_codes(s["k"])
    to, to_e = _key_parts(c, s["k_cache"])
    to[phys, :, slot], to_e[phys, :, slot] = _packed(code), e
    code, e = _to_codes(s["v"])
    to, to_e = _value_parts(c, s["v_cache"])
    to[phys, :, slot // 4, :, slot % 4] = _packed(code).unflatten(-1, (16, -1))
    to_e[phys, :, slot // 4, :, slot % 4] = e
    # the digests of every page that got a key
    row_start, start = s["row_start"].long(), s["start_pos"].long()
    end = start + row_start[1:] - row_start[:-1]
    span = (s["n_max"] + P - 2) // P + 1
    lp = torch.minimum(start[:, None] // P + torch.arange(span, device="cuda"), (end[:, None] - 1) // P)
    seq = torch.arange(c["batch"], device="cuda")[:, None].expand_as(lp)
    keys = _keys(c, s["k_cache"][s["page_table"][seq, lp].long()])
    stored = (lp[..., None] * P + torch.arange(P, device="cuda") < end[:, None, None])[:, :, None, :, None]
    lo = keys.masked_fill(~stored, math.inf).amin(3)
    hi = keys.masked_fill(~stored, -math.inf).amax(3)
    s["digest"][seq, :, lp] = torch.stack([lo, hi], dim=3).to(_TD[c["dtype"]])
    s["last_loaded"][seq, :, lp] = STEP - 1
    s["seq_lens"].copy_(end)
    return _plain_read(s, phys, slot)


def _softmax_of(score, v, shape):
    """Outputs and log-normalisers of masked scores [m][rows][L] over v [m][L][d]."""
    top = score.amax(-1, keepdim=True)
    score.sub_(top.clamp(min=torch.finfo(torch.float32).min)).exp_()
    total = score.sum(-1, keepdim=True)
    o = torch.bmm(score, v) / total.clamp(min=torch.finfo(torch.float32).tiny)
    return o.view(*shape, -1), (top + total.log()).view(shape)


def _plain_attend(s):
    c, P, d = s["case"], s["case"]["page"], s["case"]["head_dim"]
    B, hk, G = c["batch"], c["kv_heads"], c["group"]
    row_start, start, n = s["row_start"].long(), s["start_pos"].long(), s["n_max"]
    j = torch.arange(n, device="cuda")
    inside = j < (row_start[1:] - row_start[:-1])[:, None]
    row = (row_start[:-1, None] + j).clamp(max=s["rows"] - 1)
    q = s["q"][row].float().view(B, n, hk, G, d).permute(0, 2, 3, 1, 4).reshape(B * hk, G * n, d)
    pages = s["page_table"].long().clamp(min=0)
    L = pages.shape[1] * P
    k = _keys(c, s["k_cache"][pages]).permute(0, 2, 4, 1, 3).reshape(B * hk, d, L)
    v = _values(c, s["v_cache"][pages]).permute(0, 2, 1, 3, 4).reshape(B * hk, L, d)
    score = torch.bmm(q, k).view(B, hk, G, n, L).mul_(d ** -0.5)
    key = torch.arange(L, device="cuda")
    seen = (key <= (start[:, None] + j)[..., None]) & (key < s["seq_lens"][:, None, None])
    score.masked_fill_(~seen[:, None, None], -math.inf)
    o, lse = _softmax_of(score.view(B * hk, G * n, L), v, (B, hk, G, n))
    o = o.permute(0, 3, 1, 2, 4).reshape(B, n, hk * G, d)
    lse = lse.permute(0, 3, 1, 2).reshape(B, n, hk * G)
    s["out"][row[inside]] = o[inside].to(_TD[c["dtype"]])
    s["lse"][row[inside]] = lse[inside]
    return [s["out"], s["lse"]]


def _plain_window(s):
    c, P, d, W = s["case"], s["case"]["page"], s["case"]["head_dim"], s["case"]["window"]
    B, hk, G = c["batch"], c["kv_heads"], c["group"]
    q = s["q"].float().view(B, W + 1, hk, G, d).permute(0, 2, 3, 1, 4).reshape(B * hk, G * (W + 1), d)
    sel = s["selected"].long()
    seq = torch.arange(B, device="cuda")[:, None, None]
    head = torch.arange(hk, device="cuda")[None, :, None]
    phys = s["page_table"][seq, sel.clamp(min=0)].long().clamp(min=0)
    L = sel.shape[-1] * P
    k = _keys(c, s["k_cache"][phys, head]).reshape(B * hk, L, d).transpose(1, 2).contiguous()
    v = _values(c, s["v_cache"][phys, head]).reshape(B * hk, L, d)
    score = torch.bmm(q, k).view(B, hk, G, W + 1, L).mul_(d ** -0.5)
    token = sel[..., None] * P + torch.arange(P, device="cuda")
    stored = (sel >= 0)[..., None] & (token < s["seq_lens"][:, None, None, None])
    tau = STEP - W + torch.arange(W + 1, device="cuda")
    tau[W] = 1 << 30
    new = s["mask"][:, :, None] < tau[:, None]                               # [B][hk][W + 1][k]
    seen = (new[..., None] & stored[:, :, None]).flatten(-2)
    score.masked_fill_(~seen[:, :, None], -math.inf)
    o, lse = _softmax_of(score.view(B * hk, G * (W + 1), L), v, (B, hk, G, W + 1))
    s["o_part"].copy_(o.permute(0, 3, 1, 2, 4).reshape(B, W + 1, hk * G, d))
    s["lse_part"].copy_(lse.permute(0, 3, 1, 2).reshape(B, W + 1, hk * G))
    return [s["o_part"], s["lse_part"]]


def run(state):
    s = state
    if own:
        return _call(s)
    kind = s["case"]["kind"]
    if kind == "read":
        return _plain_read(s, *_places(s))
    return {"store": _plain_store, "attend": _plain_attend, "window": _plain_window}[kind](s)


# ---- the definitions in 64 bits ----------------------------------------------------------


def _exact_rounded(x):
    """x [..., d] as its codes stand for it: to the nearest multiple of the step that its size
    calls for."""
    b = x.double().unflatten(-1, (-1, 32))
    m, f = torch.frexp(b.abs().amax(-1, keepdim=True))          # top = m 2^f, 1/2 <= m < 1
    e = (f - 3 + (m >= 0.875)).clamp(-125, 125).double()
    t = b.abs() / 2.0 ** e
    step = 0.5 * 2.0 ** ((t >= 2).double() + (t >= 4).double())
    t = torch.clamp(torch.round(t / step) * step, max=6.0)
    return (torch.sign(b) * t * 2.0 ** e).flatten(-2)


def _exact_element(code):
    """Sign, exponent field and mantissa bit of a code, as a number."""
    sign, field, bit = 1 - 2 * (code >> 3).double(), (code >> 1 & 3).double(), (code & 1).double()
    return sign * torch.where(field == 0, bit / 2, (1 + bit / 2) * 2 ** (field - 1))


def _exact_tokens(c, page, values):
    """[pages * P][d] in 64 bits of one head's pages [pages][bytes], byte by byte."""
    P, d = c["page"], c["head_dim"]
    t, i = torch.arange(P, device="cuda")[:, None], torch.arange(d, device="cuda")
    part = d // 16
    if values:
        nibble = ((t // 4 * 16 + i // part) * 4 + t % 4) * part + i % part
        at_e = (t // 4 * (d // 32) + i // 32) * 4 + t % 4
    else:
        nibble, at_e = t * d + i, t * (d // 32) + i // 32
    code = page[:, nibble // 2].int() >> (nibble % 2 * 4) & 15
    e = page[:, P * d // 2 + at_e].double() - 127
    return (_exact_element(code) * 2.0 ** e).flatten(0, 1)


def exact(case, seed):
    s = prepare(case, seed)
    c, P, d, hk, G = case, case["page"], case["head_dim"], case["kv_heads"], case["group"]
    n, ctx = _lengths(c)
    table, at = s["page_table"].long(), 0
    if c["kind"] in ("store", "read"):
        keys, vals = [], []
        digest, loaded = s["digest"].double(), s["last_loaded"].clone()
        for b in range(c["batch"]):
            end, first = ctx[b] + n[b], ctx[b] // P
            pages = table[b, first:(end - 1) // P + 1]
            both = [torch.stack([_exact_tokens(c, s[x][pages, h], x == "v_cache") for h in range(hk)], dim=1)
                    for x in ("k_cache", "v_cache")]
            off = ctx[b] - first * P
            if c["kind"] == "store":
                for x, rows in zip(both, ("k", "v")):
                    x[off:off + n[b]] = _exact_rounded(s[rows][at:at + n[b]])
                for p in range(len(pages)):
                    held = both[0][p * P:min((p + 1) * P, end - first * P)]
                    digest[b, :, first + p, 0], digest[b, :, first + p, 1] = held.amin(0), held.amax(0)
                loaded[b, :, first:first + len(pages)] = STEP - 1
            keys.append(both[0][off:off + n[b]])
            vals.append(both[1][off:off + n[b]])
            at += n[b]
        out = dict(k_out=torch.cat(keys), v_out=torch.cat(vals))
        if c["kind"] == "store":
            out.update(digest=digest, last_loaded=loaded,
                       seq_lens=torch.tensor([x + y for x, y in zip(n, ctx)], dtype=torch.int32))
        return out
    if c["kind"] == "window":
        W = c["window"]
        out = torch.zeros(c["batch"], W + 1, hk * G, d, dtype=torch.float64, device="cuda")
        lse = torch.full((c["batch"], W + 1, hk * G), -math.inf, dtype=torch.float64, device="cuda")
        for b, kept in enumerate(_pages(c)):
            for h in range(hk):
                lp = s["selected"][b, h, :kept].long()
                k, v = (_exact_tokens(c, s[x][table[b, lp], h], x == "v_cache") for x in ("k_cache", "v_cache"))
                token = (lp[:, None] * P + torch.arange(P, device="cuda")).flatten()
                known = s["mask"][b, h, :kept].repeat_interleave(P)
                q = s["q"][b, :, h * G:(h + 1) * G].double()
                x = q @ k.t() / math.sqrt(d)                                 # [W + 1][G][tokens]
                row = STEP - W + torch.arange(W + 1, device="cuda")[:, None]
                hidden = (token >= ctx[b] + n[b]) | ((row < STEP) & (known >= row))
                x.masked_fill_(hidden[:, None], -math.inf)
                z = torch.logsumexp(x, dim=-1)
                some = z > -math.inf
                lse[b, :, h * G:(h + 1) * G] = z
                out[b, :, h * G:(h + 1) * G][some] = (torch.softmax(x, dim=-1) @ v)[some]
        return [out, lse]
    out = torch.empty(sum(n), hk * G, d, dtype=torch.float64, device="cuda")
    lse = torch.empty(sum(n), hk * G, dtype=torch.float64, device="cuda")
    for b in range(c["batch"]):
        end = ctx[b] + n[b]
        pages = table[b, :-(-end // P)]
        late = torch.arange(end, device="cuda") > torch.arange(ctx[b], end, device="cuda")[:, None]
        for h in range(hk):
            k, v = (_exact_tokens(c, s[x][pages, h], x == "v_cache")[:end] for x in ("k_cache", "v_cache"))
            for j in range(h * G, (h + 1) * G):
                x = s["q"][at:at + n[b], j].double() @ k.t() / math.sqrt(d)
                x.masked_fill_(late, -math.inf)
                lse[at:at + n[b], j] = torch.logsumexp(x, dim=-1)
                out[at:at + n[b], j] = torch.softmax(x, dim=-1) @ v
        at += n[b]
    return [out, lse]
