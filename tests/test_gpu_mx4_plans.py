"""What the host tells of the launches over a cache in 4 bits, against the kernels that a captured
call consists of."""
import ctypes as C
import re

import pytest
import torch

pytestmark = pytest.mark.gpu


def _kernels(call):
    """Nodes of the graph that `call` is captured into, each of them a kernel."""
    path = re.search(r"\S*libamdhip64\.so\S*", open("/proc/self/maps").read()).group(0)
    hip = C.CDLL(path)                       # (the runtime that torch has loaded)
    stream, graph, n = torch.cuda.Stream(), C.c_void_p(), C.c_size_t(0)
    torch.cuda.synchronize()
    assert hip.hipStreamBeginCapture(C.c_void_p(stream.cuda_stream), 2) == 0
    try:
        call(stream.cuda_stream)
    finally:
        assert hip.hipStreamEndCapture(C.c_void_p(stream.cuda_stream), C.byref(graph)) == 0
    assert hip.hipGraphGetNodes(graph, None, C.byref(n)) == 0
    nodes = (C.c_void_p * n.value)()
    assert hip.hipGraphGetNodes(graph, nodes, C.byref(n)) == 0
    for node in nodes:
        kind = C.c_int(-1)
        assert hip.hipGraphNodeGetType(C.c_void_p(node), C.byref(kind)) == 0 and kind.value == 0
    assert hip.hipGraphDestroy(graph) == 0
    return n.value


# KV heads, G, W, budget, pages, type, launches of a step, whether the window is split
@pytest.mark.parametrize("hk,G,W,budget,pages,dtype,launches,split",
                         [(8, 4, 16, 2048, 4100, "bf16", 5, True), (8, 4, 16, 2048, 2064, "bf16", 4, True),
                          (2, 4, 4, 128, 40, "bf16", 4, False), (2, 4, 4, 128, 40, "f32", 4, False),
                          (1, 3, 2, 4096, 300, "f32", 4, True)])
def test_launches(hk, G, W, budget, pages, dtype, launches, split):
    from paper_2508_09001_amd import binding as B
    from paper_2508_09001_amd.layer import RetroLayer
    batch = 1 if pages > 300 else 2
    lay = RetroLayer(batch=batch, num_kv_heads=hk, group=G, head_dim=128, page_size=16, budget=budget, window=W,
                     max_pages=pages, dtype=dtype, kv="mx4", reuse_interval=4)
    td = torch.bfloat16 if dtype == "bf16" else torch.float32
    q = torch.randn(batch, W + 1, hk * G, 128).to(td).cuda()
    k = torch.randn(batch, hk, 128).to(td).cuda()
    print(f"[plans] {hk, G, W, budget, pages, dtype}", flush=True)
    tiles, splits = B.retro_attend_plan(lay.dims, False)
    assert tiles in ((1, 2) if dtype == "bf16" else (1,)) and (splits > 1) == split
    assert B.retro_step_launches(lay.dims) == launches
    assert _kernels(lambda s: lay.step(4, q, k, k, s)) == launches
    assert _kernels(lambda s: lay.step(5, q, k, k, s)) == 4                    # the selection is kept
    assert _kernels(lambda s: lay.attend(4, q, s)) == (2 if split else 1)
    assert _kernels(lambda s: lay.attend_partials(4, q, s)) == 1
