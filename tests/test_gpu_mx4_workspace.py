"""Whole steps over a cache in 4 bits, whose pages are selected with counters in the workspace: a
step is the same whatever another geometry's call has left there."""
import pytest
import torch

pytestmark = pytest.mark.gpu

SMALL = dict(batch=2, num_kv_heads=2, group=4, head_dim=64, page_size=16, budget=128, window=4, max_pages=40)
# queries of one row, so that no partial result of a step is zero, and more of them than SMALL's workspace
LARGE = dict(batch=2, num_kv_heads=8, group=16, head_dim=128, page_size=16, budget=1024, window=0, max_pages=80)
STATE = ("digest", "last_loaded", "seq_lens", "selected", "mask", "num_selected", "k_cache", "v_cache", "o_out", "lse_out")


class Steps:
    """A layer with a prompt, and the inputs of its steps in buffers of their own."""

    def __init__(self, kw, seed=1, **more):
        from paper_2508_09001_amd.layer import RetroLayer
        self.lay = RetroLayer(**kw, **more)
        self.g = torch.Generator().manual_seed(seed)
        lay = self.lay
        for s in range(lay.batch):
            lay.prefill(s, *(self._rand(300 + 100 * s, lay.hk, lay.d) for _ in range(2)))
        self.q = torch.zeros(lay.batch, lay.W + 1, lay.hq, lay.d, dtype=torch.bfloat16, device="cuda")
        self.k, self.v = (torch.zeros(lay.batch, lay.hk, lay.d, dtype=torch.bfloat16, device="cuda") for _ in range(2))

    def _rand(self, *shape):
        return torch.randn(*shape, generator=self.g).bfloat16().cuda()

    def load(self):
        for x in (self.q, self.k, self.v):
            x.copy_(self._rand(*x.shape))

    def step(self, t, load=True, **kw):
        if load:
            self.load()
        self.lay.step(t, self.q, self.k, self.v, **kw)


def _same(a, b, at):
    torch.cuda.synchronize()
    for name in STATE:
        assert torch.equal(getattr(a.lay, name), getattr(b.lay, name)), (at, name)


@pytest.mark.parametrize("other", ["mx4", "dtype"])
def test_workspace_that_another_geometry_has_used(other):
    a, want, b = Steps(SMALL, kv="mx4"), Steps(SMALL, kv="mx4"), Steps(LARGE, seed=2, kv=other)
    from paper_2508_09001_amd import binding as B
    assert B.retro_step_launches(a.lay.dims) == 4      # scores and selection are one launch
    assert b.lay.ws_bytes > a.lay.ws_bytes
    a.lay.workspace = torch.zeros(b.lay.ws_bytes, dtype=torch.uint8, device="cuda")
    if other == "mx4":
        b.lay.workspace = a.lay.workspace
    else:  # attention whose partial results go to the workspace, without the one-launch step's words
        b.lay.select(0, torch.ones(2, 128, 128))
        b.lay.attend(0, torch.ones(2, 1, 128, 128))
        a.lay.workspace.copy_(b.lay.workspace)
    for t in range(4):
        print(f"[workspace] {other} step {t}", flush=True)
        if other == "mx4":
            b.step(t)
        a.step(t)
        want.step(t)
        _same(a, want, t)


def test_captured_noalloc_step_between_steps_of_another_geometry():
    a, want, b = Steps(SMALL, kv="mx4"), Steps(SMALL, kv="mx4"), Steps(LARGE, seed=2, kv="mx4")
    want.step(0)
    a.step(0, noalloc=True)
    _same(a, want, "first")
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        a.step(1, load=False, noalloc=True)
    for i in range(4):
        print(f"[noalloc] replay {i}", flush=True)
        if i != 2:
            b.step(i, noalloc=True)
        a.load()
        graph.replay()
        want.step(1)
        _same(a, want, i)
