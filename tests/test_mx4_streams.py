"""Inputs that a layer has to copy before the library reads them (a view at an odd offset of a
cache in 4 bits, another type): the copy is work of the call's stream (CPU only; on the GPU
in test_gpu_mx4_streams.py)."""
import contextlib

import pytest
import torch

from paper_2508_09001_amd import binding as B
from paper_2508_09001_amd.layer import RetroLayer

NAMES = ("retro_prefill_kv", "retro_append_kv", "retro_append_kv_tokens", "retro_select_pages", "retro_decode_attend",
         "retro_update_kv", "retro_step")


class Layer(RetroLayer):
    inside = None

    @contextlib.contextmanager
    def _on_stream(self, stream, *inputs):
        self.inside = stream
        yield
        self.inside = None


def _calls(lay, make, stream):
    hk, hq, d, b, W = lay.hk, lay.hq, lay.d, lay.batch, lay.W
    lay.prefill(0, make(3, hk, d), make(3, hk, d), stream)
    lay.append(0, make(b, hk, d), make(b, hk, d), stream)
    lay.append_tokens(0, make(2, b, hk, d), make(2, b, hk, d), stream)
    lay.select(0, make(b, hq, d), stream)
    lay.attend(0, make(b, W + 1, hq, d), stream)
    lay.update_kv(make(b, 2, hk, d), make(b, 2, hk, d), stream)
    lay.step(0, make(b, W + 1, hq, d), make(b, hk, d), make(b, hk, d), stream)


@pytest.mark.parametrize("kv,dtype", [("mx4", torch.bfloat16), ("mx4", torch.float32), ("dtype", torch.float32)])
def test_copies_are_work_of_the_calls_stream(monkeypatch, kv, dtype):
    for name in NAMES:
        monkeypatch.setattr(B, name, lambda *a: None)
    lay = Layer(batch=2, num_kv_heads=2, group=2, head_dim=64, page_size=16, budget=16, window=1, max_pages=2,
                device="cpu", kv=kv)
    copies = []
    for what in ("clone", "to"):
        def call(x, *a, what=what, real=getattr(torch.Tensor, what), **kw):
            y = real(x, *a, **kw)
            if y is not x:
                copies.append(lay.inside)
            return y
        monkeypatch.setattr(torch.Tensor, what, call)

    def make(*shape):
        n = torch.Size(shape).numel()
        return torch.zeros(n + 1, dtype=dtype)[1:].view(shape)

    _calls(lay, make, "the call's")
    assert len(copies) >= 13 and set(copies) == {"the call's"}
