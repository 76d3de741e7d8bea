"""Device buffers of one attention layer and convenience wrappers of the C ABI.

PyTorch only allocates device memory here; every step of the decode path runs in
the gfx950 library (binding.py).  Layouts are the ones documented in
include/retro.h.
"""
from __future__ import annotations

import contextlib
import math
from typing import Optional, Sequence, Tuple, Union

import torch

from . import binding as B

_TORCH_DTYPE = {"bf16": torch.bfloat16, "f32": torch.float32}
_RETRO_DTYPE = {"bf16": B.RETRO_BF16, "f32": B.RETRO_F32}


class RetroRotary:
    """Norms and rotation of a layer's queries and keys (``retro_rotary`` in the header).

    ``positions``: tokens that a position may reach, ``max_pages * page_size`` for
    ``append_chunk``; ``rot_dim``: the leading elements of a head that rotate (0: none),
    paired with those ``rot_dim / 2`` further on or, ``interleaved``, with their
    neighbours; ``q_norm`` / ``k_norm``: weights ``[d]`` of root-mean-square norms, or
    None.  ``table``: cosines and sines ``[positions][rot_dim / 2][2]`` fp32 of the
    caller's own, shared between layers (None: made from ``base``)."""

    def __init__(self, positions: int, rot_dim: int, base: float = 10000.0,
                 interleaved: bool = False, q_norm=None, k_norm=None, eps: float = 1e-6,
                 dtype: str = "bf16", device: str = "cuda", table: Optional[torch.Tensor] = None):
        self.device = torch.device(device)

        def weight(w):
            if w is None:
                return None
            if not isinstance(w, torch.Tensor):
                w = torch.from_numpy(w)
            return w.to(device=self.device, dtype=_TORCH_DTYPE[dtype]).contiguous()

        self.q_norm, self.k_norm = weight(q_norm), weight(k_norm)
        self.table = table
        if rot_dim and table is None:
            self.table = torch.empty(positions, rot_dim // 2, 2, dtype=torch.float32,
                                     device=self.device)
            with _on(self.device):
                B.retro_rotary_table(self.table, positions, rot_dim, base)
        elif rot_dim:
            if tuple(table.shape) != (positions, rot_dim // 2, 2) or \
               table.dtype != torch.float32 or not table.is_contiguous():
                raise ValueError("table must be [positions][rot_dim / 2][2] fp32, contiguous")
        self.struct = B.Rotary(B._ptr(self.table) if rot_dim else None,
                               positions if rot_dim else 0, rot_dim, 1 if interleaved else 0, eps,
                               B._ptr(self.q_norm), B._ptr(self.k_norm))


class RetroChunk:
    """A ragged batch of rows (``retro_chunk``): ``rows`` of each sequence, one sequence's
    behind the other's, from position ``start`` on."""

    def __init__(self, rows: Sequence[int], start: Sequence[int], device):
        if len(rows) != len(start) or any(n < 0 for n in rows):
            raise ValueError("rows and start must hold one entry per sequence")
        self.rows, self.start = [int(n) for n in rows], [int(n) for n in start]
        at = [0]
        for n in self.rows:
            at.append(at[-1] + n)
        self.n_rows = at[-1]
        self.reach = max((p + n for n, p in zip(self.rows, self.start) if n), default=0)
        both = torch.tensor(at + self.start, dtype=torch.int32).to(device)
        self.row_start, self.start_pos = both[:len(at)], both[len(at):]
        self.struct = B.Chunk(self.row_start.data_ptr(), self.start_pos.data_ptr(), self.n_rows,
                              max(self.rows, default=0))


def _on(device: torch.device):
    """The device current for the calls inside (they launch on the current one)."""
    return torch.cuda.device(device) if device.index is not None else contextlib.nullcontext()


def _as_stream(stream) -> torch.cuda.Stream:
    return torch.cuda.ExternalStream(stream) if isinstance(stream, int) else stream


class RetroLayer:
    """State of one layer: paged KV cache, digests, retrospective mask, selection,
    output cache, outputs and workspace, all on one device.  ``kv``: how the cache is
    held, in the layer's ``dtype`` or as "mx4" in 4 bits, which ``RETRO_FLAG_KV_MX4`` in
    ``flags`` asks for too."""

    def __init__(self, batch: int, num_kv_heads: int, group: int, head_dim: int, page_size: int,
                 budget: int, window: int, max_pages: int, dtype: str = "bf16",
                 num_phys_pages: Optional[int] = None, page_table: Optional[torch.Tensor] = None,
                 sm_scale: float = 0.0, budget_permille: int = 0, flags: int = 0,
                 reuse_interval: int = 0,
                 device: str = "cuda", kv: str = "dtype"):
        self.device = torch.device(device)
        if num_phys_pages is None:
            num_phys_pages = batch * max_pages
        if kv not in ("dtype", "mx4"):
            raise ValueError('kv must be "dtype" or "mx4"')
        if kv == "mx4" or flags & B.RETRO_FLAG_KV_MX4:
            kv = "mx4"
            flags |= B.RETRO_FLAG_KV_MX4
        self.kv = kv
        self.dims = B.Dims(batch, num_kv_heads, group, head_dim, page_size, budget, window,
                           max_pages, num_phys_pages, _RETRO_DTYPE[dtype], sm_scale,
                           budget_permille, flags, reuse_interval)
        self.k_max = B.retro_k_max(self.dims)
        self.ws_bytes = B.retro_workspace_size(self.dims)
        self.batch, self.hk, self.G, self.d = batch, num_kv_heads, group, head_dim
        self.hq, self.P, self.W = num_kv_heads * group, page_size, window
        self.dtype = _TORCH_DTYPE[dtype]
        dev, td = self.device, self.dtype
        hk, d, P = num_kv_heads, head_dim, page_size
        if kv == "mx4":  # codes, then exponents, of a page of a KV head
            page = P * d // 2 + P * d // 32
            self.k_cache = torch.zeros(num_phys_pages, hk, page, dtype=torch.uint8, device=dev)
            self.v_cache = torch.zeros_like(self.k_cache)
        else:
            self.k_cache = torch.zeros(num_phys_pages, hk, P, d, dtype=td, device=dev)
            self.v_cache = torch.zeros(num_phys_pages, hk, d, P, dtype=td, device=dev)
        # per logical page of each sequence, as the header lays it out (not per
        # physical page: the pool may hold more or fewer pages than batch * max_pages)
        self.digest = torch.zeros(batch, hk, max_pages, 2, d, dtype=td, device=dev)
        if page_table is None:
            page_table = torch.arange(batch * max_pages, dtype=torch.int32).view(batch, max_pages)
        self.page_table = page_table.to(device=dev, dtype=torch.int32).contiguous()
        # version of the table with every page mapped, so that no row is dropped (None: not so)
        full = bool(((page_table >= 0) & (page_table < num_phys_pages)).all())
        self._full_table = self._table_version() if full else None
        self.seq_lens = torch.zeros(batch, dtype=torch.int32, device=dev)
        self.last_loaded = torch.full((batch, hk, max_pages), -1, dtype=torch.int32, device=dev)
        self.selected = torch.full((batch, hk, self.k_max), -1, dtype=torch.int32, device=dev)
        self.mask = torch.full((batch, hk, self.k_max), -1, dtype=torch.int32, device=dev)
        self.num_selected = torch.zeros(batch, hk, dtype=torch.int32, device=dev)
        Wc = max(window, 1)
        self.o_cache = torch.zeros(batch, Wc, self.hq, d, dtype=torch.float32, device=dev)
        self.lse_cache = torch.full((batch, Wc, self.hq), -math.inf, dtype=torch.float32,
                                    device=dev)
        self.o_out = torch.zeros(batch, window + 1, self.hq, d, dtype=torch.float32, device=dev)
        self.lse_out = torch.zeros(batch, window + 1, self.hq, dtype=torch.float32, device=dev)
        self.o_part = torch.zeros_like(self.o_out)
        self.lse_part = torch.zeros_like(self.lse_out)
        self.workspace = torch.zeros(max(self.ws_bytes, 256), dtype=torch.uint8, device=dev)
        self.cache = B.KVCache(self.k_cache.data_ptr(), self.v_cache.data_ptr(),
                               self.digest.data_ptr(), self.page_table.data_ptr(),
                               self.seq_lens.data_ptr(), self.last_loaded.data_ptr())
        self.sel = B.Selection(self.selected.data_ptr(), self.mask.data_ptr(),
                               self.num_selected.data_ptr())
        self.ocache = B.OutputCache(self.o_cache.data_ptr(), self.lse_cache.data_ptr())
        self.chunk_ws: Optional[torch.Tensor] = None  # of attend_chunk
        self._lens = [0] * batch  # host mirror of seq_lens, for prefill positions

    @classmethod
    def for_spec(cls, spec, **kw) -> "RetroLayer":
        args = dict(batch=spec.batch, num_kv_heads=spec.num_kv_heads, group=spec.group,
                    head_dim=spec.head_dim, page_size=spec.page_size, budget=spec.budget,
                    window=spec.window, max_pages=spec.max_pages, dtype=spec.dtype,
                    budget_permille=spec.budget_permille,
                    reuse_interval=getattr(spec, "reuse_interval", 0))
        args.update(kw)
        return cls(**args)

    def _table_version(self) -> Optional[int]:
        return None if self.page_table.is_inference() else self.page_table._version

    def _may_drop(self) -> bool:
        """Whether the device may have dropped rows that ``_lens`` counts."""
        return self._full_table is None or self._full_table != self._table_version()

    def _dev(self, x, stream=None) -> torch.Tensor:
        """x as the library reads it: as it is, or a copy, which is work of the call's stream."""
        if not isinstance(x, torch.Tensor):
            x = torch.from_numpy(x)
        odd = self.kv == "mx4" and x.data_ptr() % 16
        if x.device == self.seq_lens.device and x.dtype == self.dtype and x.is_contiguous() and not odd:
            if stream is not None and x.is_cuda:  # may be freed by the caller before `stream` has read it
                x.record_stream(_as_stream(stream))
            return x
        with self._on_stream(stream, x):
            y = x.to(device=self.device, dtype=self.dtype).contiguous()
            return y.clone() if self.kv == "mx4" and y.data_ptr() % 16 else y

    # -- calls ----------------------------------------------------------------------
    def prefill(self, seq: int, k, v, stream=None) -> None:
        k, v = self._dev(k, stream), self._dev(v, stream)
        n = k.shape[0]
        B.retro_prefill_kv(self.dims, self.cache, seq, self._lens[seq], n, k, v, stream)
        self._lens[seq] += n
        self._keep = (k, v)  # keep sources alive until the copy has run

    def append(self, step: int, k_new, v_new, stream=None) -> None:
        k_new, v_new = self._dev(k_new, stream), self._dev(v_new, stream)
        B.retro_append_kv(self.dims, step, self.cache, k_new, v_new, stream)
        for b in range(self.batch):
            self._lens[b] += 1

    def append_tokens(self, step: int, k_new, v_new, stream=None) -> None:
        """Several tokens per sequence in one call: k_new / v_new [n][batch][h_k][d]."""
        k_new, v_new = self._dev(k_new, stream), self._dev(v_new, stream)
        n = int(k_new.shape[0])
        B.retro_append_kv_tokens(self.dims, step, self.cache, n, k_new, v_new, stream)
        for b in range(self.batch):
            self._lens[b] += n
        self._keep_append = (k_new, v_new)
        self._keep = (k_new, v_new)

    def select(self, step: int, q_cur, stream=None) -> None:
        q_cur = self._dev(q_cur, stream)
        B.retro_select_pages(self.dims, step, q_cur, self.cache, self.sel, self.workspace,
                             self.ws_bytes, stream)
        self._keep = q_cur

    def attend(self, step: int, q_window, stream=None) -> None:
        q_window = self._dev(q_window, stream)
        B.retro_decode_attend(self.dims, step, q_window, self.cache, self.sel, self.o_part,
                              self.lse_part, self.workspace, self.ws_bytes, stream)
        self._keep = q_window

    def attend_partials(self, step: int, q_window: torch.Tensor, stream=None) -> None:
        """Attention kernel only (partials stay in the workspace); q_window on device."""
        B.retro_decode_attend_partials(self.dims, step, q_window, self.cache, self.sel,
                                       self.workspace, self.ws_bytes, stream)

    def update_kv(self, k_upd, v_upd, stream=None) -> None:
        """UpdateKV: new keys / values [batch][n][h_k][d] for the n most recent stored
        tokens of every sequence (their pages' digests are recomputed)."""
        k_upd, v_upd = self._dev(k_upd, stream), self._dev(v_upd, stream)
        B.retro_update_kv(self.dims, self.cache, int(k_upd.shape[1]), k_upd, v_upd, stream)
        self._keep_upd = (k_upd, v_upd)

    def step_attend_partials(self, step: int, q_window: torch.Tensor, stream=None) -> None:
        """The step's launch that ends in the attention partials (scores where the step
        computes them there, selection, attention) alone; overwrites the selection
        outputs, not last_loaded."""
        B.retro_step_attend_partials(self.dims, step, q_window, self.cache, self.sel,
                                       self.workspace, self.ws_bytes, stream)

    def scores(self, stream=None) -> torch.Tensor:
        """The page scores [batch][h_k][max_pages] fp32 of the last call that computed
        them (entries past a sequence's pages are unspecified)."""
        out = torch.empty(self.batch, self.hk, self.dims.max_pages, dtype=torch.float32,
                          device=self.device)
        B.retro_copy_scores(self.dims, self.workspace, self.ws_bytes, out, stream)
        return out

    def merge(self, step: int, stream=None) -> None:
        B.retro_merge_output_cache(self.dims, step, self.o_part, self.lse_part, self.ocache,
                                   self.o_out, self.lse_out, stream)

    def step(self, step: int, q_window, k_new, v_new, stream=None, noalloc: bool = False) -> None:
        """One retro_step (noalloc: retro_step_noalloc, the library's static scratch in
        place of this layer's workspace)."""
        q_window, k_new, v_new = self._dev(q_window, stream), self._dev(k_new, stream), self._dev(v_new, stream)
        if noalloc:
            B.retro_step_noalloc(self.dims, step, q_window, k_new, v_new, self.cache, self.sel,
                                 self.ocache, self.o_out, self.lse_out, stream)
        else:
            B.retro_step(self.dims, step, q_window, k_new, v_new, self.cache, self.sel,
                         self.ocache, self.o_out, self.lse_out, self.workspace, self.ws_bytes,
                         stream)
        for b in range(self.batch):
            self._lens[b] += 1
        self._keep = (q_window, k_new, v_new)

    # -- chunks of prompts, rotated positions -----------------------------------------
    # (one at a time, like every other call of a layer; with `stream` the copies that
    # an input needs and the new tensors are that stream's too)
    @contextlib.contextmanager
    def _on_stream(self, stream, *inputs):
        """Work of a call on the cache's device and on `stream` (None: the current one)."""
        if not self.seq_lens.is_cuda:
            yield
            return
        with torch.cuda.device(self.seq_lens.device):
            if stream is None:
                yield
                return
            s = _as_stream(stream)
            with torch.cuda.stream(s):
                yield
            for x in inputs:  # may be freed by the caller before `stream` has read them
                if isinstance(x, torch.Tensor) and x.is_cuda:
                    x.record_stream(s)

    def check_rotary(self, rotary: RetroRotary) -> None:
        """ValueError unless the norms' weights and the table are this layer's to read."""
        device = self.seq_lens.device
        for w in (rotary.q_norm, rotary.k_norm):
            if w is not None and (tuple(w.shape) != (self.d,) or w.dtype != self.dtype or
                                  w.device != device):
                raise ValueError(f"norm weights must be [{self.d}] {self.dtype} on {device}")
        if rotary.table is not None and rotary.table.device != device:
            raise ValueError(f"the table must be on {device}")

    def _check_chunk(self, chunk: RetroChunk) -> None:
        if len(chunk.rows) != self.batch:
            raise ValueError("the chunk must hold one entry per sequence")
        if chunk.row_start.device != self.seq_lens.device:
            raise ValueError(f"the chunk must be on {self.seq_lens.device}")
        if chunk.n_rows > self.batch * self.dims.max_pages * self.P:
            raise ValueError("the chunk has more rows than the cache has tokens")

    def read_lens(self) -> None:
        """Takes over the sequences' lengths from the device, which is waited for.  ``chunk``
        does it where it has to; a program calls it after replays of captured calls, which
        the layer does not see, or writes to the table past its tensor."""
        if self.seq_lens.is_cuda:
            torch.cuda.synchronize(self.seq_lens.device)
        self._lens = self.seq_lens.tolist()

    def check_append(self, chunk: RetroChunk) -> None:
        """ValueError unless the chunk's rows are the next tokens and have room."""
        self._check_chunk(chunk)
        if chunk.start != self._lens and self._may_drop():
            self.read_lens()  # (rows may have been dropped here as in the chunk's layer)
        if chunk.start != self._lens:
            raise ValueError("the chunk does not begin where the sequences end")
        room = self.dims.max_pages * self.P
        if chunk.reach > room:
            raise ValueError(f"a sequence holds at most {room} tokens")

    def _rows(self, x, heads: int) -> torch.Tensor:
        """x [rows][heads][d] or [rows][heads * d] as it is where the library can read it
        (rows may be strided: parts of one projection's output), else copied."""
        if not isinstance(x, torch.Tensor):
            x = torch.from_numpy(x)
        if x.shape[0] * heads * self.d != x.numel():
            raise ValueError(f"expected [rows][{heads}][{self.d}], got {tuple(x.shape)}")
        x = x.to(device=self.device, dtype=self.dtype)
        inner = x[:1].is_contiguous() if x.shape[0] else True
        piece = 16 // x.element_size()
        if not inner or x.data_ptr() % 16 or (x.shape[0] > 1 and
                                              (x.stride(0) % piece or
                                               x.stride(0) < heads * self.d)):
            x = x.contiguous()
        return x

    def _stride(self, x: torch.Tensor, heads: int) -> int:
        return x.stride(0) if x.shape[0] > 1 else heads * self.d

    def chunk(self, rows: Sequence[int]) -> RetroChunk:
        """The next ``rows[b]`` tokens of every sequence b, behind what it holds: as counted
        by the calls of this layer, or where pages are or were not mapped (the device drops
        rows there) as on the device, which is waited for."""
        if len(rows) != self.batch:
            raise ValueError("rows must hold one entry per sequence")
        if self._may_drop():
            self.read_lens()
        return RetroChunk(rows, self._lens, self.seq_lens.device)

    def _chunk_workspace(self) -> torch.Tensor:
        if self.chunk_ws is None:
            # (a captured fill would clear the counts at replays only, not for the calls
            # in front of the first one)
            if torch.cuda.is_current_stream_capturing():
                raise RuntimeError("reserve_chunks comes before a captured attend_chunk")
            # for as many rows as the tables have tokens, or the largest call: never replaced
            # by a larger one
            most = min(self.batch * self.dims.max_pages * self.P, ((1 << 31) - 257) // self.G,
                       ((1 << 40) - 1) // (self.hq * self.d))
            self.chunk_ws = torch.zeros(B.retro_chunk_workspace_size(self.dims, most),
                                        dtype=torch.uint8, device=self.device)
        return self.chunk_ws

    def reserve_chunks(self) -> None:
        """Makes the workspace of ``attend_chunk``, ready for every stream when this returns.
        The first ``attend_chunk`` makes it too, except where it is captured into a graph
        (RuntimeError): a program that captures calls this first."""
        with torch.cuda.device(self.seq_lens.device):
            self._chunk_workspace()
            torch.cuda.current_stream().synchronize()

    def rotate(self, rotary: RetroRotary, positions: torch.Tensor, q=None, k=None,
               stream=None) -> Tuple[Optional[torch.Tensor], Optional[torch.Tensor]]:
        """Queries [rows][h_q][d] and keys [rows][h_k][d] (either may be None) normalised
        and rotated to ``positions`` [rows] (int32, on the device), as new tensors."""
        rows = int(positions.numel())
        self.check_rotary(rotary)
        with self._on_stream(stream, positions, q, k):
            positions = positions.to(device=self.device, dtype=torch.int32).contiguous()
            q = None if q is None else self._rows(q, self.hq)
            k = None if k is None else self._rows(k, self.hk)
            if any(x is not None and x.shape[0] != rows for x in (q, k)):
                raise ValueError("one position per row")
            # (rows of negative position are not written: they come out as zeros)
            qo, ko = (None if x is None else
                      torch.zeros(rows, h, self.d, dtype=self.dtype, device=self.device)
                      for x, h in ((q, self.hq), (k, self.hk)))
            B.retro_rotate_qk(self.dims, rotary.struct, positions, rows,
                              q, 0 if q is None else self._stride(q, self.hq),
                              k, 0 if k is None else self._stride(k, self.hk), qo, ko, stream)
        self._keep_rot = (positions, q, k, rotary)
        return qo, ko

    def append_chunk(self, step: int, chunk: RetroChunk, rotary: RetroRotary, k, v, q=None,
                     stream=None) -> Optional[torch.Tensor]:
        """Store the chunk's keys and values [rows][h_k][d], keys normalised and rotated on
        the way; returns the queries q [rows][h_q][d], treated likewise (None without q).
        Rows of a page that is not mapped are dropped, with those behind them."""
        self.check_rotary(rotary)
        self.check_append(chunk)
        with self._on_stream(stream, k, v, q, chunk.row_start):
            k, v = self._rows(k, self.hk), self._rows(v, self.hk)
            q = None if q is None else self._rows(q, self.hq)
            if any(x is not None and x.shape[0] != chunk.n_rows for x in (q, k, v)):
                raise ValueError("one row of q, k and v per row of the chunk")
            out = None if q is None else torch.empty(chunk.n_rows, self.hq, self.d,
                                                     dtype=self.dtype, device=self.device)
            B.retro_append_kv_rotary(self.dims, step, self.cache, chunk.struct, rotary.struct,
                                     q, 0 if q is None else self._stride(q, self.hq),
                                     k, self._stride(k, self.hk), v, self._stride(v, self.hk),
                                     out, stream)
        for b in range(self.batch):
            self._lens[b] += chunk.rows[b]
        self._keep_chunk = (q, k, v, chunk, rotary)
        return out

    def read(self, chunk: RetroChunk, keys: bool = True, values: bool = True, stream=None
             ) -> Tuple[Optional[torch.Tensor], Optional[torch.Tensor]]:
        """The chunk's rows as the cache holds them: keys and values [rows][h_k][d] (None for
        one that is not asked for), zeros for rows that are not stored."""
        self._check_chunk(chunk)
        if not keys and not values:
            return None, None
        with self._on_stream(stream, chunk.row_start):
            k, v = (torch.zeros(chunk.n_rows, self.hk, self.d, dtype=self.dtype, device=self.device)
                    if x else None for x in (keys, values))
            B.retro_read_kv(self.dims, self.cache, chunk.struct, k, v, stream)
        self._keep_read = chunk
        return k, v

    def attend_chunk(self, chunk: RetroChunk, q, lse: bool = False, stream=None
                     ) -> Union[torch.Tensor, Tuple[torch.Tensor, torch.Tensor]]:
        """Dense causal attention of the chunk's (rotated) queries [rows][h_q][d] over
        everything stored: outputs [rows][h_q][d], with ``lse`` also the natural
        log-normalisers [rows][h_q] fp32.  Captured into a graph: after ``reserve_chunks``."""
        self._check_chunk(chunk)
        with self._on_stream(stream, q, chunk.row_start):
            q = self._rows(q, self.hq)
            if q.shape[0] != chunk.n_rows:
                raise ValueError("one row of q per row of the chunk")
            out = torch.empty(chunk.n_rows, self.hq, self.d, dtype=self.dtype, device=self.device)
            z = torch.empty(chunk.n_rows, self.hq, dtype=torch.float32,
                            device=self.device) if lse else None
            ws = self._chunk_workspace()
            B.retro_chunk_attend(self.dims, self.cache, chunk.struct, q, self._stride(q, self.hq),
                                 out, z, ws, ws.numel(), stream)
        self._keep_attend = (q, chunk)
        return (out, z) if lse else out
