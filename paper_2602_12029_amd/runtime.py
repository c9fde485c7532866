"""PyTorch plumbing around the C ABI: device buffers and the current stream.

Nothing here computes: tensors are allocated with torch, raw pointers and the
stream handle go to the library, and every step of the path runs in its kernels.
"""
from __future__ import annotations

import numpy as np
import torch

from . import binding as B


# the raw handle of torch's current stream, without building a Stream object for it (3 us a launch) where torch offers that
_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None)


def _stream() -> int:
    if _raw_stream is not None:
        return _raw_stream(torch.cuda.current_device())
    return int(torch.cuda.current_stream().cuda_stream)


def to_device(bits: np.ndarray, dtype: str, device="cuda:0") -> torch.Tensor:
    """Stored bits (float32 / uint16 bf16 patterns / uint8 e4m3 codes) -> device tensor, bit for bit."""
    if dtype == "f32":
        return torch.from_numpy(np.ascontiguousarray(bits, np.float32)).to(device)
    if dtype == "bf16":
        return torch.from_numpy(np.ascontiguousarray(bits, np.uint16).view(np.int16)).to(device).view(torch.bfloat16)
    if dtype == "fp8_e4m3":
        return torch.from_numpy(np.ascontiguousarray(bits, np.uint8)).to(device)
    raise ValueError(dtype)


def from_device(t: torch.Tensor) -> np.ndarray:
    """Device tensor -> float64 numpy (bf16 widened exactly)."""
    return t.detach().to("cpu").to(torch.float64).numpy()


class Rope:
    """Norm and rotation of head rows: radians per position of every pair (float64, on the host), how elements pair up ("halves" or
    "neighbours"), the norm's weights (device tensors [head_dim] in the rows' type, None = no norm) and epsilon."""

    def __init__(self, radians, pairing="halves", q_weight: torch.Tensor | None = None, k_weight: torch.Tensor | None = None,
                 eps: float = 1e-6, device="cuda:0"):
        turns = B.ps_rope_turns(radians)
        self.turns = torch.from_numpy(turns.view(np.int64)).to(device)
        self.device = self.turns.device
        for w in (q_weight, k_weight):
            if w is not None and (not w.is_contiguous() or w.device != self.device):
                raise ValueError(f"norm weights are contiguous tensors on {self.device}")
        self.q_weight, self.k_weight = q_weight, k_weight
        self._q, self._k = ((*w.shape, w.dtype) if w is not None else None for w in (q_weight, k_weight))
        self.struct = B.ps_rope(self.turns.data_ptr() if turns.size else 0, q_weight.data_ptr() if q_weight is not None else 0,
                                k_weight.data_ptr() if k_weight is not None else 0, eps, 2 * turns.size, B.PAIRING.get(pairing, pairing))

    def check(self, device: torch.device, dim: int, q_dtype: torch.dtype | None, k_dtype: torch.dtype | None):
        """Refuses rows of another device, or weights that are not one row of their type."""
        if device != self.device:
            raise ValueError(f"the rotation's parameters are on {self.device}, the rows on {device}")
        if (q_dtype is not None and self._q not in (None, (dim, q_dtype))) or (k_dtype is not None and self._k not in (None, (dim, k_dtype))):
            raise ValueError(f"norm weights [{dim}] of the rows' type are wanted, queries {q_dtype}, keys {k_dtype}")


def _row_strides(name: str, t: torch.Tensor, dtype: torch.dtype, rows: int, heads: int, dim: int, device: int):
    """(row, head) strides of rows [rows, heads, dim] with contiguous elements; anything else is refused.  device: its index, -1 = host
    memory (comparing those takes half as long as comparing torch's device objects, which counts in front of a launch of 3 us)."""
    strides = t.stride()
    if t.dtype is not dtype or t.shape != (rows, heads, dim) or strides[2] != 1 or t.get_device() != device or (device < 0 and not t.is_cpu):
        raise ValueError(f"{name}: rows [{rows}, {heads}, {dim}] of {dtype} with contiguous elements on device {device} are wanted")
    # (of an axis of one the stride is not used, and torch's may be anything)
    return strides[0] if rows > 1 else max(strides[0], dim), strides[1] if heads > 1 else max(strides[1], dim)


def _check_positions(t: torch.Tensor, rows: int, device: int):
    if t.dtype is not torch.int32 or t.shape != (rows,) or not t.is_contiguous() or t.get_device() != device or (device < 0 and not t.is_cpu):
        raise ValueError(f"positions: a contiguous int32 tensor of {rows} on device {device} is wanted")


def _stream_of(device: torch.device) -> int:
    """The current stream, which is the current device's: tensors of another are not served from here."""
    current = torch.cuda.current_device() if device.type == "cuda" else -1
    if device.index != current:
        raise ValueError(f"the tensors are on {device}, which is not the current device")
    return _raw_stream(current) if _raw_stream is not None else int(torch.cuda.current_stream().cuda_stream)


_TORCH_DTYPE = {B.PS_F32: torch.float32, B.PS_BF16: torch.bfloat16}


def rope_rows(geometry: B.ps_geometry, rope: Rope, src: torch.Tensor, positions: torch.Tensor, out: torch.Tensor | None = None) -> torch.Tensor:
    """Queries of any number of tokens [T, Hq, d] normed and rotated; returns them contiguous (in `out` where given)."""
    dtype, n = _TORCH_DTYPE[geometry.q_dtype], src.shape[0]
    row, head = _row_strides("src", src, dtype, n, geometry.num_q_heads, geometry.head_dim, src.get_device())
    _check_positions(positions, n, src.get_device())
    if out is None:
        out = torch.empty(src.shape, dtype=dtype, device=src.device)
    elif out.shape != src.shape or out.dtype is not dtype or not out.is_contiguous() or out.device != src.device:
        raise ValueError("out: a contiguous tensor like src is wanted")
    rope.check(src.device, geometry.head_dim, dtype, None)
    B.ps_rope_rows(geometry, rope.struct, n, src.data_ptr(), row, head, positions.data_ptr(), out.data_ptr(), _stream_of(src.device))
    return out


class DecodeBatch:
    """Device-side state of one decode batch: uploaded tables, workspace, Q, output."""

    def __init__(self, layout, geometry: B.ps_geometry, num_requests: int, q: torch.Tensor, kv: torch.Tensor,
                 scales: torch.Tensor | None = None):
        if not torch.cuda.is_available():
            raise RuntimeError("a GPU is required: the attention path has no CPU fallback")
        self.layout, self.geometry, self.num_requests = layout, geometry, num_requests
        self.q, self.kv, self.scales = q, kv, scales
        self.device = q.device
        self.out = torch.empty_like(q)
        self.lse = torch.empty((num_requests, geometry.num_q_heads), dtype=torch.float32, device=self.device)
        self.tables = None
        self.workspace = None
        self._sync_plan()

    def _sync_plan(self, wait=True, tokens=None):
        # (the layout has changed: where the new tables cannot be had, the old ones must not be launched from)
        old, self.tables, self.workspace = (self.tables, self.workspace), None, None
        self._home = _stream()               # tables and workspace belong to this stream
        tables = torch.empty(B.ps_layout_device_bytes(self.layout), dtype=torch.uint8, device=self.device)
        workspace = torch.empty(B.ps_workspace_bytes(self.layout), dtype=torch.uint8, device=self.device)
        del old
        self._pending = not wait             # other streams have to wait for the upload on the GPU
        if tokens is None:
            B.ps_layout_upload(self.layout, tables.data_ptr(), _stream())
        else:
            B.ps_layout_upload_append(self.layout, tables.data_ptr(), tokens[0].data_ptr(), tokens[1].data_ptr(),
                                      self.kv.data_ptr(), self._sc(), _stream())
        self.tables, self.workspace = tables, workspace
        if wait:
            torch.cuda.current_stream().synchronize()

    def replan(self, options: B.ps_plan_options | None):
        B.ps_layout_replan(self.layout, options)
        self._sync_plan()

    def set_visible(self, prefix_visible=None):
        """Limit how much of its prompt's shared prefix every request sees (None = all of it)."""
        B.ps_layout_set_visible(self.layout, self.num_requests, prefix_visible)
        self._sync_plan()

    def _stream(self, stream: int | None = None) -> int:
        """The current stream, for a launch that reads the tables: behind their upload, whichever stream that went to, and
        they and the workspace live until the launch is done."""
        if stream is None:
            stream = _stream()
        if stream != self._home:
            current = torch.cuda.current_stream()
            # (a launch that is only recorded runs with the graph, whose replays the caller orders)
            if self._pending and not torch.cuda.is_current_stream_capturing():
                B.ps_layout_upload_wait(self.layout, stream)
            for t in (self.tables, self.workspace):
                t.record_stream(current)
        return stream

    def _sc(self):
        return self.scales.data_ptr() if self.scales is not None else 0

    def prefix_attention(self):
        B.ps_prefix_attention(self.layout, self.tables.data_ptr(), self.q.data_ptr(), self.kv.data_ptr(), self._sc(),
                              self.workspace.data_ptr(), self._stream())

    def suffix_attention(self):
        B.ps_suffix_attention(self.layout, self.tables.data_ptr(), self.q.data_ptr(), self.kv.data_ptr(), self._sc(),
                              self.workspace.data_ptr(), self._stream())

    def merge_states(self, with_lse=True):
        B.ps_merge_states(self.layout, self.tables.data_ptr(), self.workspace.data_ptr(), self.out.data_ptr(),
                          self.lse.data_ptr() if with_lse else 0, self._stream())

    def decode_attention(self, with_lse=True, kv: torch.Tensor | None = None):
        B.ps_decode_attention(self.layout, self.tables.data_ptr(), self.q.data_ptr(),
                              (self.kv if kv is None else kv).data_ptr(), self._sc(), self.workspace.data_ptr(),
                              self.out.data_ptr(), self.lse.data_ptr() if with_lse else 0, self._stream())

    def kv_ingest(self, which: int, src_k: torch.Tensor, src_v: torch.Tensor):
        """Store every segment of one kind (0 prefixes, 1 suffixes) from ragged [T, Hkv, d] sources."""
        assert src_k.stride(2) == 1 and src_v.stride() == src_k.stride()
        B.ps_kv_ingest(self.layout, self.tables.data_ptr(), which, src_k.data_ptr(), src_v.data_ptr(),
                       src_k.stride(0), src_k.stride(1), self.kv.data_ptr(), self._sc(), self._stream())

    def kv_append_rope(self, rope: Rope, q: torch.Tensor | None, k: torch.Tensor, v: torch.Tensor, positions: torch.Tensor):
        """The tokens reserved by the last append, from raw projections [R, heads, d]: queries normed and rotated into self.q (q None:
        left alone), keys normed and rotated and values into the cache."""
        rows = self._token_rows(q, k, v, positions)
        rope.check(self.device, self.geometry.head_dim, self.q.dtype if q is not None else None, k.dtype)
        stream = self._stream(_stream_of(self.device))
        B.ps_kv_append_rope(self.layout, self.tables.data_ptr(), rope.struct, rows, self.q.data_ptr() if q is not None else 0,
                            self.kv.data_ptr(), self._sc(), stream)

    def _token_rows(self, q, k, v, positions):
        g, n = self.geometry, self.num_requests
        heads, d, device = g.num_kv_heads, g.head_dim, self.q.get_device()
        dtype = torch.float32 if g.kv_dtype == B.PS_F32 else torch.bfloat16
        strides = _row_strides("k", k, dtype, n, heads, d, device)
        if _row_strides("v", v, dtype, n, heads, d, device) != strides:
            raise ValueError("k and v have the same strides")
        _check_positions(positions, n, device)
        if q is None:
            return B.ps_token_rows(0, k.data_ptr(), v.data_ptr(), 0, 0, *strides, positions.data_ptr())
        q_strides = _row_strides("q", q, _TORCH_DTYPE[g.q_dtype], n, g.num_q_heads, d, device)
        if not self.q.is_contiguous():
            raise ValueError("the batch's queries are a contiguous tensor")
        return B.ps_token_rows(q.data_ptr(), k.data_ptr(), v.data_ptr(), *q_strides, *strides, positions.data_ptr())

    def kv_ingest_rope(self, which: int, rope: Rope, src_k: torch.Tensor, src_v: torch.Tensor, positions: torch.Tensor):
        """kv_ingest of raw projections [T, Hkv, d]: keys normed and rotated on their way; positions int32 [T]."""
        g, n = self.geometry, self._segment_tokens(which)
        heads, d, device = g.num_kv_heads, g.head_dim, self.q.get_device()
        dtype = torch.float32 if g.kv_dtype == B.PS_F32 else torch.bfloat16
        strides = _row_strides("src_k", src_k, dtype, n, heads, d, device)
        if _row_strides("src_v", src_v, dtype, n, heads, d, device) != strides:
            raise ValueError("src_k and src_v have the same strides")
        _check_positions(positions, n, device)
        rope.check(self.device, d, None, dtype)
        stream = self._stream(_stream_of(self.device))
        B.ps_kv_ingest_rope(self.layout, self.tables.data_ptr(), which, rope.struct, src_k.data_ptr(), src_v.data_ptr(), *strides,
                            positions.data_ptr(), self.kv.data_ptr(), self._sc(), stream)

    def kv_gather(self, which: int, dst_k: torch.Tensor, dst_v: torch.Tensor):
        """The stored segments of one kind back into [T, Hkv, d] tensors, bf16 or float32 (kv_ingest the other way round)."""
        g, n, dtype = self.geometry, self._segment_tokens(which), dst_k.dtype
        heads, d, device = g.num_kv_heads, g.head_dim, self.q.get_device()
        if dtype is not torch.bfloat16 and dtype is not torch.float32:
            raise ValueError("dst_k, dst_v: bf16 or float32 tensors are wanted")
        strides = _row_strides("dst_k", dst_k, dtype, n, heads, d, device)
        if _row_strides("dst_v", dst_v, dtype, n, heads, d, device) != strides:
            raise ValueError("dst_k and dst_v have the same strides")
        stream = self._stream(_stream_of(self.device))
        B.ps_kv_gather(self.layout, self.tables.data_ptr(), which, self.kv.data_ptr(), self._sc(),
                       B.PS_F32 if dtype is torch.float32 else B.PS_BF16, dst_k.data_ptr(), dst_v.data_ptr(), *strides, stream)

    def _segment_tokens(self, which: int) -> int:
        """Tokens that an ingest of one kind of segment takes (adopted blocks aside)."""
        return B.ps_ingest_tokens(self.layout, which)

    def block_summaries(self, which: int, summaries: torch.Tensor, summary_scales: torch.Tensor):
        """Eight-bit bounds of every block's keys: summaries int8 [num_blocks, Hkv, 2, d], summary_scales float32 [num_blocks, Hkv]."""
        self._check_summaries(summaries, summary_scales)
        stream = self._stream(_stream_of(self.device))
        B.ps_block_summaries(self.layout, self.tables.data_ptr(), which, self.kv.data_ptr(), self._sc(), summaries.data_ptr(),
                             summary_scales.data_ptr(), stream)

    def _check_summaries(self, summaries, summary_scales):
        heads, n = self.geometry.num_kv_heads, summaries.shape[0]
        if (summaries.dtype is not torch.int8 or summary_scales.dtype is not torch.float32 or summaries.shape != (n, heads, 2, self.geometry.head_dim) or
                summary_scales.shape != (n, heads) or not summaries.is_contiguous() or not summary_scales.is_contiguous() or
                summaries.device != self.device or summary_scales.device != self.device):
            raise ValueError(f"summaries: contiguous int8 [num_blocks, Hkv, 2, d] and float32 [num_blocks, Hkv] on {self.device} are wanted")

    def select(self, blocks: int, keep_first: int = 1, keep_last: int = 2) -> "SelectedBatch":
        """A step over `blocks` blocks of every request's shared context and its private tokens, chosen by the queries."""
        return SelectedBatch(self, blocks, keep_first, keep_last)

    def append_step(self, pool, new_k: torch.Tensor, new_v: torch.Tensor, active=None):
        """One decode step of cache growth: tables grow on the host and are uploaded again, then the new
        tokens ([R, Hkv, d], contiguous) are stored.  Returns the destinations the host chose."""
        if torch.cuda.is_current_stream_capturing():
            raise RuntimeError("append_step changes the tables on the host: it cannot be recorded into a graph")
        if not (new_k.is_contiguous() and new_v.is_contiguous()):
            raise ValueError("append_step stores tokens from contiguous tensors")
        dest = B.ps_layout_append(pool, self.layout, self.num_requests, active)
        # No wait on the host for the upload: it is ordered in front of what follows on this stream, and launches of this
        # batch on other streams wait for it there.
        self._sync_plan(wait=False, tokens=(new_k, new_v))
        return dest

    def stage_out(self, image: torch.Tensor):
        """Copy the batch's blocks (and e4m3 scales) into `image`: uint8, device memory or pinned host memory."""
        B.ps_kv_stage_out(self.layout, self.tables.data_ptr(), self.kv.data_ptr(), self._sc(), image.data_ptr(), self._stream())

    def stage_in(self, image: torch.Tensor):
        B.ps_kv_stage_in(self.layout, self.tables.data_ptr(), image.data_ptr(), self.kv.data_ptr(), self._sc(), self._stream())

    def park(self, pool):
        """Hand the batch's blocks back to the pool (after stage_out has completed)."""
        torch.cuda.current_stream().synchronize()
        B.ps_layout_park(pool, self.layout)

    def resume(self, pool):
        """Take blocks again and upload the new tables; stage_in then restores the contents."""
        B.ps_layout_resume(pool, self.layout)
        self._sync_plan()

    def workspace_views(self):
        """(o [slots, Hq, d] fp32, lse [slots, Hq] fp32) views of the partial-state workspace."""
        slots, off = B.ps_workspace_layout(self.layout)
        g = self.geometry
        o = self.workspace[:off].view(torch.float32).view(slots, g.num_q_heads, g.head_dim)
        lse = self.workspace[off:off + slots * g.num_q_heads * 4].view(torch.float32).view(slots, g.num_q_heads)
        return o, lse


class SelectedBatch(DecodeBatch):
    """A selection over a DecodeBatch: its queries and cache, block lists of its own.  select_blocks() chooses, decode_attention() and
    its parts attend; after append_step, set_visible or replan of the base, follow().  A follow or a replan starts the lists anew:
    the next step chooses first.  Calls on one selection are ordered by the caller: they share its lists and its scratch memory."""

    def __init__(self, base: DecodeBatch, blocks: int, keep_first: int = 1, keep_last: int = 2):
        self.base, self.scratch, self._lists = base, None, None
        layout = B.ps_layout_select(base.layout, blocks, keep_first, keep_last)
        super().__init__(layout, base.geometry, base.num_requests, base.q, base.kv, base.scales)

    @property
    def q(self) -> torch.Tensor:
        return self.base.q

    @q.setter
    def q(self, q: torch.Tensor):
        self.base.q = q

    def _sync_plan(self, wait=True, tokens=None):
        super()._sync_plan(wait, tokens)
        self.scratch = torch.empty(B.ps_select_workspace_bytes(self.layout), dtype=torch.uint8, device=self.device)
        indptr, stride = B.ps_select_lists(self.layout, self.num_requests)
        self._lists = self.tables.view(torch.int32).as_strided((self.geometry.num_kv_heads, int(indptr[-1])), (stride, 1))

    def _stream(self, stream: int | None = None) -> int:
        stream = super()._stream(stream)
        if stream != self._home:
            self.scratch.record_stream(torch.cuda.current_stream())
        return stream

    def select_blocks(self, summaries: torch.Tensor, summary_scales: torch.Tensor):
        """Scores every block of the shared contexts against the base's queries and writes the lists of the highest."""
        self._check_summaries(summaries, summary_scales)
        base, stream = self.base, _stream_of(self.device)
        base._stream(stream)                 # (the base's tables, too, behind their upload)
        self._stream(stream)
        B.ps_select_blocks(base.layout, base.tables.data_ptr(), self.layout, self.tables.data_ptr(), base.q.data_ptr(), summaries.data_ptr(),
                           summary_scales.data_ptr(), self.scratch.data_ptr(), stream)

    def follow(self):
        """In line with the base again.  Like the base's append_step it does not wait on the host."""
        if torch.cuda.is_current_stream_capturing():
            raise RuntimeError("follow changes the tables on the host: it cannot be recorded into a graph")
        B.ps_layout_select_follow(self.base.layout, self.layout)
        self._sync_plan(wait=False)

    def lists(self) -> torch.Tensor:
        """The chosen blocks, int32 [Hkv, sum of the list lengths] (requests one behind another, see list_indptr()): a view."""
        return self._lists

    def list_indptr(self) -> np.ndarray:
        return B.ps_select_lists(self.layout, self.num_requests)[0]
