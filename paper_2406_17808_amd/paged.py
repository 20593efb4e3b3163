"""Norms of queries and keys per head, and a paged cache held in 4 bits, for callers that hold torch tensors.

Like cache.py this owns device memory and passes data pointers and the current stream to the C ABI; no arithmetic
happens here.
"""
from __future__ import annotations

from typing import Optional, Tuple

import torch

from . import binding as B

_TYPES = {torch.bfloat16: B.CASCADE_BF16, torch.float32: B.CASCADE_F32}


# The current stream as a number, without the stream object around it (0.1 instead of 2 us of a call's host time).
_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None)


_current_device = getattr(torch._C, "_cuda_getDevice", torch.cuda.current_device)


def _like(x: torch.Tensor) -> torch.Tensor:
    """A contiguous array of x's shape (half the host time of torch.empty with all of its arguments)."""
    return torch.empty_like(x, memory_format=torch.contiguous_format)


def _numbered(device) -> torch.device:
    """The device that tensors made on `device` report: "cuda" is the current one."""
    device = torch.device(device)
    return torch.device("cuda", _current_device()) if device.type == "cuda" and device.index is None else device


def _stream(device: torch.device) -> int:
    if _raw_stream is not None:
        return _raw_stream(device.index)
    return torch.cuda.current_stream(device).cuda_stream


def _rows(x: torch.Tensor, device, dtype, tokens: int, heads: int, head_dim: int) -> int:
    """Checks [tokens, heads, head_dim] with the heads of a token next to each other; returns how far apart the tokens lie (0: next to each other)."""
    strides = x.stride()
    if x.dtype is not dtype or x.device != device or x.shape != (tokens, heads, head_dim) or strides[1:] != (head_dim, 1):
        # strides of dimensions of one element say nothing
        fits = x.dtype is dtype and x.device == device and x.shape == (tokens, heads, head_dim)
        assert fits and ((strides[2] == 1 or head_dim == 1) and (strides[1] == head_dim or heads == 1) or x.numel() == 0), \
            (x.device, x.dtype, tuple(x.shape), strides, "wanted", device, dtype, (tokens, heads, head_dim))
    if tokens < 2:
        return 0
    assert strides[0] >= heads * head_dim, ("tokens of an array must not share memory", tuple(x.shape), strides)      # (an expanded one; 0 would stand for contiguous)
    return strides[0]


def _serving_only(*inputs: Optional[torch.Tensor]) -> None:
    if torch.is_grad_enabled():
        for x in inputs:
            if x is not None and x.requires_grad:
                raise RuntimeError("norms and the paged cache have no backward pass: call them under torch.no_grad(), or with inputs that require no gradient")


class RopeTable:
    """Cosines and sines of the positions below n_positions (pairs (i, i + head_dim / 2), angles p * base^(-2i / head_dim))."""

    def __init__(self, n_positions: int, head_dim: int, base: float, device: str = "cuda:0"):
        self.n_positions, self.head_dim, self.base = n_positions, head_dim, base
        self.device = _numbered(device)
        nbytes = B.cascade_rope_table_bytes(n_positions, head_dim)
        self.table = torch.empty(max(nbytes, 16), dtype=torch.uint8, device=self.device)
        with torch.cuda.device(self.device):
            B.cascade_rope_table(self.table.data_ptr(), nbytes, n_positions, head_dim, base, _stream(self.device))


def qk_norm_rope(q: torch.Tensor, k: Optional[torch.Tensor] = None, q_weight: Optional[torch.Tensor] = None,
                 k_weight: Optional[torch.Tensor] = None, eps: float = 1e-6, norm: bool = True, positions: Optional[torch.Tensor] = None,
                 rope: Optional[RopeTable] = None, q_out: Optional[torch.Tensor] = None,
                 k_out: Optional[torch.Tensor] = None) -> Tuple[torch.Tensor, Optional[torch.Tensor]]:
    """RMS norm over head_dim of q [tokens, q heads, head_dim] and k [tokens, k heads, head_dim] with the rotation to `positions`
    [tokens] (int32; None: not rotated, as CascadeKVCache takes them) in the same pass.  norm=False rotates only.  Tokens
    of q and k may lie apart (views of a fused projection).  q_out / k_out may be q / k.  For serving: inputs that require a gradient are refused."""
    if q.requires_grad or k is not None and k.requires_grad or q_weight is not None and q_weight.requires_grad or k_weight is not None and k_weight.requires_grad:
        _serving_only(q, k, q_weight, k_weight)
    device, dtype, (tokens, hq, d) = q.device, q.dtype, q.shape
    assert q.is_cuda and dtype in _TYPES and tokens < 1 << 31, (device, dtype, tokens)
    q_stride, q_out_stride, hk, k_stride, k_out_stride = _rows(q, device, dtype, tokens, hq, d), 0, 0, 0, 0
    if q_out is None:
        q_out = _like(q)
    else:
        q_out_stride = _rows(q_out, device, dtype, tokens, hq, d)
    if k is not None:
        hk = k.shape[1]
        k_stride = _rows(k, device, dtype, tokens, hk, d)
        if k_out is None:
            k_out = _like(k)
        else:
            k_out_stride = _rows(k_out, device, dtype, tokens, hk, d)
    else:
        assert k_out is None and k_weight is None
    for w in (q_weight, k_weight):
        assert w is None or (norm and w.device == device and w.dtype == dtype and w.shape == (d,) and w.is_contiguous())
    if positions is not None:
        assert positions.device == device and positions.dtype == torch.int32 and positions.shape == (tokens,) and positions.is_contiguous()
        assert rope is not None and rope.device == device and rope.head_dim == d, "positions need a RopeTable of this head_dim"
    args = B.cascade_norm_rope_args(
        _TYPES[dtype], d, tokens, hq, hk, norm, eps, 0, q.data_ptr(), k.data_ptr() if hk else None, q_out.data_ptr(), k_out.data_ptr() if hk else None,
        q_stride, k_stride, q_out_stride, k_out_stride, None if q_weight is None else q_weight.data_ptr(), None if k_weight is None else k_weight.data_ptr(),
        *((None, None, 0) if positions is None else (positions.data_ptr(), rope.table.data_ptr(), rope.n_positions)))
    if _current_device() == device.index:
        B.cascade_norm_rope(args, _stream(device))
    else:
        with torch.cuda.device(device):
            B.cascade_norm_rope(args, _stream(device))
    return q_out, k_out


def _batch_bounds(n_tokens: int, max_new: int, max_length: int) -> Tuple[int, int, int]:
    bounds = int(n_tokens), int(max_new), int(max_length)
    B.check_int32(B.CASCADE_E_BAD_ARG, n_tokens=bounds[0], max_new=bounds[1], max_length=bounds[2])
    return bounds


class PagedBatch:
    """The sequences of one call (see cascade_paged_batch): lengths [n] tokens before the new ones, new_offsets [n + 1] rows of the new tokens,
    page_table [n, pages], int32 on the device, and the host's bounds on what they hold.  The arrays are read when the kernels run, so a
    captured step follows lengths that are advanced in place."""

    def __init__(self, lengths: torch.Tensor, new_offsets: torch.Tensor, page_table: torch.Tensor, n_tokens: int, max_new: int, max_length: int):
        n = lengths.shape[0]
        for x in (lengths, new_offsets, page_table):
            assert x.is_cuda and x.dtype == torch.int32 and x.device == lengths.device, (x.device, x.dtype)
        assert lengths.dim() == 1 and lengths.is_contiguous() and tuple(new_offsets.shape) == (n + 1,) and new_offsets.is_contiguous()
        assert page_table.dim() == 2 and page_table.shape[0] == n and page_table.is_contiguous()
        self.device = lengths.device
        self.lengths, self.new_offsets, self.page_table = lengths, new_offsets, page_table
        self.n_tokens, self.max_new, self.max_length = _batch_bounds(n_tokens, max_new, max_length)
        self.c = B.cascade_paged_batch(n_seqs=n, n_tokens=self.n_tokens, max_new=self.max_new, max_length=self.max_length,
                                       dev_lengths=lengths.data_ptr(), dev_new_offsets=new_offsets.data_ptr(),
                                       dev_page_table=page_table.data_ptr(), table_stride=page_table.shape[1])


class PagedKVCache:
    """Pages of keys and values in 4 bits (see cascade_paged_config for the numbers and bytes).  `pages` [n_pages, page bytes] uint8 may be handed in;
    with `rope` append rotates keys, and the queries given to it, to their positions.  One attend at a time: its partial results lie in the workspace.  `workspace` (uint8, workspace_size(cfg) bytes) may be shared by layers
    whose calls follow each other."""

    def __init__(self, cfg: B.cascade_paged_config, device: str = "cuda:0", pages: Optional[torch.Tensor] = None, rope: Optional[RopeTable] = None,
                 workspace: Optional[torch.Tensor] = None):
        self.cfg, self.rope = cfg, rope
        self.n_q_heads, self.n_kv_heads, self.head_dim = cfg.n_q_heads, cfg.n_kv_heads, cfg.head_dim
        self.device = _numbered(device)
        self.torch_dtype = torch.bfloat16 if cfg.dtype == B.CASCADE_BF16 else torch.float32
        self.page_bytes = B.cascade_paged_page_bytes(cfg)
        self.workspace_bytes = B.cascade_paged_workspace_bytes(cfg)
        if self.workspace_bytes == 0:
            B.cascade_paged_init(cfg, 256, 256, 0)      # reports why
        if pages is None:
            pages = torch.empty((cfg.n_pages, self.page_bytes), dtype=torch.uint8, device=self.device)
        assert pages.device == self.device and pages.dtype == torch.uint8 and tuple(pages.shape) == (cfg.n_pages, self.page_bytes) and pages.is_contiguous()
        assert rope is None or (rope.device == self.device and rope.head_dim == cfg.head_dim)
        self.pages = pages
        if workspace is None:
            workspace = torch.empty(self.workspace_size(cfg), dtype=torch.uint8, device=self.device)
        assert workspace.device == self.device and workspace.dtype == torch.uint8 and workspace.is_contiguous()
        assert workspace.numel() >= self.workspace_size(cfg), "the workspace is smaller than workspace_size(cfg)"
        self.workspace = workspace
        self._streams = set()
        with torch.cuda.device(self.device):
            self.ctx = B.cascade_paged_init(cfg, pages.data_ptr(), (self.workspace.data_ptr() + 255) & ~255, self.workspace_bytes,
                                            rope.table.data_ptr() if rope is not None else 0, rope.n_positions if rope is not None else 0)

    @staticmethod
    def workspace_size(cfg: B.cascade_paged_config) -> int:
        return B.cascade_paged_workspace_bytes(cfg) + 256      # the workspace begins at a multiple of 256

    def _first_use(self, stream: int) -> None:
        """The allocator is told of each stream that the cache's arrays are used on, so that they are not handed out again before its work is done, whenever
        the cache is dropped."""
        now = torch.cuda.current_stream(self.device)
        for x in (self.pages, self.workspace) + ((self.rope.table,) if self.rope is not None else ()):
            x.record_stream(now)
        self._streams.add(stream)

    def close(self):
        """Ends the context, a structure of the host: nothing is waited for, so that a cache may also be collected while a stream is being captured.
        (A graph that was captured with the cache needs its arrays for as long as it is replayed.)"""
        if getattr(self, "ctx", None):
            B.cascade_paged_destroy(self.ctx)
            self.ctx = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    def append(self, batch: PagedBatch, k: torch.Tensor, v: torch.Tensor, q: Optional[torch.Tensor] = None,
               q_out: Optional[torch.Tensor] = None) -> Optional[torch.Tensor]:
        """Stores k, v [n_tokens, kv heads, head_dim] of the batch's new tokens; q [n_tokens, q heads, head_dim] is rotated into q_out, which is returned.
        Rows of no sequence (n_tokens above what the offsets reach, as in a padded step) are left as they are in q_out; in one made here they hold anything."""
        if k.requires_grad or v.requires_grad or q is not None and q.requires_grad:
            _serving_only(k, v, q)
        n, d, device, dtype = batch.n_tokens, self.head_dim, self.device, self.torch_dtype
        assert batch.device == device
        stream = _stream(device)
        if stream not in self._streams:
            self._first_use(stream)
        k_stride, v_stride = _rows(k, device, dtype, n, self.n_kv_heads, d), _rows(v, device, dtype, n, self.n_kv_heads, d)
        if q is None:
            assert q_out is None
            B.cascade_paged_append(self.ctx, batch.c, k.data_ptr(), k_stride, v.data_ptr(), v_stride, 0, 0, 0, stream)
            return None
        q_stride = _rows(q, device, dtype, n, self.n_q_heads, d)
        if q_out is None:
            q_out = _like(q)
        else:
            _rows(q_out, device, dtype, n, self.n_q_heads, d)
            assert q_out.is_contiguous()
        B.cascade_paged_append(self.ctx, batch.c, k.data_ptr(), k_stride, v.data_ptr(), v_stride, q.data_ptr(), q_stride, q_out.data_ptr(), stream)
        return q_out

    def attend(self, batch: PagedBatch, q: torch.Tensor, out: Optional[torch.Tensor] = None) -> torch.Tensor:
        """Attention of q [n_tokens, q heads, head_dim], rotated, over the cache, the batch's new tokens included.  Rows of no sequence are left as they are in
        `out`; in one made here they hold anything (hand in an array of zeros where they are looked at)."""
        if q.requires_grad:
            _serving_only(q)
        n, d, device, dtype = batch.n_tokens, self.head_dim, self.device, self.torch_dtype
        assert batch.device == device
        q_stride = _rows(q, device, dtype, n, self.n_q_heads, d)
        stream = _stream(device)
        if stream not in self._streams:
            self._first_use(stream)
        if out is None:
            out = _like(q)
        else:
            _rows(out, device, dtype, n, self.n_q_heads, d)
            assert out.is_contiguous()
        B.cascade_paged_attend(self.ctx, batch.c, q.data_ptr(), q_stride, out.data_ptr(), stream)
        return out

    def read(self, batch: PagedBatch) -> Tuple[torch.Tensor, torch.Tensor]:
        """The rows that the batch calls new, as the values their codes stand for (rows of no sequence hold anything)."""
        assert batch.device == self.device
        k = torch.empty((batch.n_tokens, self.n_kv_heads, self.head_dim), dtype=self.torch_dtype, device=self.device)
        v = _like(k)
        stream = _stream(self.device)
        if stream not in self._streams:
            self._first_use(stream)
        B.cascade_paged_read(self.ctx, batch.c, k.data_ptr(), v.data_ptr(), stream)
        return k, v
