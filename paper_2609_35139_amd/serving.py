"""Torch-side marshalling of answering over a paged cache (``cr_append_kv``,
``cr_attend``): device buffers and streams only, like :mod:`repairer`.

:class:`PagedCache` wraps the block pool that a paged repair writes
(``binding.paged_layout``); :meth:`PagedCache.sequences` describes a batch and
is reused by every layer (and, as the lengths and the table are read on the
device, by every replay of a captured step)::

    cache = PagedCache(pool)                        # [L][2][n_blocks][block_size][H][d_h]
    step = cache.sequences(block_table, kv_lens)    # one new token per sequence
    for layer in range(L):
        cache.append(layer, step, k, v, q=q, q_out=q, rope={"theta": 1e6})
        o = cache.attend(layer, step, q)

Calls go to ``stream``, or to torch's current stream on the cache's device.
Where that is not the stream that a tensor was allocated on, the caller orders
the two and keeps the tensor (or calls its ``record_stream``) until the call
has run, as for any torch operation on another stream.
"""
from __future__ import annotations

import ctypes
from typing import Optional, Sequence

import numpy as np
import torch

from . import binding as B

# handle of torch's current stream on a device (the Stream object that
# torch.cuda.current_stream makes costs more than a launch's other checks)
_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream",
                      lambda i: torch.cuda.current_stream(i).cuda_stream)
_DTYPE = {torch.bfloat16: B.CR_DTYPE_BF16, torch.float32: B.CR_DTYPE_F32}


class Sequences:
    """A batch of sequences of a :class:`PagedCache` (cr_sequences)."""

    def __init__(self, cache: "PagedCache", block_table: torch.Tensor, kv_lens: torch.Tensor,
                 query_offsets: Optional[Sequence[int]]):
        for t, dims, name in ((block_table, 2, "block_table"), (kv_lens, 1, "kv_lens")):
            if t.dtype != torch.int32 or t.dim() != dims or not t.is_contiguous():
                raise TypeError(f"{name} must be a contiguous {dims}-d int32 tensor")
            if t.device != cache.pool.device:
                raise ValueError(f"{name} must be on the cache's device")
        n = kv_lens.shape[0]
        if block_table.shape[0] != n:
            raise ValueError("block_table needs one row per sequence")
        self.cache = cache
        self.block_table, self.kv_lens = block_table, kv_lens        # keeps them alive
        self.struct, self._offsets = B.sequences_struct(
            n, kv_lens.data_ptr(), block_table.data_ptr(), block_table.shape[1], cache.block_size,
            cache.n_blocks, cache.stride_block, query_offsets)
        self.n_tokens = n if query_offsets is None else int(self._offsets[-1])
        self.workspace_bytes = {}                                    # by (heads, shared_len)


class PagedCache:
    """Block pool [n_layers][2][n_blocks][block_size][n_kv_heads][head_dim]
    (any strides that cr_kv_layout and stride_block can describe)."""

    def __init__(self, pool: torch.Tensor):
        if pool.dim() != 6 or pool.shape[1] != 2 or pool.dtype not in _DTYPE:
            raise TypeError("pool must be a bf16 or fp32 [L][2][n_blocks][block_size][H][d_h] tensor")
        if not pool.is_cuda or pool.stride(5) != 1:
            raise ValueError("pool must be device memory whose last dimension is contiguous")
        self.pool, self.device = pool, pool.device
        L, _, self.n_blocks, self.block_size, H, d = pool.shape
        # (the stride of a dimension of one element addresses nothing)
        st = [x if n > 1 else 0 for x, n in zip(pool.stride(), pool.shape)]
        self.stride_block = st[2]
        self.layout = B.cr_kv_layout(L, H, d, _DTYPE[pool.dtype], st[0], st[1], st[3], st[4])
        self.n_kv_heads, self.head_dim = H, d

    def sequences(self, block_table: torch.Tensor, kv_lens: torch.Tensor,
                  query_offsets: Optional[Sequence[int]] = None) -> Sequences:
        """block_table: device int32 [n_seqs][max_blocks]; kv_lens: device int32
        [n_seqs], the new tokens included; query_offsets: host offsets of each
        sequence's new tokens, or None for one each."""
        return Sequences(self, block_table, kv_lens, query_offsets)

    def _tokens(self, seqs: Sequences) -> int:
        if seqs.cache is not self:
            raise ValueError("the sequences were made by another cache")
        return seqs.n_tokens

    def _rows(self, t: torch.Tensor, n: int, heads: int, name: str) -> B.cr_rows:
        if t.dtype is not self.pool.dtype or t.device != self.device:
            raise TypeError(f"{name} must have the cache's dtype and device")
        if t.shape != (n, heads, self.head_dim):
            raise ValueError(f"{name}: shape {tuple(t.shape)}, expected {(n, heads, self.head_dim)}")
        st = t.stride()
        if st[2] != 1:
            raise ValueError(f"{name}: the last dimension must be contiguous")
        return B.cr_rows(t.data_ptr(), st[0] if n > 1 else 0, st[1] if heads > 1 else 0)

    def _index(self, t: Optional[torch.Tensor], n: int, name: str) -> Optional[int]:
        if t is None:
            return None
        if t.dtype is not torch.int32 or t.device != self.device or t.shape != (n,) or \
                not t.is_contiguous():
            raise TypeError(f"{name} must be a contiguous int32 [{n}] tensor on the cache's device")
        return t.data_ptr()

    def _on(self, stream: Optional[torch.cuda.Stream], call) -> None:
        """call(stream handle) with the cache's device and the call's stream as
        torch's current ones: the library launches on the current device, and a
        workspace or result allocated here belongs to the stream that uses it."""
        if stream is not None:
            if stream.device != self.device:
                raise ValueError("the stream must be on the cache's device")
            with torch.cuda.stream(stream):
                call(stream.cuda_stream)
        elif torch.cuda.current_device() == self.device.index:
            call(_raw_stream(self.device.index))
        else:
            with torch.cuda.device(self.device):
                call(_raw_stream(self.device.index))

    def append(self, layer: int, seqs: Sequences, k: torch.Tensor, v: torch.Tensor,
               q: Optional[torch.Tensor] = None, q_out: Optional[torch.Tensor] = None,
               rope: Optional[dict] = None, positions: Optional[torch.Tensor] = None,
               stream: Optional[torch.cuda.Stream] = None) -> Optional[torch.Tensor]:
        """K <- R(p) k and V <- v in the new tokens' slots, q_out <- R(p) q
        (cr_append_kv).  k, v: [n_tokens, n_kv_heads, head_dim]; q, q_out:
        [n_tokens, n_heads, head_dim] (q_out None: a new tensor); rope: as
        Repairer.rotate_keys, or None; positions: device int32, or None for the
        slots.  Returns q_out."""
        n = self._tokens(seqs)
        kr, vr = self._rows(k, n, self.n_kv_heads, "k"), self._rows(v, n, self.n_kv_heads, "v")
        pos = self._index(positions, n, "positions")
        rs, keep = (None, None) if rope is None else B.rope_struct(**rope)
        if keep is not None and len(keep) != self.head_dim // 2:
            raise ValueError("inv_freq needs head_dim / 2 entries")
        heads = 0 if q is None else q.shape[1]
        qr = None if q is None else self._rows(q, n, heads, "q")
        if q is None and q_out is not None:
            raise ValueError("q_out without q")
        result = q_out

        def call(handle):
            nonlocal result
            if q is not None and result is None:
                result = torch.empty(q.shape, dtype=q.dtype, device=q.device)
            qo = None if q is None else self._rows(result, n, heads, "q_out")
            B.cr_append_kv(self.pool.data_ptr(), self.layout, layer, seqs.struct, kr, vr, qr, qo,
                           heads, rs, pos, handle)

        self._on(stream, call)
        return result

    def workspace(self, seqs: Sequences, n_heads: int, shared_len: int = 0) -> torch.Tensor:
        """Device scratch for :meth:`attend` with these arguments."""
        self._tokens(seqs)
        return torch.empty(max(self._workspace_bytes(seqs, n_heads, shared_len), 256),
                           dtype=torch.uint8, device=self.pool.device)

    def _workspace_bytes(self, seqs: Sequences, n_heads: int, shared_len: int) -> int:
        n = seqs.workspace_bytes.get((n_heads, shared_len))
        if n is None:
            n = B.cr_attend_workspace_bytes(self.layout, seqs.struct, n_heads, shared_len)
            seqs.workspace_bytes[n_heads, shared_len] = n
        return n

    def attend(self, layer: int, seqs: Sequences, q: torch.Tensor,
               out: Optional[torch.Tensor] = None, scale: float = 0.0, softcap: float = 0.0,
               slopes: Optional[Sequence[float]] = None, lo: Optional[torch.Tensor] = None,
               hi: Optional[torch.Tensor] = None, shared_len: int = 0,
               lse: Optional[torch.Tensor] = None, workspace: Optional[torch.Tensor] = None,
               stream: Optional[torch.cuda.Stream] = None) -> torch.Tensor:
        """Attention of the new tokens' queries over the pages (cr_attend): out
        [n_tokens, n_heads, head_dim] (None: a new tensor).  The options are
        those of cr_attend_options; slopes is a host sequence, lo, hi (int32)
        and lse (fp32 [n_tokens, n_heads]) are device tensors."""
        n, heads = self._tokens(seqs), q.shape[1]
        qr = self._rows(q, n, heads, "q")
        o = B.cr_attend_options(scale, softcap)
        if slopes is not None:
            sl = np.ascontiguousarray(slopes, dtype=np.float32)
            if sl.shape != (heads,):
                raise ValueError("slopes needs one entry per query head")
            o.slopes = sl.ctypes.data_as(ctypes.POINTER(ctypes.c_float))
        o.lo, o.hi = self._index(lo, n, "lo"), self._index(hi, n, "hi")
        o.shared_len = shared_len
        if lse is not None:
            if lse.dtype is not torch.float32 or lse.shape != (n, heads) or \
                    not lse.is_contiguous() or lse.device != self.device:
                raise TypeError(f"lse must be a contiguous fp32 [{n}, {heads}] tensor on the "
                                "cache's device")
            o.lse = lse.data_ptr()
        need = self._workspace_bytes(seqs, heads, shared_len)
        if workspace is not None and (workspace.device != self.device or
                                      not workspace.is_contiguous()):
            raise ValueError("workspace must be a contiguous tensor on the cache's device")
        result = out

        def call(handle):
            nonlocal result
            if result is None:
                result = torch.empty(q.shape, dtype=q.dtype, device=q.device)
            ws = workspace
            if ws is None and need:
                ws = torch.empty(need, dtype=torch.uint8, device=self.device)
            B.cr_attend(self.pool.data_ptr(), self.layout, layer, seqs.struct, qr,
                        self._rows(result, n, heads, "out"), heads, o,
                        None if ws is None else ws.data_ptr(),
                        0 if ws is None else ws.numel() * ws.element_size(), handle)

        self._on(stream, call)
        return result
