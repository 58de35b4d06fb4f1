"""Operators over a paged cache (via_paged_*), for layers of the caller's own.

``PagedCache`` describes pages of this library's layout (a pool of one's own, or
one of a KV handle's, ``PagedCache.of_handle``) and the page table of the
sequences; ``PagedBatch`` the rows of one step or prompt chunk.  For every layer
a program appends the rows and attends::

    q = batch.append(slot, qkv, n_heads, q_gain=gq, k_gain=gk)
    out = batch.attend(slot, q)

and, where contexts are long, keeps the mean key of every whole block and reads
chosen blocks only::

    batch.block_means(slot, means)
    sel = batch.select_blocks(q, means, n_sel=32)
    out = batch.attend_blocks(slot, q, sel)

The page table, row starts and lengths stay on the device and are read by the
kernels, so a captured HIP graph follows them from replay to replay.  Calls run on
the current stream of the cache's device.  Rows behind the last sequence keep
what the output held (an output the call allocates holds nothing there).  They are for
inference: none has a gradient.
"""
from __future__ import annotations

import ctypes as C

import torch
import torch.autograd.forward_ad as forward_ad

from . import via

_DTYPES = {torch.float32: via.DTYPE_F32, torch.bfloat16: via.DTYPE_BF16}


def _expect(cond, what):
    if not cond:
        raise ValueError(what)


def _int32(*values):
    for v in values:
        if not -(1 << 31) <= v < 1 << 31:
            raise ValueError(f"{v} is out of range")


def _no_gradient(t, what):
    """Refuses a tensor that a derivative is asked of, backward or forward: the result would have none."""
    if t.requires_grad and torch.is_grad_enabled():
        raise ValueError(f"{what} requires a gradient; the operators have none (call them under torch.no_grad)")
    # (asking a tensor for its tangent costs 1 us: only within a level of forward derivatives)
    if forward_ad._current_level >= 0 and t.is_floating_point() and forward_ad.unpack_dual(t).tangent is not None:
        raise ValueError(f"{what} has a forward-mode tangent; the operators have none")


class PagedCache:
    """``pool``: contiguous device tensor [n_slots, n_kv_heads, n_blocks, 2, 16 * head_dim]
    (or that many elements flat, with ``n_slots``), fp32 or bf16.  ``table``: int32 [n_seqs,
    pages] on the same device, rows contiguous; entries outside the pool name no page."""

    def __init__(self, pool, n_kv_heads, head_dim, table, n_slots=None):
        _expect(pool.is_cuda and pool.is_contiguous() and not pool.requires_grad,
                "the pool must be a contiguous device tensor without a gradient")
        _no_gradient(pool, "the pool")
        _expect(pool.dtype in _DTYPES, f"a pool of {pool.dtype} (float32 or bfloat16)")
        _expect(n_kv_heads >= 1 and head_dim >= 1, "n_kv_heads and head_dim must be positive")
        n_slots = n_slots if n_slots is not None else (pool.shape[0] if pool.dim() == 5 else 1)
        per_block = n_slots * n_kv_heads * 2 * via.BLOCK * head_dim
        _expect(n_slots >= 1 and pool.numel() % per_block == 0, "the pool holds no whole blocks of these sizes")
        self.pool, self.n_kv_heads, self.head_dim, self.n_slots = pool, n_kv_heads, head_dim, n_slots
        self.n_blocks = pool.numel() // per_block
        if pool.dim() == 5:
            _expect(tuple(pool.shape) == (n_slots, n_kv_heads, self.n_blocks, 2, via.BLOCK * head_dim),
                    f"a pool of shape {tuple(pool.shape)}")
        self.device, self.dtype = pool.device, pool.dtype
        self.set_table(table)

    def set_table(self, table):
        """Another page table (batches made from now on read it)."""
        _expect(table.dim() == 2 and table.dtype == torch.int32 and table.device == self.device,
                "the table must be an int32 matrix on the pool's device")
        _expect(table.stride(1) == 1 and table.stride(0) >= table.shape[1], "the table's rows must be contiguous")
        self.table = table

    @classmethod
    def of_handle(cls, kv: via.KV, cache, seq_ids, pages=None):
        """The full or slim cache of a KV handle, with the block tables its sequences have now
        (``pages`` columns at least)."""
        m = kv.model.desc
        tables = [kv.seq_info(s, cache)[1] for s in seq_ids]
        width = max([1, pages or 1] + [len(t) for t in tables])
        host = torch.full((len(tables), width), -1, dtype=torch.int32)
        for i, t in enumerate(tables):
            host[i, :len(t)] = torch.tensor(t, dtype=torch.int32)
        pool = kv.pool_view(cache)
        return cls(pool, m["n_kv_heads"], m["head_dim"], host.to(pool.device))


class PagedBatch:
    """Rows of a batch: sequence s has rows row_start[s] .. row_start[s + 1] - 1 (device int32
    [n_seqs + 1]) and kv_len[s] cached positions, those rows included (device int32 [n_seqs]).
    ``rows`` and ``max_kv`` bound the rows and the lengths."""

    def __init__(self, cache: PagedCache, row_start, kv_len, rows, max_kv):
        n = cache.table.shape[0]
        for t, shape in ((row_start, (n + 1,)), (kv_len, (n,))):
            _expect(t.dtype == torch.int32 and t.device == cache.device and tuple(t.shape) == shape
                    and t.is_contiguous(), f"row_start and kv_len must be int32 [{n + 1}] and [{n}] on the pool's device")
        self.cache, self.row_start, self.kv_len, self.table = cache, row_start, kv_len, cache.table
        # (a table that is part of a wider one: no more than its own columns)
        _int32(rows, cache.n_blocks, cache.n_slots, self.table.stride(0))
        self.rows, self.max_kv, self.n_seqs = int(rows), min(int(max_kv), self.table.shape[1] * via.BLOCK), n
        _int32(self.max_kv)
        self.c = via.Paged(cache.pool.data_ptr(), _DTYPES[cache.dtype], cache.n_slots, cache.n_blocks, cache.n_kv_heads,
                           cache.head_dim, self.table.data_ptr(), max(1, self.table.stride(0)), n, row_start.data_ptr(),
                           kv_len.data_ptr(), self.rows, self.max_kv)
        self._c = C.byref(self.c)
        self._sizes = {}  # workspace sizes by the arguments they depend on

    # ---- arguments
    def _call(self, f, *args):
        _no_gradient(self.cache.pool, "the pool")
        dev = self.cache.device.index
        stream = torch._C._cuda_getCurrentRawStream(dev)  # (torch.cuda.current_stream builds an object: 2 us)
        if torch.cuda.current_device() == dev:
            st = f(self._c, *args, stream)
        else:
            with torch.cuda.device(dev):
                st = f(self._c, *args, stream)
        if st != via.OK:
            via.check(st)

    def _rows_of(self, t, heads, what):
        """Address and row length of a [rows, heads, head_dim] (or [rows, heads * head_dim]) tensor."""
        hd, shape, stride = self.cache.head_dim, t.shape, t.stride()
        if t.dtype != self.cache.dtype or t.device != self.cache.device:
            raise ValueError(f"{what} must be {self.cache.dtype} on {self.cache.device}, as the pool is")
        _no_gradient(t, what)
        if len(shape) == 3:
            ok = shape[1] == heads and shape[2] == hd and stride[2] == 1 and (heads == 1 or stride[1] == hd)
        else:
            ok = len(shape) == 2 and shape[1] == heads * hd and stride[1] == 1
        if not ok or shape[0] != self.rows:
            raise ValueError(f"{what} of shape {tuple(shape)}: {self.rows} rows of {heads} heads of {hd}, a row contiguous")
        ld = stride[0] if self.rows > 1 else heads * hd
        if ld >= 1 << 31:
            raise ValueError(f"{what}: rows {ld} elements apart (less than 2^31)")
        return t.data_ptr(), ld

    def _heads_of(self, q):
        hd = self.cache.head_dim
        if q.dim() not in (2, 3) or q.shape[-1] % hd:
            raise ValueError(f"q of shape {tuple(q.shape)}")
        return q.shape[1] if q.dim() == 3 else q.shape[1] // hd

    def _vector(self, t, dtype, shape, what):
        if t is None:
            return None
        if t.dtype != dtype or t.device != self.cache.device or t.shape != shape or not t.is_contiguous():
            raise ValueError(f"{what} must be contiguous {dtype} {list(shape)} on {self.cache.device}")
        _no_gradient(t, what)
        return t.data_ptr()

    def _apart(self, src, ld, heads, dst, out_ld, out_heads):
        """Refuses an output that lies over its input but in its own place (the same start and rows)."""
        n, size, hd = self.rows, self.cache.pool.element_size(), self.cache.head_dim
        if n == 0 or (dst == src and (out_ld == ld or n == 1)):
            return
        w, out_w = heads * hd, out_heads * hd
        if dst >= src + ((n - 1) * ld + w) * size or src >= dst + ((n - 1) * out_ld + out_w) * size:
            return
        at = (dst - src) // size % ld  # side by side in the same rows
        _expect(out_ld == ld and at >= w and at + out_w <= ld, "out overlaps the input")

    def _workspace(self, f, *args):
        """A workspace (None if none is needed) and its size.  It is the call's own: two calls in flight
        (streams, captured graphs) never share one."""
        key = (f.__name__, args)
        n = self._sizes.get(key)
        if n is None:
            n = self._sizes[key] = f(self._c, *args)
        return (torch.empty(n, dtype=torch.uint8, device=self.cache.device) if n else None), n

    # ---- operators
    def append(self, slot, qkv, n_heads, pos=None, q_gain=None, k_gain=None, eps=1e-5, theta=10000.0, out=None):
        """Cache the rows' keys and values, heads normalised (with gains) and rotated; returns the
        queries [rows, n_heads, head_dim].  ``qkv`` [rows, (n_heads + 2 n_kv_heads) * head_dim];
        ``pos`` int32 [rows]: rotary positions other than the cache's; ``out``: where the queries
        go, qkv[:, :n_heads * head_dim] among others."""
        _int32(slot, n_heads)
        hd = self.cache.head_dim
        src, ld = self._rows_of(qkv, n_heads + 2 * self.cache.n_kv_heads, "qkv")
        if out is None:
            out = torch.empty((self.rows, n_heads, hd), dtype=qkv.dtype, device=qkv.device)
            dst, out_ld = out.data_ptr(), n_heads * hd
        else:
            dst, out_ld = self._rows_of(out, n_heads, "out")
            self._apart(src, ld, n_heads + 2 * self.cache.n_kv_heads, dst, out_ld, n_heads)
            if dst == src and self.rows == 1:
                out_ld = ld
        self._call(via.via_paged_append, slot, src, ld, n_heads, self._vector(pos, torch.int32, (self.rows,), "pos"),
                   self._vector(q_gain, self.cache.dtype, (hd,), "q_gain"),
                   self._vector(k_gain, self.cache.dtype, (hd,), "k_gain"), eps, theta, dst, out_ld)
        return out

    def _attend(self, f, q, heads, out, return_lse, head_args, tail_args, workspace):
        src, ld = self._rows_of(q, heads, "q")
        if out is None:
            out = torch.empty(q.shape, dtype=q.dtype, device=q.device)
            dst, out_ld = out.data_ptr(), heads * self.cache.head_dim
        else:
            dst, out_ld = self._rows_of(out, heads, "out")
            self._apart(src, ld, heads, dst, out_ld, heads)
        lse = torch.empty((self.rows, heads), dtype=torch.float32, device=q.device) if return_lse else None
        ws, nbytes = self._workspace(*workspace)
        self._call(f, head_args[0], src, ld, heads, *head_args[1:], *tail_args, dst, out_ld,
                   lse.data_ptr() if return_lse else None, ws.data_ptr() if nbytes else None, nbytes)
        return (out, lse) if return_lse else out

    def attend(self, slot, q, scale=None, window=0, row_mask=None, out=None, return_lse=False):
        """Attention of the rows over their cached sequences: causal, the last ``window`` positions
        (0: all), or with ``row_mask`` (int64 [rows], bit o: the batch's own position o) a token
        tree.  ``scale`` defaults to head_dim ** -0.5."""
        _int32(slot, window)
        heads = self._heads_of(q)
        mask = self._vector(row_mask, torch.int64, (self.rows,), "row_mask")
        scale = self.cache.head_dim ** -0.5 if scale is None else scale
        return self._attend(via.via_paged_attend, q, heads, out, return_lse, (slot, scale), (window, mask),
                            (via.via_paged_attend_bytes, heads, window))

    def block_means(self, slot, means, block=64):
        """Mean keys of the blocks the rows complete, into ``means`` (fp32 [n_seqs, n_kv_heads,
        blocks, head_dim]); returns it."""
        _int32(slot, block)
        n = means.shape[2] if means.dim() == 4 else 0
        addr = self._vector(means, torch.float32, (self.n_seqs, self.cache.n_kv_heads, n, self.cache.head_dim), "means")
        self._call(via.via_paged_block_means, slot, block, addr, n)
        return means

    def select_blocks(self, q, means, n_sel, block=64, n_first=1, n_last=2, out=None):
        """The blocks each row reads: int32 [rows, n_kv_heads, n_sel], ascending, then -1."""
        _int32(n_sel, block, n_first, n_last)
        heads, kvh = self._heads_of(q), self.cache.n_kv_heads
        src, ld = self._rows_of(q, heads, "q")
        n = means.shape[2] if means.dim() == 4 else 0
        addr = self._vector(means, torch.float32, (self.n_seqs, kvh, n, self.cache.head_dim), "means")
        if out is None:
            out = torch.empty((self.rows, kvh, n_sel), dtype=torch.int32, device=q.device)
        dst = self._vector(out, torch.int32, (self.rows, kvh, n_sel), "out")
        ws, nbytes = self._workspace(via.via_paged_select_bytes, block)
        self._call(via.via_paged_select, src, ld, heads, addr, n, block, n_first, n_last, n_sel, dst,
                   ws.data_ptr() if nbytes else None, nbytes)
        return out

    def attend_blocks(self, slot, q, sel, block=64, scale=None, out=None, return_lse=False):
        """``attend`` over the blocks listed in ``sel`` (int32 [rows, n_kv_heads, n_sel])."""
        _int32(slot, block)
        heads = self._heads_of(q)
        n_sel = sel.shape[2] if sel.dim() == 3 else 0
        lists = self._vector(sel, torch.int32, (self.rows, self.cache.n_kv_heads, n_sel), "sel")
        scale = self.cache.head_dim ** -0.5 if scale is None else scale
        return self._attend(via.via_paged_attend_blocks, q, heads, out, return_lse, (slot, scale), (block, lists, n_sel),
                            (via.via_paged_attend_blocks_bytes, heads, block, n_sel))
