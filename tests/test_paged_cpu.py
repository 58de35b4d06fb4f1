"""Refusals and sizes of the paged-cache operators (include/via.h): a call with
bad arguments returns its status before it touches a device, so no GPU is
needed.  And the binding's own checks that need none."""
import ctypes as C
import math

import pytest

from paper_2606_12243_amd import via

A = 1 << 20  # an address that is aligned and never read


def desc(**kw):
    d = dict(pool=A, dtype=via.DTYPE_BF16, n_slots=2, n_blocks=10, n_kv_heads=2, head_dim=64, table=A, table_ld=4, n_seqs=2,
             row_start=A, kv_len=A, rows=3, max_kv=60)
    d.update(kw)
    return via.Paged(*[d[n] for n, _ in via.Paged._fields_])


def call(op, d, **kw):
    c = C.byref(d) if d is not None else None
    a = dict(slot=1, qkv=A, qkv_ld=512, q=A, q_ld=256, H=4, scale=0.1, window=0, mask=None, out=A, out_ld=256, lse=None, ws=A,
             ws_bytes=1 << 40, pos=None, eps=1e-5, theta=1e4, block=64, means=A, nb=2, first=1, last=2, n_sel=4, sel=A)
    a.update(kw)
    g = lambda *names: [a[n] for n in names]
    if op == "append":
        return via.via_paged_append(c, *g("slot", "qkv", "qkv_ld", "H", "pos"), None, None, *g("eps", "theta", "out", "out_ld"), None)
    if op == "attend":
        return via.via_paged_attend(c, *g("slot", "q", "q_ld", "H", "scale", "window", "mask", "out", "out_ld", "lse", "ws", "ws_bytes"), None)
    if op == "means":
        return via.via_paged_block_means(c, *g("slot", "block", "means", "nb"), None)
    if op == "select":
        return via.via_paged_select(c, *g("q", "q_ld", "H", "means", "nb", "block", "first", "last", "n_sel", "sel", "ws", "ws_bytes"), None)
    return via.via_paged_attend_blocks(c, *g("slot", "q", "q_ld", "H", "scale", "block", "sel", "n_sel", "out", "out_ld", "lse", "ws", "ws_bytes"), None)


OPS = ["append", "attend", "means", "select", "blocks"]


@pytest.mark.parametrize("op", OPS)
@pytest.mark.parametrize("bad,status", [
    (None, via.EINVAL), (dict(dtype=5), via.EINVAL), (dict(n_slots=0), via.EINVAL), (dict(n_blocks=0), via.EINVAL),
    (dict(n_kv_heads=0), via.EINVAL), (dict(table_ld=0), via.EINVAL), (dict(n_seqs=-1), via.EINVAL), (dict(rows=-1), via.EINVAL),
    (dict(max_kv=-1), via.EINVAL), (dict(head_dim=96), via.EUNSUPPORTED), (dict(n_seqs=65536), via.EUNSUPPORTED),
    (dict(pool=None), via.EINVAL), (dict(table=None), via.EINVAL), (dict(row_start=None), via.EINVAL),
    (dict(kv_len=None), via.EINVAL), (dict(pool=A + 8), via.EINVAL)])
def test_bad_batches(op, bad, status):
    assert call(op, None if bad is None else desc(**bad)) == status
    assert via.via_last_error()


@pytest.mark.parametrize("op,bad,status", [
    (op, bad, st) for ops, bad, st in [
        (["append", "attend", "means", "blocks"], dict(slot=2), via.EINVAL),
        (["append", "attend", "means", "blocks"], dict(slot=-1), via.EINVAL),
        (["append", "attend", "select", "blocks"], dict(H=3), via.EINVAL),
        (["append", "attend", "select", "blocks"], dict(H=0), via.EINVAL),
        (["append"], dict(qkv=None), via.EINVAL), (["append"], dict(qkv=A + 4), via.EINVAL),
        (["append"], dict(qkv_ld=511), via.EINVAL), (["append"], dict(qkv_ld=516), via.EINVAL),
        (["append"], dict(qkv_ld=256), via.EINVAL), (["append"], dict(theta=0.0), via.EINVAL),
        (["append"], dict(theta=math.inf), via.EINVAL), (["append"], dict(eps=-1.0), via.EINVAL),
        (["append"], dict(eps=math.nan), via.EINVAL), (["append"], dict(out=A, out_ld=256, qkv=A), via.EINVAL),
        (["attend", "select", "blocks"], dict(q=None), via.EINVAL), (["attend", "select", "blocks"], dict(q=A + 2), via.EINVAL),
        (["attend", "select", "blocks"], dict(q_ld=248), via.EINVAL), (["attend", "select", "blocks"], dict(q_ld=257), via.EINVAL),
        (["append", "attend", "blocks"], dict(out=None), via.EINVAL), (["append", "attend", "blocks"], dict(out=A + 8), via.EINVAL),
        (["append", "attend", "blocks"], dict(out_ld=128), via.EINVAL),
        (["attend", "blocks"], dict(out=A, q=A, out_ld=264), via.EINVAL),
        (["attend", "blocks"], dict(scale=0.0), via.EINVAL), (["attend", "blocks"], dict(scale=-1.0), via.EINVAL),
        (["attend", "blocks"], dict(scale=math.nan), via.EINVAL), (["attend", "blocks"], dict(scale=math.inf), via.EINVAL),
        (["attend", "blocks"], dict(scale=1e-42), via.EINVAL),
        (["attend"], dict(window=-1), via.EINVAL), (["attend"], dict(window=4, mask=A), via.EINVAL),
        (["means", "select", "blocks"], dict(block=16), via.EUNSUPPORTED), (["means", "select", "blocks"], dict(block=0), via.EUNSUPPORTED),
        (["means", "select"], dict(means=None), via.EINVAL), (["means", "select"], dict(means=A + 4), via.EINVAL),
        (["means", "select"], dict(nb=0), via.EINVAL),
        (["select"], dict(block=32, nb=1), via.EINVAL), (["select"], dict(first=-1), via.EINVAL), (["select"], dict(last=0), via.EINVAL),
        (["select"], dict(n_sel=2), via.EINVAL), (["select"], dict(first=2 ** 31 - 1, last=2 ** 31 - 1), via.EINVAL),
        (["select", "blocks"], dict(sel=None), via.EINVAL), (["blocks"], dict(n_sel=0), via.EINVAL),
        (["blocks"], dict(n_sel=2 ** 30, block=128), via.EINVAL),
        (["select"], dict(ws=None, ws_bytes=0), via.ENOMEM), (["select"], dict(ws_bytes=8), via.ENOMEM),
        (["select"], dict(ws=A + 8), via.EINVAL)] for op in ops])
def test_bad_arguments(op, bad, status):
    assert call(op, desc(), **bad) == status
    assert via.via_last_error()


@pytest.mark.parametrize("op", OPS)
def test_nothing_to_do(op):
    for kw in (dict(rows=0), dict(n_seqs=0)):
        d = desc(pool=None, table=None, row_start=None, kv_len=None, **kw)
        assert call(op, d, qkv=None, q=None, out=None, means=None, sel=None, ws=None, ws_bytes=0) == via.OK


def test_long_keys_need_a_workspace():
    """One row over a long context is split; its workspace is asked for, and refused if it is short or misaligned."""
    d = desc(table_ld=4096, max_kv=60000, rows=1, n_seqs=1)
    n = via.via_paged_attend_bytes(C.byref(d), 4, 0)
    assert n > 0 and n % (4 * (64 + 2) * 4) == 0  # a partial output, maximum and sum per split, row and head
    assert call("attend", d, ws_bytes=n - 1) == via.ENOMEM
    assert call("attend", d, ws=None, ws_bytes=0) == via.ENOMEM
    assert call("attend", d, ws=A + 16, ws_bytes=n) == via.EINVAL
    m = via.via_paged_attend_blocks_bytes(C.byref(d), 4, 64, 32)
    assert m > 0 and call("blocks", d, n_sel=32, ws_bytes=m - 1) == via.ENOMEM
    assert via.via_paged_attend_bytes(C.byref(d), 4, 100) <= n  # a window reads less
    for bad in (via.via_paged_attend_bytes(C.byref(d), 3, 0), via.via_paged_attend_bytes(C.byref(d), 4, -1),
                via.via_paged_attend_bytes(None, 4, 0), via.via_paged_attend_blocks_bytes(C.byref(d), 4, 60, 32),
                via.via_paged_select_bytes(C.byref(d), 16)):
        assert bad == 0
    assert via.via_paged_select_bytes(C.byref(d), 64) == 2 * -(-60000 // 64) * 8


def test_a_launch_has_an_end():
    d = desc(rows=2 ** 31 - 1, n_seqs=1, table_ld=4, max_kv=60)
    assert call("attend", d) == via.EUNSUPPORTED
    assert call("blocks", d) == via.EUNSUPPORTED
    for op in ("attend", "select", "blocks"):
        assert call(op, desc(rows=1 << 24, n_seqs=1)) == via.EUNSUPPORTED, op


def test_binding_refuses_what_it_cannot_pass():
    torch = pytest.importorskip("torch")
    from paper_2606_12243_amd import paged
    table = torch.zeros((1, 4), dtype=torch.int32)
    with pytest.raises(ValueError):  # not on a device
        paged.PagedCache(torch.zeros((1, 2, 4, 2, 1024)), 2, 64, table)
    with pytest.raises(ValueError):
        paged.PagedCache(torch.zeros((1, 2, 4, 2, 1024), dtype=torch.float64), 2, 64, table)


@pytest.mark.parametrize("rows,n_seqs,max_kv", [(8192, 2, 131072), (32768, 8, 131072), (8188, 4, 1 << 20), (65535, 65535, 400000),
                                                (4000, 4, 32768), (1 << 17, 3, 1 << 29)])
def test_many_rows_of_several_sequences_need_no_large_workspace(rows, n_seqs, max_kv):
    """max_kv is a bound: partial results of every row for each 8192 keys of it would take gigabytes."""
    d = desc(rows=rows, n_seqs=n_seqs, max_kv=max_kv, table_ld=max_kv // 16 + 1, n_kv_heads=8, head_dim=128)
    for window in (0, 100000):
        assert via.via_paged_attend_bytes(C.byref(d), 32, window) <= 256 << 20
    few = desc(rows=8, n_seqs=2, max_kv=max_kv, table_ld=max_kv // 16 + 1, n_kv_heads=8, head_dim=128)
    assert via.via_paged_attend_bytes(C.byref(few), 32, 0) > 0  # few rows are still split


def test_splits_do_not_outgrow_a_launch():
    """As many sequences as there may be, over contexts of 2^20: the call wants its workspace, it is not refused."""
    d = desc(rows=65535, n_seqs=65535, max_kv=1 << 20, table_ld=1 << 16, n_kv_heads=4, head_dim=64)
    assert 0 < via.via_paged_attend_bytes(C.byref(d), 4, 0) <= 256 << 20
    assert call("attend", d, ws=None, ws_bytes=0) == via.ENOMEM
    # sizes that the call refuses: the product of rows, heads and bytes passes 64 bits
    for rows, heads in ((1 << 27, 2 ** 31 - 4), (1 << 27, 1 << 30), (1 << 25, 1 << 30)):
        d = desc(rows=rows, n_seqs=2, max_kv=1 << 20, table_ld=1 << 16, n_kv_heads=4, head_dim=128)
        via.via_paged_attend_bytes(C.byref(d), heads, 0)
        assert call("attend", d, H=heads, q_ld=2 ** 31 - 8, out_ld=2 ** 31 - 8) == via.EINVAL  # (no row holds them)


def test_no_derivative_is_dropped():
    """Tensors that a backward or forward derivative is asked of are refused."""
    torch = pytest.importorskip("torch")
    import torch.autograd.forward_ad as forward_ad
    from paper_2606_12243_amd import paged
    x = torch.zeros(4)
    paged._no_gradient(x, "x")
    with pytest.raises(ValueError, match="x requires a gradient"):
        paged._no_gradient(torch.zeros(4, requires_grad=True), "x")
    with forward_ad.dual_level():
        paged._no_gradient(x, "x")
        paged._no_gradient(torch.zeros(4, dtype=torch.int32), "x")
        dual = forward_ad.make_dual(x, torch.ones(4))
        for t in (dual, dual[:2], dual.view(2, 2)):
            with torch.no_grad(), pytest.raises(ValueError, match="x has a forward-mode tangent"):
                paged._no_gradient(t, "x")


def test_sequences_times_heads_have_an_end():
    for op in ("attend", "blocks"):
        d = desc(rows=1 << 17, n_seqs=65535, n_kv_heads=256, head_dim=64)
        assert call(op, d, H=256, q_ld=1 << 14, out_ld=1 << 14) == via.EUNSUPPORTED, op
    d = desc(rows=65535, n_seqs=65535, n_kv_heads=257, head_dim=64)
    assert call("attend", d, H=257, q_ld=1 << 15, out_ld=1 << 15) == via.EUNSUPPORTED
    d = desc(rows=1, n_seqs=65535, n_kv_heads=257, head_dim=64)  # one row, as many sequences
    assert call("attend", d, H=257, q_ld=1 << 15, out_ld=1 << 15) == via.EUNSUPPORTED
