"""The paged-cache operators, as cases that can be timed and checked.

A program that runs layers of its own over this library's page layout does, for
every layer: append the batch's keys and values (heads normalised and rotated on
the way), attend to the pages, and -- where contexts are long -- keep the mean
key of every completed block, let each query choose blocks by it, and attend to
those alone.  Sizes are those of the workload configurations and the benchmark;
``draw`` spreads them over the ranges between.

A page holds 16 tokens of one K/V head: keys as [head_dim/8][16][8], values
transposed as [head_dim][16]; pool[slot][kv_head][block][K|V][page].
"""
from __future__ import annotations

import math
import random

import torch

own = False

_PAGE = 16
_EPS = 1e-6
# heads, K/V heads, head size, type
_HEADS = {
    "tiny_fp32": (4, 4, 64, "f32"),
    "micro_f32": (2, 1, 64, "f32"),
    "micro_bf16": (4, 2, 64, "bf16"),
    "small_bf16_hd128": (8, 2, 128, "bf16"),
    "1b_bf16": (16, 4, 128, "bf16"),
    "8b_bf16": (32, 8, 128, "bf16"),
}


def _case(name, kind, model, batch, rows, ctx, **kw):
    """batch sequences; (least, most) new rows and (least, most) cached positions before them."""
    c = dict(kind=kind, model=model, batch=batch, rows_lo=rows[0], rows_hi=rows[1], ctx_lo=ctx[0], ctx_hi=ctx[1], **kw)
    return dict(name=name, **c) if name else c


def listed():
    return [
        # a verification window of the headline workload entering the cache, heads normalised
        _case("append_window", "append", "8b_bf16", 4, (8, 8), (2048, 2048), norm=True, theta=10000.0),
        # four prompts entering it, far rotations
        _case("append_prompts", "append", "8b_bf16", 4, (2047, 2047), (0, 0), norm=True, theta=1000000.0),
        # the smallest model's short window: launches and latency
        _case("attend_tiny_fp32", "attend", "tiny_fp32", 1, (4, 4), (32, 32), window=0, tree=False),
        # one token each of a long-context batch
        _case("attend_tokens", "attend", "8b_bf16", 16, (1, 1), (4096, 8192), window=0, tree=False),
        # four prompts
        _case("attend_prompts", "attend", "8b_bf16", 4, (2047, 2047), (0, 0), window=0, tree=False),
        # a chunk of a long document after what is cached of it
        _case("attend_chunk", "attend", "8b_bf16", 1, (1000, 1000), (15000, 15000), window=0, tree=False),
        # the blocks a window of the long-context batch completes ...
        _case("means_window", "means", "8b_bf16", 16, (6, 6), (4096, 8191), block=32),
        # ... and those of its prompts
        _case("means_prompts", "means", "8b_bf16", 16, (4096, 8192), (0, 0), block=64),
        # blocks chosen for the windows of a batch of long documents
        _case("select_windows", "select", "8b_bf16", 16, (6, 6), (16384, 32768), block=64, n_sel=32),
        # blocks chosen for a chunk of a prompt
        _case("select_chunk", "select", "8b_bf16", 1, (1000, 1000), (31000, 31000), block=64, n_sel=32),
        # attention of one token of a long document to its blocks
        _case("blocks_token", "blocks", "8b_bf16", 1, (1, 1), (32000, 32000), block=64, n_sel=32),
        # ... and of the batch's windows
        _case("blocks_windows", "blocks", "8b_bf16", 16, (6, 6), (16384, 32768), block=64, n_sel=32),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["append", "attend", "attend", "attend", "means", "select", "blocks", "blocks"])
    model = rng.choice(["8b_bf16", "8b_bf16", "8b_bf16", "1b_bf16", "1b_bf16", "small_bf16_hd128", "micro_bf16",
                        "tiny_fp32", "micro_f32"])
    small = model in ("tiny_fp32", "micro_f32")
    batch = _log_int(rng, 1, 16)
    prompts = rng.random() < 0.4
    if kind == "append":
        hi = _log_int(rng, 1, 8000 // batch) if prompts else rng.randint(1, 16)
        ctx = _log_int(rng, 1, 8192) - 1
        return _case(None, kind, model, batch, (rng.choice([hi, max(1, hi // 3)]), hi), (ctx // 2, ctx),
                     norm=rng.random() < 0.7, theta=rng.choice([10000.0, 500000.0, 1000000.0]))
    if kind == "attend":
        top = 2048 if small else 16384
        if prompts:
            hi = _log_int(rng, 17, min(2047, 4000 // batch) if not small else 500)
            ctx = _log_int(rng, 1, max(2, min(top, 12000000 // (hi * batch)))) - 1
        else:
            hi = rng.randint(1, 12)
            ctx = _log_int(rng, 1, min(top, 8192)) - 1
        tree = not prompts and rng.random() < 0.3
        window = rng.choice([0, 0, _log_int(rng, 1, 4096)]) if not tree else 0
        return _case(None, kind, model, batch, (rng.choice([hi, max(1, hi // 2)]), hi), (ctx // 2, ctx), window=window,
                     tree=tree)
    block = rng.choice([32, 64, 128])
    if kind == "means":
        hi = _log_int(rng, 17, 8192) if prompts else rng.randint(1, 64)
        ctx = rng.choice([0, _log_int(rng, 1, 8192)])
        return _case(None, kind, model, batch, (max(1, hi // 2), hi), (ctx // 2, ctx), block=block)
    n_sel = rng.choice([4, 8, 16, 32, 48])
    hi = _log_int(rng, 17, 800 // batch) if prompts else rng.randint(1, 8)
    if kind == "select":  # enough blocks that there is a choice
        ctx = _log_int(rng, 3 * n_sel * block, 32768)
    else:
        ctx = _log_int(rng, 1, 8192 if small or prompts else 32768) - 1
    return _case(None, kind, model, batch, (max(1, hi // 2), hi), (ctx // 2, ctx), block=block, n_sel=n_sel)


# ------------------------------------------------------------------ inputs
class _State:
    pass


def _sizes(case):
    """Ragged new rows and lengths before them (the case's own, not the seed's: they give the outputs' shapes)."""
    r = random.Random("%s %s %s" % (case["batch"], case["rows_hi"], case["ctx_hi"]))
    rows = [r.randint(case["rows_lo"], case["rows_hi"]) for _ in range(case["batch"])]
    ctx = [r.randint(case["ctx_lo"], case["ctx_hi"]) for _ in range(case["batch"])]
    return rows, [a + b for a, b in zip(rows, ctx)]


def _blocks(n, size):
    return (n + size - 1) // size


def _tree_masks(rows, rng):
    """Visible window rows of every row of a random token tree: itself, its ancestors and the root (bits)."""
    masks = []
    for n in rows:
        seen = []
        for i in range(n):
            seen.append((seen[rng.randint(max(0, i - 8), i - 1)] if i else 0) | (1 << i))
        masks += seen
    return [m - (1 << 64) if m >> 63 else m for m in masks]


def _inputs(case, seed):
    st = _State()
    st.case = case
    H, KVH, hd, dt = _HEADS[case["model"]]
    st.H, st.KVH, st.hd = H, KVH, hd
    st.dtype = torch.float32 if dt == "f32" else torch.bfloat16
    st.rows, st.len = _sizes(case)
    T = sum(st.rows)
    kind = case["kind"]
    g = torch.Generator(device="cuda").manual_seed(seed)
    rng = random.Random(seed)

    def normal(*shape, dtype=st.dtype):
        return torch.empty(shape, dtype=dtype, device="cuda").normal_(0.0, 1.0, generator=g)

    st.start = [0]
    for n in st.rows:
        st.start.append(st.start[-1] + n)
    i32 = dict(dtype=torch.int32, device="cuda")
    st.row_start = torch.tensor(st.start, **i32)
    st.kv_len = torch.tensor(st.len, **i32)
    # pages in the order that long serving leaves them in; two layers, the second is used (the choice of
    # blocks reads none)
    need = [_blocks(n, _PAGE) for n in st.len]
    n_pages = sum(need) + 3
    order = torch.randperm(n_pages, generator=g, device="cuda").to(torch.int32)
    st.table = torch.full((case["batch"], max(need) + 1), -1, **i32)
    at = 0
    for b, n in enumerate(need):
        st.table[b, :n] = order[at:at + n]
        at += n
    st.slot = 1
    shape = (2, KVH, n_pages, 2, _PAGE * hd)
    st.pool = torch.empty(shape, dtype=st.dtype, device="cuda") if kind == "select" else normal(*shape)
    if kind == "append":
        # a fused projection's rows: queries, keys, values
        st.qkv = normal(T, (H + 2 * KVH) * hd).mul_(1.3)
        st.q_gain = st.k_gain = None
        if case["norm"]:
            st.q_gain, st.k_gain = (1.0 + 0.1 * normal(hd)).to(st.dtype), (1.0 + 0.1 * normal(hd)).to(st.dtype)
        return st
    if kind != "means":
        st.q = normal(T, H, hd)
    if kind == "attend":
        st.mask = None
        if case["tree"]:
            st.mask = torch.tensor(_tree_masks(st.rows, rng), dtype=torch.int64, device="cuda")
    if kind in ("means", "select"):
        # mean keys of every block a sequence can have; those of blocks that are not complete hold what was there
        st.n_means = max(_blocks(n, case["block"]) for n in st.len)
        st.means = normal(case["batch"], KVH, st.n_means, hd, dtype=torch.float32).mul_(case["block"] ** -0.5)
    if kind == "blocks":
        # the first block, the last two and distinct others, ascending; -1 where there are fewer
        n_sel, size = case["n_sel"], case["block"]
        own_block = torch.cat([torch.arange(n - r, n, device="cuda") for r, n in zip(st.rows, st.len)]) // size
        nb = max(_blocks(n, size) for n in st.len)
        key = torch.rand((T, KVH, nb), generator=g, device="cuda")
        b = torch.arange(nb, device="cuda")
        key += 2.0 * ((b < 1) | (b > own_block[:, None, None] - 2)).float()
        key -= 8.0 * (b > own_block[:, None, None]).float()
        top = key.topk(min(n_sel, nb), -1)
        sel = torch.where(top.values < -1.0, nb, top.indices).sort(-1).values
        st.sel = torch.full((T, KVH, n_sel), -1, **i32)
        st.sel[..., :sel.shape[-1]] = torch.where(sel == nb, -1, sel).to(torch.int32)
    return st


def prepare(case, seed):
    st = _inputs(case, seed)
    if own:
        from paper_2606_12243_amd import paged
        # what a program keeps for a batch: the pool's geometry, the tables and lengths on the device
        cache = paged.PagedCache(st.pool, st.KVH, st.hd, st.table)
        st.batch = paged.PagedBatch(cache, st.row_start, st.kv_len, rows=sum(st.rows), max_kv=max(st.len))
    return st


# ------------------------------------------------------------- plain forms
def _read(pool, table, n, hd):
    """Keys and values [KVH, n, hd] of a sequence, in 32 bits."""
    pages = table[:_blocks(n, _PAGE)].long()
    kvh = pool.shape[0]
    k = pool[:, pages, 0].view(kvh, -1, hd // 8, _PAGE, 8).permute(0, 1, 3, 2, 4).reshape(kvh, -1, hd)
    v = pool[:, pages, 1].view(kvh, -1, hd, _PAGE).permute(0, 1, 3, 2).reshape(kvh, -1, hd)
    return k[:, :n].float(), v[:, :n].float()


def _softmax_v(s, v):
    """Softmax over the last axis (rows may see nothing) times v, and the log of the sum."""
    m = s.amax(-1, keepdim=True)
    p = torch.exp(s - torch.where(torch.isinf(m), torch.zeros_like(m), m))
    l = p.sum(-1, keepdim=True)
    o = torch.matmul(p, v) / torch.where(l == 0, torch.ones_like(l), l)
    return o, (m + torch.log(l)).squeeze(-1)


def _plain_append(st):
    case, H, KVH, hd = st.case, st.H, st.KVH, st.hd
    T = st.qkv.shape[0]
    x = st.qkv.view(T, H + 2 * KVH, hd).float()
    q, k, v = x[:, :H], x[:, H:H + KVH], st.qkv.view(T, H + 2 * KVH, hd)[:, H + KVH:]
    if case["norm"]:
        q = q * torch.rsqrt((q * q).mean(-1, keepdim=True) + _EPS) * st.q_gain.float()
        k = k * torch.rsqrt((k * k).mean(-1, keepdim=True) + _EPS) * st.k_gain.float()
    slot = torch.cat([torch.arange(n - r, n, device="cuda") for r, n in zip(st.rows, st.len)])
    seq = torch.cat([torch.full((r,), b, device="cuda") for b, r in enumerate(st.rows)])
    i = torch.arange(hd // 2, dtype=torch.float64, device="cuda")
    angle = slot.double()[:, None] * torch.exp(i * (-2.0 / hd * math.log(case["theta"])))
    c, s = torch.cos(angle).float()[:, None], torch.sin(angle).float()[:, None]

    def rotate(y):
        a, b = y[..., :hd // 2], y[..., hd // 2:]
        return torch.cat([a * c - b * s, b * c + a * s], -1).to(st.dtype)

    page, tok = st.table[seq, slot // _PAGE].long(), slot % _PAGE
    layer = st.pool[st.slot]
    layer[:, :, 0].view(KVH, -1, hd // 8, _PAGE, 8)[:, page, :, tok] = rotate(k).view(T, KVH, hd // 8, 8)
    layer[:, :, 1].view(KVH, -1, hd, _PAGE)[:, page, :, tok] = v
    return dict(q=rotate(q), pool=st.pool)


def _plain_attend(st):
    case, H, KVH, hd = st.case, st.H, st.KVH, st.hd
    G = H // KVH
    out, lse = torch.empty_like(st.q), torch.empty(st.q.shape[:2], device="cuda")
    for b, (r, n) in enumerate(zip(st.rows, st.len)):
        at = slice(st.start[b], st.start[b + 1])
        k, v = _read(st.pool[st.slot], st.table[b], n, hd)
        q = st.q[at].float().view(r, KVH, G, hd).transpose(0, 1).reshape(KVH, r * G, hd)
        s = torch.matmul(q, k.transpose(1, 2)) * hd ** -0.5
        key, pos = torch.arange(n, device="cuda"), torch.arange(n - r, n, device="cuda")[:, None]
        if case["tree"]:
            o = (key - (n - r)).clamp(min=0)
            seen = (key < n - r) | (((st.mask[at][:, None] >> o) & 1) == 1)
        else:
            seen = key <= pos
            if case["window"]:
                seen &= key > pos - case["window"]
        s = s.masked_fill(~seen.repeat_interleave(G, 0), float("-inf"))
        o, z = _softmax_v(s, v)
        out[at] = o.view(KVH, r, G, hd).transpose(0, 1).reshape(r, H, hd).to(st.dtype)
        lse[at] = z.view(KVH, r, G).transpose(0, 1).reshape(r, H)
    return dict(out=out, lse=lse)


def _plain_means(st):
    size = st.case["block"]
    for b, (r, n) in enumerate(zip(st.rows, st.len)):
        lo, hi = (n - r) // size, n // size
        if hi > lo:
            k, _ = _read(st.pool[st.slot], st.table[b], n, st.hd)
            st.means[b, :, lo:hi] = k[:, lo * size:hi * size].view(st.KVH, hi - lo, size, st.hd).mean(2)
    return st.means


def _plain_select(st):
    case, KVH, hd = st.case, st.KVH, st.hd
    sel = torch.full((st.q.shape[0], KVH, case["n_sel"]), -1, dtype=torch.int32, device="cuda")
    for b, (r, n) in enumerate(zip(st.rows, st.len)):
        at = slice(st.start[b], st.start[b + 1])
        q = st.q[at].double().view(r, KVH, -1, hd).sum(2).transpose(0, 1)
        score = torch.matmul(q, st.means[b].double().transpose(1, 2)).transpose(0, 1)
        block = torch.arange(st.n_means, device="cuda")
        last = (torch.arange(n - r, n, device="cuda") // case["block"])[:, None, None]
        score = score.masked_fill((block < 1) | (block > last - 2), float("inf"))
        score = score.masked_fill(block > last, float("-inf"))
        # highest first, equal ones in block order; then the chosen ones in block order
        pick = torch.sort(score, dim=-1, descending=True, stable=True).indices[..., :case["n_sel"]]
        pick = torch.where(pick > last, st.n_means, pick).sort(-1).values
        sel[at, :, :pick.shape[-1]] = torch.where(pick == st.n_means, -1, pick).to(torch.int32)
    return sel


def _plain_blocks(st):
    case, H, KVH, hd = st.case, st.H, st.KVH, st.hd
    size, G = case["block"], H // KVH
    out, lse = torch.empty_like(st.q), torch.empty(st.q.shape[:2], device="cuda")
    for b, (r, n) in enumerate(zip(st.rows, st.len)):
        k, v = _read(st.pool[st.slot], st.table[b], n, hd)
        pad = (0, 0, 0, _blocks(n, size) * size - n)
        k = torch.nn.functional.pad(k, pad).view(KVH, -1, size, hd)
        v = torch.nn.functional.pad(v, pad).view(KVH, -1, size, hd)
        head = torch.arange(KVH, device="cuda")[:, None]
        for r0 in range(0, r, 64):  # the rows' own copies of their blocks, 64 rows at a time
            m = min(64, r - r0)
            at = slice(st.start[b] + r0, st.start[b] + r0 + m)
            sel = st.sel[at].long()
            kk = k[head, sel.clamp(min=0)].view(m, KVH, -1, hd)
            vv = v[head, sel.clamp(min=0)].view(m, KVH, -1, hd)
            key = (sel[..., None] * size + torch.arange(size, device="cuda")).view(m, KVH, 1, -1)
            pos = torch.arange(n - r + r0, n - r + r0 + m, device="cuda").view(m, 1, 1, 1)
            s = torch.matmul(st.q[at].float().view(m, KVH, G, hd), kk.transpose(2, 3)) * hd ** -0.5
            s = s.masked_fill((key > pos) | (key < 0), float("-inf"))
            o, z = _softmax_v(s, vv)
            out[at], lse[at] = o.reshape(m, H, hd).to(st.dtype), z.reshape(m, H)
    return dict(out=out, lse=lse)


_PLAIN = dict(append=_plain_append, attend=_plain_attend, means=_plain_means, select=_plain_select, blocks=_plain_blocks)


def run(st):
    case = st.case
    kind = case["kind"]
    if not own:
        return _PLAIN[kind](st)
    if kind == "append":
        q = st.batch.append(st.slot, st.qkv, st.H, q_gain=st.q_gain, k_gain=st.k_gain, eps=_EPS, theta=case["theta"])
        return dict(q=q, pool=st.pool)
    if kind == "attend":
        out, lse = st.batch.attend(st.slot, st.q, window=case["window"], row_mask=st.mask, return_lse=True)
        return dict(out=out, lse=lse)
    if kind == "means":
        return st.batch.block_means(st.slot, st.means, block=case["block"])
    if kind == "select":
        return st.batch.select_blocks(st.q, st.means, case["n_sel"], block=case["block"], n_first=1, n_last=2)
    out, lse = st.batch.attend_blocks(st.slot, st.q, st.sel, block=case["block"], return_lse=True)
    return dict(out=out, lse=lse)


# -------------------------------------------------------------------- work
def work(case):
    H, KVH, hd, dt = _HEADS[case["model"]]
    e = 4 if dt == "f32" else 2
    rows, lens = _sizes(case)
    T = sum(rows)
    kind = case["kind"]
    if kind == "append":
        n = T * (H + 2 * KVH) * hd
        return dict(bytes=2 * n * e, flops=10 * n)
    qo = 2 * T * H * hd * e + 4 * T * H
    if kind == "attend":
        keys, seen = 0, 0
        for r, n in zip(rows, lens):
            w = case["window"] or n
            keys += min(n, w + r - 1)
            seen += sum(min(p + 1, w) for p in range(n - r, n))
        return dict(bytes=qo + 2 * keys * KVH * hd * e, flops=4 * seen * H * hd)
    size = case["block"]
    if kind == "means":
        nb = sum(n // size - (n - r) // size for r, n in zip(rows, lens))
        return dict(bytes=nb * KVH * hd * (size * e + 4), flops=nb * KVH * hd * size)
    nb = sum((n - 1) // size + 1 for n in lens)
    scored = sum(r * ((n - 1) // size + 1) for r, n in zip(rows, lens))
    if kind == "select":
        return dict(bytes=nb * KVH * hd * 4 + T * (H * hd * e + KVH * case["n_sel"] * 4), flops=2 * scored * KVH * hd)
    read = sum(min(n, r * case["n_sel"] * size) for r, n in zip(rows, lens))
    seen = sum(r * min(n, case["n_sel"] * size) for r, n in zip(rows, lens))
    return dict(bytes=qo + T * KVH * case["n_sel"] * 4 + 2 * read * KVH * hd * e, flops=4 * seen * H * hd)


# ------------------------------------------------------------------- exact
def _cached(st, b):
    """Keys and values [n, KVH, hd] of sequence b in float64, read token by token."""
    t = torch.arange(st.len[b], device="cuda")
    page, tok = st.table[b].long()[t // _PAGE], t % _PAGE
    d = torch.arange(st.hd, device="cuda")
    layer = st.pool[st.slot]
    k = layer[:, page, 0].gather(2, ((d // 8) * 128 + tok[:, None] * 8 + d % 8).expand(st.KVH, -1, -1))
    v = layer[:, page, 1].gather(2, (d * _PAGE + tok[:, None]).expand(st.KVH, -1, -1))
    return k.transpose(0, 1).double(), v.transpose(0, 1).double()


def _exact_attention(st, seen_of):
    """seen_of(b, g): the keys [rows, n] that the rows of sequence b see under K/V head g."""
    G = st.H // st.KVH
    out = torch.zeros(st.q.shape, dtype=torch.float64, device="cuda")
    lse = torch.zeros(st.q.shape[:2], dtype=torch.float64, device="cuda")
    for b in range(len(st.rows)):
        k, v = _cached(st, b)
        at = slice(st.start[b], st.start[b + 1])
        for h in range(st.H):
            g = h // G
            z = st.q[at, h].double() @ k[:, g].t().contiguous() / math.sqrt(st.hd)
            z = torch.where(seen_of(b, g), z, torch.full_like(z, -math.inf))
            lse[at, h] = torch.logsumexp(z, -1)
            out[at, h] = torch.nan_to_num(torch.softmax(z, -1)) @ v[:, g].contiguous()
    return dict(out=out, lse=lse)


def exact(case, seed):
    st = _inputs(case, seed)
    kind = case["kind"]
    pos = [torch.arange(n - r, n, device="cuda") for r, n in zip(st.rows, st.len)]
    if kind == "append":
        T, hd = st.qkv.shape[0], st.hd
        x = st.qkv.double().view(T, -1, hd)
        pool = st.pool.double()
        p = torch.cat(pos).double()
        j = torch.arange(hd // 2, device="cuda").double()
        turn = torch.polar(torch.ones((T, 1, hd // 2), dtype=torch.float64, device="cuda"),
                           (p[:, None] / torch.pow(case["theta"], 2.0 * j / hd))[:, None])

        def head(y, gain):
            if gain is not None:
                y = y / torch.sqrt(y.square().sum(-1, keepdim=True) / hd + _EPS) * gain.double()
            z = torch.complex(y[..., :hd // 2].contiguous(), y[..., hd // 2:].contiguous()) * turn
            return torch.cat([z.real, z.imag], -1)

        q = head(x[:, :st.H], st.q_gain)
        k, v = head(x[:, st.H:st.H + st.KVH], st.k_gain), x[:, st.H + st.KVH:]
        d = torch.arange(hd, device="cuda")
        for b in range(case["batch"]):
            at = slice(st.start[b], st.start[b + 1])
            page, tok = st.table[b].long()[pos[b] // _PAGE], (pos[b] % _PAGE)[:, None]
            for g in range(st.KVH):
                pool[st.slot, g, page[:, None], 0, (d // 8) * 128 + tok * 8 + d % 8] = k[at, g]
                pool[st.slot, g, page[:, None], 1, d * _PAGE + tok] = v[at, g]
        return dict(q=q, pool=pool)
    if kind == "attend":
        def seen(b, g):
            n, key = st.len[b], torch.arange(st.len[b], device="cuda")
            if case["tree"]:
                m = st.mask[st.start[b]:st.start[b + 1], None]
                o = key - (n - st.rows[b])
                return (o < 0) | ((o >= 0) & ((m >> o.clamp(0, 63)) % 2 != 0))
            ago = pos[b][:, None] - key
            return (ago >= 0) & (ago < (case["window"] or n))
        return _exact_attention(st, seen)
    size = case["block"]
    if kind == "means":
        means = st.means.double()
        for b, (r, n) in enumerate(zip(st.rows, st.len)):
            k, _ = _cached(st, b)
            for i in range((n - r) // size, n // size):
                means[b, :, i] = k[i * size:(i + 1) * size].sum(0) / size
        return means
    if kind == "select":
        n_sel = case["n_sel"]
        sel = torch.full((st.q.shape[0], st.KVH, n_sel), -1, dtype=torch.int64, device="cuda")
        for b in range(case["batch"]):
            last = pos[b] // size
            for g in range(st.KVH):
                q = st.q[st.start[b]:st.start[b + 1], g * (st.H // st.KVH):(g + 1) * (st.H // st.KVH)].double().sum(1)
                score = torch.stack([q @ m for m in st.means[b, g].double()], 1)
                i = torch.arange(st.n_means, device="cuda")
                keep = (i[None] == 0) | (i[None] >= last[:, None] - 1)
                score = torch.where(keep, torch.full_like(score, math.inf), score)
                score = torch.where(i[None] > last[:, None], torch.full_like(score, -math.inf), score)
                # a block's rank: how many stand before it
                for r0 in range(0, q.shape[0], 32):
                    z = score[r0:r0 + 32]
                    rank = ((z[:, None] > z[..., None]) | ((z[:, None] == z[..., None]) & (i < i[:, None]))).sum(-1)
                    chosen = (rank < n_sel) & (i <= last[r0:r0 + 32, None])
                    for r, c in enumerate(chosen):
                        c = c.nonzero()[:, 0]
                        sel[st.start[b] + r0 + r, g, :len(c)] = c
        return sel

    def listed_keys(b, g):
        at = slice(st.start[b], st.start[b + 1])
        key = torch.arange(st.len[b], device="cuda")
        member = torch.zeros((st.rows[b], max(_blocks(st.len[b], size), 1) + 1), dtype=torch.bool, device="cuda")
        member.scatter_(1, st.sel[at, g].long() + 1, True)  # column 0: the places that list nothing
        return member[:, 1 + key // size] & (key <= pos[b][:, None])
    return _exact_attention(st, listed_keys)
