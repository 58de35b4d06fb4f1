"""The paged-cache operators (via_paged_*, paper_2606_12243_amd.paged) against
plain float64 arithmetic (tests/paged_cases.py), where they can go wrong: no
rows, empty sequences, negative positions, single tokens to ragged prompts,
odd group sizes, padded batches, absent pages, windows, token trees, values
that no row may see, ties, other streams and captured graphs.

Tolerances: one rounding to the type (half a step) plus bounds of the 32-bit
arithmetic before it, see paged_cases.bounds and beside each test.
"""
import ctypes as C
import math

import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

if not torch.cuda.is_available():  # pragma: no cover
    pytest.skip("needs a GPU", allow_module_level=True)

import paged_cases as ref  # noqa: E402
from paper_2606_12243_amd import paged, via  # noqa: E402

BF16, F32 = torch.bfloat16, torch.float32


def on_gpu(b):
    """PagedBatch of a reference batch, its pool copied to the device."""
    cache = paged.PagedCache(b.pool.cuda(), b.KVH, b.hd, b.table.cuda())
    return paged.PagedBatch(cache, b.row_start.cuda(), b.kv_len.cuda(), b.T, b.max_kv)


def say(*what):
    print("[case]", *what, flush=True)


def weight_bits(b):
    """bf16 calls of 128 queries a K/V head and sequence or more hold their weights as one bf16 value (to
    nearest: 2^-8 of each at most), others as two (2^-15)."""
    many = -(-b.T // len(b.rows)) * (b.H // b.KVH) >= 128
    return 22 if b.dtype == F32 else 8 if many else 15


def check_attention(b, q, got, lse, n, scale, p_bits=None, **kw):
    want, z, pv, amp = ref.attend(b, q, scale, **kw)
    live = torch.zeros(b.T, dtype=torch.bool)
    live[:b.start[-1]] = True
    tol, ztol = ref.bounds(b.dtype, b.hd, n, want, torch.nan_to_num(z, neginf=0.0), pv, amp,
                           p_bits or (weight_bits(b) if kw.get("sel") is None else 22 if b.dtype == F32 else 15))
    err = (got.double().cpu() - want).abs()
    assert (err <= tol)[live].all(), float((err / tol)[live].max())
    zz = lse.double().cpu()
    none = torch.isinf(z)
    assert (zz[live & none.all(-1)] == -math.inf).all()
    assert ((zz - z).abs() <= ztol)[live][~none[live]].all()
    assert (got.cpu()[live][none[live]] == 0).all()


SHAPES = [(BF16, 8, 2, 128), (BF16, 4, 2, 64), (BF16, 3, 3, 128), (BF16, 12, 1, 64), (F32, 4, 4, 64), (F32, 6, 2, 128),
          (BF16, 3, 1, 64), (F32, 1, 1, 64), (BF16, 40, 1, 128)]
BATCHES = [
    ([1], [1]),                           # the first token
    ([1, 1, 1], [17, 300, 64]),           # single tokens
    ([4], [36]),
    ([0, 5, 0, 33, 1], [50, 5, 0, 130, 16]),  # sequences without rows, one without anything
    ([7, 3], [4, 0]),                     # more rows than positions: negative ones see nothing
    ([40, 77], [40, 500]),                # prompts and a chunk
    ([2], [2501]),                        # split over work-groups, and a length past a page lookup's chunk
    ([1], [5000]),
]


@pytest.mark.parametrize("rows,lens", BATCHES)
@pytest.mark.parametrize("dtype,H,KVH,hd", SHAPES)
def test_attend(dtype, H, KVH, hd, rows, lens):
    say("attend", dtype, H, KVH, hd, rows, lens)
    b = ref.Batch(dtype, H, KVH, hd, rows, lens, seed=len(rows) * 100 + lens[0])
    q = b.randn(b.T, H, hd).to(dtype)
    out, lse = on_gpu(b).attend(b.slot, q.cuda(), return_lse=True)
    torch.cuda.synchronize()
    check_attention(b, q, out, lse, b.max_kv, hd ** -0.5)


@pytest.mark.parametrize("dtype,H,KVH,hd", [(BF16, 8, 2, 128), (F32, 4, 4, 64)])
@pytest.mark.parametrize("rows,lens,window", [([3, 1], [40, 700], 1), ([3, 1], [40, 700], 33), ([50], [1300], 200),
                                              ([20], [10], 4), ([9], [2000], 5000)])
def test_window(dtype, H, KVH, hd, rows, lens, window):
    say("window", dtype, rows, lens, window)
    b = ref.Batch(dtype, H, KVH, hd, rows, lens, seed=window)
    q = b.randn(b.T, H, hd).to(dtype)
    out, lse = on_gpu(b).attend(b.slot, q.cuda(), scale=0.2, window=window, return_lse=True)
    torch.cuda.synchronize()
    check_attention(b, q, out, lse, window + 1, 0.2, window=window)


@pytest.mark.parametrize("dtype,H,KVH,hd", [(BF16, 8, 2, 128), (F32, 2, 1, 64)])
@pytest.mark.parametrize("rows,lens", [([5, 9], [21, 900]), ([64], [64]), ([70], [100]), ([6], [6]), ([3, 2], [1, 2])])
def test_tree_masks(dtype, H, KVH, hd, rows, lens):
    """Masks with bits past the rows, the 64th bit, and none at all (with no context: an empty row)."""
    say("tree", dtype, rows, lens)
    b = ref.Batch(dtype, H, KVH, hd, rows, lens, seed=rows[0])
    masks = torch.randint(-2 ** 63, 2 ** 63 - 1, (b.T,), generator=b.g, dtype=torch.int64)
    masks[0], masks[b.T // 2], masks[-1] = 0, 1, -2 ** 63
    q = b.randn(b.T, H, hd).to(dtype)
    out, lse = on_gpu(b).attend(b.slot, q.cuda(), row_mask=masks.cuda(), return_lse=True)
    torch.cuda.synchronize()
    check_attention(b, q, out, lse, b.max_kv, hd ** -0.5, masks=masks.tolist())


@pytest.mark.parametrize("dtype,H,KVH,hd", [(BF16, 8, 2, 128), (BF16, 2, 1, 64), (F32, 4, 2, 64)])
@pytest.mark.parametrize("rows,lens", [([3, 2], [37, 401]), ([80, 1], [80, 33])])
def test_values_no_row_may_see(dtype, H, KVH, hd, rows, lens):
    """NaN and infinities behind the last position, in keys after a row's own, and in spare pages
    change nothing for the rows that do not see them; rows that do get them."""
    say("unseen values", dtype, rows, lens)
    b = ref.Batch(dtype, H, KVH, hd, rows, lens, seed=3)
    clean = b.pool.clone()
    q = b.randn(b.T, H, hd).to(dtype)
    used = torch.zeros(b.n_blocks, dtype=torch.bool)
    k_pages = b.pool[b.slot][:, :, 0].view(KVH, b.n_blocks, hd // 8, 16, 8)
    v_pages = b.pool[b.slot][:, :, 1].view(KVH, b.n_blocks, hd, 16)
    for s, n in enumerate(lens):
        for j in range(-(-n // 16)):
            used[b.page(s, j * 16)] = True
        if n % 16:  # the rest of the last page
            p = b.page(s, n - 1)
            k_pages[:, p, :, n % 16:] = math.nan
            v_pages[:, p, :, n % 16:] = math.inf
    b.pool[:, :, ~used] = math.nan
    # the last row's own key and value of sequence 0: earlier rows do not see them
    p0, t0 = b.page(0, lens[0] - 1), (lens[0] - 1) % 16
    v_pages[:, p0, 1, t0], v_pages[:, p0, 2, t0], v_pages[:, p0, hd - 1, t0] = math.nan, math.inf, -math.inf
    out, lse = on_gpu(b).attend(b.slot, q.cuda(), return_lse=True)
    torch.cuda.synchronize()
    last = b.start[1] - 1
    odd = out[last].float().cpu()
    assert torch.isnan(odd[:, 1]).all() and (odd[:, 2] == math.inf).all() and (odd[:, hd - 1] == -math.inf).all()
    assert torch.isfinite(odd[:, [0, 3, 4, hd - 2]]).all()
    b.pool = clean
    # that row is compared where its values are finite
    out[last, :, 1], out[last, :, 2], out[last, :, hd - 1] = (
        x[last].cuda() for x in (ref.attend(b, q, hd ** -0.5)[0][..., i].to(dtype) for i in (1, 2, hd - 1)))
    check_attention(b, q, out, lse, b.max_kv, hd ** -0.5)


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_absent_pages_and_padded_rows(dtype):
    """Table entries outside the pool name no page; positions at or past max_kv do not exist; padded
    rows and what lies between the rows of a wider output stay as they were."""
    say("absent pages", dtype)
    H, KVH, hd = 4, 2, 64
    b = ref.Batch(dtype, H, KVH, hd, [4, 3], [200, 90], seed=8, pad=5)
    b.table[0, 2], b.table[0, 5], b.table[1, 0] = -7, b.n_blocks, 1 << 30
    b.max_kv = 180
    wide = b.randn(b.T, (H + 3) * hd).to(dtype).cuda()
    q = wide[:, hd:(H + 1) * hd]
    room = torch.full((b.T, (H + 2) * hd), 7.0, dtype=dtype, device="cuda")
    out, lse = on_gpu(b).attend(b.slot, q, out=room[:, :H * hd], return_lse=True)
    torch.cuda.synchronize()
    assert (room[b.start[-1]:] == 7).all() and (room[:, H * hd:] == 7).all()
    check_attention(b, q.reshape(b.T, H, hd).cpu(), out.reshape(b.T, H, hd), lse, 200, hd ** -0.5)
    n_sel = 3
    sel = torch.tensor([[[2, 0, 1], [0, 5, -1]]] * b.T, dtype=torch.int32)
    out, lse = on_gpu(b).attend_blocks(b.slot, q, sel.cuda(), block=32, out=room[:, :H * hd], return_lse=True)
    torch.cuda.synchronize()
    assert (room[b.start[-1]:] == 7).all() and (room[:, H * hd:] == 7).all()
    check_attention(b, q.reshape(b.T, H, hd).cpu(), out.reshape(b.T, H, hd), lse, n_sel * 32, hd ** -0.5, sel=sel, block=32)


@pytest.mark.parametrize("dtype,H,KVH,hd", SHAPES + [(BF16, 80, 2, 64)])
@pytest.mark.parametrize("rows,lens,block,n_sel", [([1, 1], [1, 700], 64, 4), ([3, 0, 2], [300, 9, 31], 32, 5),
                                                   ([37], [260], 128, 2), ([1], [6000], 64, 48)])
def test_attend_blocks(dtype, H, KVH, hd, rows, lens, block, n_sel):
    """Lists in any order, with repeats (which count again), blocks past the row's own and negative entries."""
    say("attend blocks", dtype, H, KVH, hd, rows, lens, block, n_sel)
    b = ref.Batch(dtype, H, KVH, hd, rows, lens, seed=block + n_sel)
    q = b.randn(b.T, H, hd).to(dtype)
    sel = torch.randint(-1, -(-max(lens) // block) + 1, (b.T, KVH, n_sel), generator=b.g, dtype=torch.int32)
    sel[0, 0] = -1  # nothing listed
    sel[-1, -1, 1] = sel[-1, -1, 0]
    out, lse = on_gpu(b).attend_blocks(b.slot, q.cuda(), sel.cuda(), block=block, return_lse=True)
    torch.cuda.synchronize()
    check_attention(b, q, out, lse, n_sel * block, hd ** -0.5, sel=sel, block=block)


# ------------------------------------------------------------------- append
def check_append(b, step, qkv, theta, eps, gains, pos, out=None):
    """32-bit arithmetic before the rounding: at most 24 half steps of the pair's magnitude (sum of squares
    12, root and reciprocal 3, gains 2, sine and cosine with the angle's fraction 4, rotation 3)."""
    qg, kg = gains
    want, mag, pool, pool_mag = ref.append(b, qkv, theta, eps, qg, kg, pos)
    dev = lambda t: None if t is None else t.cuda()
    got = step.append(b.slot, qkv if qkv.is_cuda else qkv.cuda(), b.H, pos=dev(pos), q_gain=dev(qg), k_gain=dev(kg), eps=eps,
                      theta=theta, out=out)
    torch.cuda.synchronize()
    half = torch.finfo(b.dtype).eps / 2
    live = slice(0, b.start[-1])
    err = (got.reshape(b.T, b.H, b.hd).double().cpu() - want).abs()[live]
    assert (err <= half * want.abs()[live] + 2.0 ** -19 * mag[live]).all(), float(err.max())
    err = (step.cache.pool.double().cpu() - pool).abs()
    assert (err <= half * pool.abs() * (pool_mag > 0) + 2.0 ** -19 * pool_mag).all(), float(err.max())
    return got


@pytest.mark.parametrize("dtype,H,KVH,hd", SHAPES)
@pytest.mark.parametrize("rows,lens,norm", [([1], [1], "qk"), ([4, 0, 30], [40, 3, 30], "qk"), ([17, 5], [100, 3], ""),
                                            ([2, 65], [900, 70], "k")])
def test_append(dtype, H, KVH, hd, rows, lens, norm):
    say("append", dtype, H, KVH, hd, rows, lens, norm)
    b = ref.Batch(dtype, H, KVH, hd, rows, lens, seed=lens[0])
    qkv = (b.randn(b.T, (H + 2 * KVH) * hd) * 1.5).to(dtype)
    gains = [(1 + 0.2 * b.randn(hd)).to(dtype) if c in norm else None for c in "qk"]
    check_append(b, on_gpu(b), qkv, 10000.0, 1e-5, gains, None)


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_append_far_positions_padding_and_place(dtype):
    """Given positions up to 2^31 - 1 (and a negative one), absent pages, padded rows, a strided projection,
    queries written over themselves."""
    say("append far", dtype)
    H, KVH, hd = 4, 2, 64
    b = ref.Batch(dtype, H, KVH, hd, [5, 3], [37, 20], seed=4, pad=3)
    b.table[1, 1] = -1
    b.max_kv = 36
    pos = torch.tensor([0, 1, 2 ** 31 - 1, 1000003, -5, 7, 123456789, 3] + [0] * 3, dtype=torch.int32)
    wide = b.randn(b.T, (H + 2 * KVH + 1) * hd).to(dtype).cuda()
    qkv = wide[:, :(H + 2 * KVH) * hd]
    before, held = wide.clone(), qkv.cpu().clone()
    gains = [(1 + 0.2 * b.randn(hd)).to(dtype) for _ in "qk"]
    step = on_gpu(b)
    kept = check_append(b, step, held, 500000.0, 1e-6, gains, pos).clone()
    step.cache.pool.copy_(b.pool)
    got = step.append(b.slot, qkv, H, pos=pos.cuda(), q_gain=gains[0].cuda(), k_gain=gains[1].cuda(), eps=1e-6,
                      theta=500000.0, out=wide[:, :H * hd])
    torch.cuda.synchronize()
    n = b.start[-1]
    assert torch.equal(got[:n].reshape(n, H, hd), kept[:n])
    assert torch.equal(wide[n:], before[n:]) and torch.equal(wide[:, H * hd:], before[:, H * hd:])


# ------------------------------------------------------- means and selection
@pytest.mark.parametrize("dtype,H,KVH,hd", SHAPES)
@pytest.mark.parametrize("rows,lens,block", [([1, 1, 1], [32, 33, 64], 32), ([200, 0, 7], [200, 100, 70], 64),
                                             ([300], [300], 128), ([9], [5], 32), ([40], [1064], 64)])
def test_block_means(dtype, H, KVH, hd, rows, lens, block):
    """At most block / 16 + 5 roundings to 32 bits of sums that the mean |k| bounds."""
    say("means", dtype, KVH, hd, rows, lens, block)
    b = ref.Batch(dtype, H, KVH, hd, rows, lens, seed=block)
    if len(rows) == 1 and lens[0] == 300:
        b.table[0, 9] = -1  # a block with an absent page keeps its mean
    nb = max(1, max(lens) // block)
    if lens[0] == 1064:
        nb -= 1  # fewer than the sequence has
    old = b.randn(len(rows), KVH, nb, hd)
    got = on_gpu(b).block_means(b.slot, old.cuda(), block=block)
    torch.cuda.synchronize()
    want, mag = ref.means(b, old, block)
    assert ((got.double().cpu() - want).abs() <= (block // 16 + 5) * 2.0 ** -24 * mag).all()


@pytest.mark.parametrize("dtype,H,KVH,hd", SHAPES)
@pytest.mark.parametrize("rows,lens,block,n_sel,first,last", [
    ([1], [1], 64, 3, 1, 2), ([1, 2], [2100, 300], 32, 8, 1, 2), ([19, 0, 3], [700, 9, 2], 64, 4, 0, 1),
    ([33], [5000], 32, 16, 2, 3), ([5], [3], 128, 6, 3, 3), ([2], [9000], 32, 40, 0, 1)])
def test_select(dtype, H, KVH, hd, rows, lens, block, n_sel, first, last):
    """Blocks are whole numbers: equal to the reference's.  Equal means (ties) and NaN among them."""
    say("select", dtype, H, KVH, hd, rows, lens, block, n_sel)
    b = ref.Batch(dtype, H, KVH, hd, rows, lens, seed=n_sel + lens[0])
    nb = -(-max(lens) // block) + 1
    m = b.randn(len(rows), KVH, nb, hd)
    m[:, :, 4:nb:3] = m[:, :, :1].clone()  # equal scores in many places
    if nb > 8:
        m[:, 0, 7, 0] = math.nan
        m[:, 0, 6, 3] = math.inf
    q = b.randn(b.T, H, hd).to(dtype)
    got = on_gpu(b).select_blocks(q.cuda(), m.cuda(), n_sel, block=block, n_first=first, n_last=last)
    torch.cuda.synchronize()
    assert torch.equal(got.cpu(), ref.select(b, q, m, n_sel, block, first, last))


def test_select_small_differences_and_padding():
    """Scores that differ by less than 32 bits hold are still ordered; padded rows keep their lists."""
    say("select near ties")
    b = ref.Batch(F32, 2, 1, 64, [2], [64 * 40], seed=1, pad=3)
    q = torch.ones(b.T, 2, 64)
    m = torch.full((1, 1, 41, 64), 1.0)
    m[0, 0, :, 0] = 1000.0
    m[0, 0, :, 1] = torch.randperm(41, generator=b.g).float() * 2.0 ** -20  # 2^-30 of the sum
    out = torch.full((b.T, 1, 6), 99, dtype=torch.int32, device="cuda")
    on_gpu(b).select_blocks(q.cuda(), m.cuda(), 6, block=64, n_first=0, n_last=1, out=out)
    torch.cuda.synchronize()
    assert torch.equal(out[:2].cpu(), ref.select(b, q, m, 6, 64, 0, 1)[:2]) and (out[2:] == 99).all()


# ------------------------------------------------------------ used together
def test_layers_together():
    """Two layers of a prompt, its tail and single tokens, as a program runs them; every block chosen, the
    sparse form gives the dense form's result."""
    say("together")
    H, KVH, hd = 8, 2, 128
    g = torch.Generator().manual_seed(2)
    b = ref.Batch(BF16, H, KVH, hd, [0, 0], [420, 130], seed=6)
    cache = paged.PagedCache(b.pool.cuda(), KVH, hd, b.table.cuda())
    gains = [(1 + 0.1 * torch.randn(hd, generator=g)).to(BF16) for _ in "qk"]
    means = torch.zeros(2, 2, KVH, 14, hd, device="cuda")
    steps = [([300, 129], [300, 129]), ([119, 0], [419, 129]), ([1, 1], [420, 130])]
    for rows, lens in steps:
        b.rows, b.lens, b.T = rows, lens, sum(rows)
        b.start = [0, rows[0], sum(rows)]
        step = paged.PagedBatch(cache, torch.tensor(b.start, dtype=torch.int32).cuda(),
                                torch.tensor(lens, dtype=torch.int32).cuda(), b.T, 500)
        for slot in (0, 1):
            b.slot = slot
            b.pool = cache.pool.cpu()
            qkv = (torch.randn(b.T, (H + 2 * KVH) * hd, generator=g)).to(BF16)
            q = check_append(b, step, qkv, 10000.0, 1e-5, gains, None)
            b.pool = cache.pool.cpu()
            out, lse = step.attend(slot, q, return_lse=True)
            check_attention(b, q.cpu(), out, lse, 420, hd ** -0.5)
            before = means[slot].clone()
            step.block_means(slot, means[slot], block=32)
            torch.cuda.synchronize()
            want, mag = ref.means(b, before, 32)
            assert ((means[slot].double().cpu() - want).abs() <= 7 * 2.0 ** -24 * mag).all()
            b.max_kv = 420
            some = step_of(cache, b).select_blocks(q, means[slot], 4, block=32)
            assert torch.equal(some.cpu(), ref.select(b, q.cpu(), means[slot].cpu(), 4, 32, 1, 2))
            out, lse = step.attend_blocks(slot, q, some, block=32, return_lse=True)
            check_attention(b, q.cpu(), out, lse, 128, hd ** -0.5, sel=some.cpu(), block=32)
            every = step_of(cache, b).select_blocks(q, means[slot], 14, block=32)
            out, lse = step.attend_blocks(slot, q, every, block=32, return_lse=True)
            check_attention(b, q.cpu(), out, lse, 448, hd ** -0.5)


def step_of(cache, b):
    return paged.PagedBatch(cache, torch.tensor(b.start, dtype=torch.int32).cuda(),
                            torch.tensor(b.lens, dtype=torch.int32).cuda(), b.T, b.max_kv)


@pytest.mark.parametrize("name", ["micro_bf16", "micro_f32"])
def test_a_handles_cache(name):
    """Attention over the cache that a KV handle's prefill filled."""
    say("handle", name)
    from workload import configs, gen
    cfg = configs.get(name)
    md = cfg["model"]
    model = via.Model(md, gen.model_weights(cfg), cfg["route"])
    kv = via.KV(model, max_seqs=3, max_blocks_per_seq=8, blocks_full=20, blocks_slim=20, max_rows=128, max_batch=2,
                max_drafts=4)
    try:
        sp = C.c_void_p(torch.cuda.current_stream().cuda_stream)
        lens = [70, 33]
        toks, tp = via._i32([i * 7 % md["vocab"] for i in range(sum(lens))])
        ids, ip = via._i32([0, 2])
        ln, lp = via._i32(lens)
        via.check(via.via_prefill_batch(model.h, kv.h, 2, ip, lp, tp, sp))
        torch.cuda.synchronize()
        cache = paged.PagedCache.of_handle(kv, via.CACHE_FULL, [0, 2])
        dtype = BF16 if md["dtype"] == "bf16" else F32
        b = ref.Batch(dtype, md["n_heads"], md["n_kv_heads"], md["head_dim"], [2, 1], lens, slot=2)
        b.pool, b.table, b.n_blocks = cache.pool.cpu(), cache.table.cpu(), cache.n_blocks
        q = b.randn(b.T, b.H, b.hd).to(dtype)
        out, lse = step_of(cache, b).attend(2, q.cuda(), return_lse=True)
        torch.cuda.synchronize()
        check_attention(b, q, out, lse, 70, b.hd ** -0.5)
    finally:
        kv.close()
        model.close()


def test_streams_and_captured_graphs():
    """The operators on another stream than the default, and captured: a graph follows the lengths,
    tables and queries it finds on replay, with the program's eager work in between; two captured
    graphs do not share a workspace."""
    say("graphs")
    H, KVH, hd = 8, 2, 128
    b = ref.Batch(BF16, H, KVH, hd, [1, 1], [900, 1500], seed=9)
    gains = [(1 + 0.1 * b.randn(hd)).to(BF16) for _ in "qk"]
    step = on_gpu(b)
    qkv = b.randn(b.T, (H + 2 * KVH) * hd).to(BF16).cuda()
    means = torch.zeros(2, KVH, 24, hd, device="cuda")
    gg = [t.cuda() for t in gains]

    def work():
        q = step.append(1, qkv, H, q_gain=gg[0], k_gain=gg[1])
        step.block_means(1, means)
        sel = step.select_blocks(q, means, 8)
        return q, step.attend(1, q), sel, step.attend_blocks(1, q, sel)

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        eager = work()
    side.synchronize()
    first = [t.clone() for t in work()]
    torch.cuda.synchronize()
    assert all(torch.equal(x, y) for x, y in zip(eager, first))
    pool0, means0 = step.cache.pool.clone(), means.clone()
    graphs, outs = [], []
    for _ in range(2):
        gr = torch.cuda.CUDAGraph()
        with torch.cuda.graph(gr):
            outs.append(work())
        graphs.append(gr)
    other = torch.cuda.Stream()
    for i in range(3):
        step.kv_len.copy_(torch.tensor([900 - i * 64, 1500 - i * 100], dtype=torch.int32))
        qkv.normal_()
        step.cache.pool.copy_(pool0)
        means.copy_(means0)
        want = [t.clone() for t in work()]
        step.cache.pool.copy_(pool0)
        means.copy_(means0)
        torch.cuda.synchronize()
        graphs[0].replay()
        with torch.cuda.stream(other):  # the same values go to the same places
            graphs[1].replay()
        torch.cuda.synchronize()
        for o in outs:
            assert all(torch.equal(x, y) for x, y in zip(o, want)), i


def test_more_than_32_bits_of_elements():
    """Pages more than 2^31 elements into the pool."""
    say("far pages")
    H, KVH, hd = 4, 2, 128
    n_blocks = 530000  # K/V head 1 starts 2.17e9 elements in
    pool = torch.empty((1, KVH, n_blocks, 2, 16 * hd), dtype=BF16, device="cuda")
    b = ref.Batch(BF16, H, KVH, hd, [3], [40], seed=12, slot=0)
    far = [n_blocks - 1, 7, n_blocks - 9]
    small = b.pool[0]
    for j, p in enumerate(far):
        pool[0, :, p] = small[:, int(b.table[0, j])].cuda()
    table = torch.full((1, 5), -1, dtype=torch.int32)
    table[0, :3] = torch.tensor(far)
    step = paged.PagedBatch(paged.PagedCache(pool, KVH, hd, table.cuda()), b.row_start.cuda(), b.kv_len.cuda(), b.T, 40)
    q = b.randn(b.T, H, hd).to(BF16)
    out, lse = step.attend(0, q.cuda(), return_lse=True)
    qkv = b.randn(b.T, (H + 2 * KVH) * hd).to(BF16)
    torch.cuda.synchronize()
    check_attention(b, q, out, lse, 40, hd ** -0.5)
    step.append(0, qkv.cuda(), H)
    torch.cuda.synchronize()
    _, _, want, mag = ref.append(b, qkv, 10000.0, 1e-5, None, None)
    for j, p in enumerate(far):
        w, m = want[0, :, int(b.table[0, j])], mag[0, :, int(b.table[0, j])]
        assert ((pool[0, :, p].double().cpu() - w).abs() <= 2.0 ** -8 * w.abs() * (m > 0) + 2.0 ** -19 * m).all()


@pytest.mark.parametrize("H,KVH,hd", [(8, 2, 128), (4, 2, 64), (5, 5, 128), (32, 1, 64)])
@pytest.mark.parametrize("rows,lens,kw", [
    ([128, 131], [128, 1000], {}),             # prompt and chunk, whole and partial tiles
    ([200, 0, 260], [100, 5, 330], {}),        # more rows than positions
    ([300], [9000], {}),                       # split
    ([150, 128], [700, 150], dict(window=70)),
    ([130], [2000], dict(tree=True)),          # only its first 64 positions have bits
    ([34], [4130], dict(tree=True)),           # fewer rows: two terms a weight
    ([20, 33, 41], [20, 1100, 3000], {}),
    ([3, 60], [9000, 60], {}),                 # uneven: split all the same
])
def test_attend_many_rows(H, KVH, hd, rows, lens, kw):
    """The kernel for more than 32 queries."""
    say("many rows", H, KVH, hd, rows, lens, kw)
    b = ref.Batch(BF16, H, KVH, hd, rows, lens, seed=lens[0], pad=3)
    q = (b.randn(b.T, H, hd) * 2).to(BF16)
    masks = torch.randint(-2 ** 63, 2 ** 63 - 1, (b.T,), generator=b.g, dtype=torch.int64) if "tree" in kw else None
    window = kw.get("window", 0)
    out = torch.full((b.T, H, hd), 7.0, dtype=BF16, device="cuda")
    _, lse = on_gpu(b).attend(b.slot, q.cuda(), window=window, row_mask=None if masks is None else masks.cuda(), out=out,
                              return_lse=True)
    torch.cuda.synchronize()
    assert (out[b.start[-1]:] == 7).all()
    check_attention(b, q, out, lse, b.max_kv, hd ** -0.5, window=window,
                    masks=None if masks is None else masks.tolist())


def test_values_no_row_may_see_many_rows():
    say("unseen values, many rows")
    H, KVH, hd = 8, 2, 128
    b = ref.Batch(BF16, H, KVH, hd, [200], [333], seed=5)
    b.table[0, 3] = -1
    q = b.randn(b.T, H, hd).to(BF16)
    clean = b.pool.clone()
    v = b.pool[b.slot][:, :, 1].view(KVH, b.n_blocks, hd, 16)
    for pos, dim, x in ((250, 9, math.nan), (251, 10, math.inf), (252, 127, -math.inf), (252, 64, math.inf), (253, 64, -math.inf)):
        v[:, b.page(0, pos), dim, pos % 16] = x
    last = b.page(0, 332)
    v[:, last, :, 333 % 16:] = math.nan
    b.pool[b.slot][:, :, 0].view(KVH, b.n_blocks, hd // 8, 16, 8)[:, last, :, 333 % 16:] = math.inf
    out, lse = on_gpu(b).attend(b.slot, q.cuda(), return_lse=True)
    torch.cuda.synchronize()
    o = out.float().cpu()
    first = 333 - 200  # row r is position first + r
    for dim, pos, test in ((9, 250, torch.isnan), (10, 251, lambda t: t == math.inf), (127, 252, lambda t: t == -math.inf),
                           (64, 253, torch.isnan)):
        assert test(o[pos - first:, :, dim]).all()
    assert (o[252 - first, :, 64] == math.inf).all()
    b.pool = clean
    want = ref.attend(b, q, hd ** -0.5)[0].to(BF16).cuda()
    for dim, pos in ((9, 250), (10, 251), (127, 252), (64, 252)):
        assert torch.isfinite(o[:pos - first, :, dim]).all()
        out[pos - first:, :, dim] = want[pos - first:, :, dim]
    check_attention(b, q, out, lse, b.max_kv, hd ** -0.5)


@pytest.mark.parametrize("len_,n_sel", [(32 * 2048, 40), (32 * 2049 + 5, 7), (32 * 3000, 100)])
def test_select_of_many_blocks(len_, n_sel):
    """Around the number of blocks whose scores a wave holds, with ties across it."""
    say("select many", len_, n_sel)
    b = ref.Batch(BF16, 2, 1, 64, [2], [16], seed=n_sel)
    b.lens, b.max_kv = [len_], len_
    b.kv_len = torch.tensor([len_], dtype=torch.int32)
    b.table = torch.zeros((1, len_ // 16 + 1), dtype=torch.int32)
    nb = -(-len_ // 32)
    m = b.randn(1, 1, nb, 64)
    m[0, 0, 100::500] = m[0, 0, 100].clone()
    m[0, 0, 100::500, :2] += 3
    q = b.randn(b.T, 2, 64).to(BF16)
    q[:, :, :2] = 2
    got = on_gpu(b).select_blocks(q.cuda(), m.cuda(), n_sel, block=32)
    torch.cuda.synchronize()
    assert torch.equal(got.cpu(), ref.select(b, q, m, n_sel, 32, 1, 2))


def test_select_with_nan_scores_only():
    say("select nan")
    b = ref.Batch(BF16, 2, 1, 64, [3], [640], seed=1)
    m = b.randn(1, 1, 20, 64)
    m[:, :, 2:15] = math.nan
    q = b.randn(b.T, 2, 64).to(BF16)
    q[1] = math.nan
    for n_sel in (4, 12, 18, 30):
        got = on_gpu(b).select_blocks(q.cuda(), m.cuda(), n_sel, block=32)
        torch.cuda.synchronize()
        assert torch.equal(got.cpu(), ref.select(b, q, m, n_sel, 32, 1, 2)), n_sel


@pytest.mark.parametrize("case", ["all equal", "64 equal", "65 equal", "zero", "small", "tiny", "large", "huge", "wide", "close",
                                  "one infinite"])
@pytest.mark.parametrize("dtype,hd", [(BF16, 128), (F32, 64)])
def test_select_where_32_bits_do_not_decide(dtype, hd, case):
    """Equal and nearly equal scores, few and many of them around the last place, and sizes at which 32-bit
    products, squares or sums underflow or overflow: the blocks are those of the 64-bit scores."""
    say("select undecided", dtype, hd, case)
    H, KVH, block, n_sel = 4, 2, 32, 40
    b = ref.Batch(dtype, H, KVH, hd, [3], [16], seed=len(case))
    b.lens, b.max_kv = [32 * 300 + 3], 32 * 300 + 3
    b.kv_len = torch.tensor(b.lens, dtype=torch.int32)
    b.table = torch.zeros((1, 700), dtype=torch.int32)
    m = b.randn(1, KVH, 301, hd)
    q = b.randn(b.T, H, hd).to(dtype)
    best = q.float().view(b.T, KVH, -1, hd).sum(2)[1]  # a mean along the queries of row 1
    if case == "all equal":
        m[:] = m[:, :, :1].clone()
    elif "equal" in case:  # 30 better ones, then as many equal ones as it says
        n = int(case.split()[0])
        at = torch.randperm(280, generator=b.g)[:n + 30] + 5
        m *= 0.01
        m[0, :, at[:30]] = best[:, None] * (2 + 0.01 * torch.arange(30.0)[:, None])
        m[0, :, at[30:]] = best[:, None]
    elif case == "zero":
        m[:] = 0
    elif case == "wide":
        m *= torch.exp(b.randn(1, KVH, 301, 1) * 20)
    elif case == "close":  # steps of 2^-26 of the score
        m[:] = best[:, None] * 1024
        step = torch.randperm(301, generator=b.g).float() * 2.0 ** -17
        m[0, :, :, 0] += step * best[:, :1].sign()
    elif case == "one infinite":
        m[0, 0, 77, 3], m[0, 1, 78, 5] = math.inf, -math.inf
    else:
        m *= {"small": 1e-19, "tiny": 1e-38, "large": 1e18, "huge": 1e36}[case]
        q = (q.float() * {"small": 1e-3, "tiny": 1e-2, "large": 1e3, "huge": 1e3}[case]).to(dtype)
    got = on_gpu(b).select_blocks(q.cuda(), m.cuda(), n_sel, block=block, n_first=1, n_last=2)
    torch.cuda.synchronize()
    assert torch.equal(got.cpu(), ref.select(b, q, m, n_sel, block, 1, 2))


@pytest.mark.parametrize("rows,lens", [([1, 2], [900, 40]), ([60, 5], [60, 700])])
def test_output_over_the_queries(rows, lens):
    say("in place", rows, lens)
    b = ref.Batch(BF16, 8, 2, 128, rows, lens, seed=3)
    q = b.randn(b.T, 8, 128).to(BF16)
    step = on_gpu(b)
    sel = torch.arange(3, dtype=torch.int32, device="cuda").expand(b.T, 2, 3).contiguous()
    for f in (lambda t, o: step.attend(b.slot, t, out=o), lambda t, o: step.attend_blocks(b.slot, t, sel, block=32, out=o)):
        apart = f(q.cuda(), None)
        t = q.cuda()
        f(t, t)
        torch.cuda.synchronize()
        assert torch.equal(t, apart)


def test_binding_refuses():
    b = ref.Batch(BF16, 4, 2, 64, [3], [40], seed=1)
    step = on_gpu(b)
    q = b.randn(b.T, 4, 64).to(BF16).cuda()
    means = torch.zeros(1, 2, 3, 64, device="cuda")
    sel = torch.zeros(3, 2, 2, dtype=torch.int32, device="cuda")
    bad = [
        lambda: step.attend(1, q.float()), lambda: step.attend(1, q.cpu()), lambda: step.attend(1, q[:2]),
        lambda: step.attend(1, q[:, :, :32]), lambda: step.attend(1, q.transpose(1, 2)),
        lambda: step.attend(1, q.clone().requires_grad_()), lambda: step.attend(1, q, out=q[:, :2]),
        lambda: step.attend(1, q, row_mask=torch.zeros(3, dtype=torch.int32, device="cuda")),
        lambda: step.append(1, q, 4), lambda: step.append(1, q.reshape(3, 256), 2, pos=torch.zeros(2, dtype=torch.int32, device="cuda")),
        lambda: step.append(1, q.new_zeros(3, 512), 4, q_gain=q.new_zeros(32)),
        lambda: step.block_means(1, means.double()), lambda: step.block_means(1, means[:, :1]),
        lambda: step.select_blocks(q, means[0], 4), lambda: step.select_blocks(q, means, 4, out=sel),
        lambda: step.attend_blocks(1, q, sel.long()), lambda: step.attend_blocks(1, q, sel[:2]),
        lambda: paged.PagedBatch(step.cache, step.row_start, step.kv_len.long(), 3, 40),
        lambda: paged.PagedBatch(step.cache, step.kv_len, step.kv_len, 3, 40),
        lambda: paged.PagedCache(step.cache.pool, 2, 64, step.table.cpu()),
        lambda: paged.PagedCache(step.cache.pool, 3, 64, step.table),
        lambda: paged.PagedCache(step.cache.pool[..., ::2], 2, 64, step.table),
    ]
    for i, f in enumerate(bad):
        with pytest.raises(ValueError):
            f()
            pytest.fail(f"call {i} was not refused")
    for f in (lambda: step.attend(2, q), lambda: step.attend(1, q, scale=0.0), lambda: step.attend(1, q, window=-1),
              lambda: step.attend_blocks(1, q, sel, block=48), lambda: step.select_blocks(q, means[:, :, :1].contiguous(), 4, block=32)):
        with pytest.raises(via.ViaError):
            f()
    # part of a wider table, at its end
    wide = torch.full((1, 9), -1, dtype=torch.int32, device="cuda")
    wide[:, 5:8] = step.table[:, :3]
    part = paged.PagedBatch(paged.PagedCache(step.cache.pool, 2, 64, wide[:, 5:8]), step.row_start, step.kv_len, 3, 1000)
    assert torch.equal(part.attend(1, q), step.attend(1, q))


@pytest.mark.parametrize("dtype,H,KVH,hd,most", [(BF16, 4, 2, 64, 3), (F32, 2, 1, 64, 2), (BF16, 8, 1, 64, 12)])
@pytest.mark.parametrize("n_seqs", [64, 65, 131])
def test_many_sequences(dtype, H, KVH, hd, most, n_seqs):
    """More sequences than a wave has lanes, those without rows among them, through every operator."""
    say("many sequences", dtype, H, KVH, hd, most, n_seqs)
    g = torch.Generator().manual_seed(n_seqs)
    rows = torch.randint(0, most + 1, (n_seqs,), generator=g).tolist()
    lens = [n + int(c) for n, c in zip(rows, torch.randint(0, 90, (n_seqs,), generator=g))]
    rows[0], lens[0], rows[-1], lens[-1], rows[63], lens[63] = 0, 0, most, 300, most, most
    b = ref.Batch(dtype, H, KVH, hd, rows, lens, seed=most, pad=2)
    step = on_gpu(b)
    qkv = b.randn(b.T, (H + 2 * KVH) * hd).to(dtype)
    q = check_append(b, step, qkv, 10000.0, 1e-5, [None, None], None)
    b.pool = step.cache.pool.cpu()
    out, lse = step.attend(b.slot, q, return_lse=True)
    torch.cuda.synchronize()
    check_attention(b, q.cpu(), out, lse, b.max_kv, hd ** -0.5)
    old = b.randn(n_seqs, KVH, 11, hd)
    got = step.block_means(b.slot, old.cuda(), block=32)
    torch.cuda.synchronize()
    want, mag = ref.means(b, old, 32)
    assert ((got.double().cpu() - want).abs() <= 7 * 2.0 ** -24 * mag).all()
    sel = step.select_blocks(q, got, 3, block=32)
    torch.cuda.synchronize()
    n = b.start[-1]
    assert torch.equal(sel[:n].cpu(), ref.select(b, q.cpu(), got.cpu(), 3, 32, 1, 2)[:n])
    out, lse = step.attend_blocks(b.slot, q, sel, block=32, return_lse=True)
    torch.cuda.synchronize()
    check_attention(b, q.cpu(), out, lse, 96, hd ** -0.5, sel=sel.cpu(), block=32)


@pytest.mark.parametrize("dtype,H,KVH,hd,rows", [(BF16, 8, 2, 128, 1), (F32, 2, 1, 64, 3), (BF16, 8, 2, 64, 50), (BF16, 32, 1, 128, 70)])
def test_values_outside_a_window(dtype, H, KVH, hd, rows):
    """NaN and infinities in keys and values that the window leaves behind, inside a page and whole pages."""
    say("outside a window", dtype, H, KVH, hd, rows)
    window, len_ = 45, 700
    b = ref.Batch(dtype, H, KVH, hd, [rows], [len_], seed=rows)
    q = b.randn(b.T, H, hd).to(dtype)
    first = len_ - rows - window + 1  # the first key of the first row
    pool = b.pool.clone()
    k = pool[b.slot][:, :, 0].view(KVH, b.n_blocks, hd // 8, 16, 8)
    v = pool[b.slot][:, :, 1].view(KVH, b.n_blocks, hd, 16)
    for pos in range(first):
        p = b.page(0, pos)
        k[:, p, :, pos % 16] = (math.nan, math.inf, -math.inf)[pos % 3]
        v[:, p, :, pos % 16] = (-math.inf, math.nan, math.inf)[pos % 3]
    clean, b.pool = b.pool, pool
    out, lse = on_gpu(b).attend(b.slot, q.cuda(), window=window, return_lse=True)
    torch.cuda.synchronize()
    b.pool = clean
    check_attention(b, q, out, lse, window + 1, hd ** -0.5, window=window)


@pytest.mark.parametrize("dtype,H,KVH,hd,rows", [(BF16, 8, 2, 128, 2), (F32, 2, 1, 64, 2), (BF16, 4, 2, 64, 20), (BF16, 8, 2, 128, 90)])
@pytest.mark.parametrize("grow", [0.5, 6.0, 40.0, -6.0])
def test_scores_that_climb(dtype, H, KVH, hd, rows, grow):
    """The running maximum moves a little, much, or never after the first keys: scores climb (or fall) by
    ``grow`` every 64 keys, the largest ones far from zero."""
    say("climb", dtype, H, KVH, hd, rows, grow)
    len_ = 900
    b = ref.Batch(dtype, H, KVH, hd, [rows], [len_], seed=rows)
    k = b.pool[b.slot][:, :, 0].view(KVH, b.n_blocks, hd // 8, 16, 8)
    for pos in range(len_):
        k[:, b.page(0, pos), 0, pos % 16, 0] = pos * grow / 64
    q = b.randn(b.T, H, hd).to(dtype)
    q[:, :, 0] = hd ** 0.5
    out, lse = on_gpu(b).attend(b.slot, q.cuda(), return_lse=True)
    torch.cuda.synchronize()
    check_attention(b, q, out, lse, b.max_kv, hd ** -0.5)


@pytest.mark.parametrize("dtype,H,KVH,hd", [(BF16, 8, 2, 128), (F32, 2, 1, 64)])
@pytest.mark.parametrize("rows", [3, 60])
@pytest.mark.parametrize("window", [2 ** 31 - 1, 2 ** 31 - 2, 2 ** 30])
def test_window_of_all_positions(dtype, H, KVH, hd, rows, window):
    """The largest windows, with rows at negative positions before them."""
    say("largest window", dtype, rows, window)
    b = ref.Batch(dtype, H, KVH, hd, [rows, 2], [rows - 2, 700], seed=rows)
    q = b.randn(b.T, H, hd).to(dtype)
    out, lse = on_gpu(b).attend(b.slot, q.cuda(), window=window, return_lse=True)
    torch.cuda.synchronize()
    check_attention(b, q, out, lse, b.max_kv, hd ** -0.5, window=window)


@pytest.mark.parametrize("dtype,H,KVH,hd", [(BF16, 8, 2, 128), (F32, 2, 1, 64)])
@pytest.mark.parametrize("rows", [3, 60])
@pytest.mark.parametrize("window", [0, 100, 2 ** 31 - 1])
def test_lengths_far_past_the_bound(dtype, H, KVH, hd, rows, window):
    """A length up to 2^31 - 1 on the device: its rows cache nothing and see what max_kv leaves of their keys."""
    say("far lengths", dtype, rows, window)
    far = 2 ** 31 - 1
    b = ref.Batch(dtype, H, KVH, hd, [rows, 2], [700, 40], seed=rows)
    b.lens[0] = far
    b.kv_len = torch.tensor(b.lens, dtype=torch.int32)
    b.max_kv = 650
    step = on_gpu(b)
    q = b.randn(b.T, H, hd).to(dtype)
    out, lse = step.attend(b.slot, q.cuda(), window=window, return_lse=True)
    torch.cuda.synchronize()
    check_attention(b, q, out, lse, b.max_kv, hd ** -0.5, window=window)
    old = b.randn(2, KVH, 21, hd)
    got = step.block_means(b.slot, old.cuda(), block=32)
    sel = step.select_blocks(q.cuda(), got, 5, block=32)
    torch.cuda.synchronize()
    assert torch.equal(got[0].cpu(), old[0])
    assert torch.equal(sel.cpu(), ref.select(b, q, got.cpu(), 5, 32, 1, 2))
    out, lse = step.attend_blocks(b.slot, q.cuda(), sel, block=32, return_lse=True)
    torch.cuda.synchronize()
    check_attention(b, q, out, lse, 160, hd ** -0.5, sel=sel.cpu(), block=32)
    before = step.cache.pool.clone()
    step.append(b.slot, b.randn(b.T, (H + 2 * KVH) * hd).to(dtype).cuda(), H)
    torch.cuda.synchronize()
    changed = (step.cache.pool != before).flatten(3).any(-1).any(1).any(0)
    assert changed.nonzero()[:, 0].tolist() == sorted({b.page(1, 38), b.page(1, 39)})


def test_binding_refuses_overlaps_gradients_and_numbers_out_of_range():
    b = ref.Batch(BF16, 4, 2, 64, [3], [40], seed=1)
    step = on_gpu(b)
    flat = torch.zeros(4000, dtype=BF16, device="cuda")
    qkv = flat[:3 * 600].view(3, 600)[:, :512]
    q = qkv[:, :256]
    gain = torch.nn.Parameter(torch.ones(64, dtype=BF16, device="cuda"))
    sel = torch.zeros(3, 2, 2, dtype=torch.int32, device="cuda")
    means = torch.zeros(1, 2, 2, 64, device="cuda")
    bad = [
        lambda: step.append(1, qkv, 4, out=flat[:768].view(3, 256)),  # the same start, other rows
        lambda: step.append(1, qkv, 4, out=qkv[:, 8:264]), lambda: step.append(1, qkv, 4, out=qkv[:, 256:]),
        lambda: step.append(1, qkv, 4, out=flat[600:].narrow(0, 0, 1800).view(3, 600)[:, :256]),
        lambda: step.append(1, qkv, 4, q_gain=gain), lambda: step.append(1 << 32, qkv, 4),
        lambda: step.attend(1, q, out=qkv[:, 128:384]), lambda: step.attend(1, q, out=flat[:768].view(3, 256)),
        lambda: step.attend(1, q, window=1 << 32), lambda: step.attend_blocks(1, q, sel, block=(1 << 32) + 32),
        lambda: step.attend_blocks(1, q, sel, block=32, out=qkv[:, 8:264]),
        lambda: step.select_blocks(q, means, 4, block=32, n_first=1 << 32),
        lambda: step.block_means(1, means, block=(1 << 32) + 32),
        lambda: paged.PagedBatch(step.cache, step.row_start, step.kv_len, (1 << 32) + 3, 40),
        lambda: paged.PagedCache(step.cache.pool.clone().requires_grad_(), 2, 64, step.table),
    ]
    for i, f in enumerate(bad):
        with pytest.raises(ValueError):
            f()
            pytest.fail(f"call {i} was not refused")
    with torch.no_grad():
        step.append(1, qkv, 4, q_gain=gain)
    # side by side in the same rows, and behind each other, are apart
    want = step.attend(1, q)
    assert torch.equal(step.attend(1, q, out=qkv[:, 256:]), want)
    assert torch.equal(step.attend(1, q, out=flat[1800:].narrow(0, 0, 768).view(3, 256)), want)


def test_thousands_of_sequences():
    """A search of three steps, with sequences without rows and runs of them."""
    say("thousands")
    n_seqs = 4200
    g = torch.Generator().manual_seed(5)
    rows = torch.randint(0, 3, (n_seqs,), generator=g)
    rows[100:400], rows[4100:] = 0, 0
    lens = (rows + torch.randint(0, 40, (n_seqs,), generator=g)).tolist()
    b = ref.Batch(F32, 1, 1, 64, rows.tolist(), lens, seed=5, pad=1)
    step = on_gpu(b)
    qkv = b.randn(b.T, 3 * 64)
    q = check_append(b, step, qkv, 10000.0, 1e-5, [None, None], None)
    b.pool = step.cache.pool.cpu()
    out, lse = step.attend(b.slot, q, return_lse=True)
    means = torch.zeros(n_seqs, 1, 2, 64, device="cuda")
    sel = step.select_blocks(q, step.block_means(b.slot, means, block=32), 2, block=32, n_first=0, n_last=1)
    some, some_lse = step.attend_blocks(b.slot, q, sel, block=32, return_lse=True)
    torch.cuda.synchronize()
    check_attention(b, q.cpu(), out, lse, b.max_kv, 0.125)
    want, mag = ref.means(b, torch.zeros(n_seqs, 1, 2, 64), 32)
    assert ((means.double().cpu() - want).abs() <= 7 * 2.0 ** -24 * mag).all()
    n = b.start[-1]
    assert torch.equal(sel[:n].cpu(), ref.select(b, q.cpu(), means.cpu(), 2, 32, 0, 1)[:n])
    check_attention(b, q.cpu(), some, some_lse, 64, 0.125, sel=sel.cpu(), block=32)


@pytest.mark.parametrize("dtype,H,KVH,hd", [(BF16, 8, 2, 128), (F32, 2, 1, 64)])
def test_empty_calls(dtype, H, KVH, hd):
    """No sequences, no rows, no positions, lengths below 0: outputs of rows with a sequence are those of an
    empty cache, others stay, and nothing enters the pool."""
    say("empty", dtype)
    b = ref.Batch(dtype, H, KVH, hd, [3, 2], [40, 20], seed=1)
    pool = b.pool.cuda()
    ints = lambda *v: torch.tensor(v, dtype=torch.int32, device="cuda")
    table = b.table.cuda()
    for n_seqs, rows, lens, max_kv in ((0, 5, (), 40), (2, 0, (40, 20), 40), (2, 5, (40, 20), 0), (2, 5, (-3, -2 ** 31), 40)):
        say(n_seqs, rows, lens, max_kv)
        cache = paged.PagedCache(pool, KVH, hd, table[:n_seqs])
        step = paged.PagedBatch(cache, ints(*[0, 3, 5][:n_seqs + 1]) if rows else ints(0, 0, 0), ints(*lens), rows, max_kv)
        qkv = b.randn(rows, (H + 2 * KVH) * hd).to(dtype).cuda()
        q = torch.full((rows, H, hd), 7.0, dtype=dtype, device="cuda")
        step.append(1, qkv, H, out=q)
        live = n_seqs and rows
        assert not live or (q != 7).any(-1).any(-1).all()
        means = torch.full((n_seqs, KVH, 2, hd), 7.0, device="cuda")
        sel = torch.full((rows, KVH, 4), 7, dtype=torch.int32, device="cuda")
        step.block_means(1, means, block=32)
        step.select_blocks(q, means, 4, block=32, out=sel)
        lists = torch.zeros_like(sel)
        outs = []
        for f in (lambda o: step.attend(1, q, out=o, return_lse=True), lambda o: step.attend(1, q, window=9, out=o, return_lse=True),
                  lambda o: step.attend_blocks(1, q, lists, block=32, out=o, return_lse=True)):
            outs.append(f(torch.full((rows, H, hd), 7.0, dtype=dtype, device="cuda")))
        torch.cuda.synchronize()
        assert (means == 7).all()
        if live:
            # with max_kv 0 a row has a position still, and sees no block of those that there are
            assert (sel == -1).all()
            assert all((o == 0).all() and (z == -math.inf).all() for o, z in outs)
        else:
            assert (sel == 7).all() and all((o == 7).all() for o, _ in outs)
    assert torch.equal(pool.cpu(), b.pool)


@pytest.mark.parametrize("rows,lens,max_kv", [([5000, 3600], [9000, 8300], 9000), ([8300, 2], [8300, 20000], 20000)])
def test_many_rows_of_sequences_too_large_to_split(rows, lens, max_kv):
    """More partial results than a call asks room for: spans are longer instead.  The last three rows of the
    first sequence and the last two of the other."""
    say("too large to split", rows, lens)
    H, KVH, hd = 64, 2, 128
    b = ref.Batch(BF16, H, KVH, hd, rows, lens, seed=rows[1])
    b.max_kv = max_kv
    step = on_gpu(b)
    assert via.via_paged_attend_bytes(C.byref(step.c), H, 0) == 0
    q = torch.randn((b.T, H, hd), dtype=torch.float32, generator=torch.Generator("cuda").manual_seed(1), device="cuda").to(BF16)
    out, lse = step.attend(b.slot, q, return_lse=True)
    torch.cuda.synchronize()
    at = [rows[0] - 3, rows[0] - 2, rows[0] - 1, b.T - 2, b.T - 1]
    b.rows, b.T, b.start = [3, 2], 5, [0, 3, 5]
    check_attention(b, q[at].cpu(), out[at], lse[at], max_kv, hd ** -0.5, p_bits=8)


def test_binding_refuses_forward_tangents():
    import torch.autograd.forward_ad as forward_ad
    b = ref.Batch(BF16, 4, 2, 64, [3], [40], seed=1)
    step = on_gpu(b)
    qkv, gain = torch.zeros(3, 512, dtype=BF16, device="cuda"), torch.ones(64, dtype=BF16, device="cuda")
    q, means = qkv[:, :256], torch.zeros(1, 2, 2, 64, device="cuda")
    sel = torch.zeros(3, 2, 4, dtype=torch.int32, device="cuda")
    with forward_ad.dual_level():
        dual = lambda t: forward_ad.make_dual(t, torch.ones_like(t))
        room = torch.zeros(3, 256, dtype=BF16, device="cuda")
        bad = [
            lambda: step.append(1, dual(qkv), 4), lambda: step.append(1, qkv, 4, q_gain=dual(gain)),
            lambda: step.append(1, qkv, 4, k_gain=dual(gain)), lambda: step.attend(1, dual(q)),
            lambda: step.attend(1, q, out=dual(room)), lambda: step.block_means(1, dual(means), block=32),
            lambda: step.select_blocks(dual(q), means, 4, block=32), lambda: step.select_blocks(q, dual(means), 4, block=32),
            lambda: step.attend_blocks(1, dual(q), sel, block=32), lambda: paged.PagedCache(dual(step.cache.pool), 2, 64, step.table),
        ]
        for i, f in enumerate(bad):
            with pytest.raises(ValueError):
                f()
                pytest.fail(f"call {i} was not refused")
        step.append(1, qkv, 4)  # tensors without a tangent are taken
        step.cache.pool.copy_(dual(step.cache.pool.clone()))
        with pytest.raises(ValueError):
            step.attend(1, q)


def test_binding_refuses_bounds_past_32_bits():
    b = ref.Batch(BF16, 4, 2, 64, [3], [40], seed=1)
    step = on_gpu(b)
    q = torch.ones(3, 4, 64, dtype=BF16, device="cuda")
    for max_kv in (-(1 << 32), -(1 << 31) - 1):  # (32 bits of the first: 0, an empty cache)
        with pytest.raises(ValueError):
            paged.PagedBatch(step.cache, step.row_start, step.kv_len, 3, max_kv)
    most = paged.PagedBatch(step.cache, step.row_start, step.kv_len, 3, 1 << 40)  # the table's columns bound it
    assert torch.equal(most.attend(1, q), step.attend(1, q))


@pytest.mark.parametrize("dtype,H,KVH,hd,rows,lens", [(BF16, 8, 2, 128, [3, 2], [40, 700]), (F32, 2, 1, 64, [3, 2], [40, 700]),
                                                      (BF16, 8, 2, 64, [60, 60], [60, 700])])
def test_scores_of_minus_infinity(dtype, H, KVH, hd, rows, lens):
    """Keys of -infinity have no weight; a row that sees no others gets zeros, as one that sees none."""
    say("minus infinity", dtype, H, KVH, hd, rows, lens)
    b = ref.Batch(dtype, H, KVH, hd, rows, lens, seed=lens[1])
    clean = b.pool.clone()
    k = b.pool[b.slot][:, :, 0].view(KVH, b.n_blocks, hd // 8, 16, 8)
    for pos in range(lens[0]):
        k[:, b.page(0, pos), 0, pos % 16, 0] = -math.inf
    for pos in range(lens[1] - 3):
        k[:, b.page(1, pos), 0, pos % 16, 0] = -math.inf
    q = b.randn(b.T, H, hd).to(dtype)
    q[:, :, 0] = 1.0
    out, lse = on_gpu(b).attend(b.slot, q.cuda(), return_lse=True)
    torch.cuda.synchronize()
    n = rows[0]
    assert (out[:n] == 0).all() and (lse[:n] == -math.inf).all()
    blind = n + rows[1] - 3 if rows[1] > 3 else n  # rows of the other that see only such keys
    assert (out[n:blind] == 0).all() and (lse[n:blind] == -math.inf).all()
    # the others see the last keys alone, as a window would have it
    b.pool = clean
    at = list(range(blind, b.T))
    last = ref.Batch(dtype, H, KVH, hd, rows, lens, seed=lens[1])
    last.rows, last.T, last.start, last.pool = [0, len(at)], len(at), [0, 0, len(at)], clean
    for i, t in enumerate(at):
        last.rows, last.T, last.start, last.lens = [0, 1], 1, [0, 0, 1], [lens[0], lens[1] - len(at) + 1 + i]
        window = last.lens[1] - (lens[1] - 3)
        check_attention(last, q[t:t + 1], out[t:t + 1], lse[t:t + 1], 3, hd ** -0.5, p_bits=weight_bits(b),
                        window=window)


def test_spans_longer_than_usual():
    """Partial results limited to fewer, longer spans: two of 15104 keys here instead of four."""
    say("longer spans")
    H, KVH, hd = 64, 2, 128
    rows, lens = [2500, 200], [30000, 9000]
    b = ref.Batch(BF16, H, KVH, hd, rows, lens, seed=4)
    step = on_gpu(b)
    assert via.via_paged_attend_bytes(C.byref(step.c), H, 0) == 2 * b.T * H * (hd + 2) * 4
    q = torch.randn((b.T, H, hd), dtype=torch.float32, generator=torch.Generator("cuda").manual_seed(2), device="cuda").to(BF16)
    out, lse = step.attend(b.slot, q, return_lse=True)
    torch.cuda.synchronize()
    at = [rows[0] - 2, rows[0] - 1, b.T - 2, b.T - 1]
    b.rows, b.T, b.start = [2, 2], 4, [0, 2, 4]
    check_attention(b, q[at].cpu(), out[at], lse[at], b.max_kv, hd ** -0.5, p_bits=8)
