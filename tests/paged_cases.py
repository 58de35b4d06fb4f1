"""Batches over a paged cache and a plain float64 reference of the via_paged
operators (position by position, from the documented page layout), shared by
their tests."""
import math

import torch

PAGE = 16


class Batch:
    """Sequences with rows[s] new rows and len[s] cached positions (those included; a row of a
    shorter sequence has a negative position), pages shuffled over a pool of two layers."""

    def __init__(self, dtype, H, KVH, hd, rows, lens, seed=0, pad=0, spare=2, slot=1, device="cpu"):
        g = torch.Generator().manual_seed(seed)
        self.g, self.dtype, self.H, self.KVH, self.hd, self.slot = g, dtype, H, KVH, hd, slot
        self.rows, self.lens, self.pad = list(rows), list(lens), pad
        self.T = sum(rows) + pad
        need = [-(-n // PAGE) for n in lens]
        self.n_blocks = sum(need) + 3
        order = torch.randperm(self.n_blocks, generator=g).tolist()
        self.table = torch.full((len(rows), max(need + [0]) + spare), -1, dtype=torch.int32)
        for s, n in enumerate(need):
            for j in range(n):
                self.table[s, j] = order.pop()
        self.pool = torch.randn((2, KVH, self.n_blocks, 2, PAGE * hd), generator=g).to(dtype)
        self.start = [0]
        for n in rows:
            self.start.append(self.start[-1] + n)
        self.row_start = torch.tensor(self.start, dtype=torch.int32)
        self.kv_len = torch.tensor(lens, dtype=torch.int32)
        self.max_kv = max(list(lens) + [1])

    def randn(self, *shape):
        return torch.randn(shape, generator=self.g)

    def positions(self):
        """(row, sequence, position) of every row that belongs to a sequence."""
        for s, (n, ln) in enumerate(zip(self.rows, self.lens)):
            for r in range(n):
                yield self.start[s] + r, s, ln - n + r

    def page(self, s, pos):
        if pos < 0 or pos >= self.max_kv or pos // PAGE >= self.table.shape[1]:
            return None
        p = int(self.table[s, pos // PAGE])
        return p if 0 <= p < self.n_blocks else None

    def cached(self, s, pool=None):
        """Keys and values [n, KVH, hd] (float64) and which positions have a page."""
        pool = (self.pool if pool is None else pool)[self.slot].cpu()
        n = min(self.lens[s], self.max_kv)
        k = torch.zeros((n, self.KVH, self.hd), dtype=torch.float64)
        v, have = torch.zeros_like(k), torch.zeros(n, dtype=torch.bool)
        kp = pool[:, :, 0].view(self.KVH, self.n_blocks, self.hd // 8, PAGE, 8)
        vp = pool[:, :, 1].view(self.KVH, self.n_blocks, self.hd, PAGE)
        for j in range(-(-n // PAGE)):
            p = self.page(s, j * PAGE)
            m = min(PAGE, n - j * PAGE)
            if p is not None:
                at = slice(j * PAGE, j * PAGE + m)
                have[at] = True
                k[at] = kp[:, p].permute(2, 0, 1, 3).reshape(PAGE, self.KVH, self.hd)[:m].double()
                v[at] = vp[:, p].permute(2, 0, 1)[:m].double()
        return k, v, have


def see(b, s, r, pos, n_keys, window, mask):
    """Positions that row r (of its sequence) at ``pos`` sees."""
    key = torch.arange(n_keys)
    if mask is None:
        seen = key <= pos
        return seen & (key > pos - window) if window else seen
    base = b.lens[s] - b.rows[s]
    bits = int(mask) & ((1 << 64) - 1)
    own = torch.tensor([0 <= k - base < min(64, b.rows[s]) and (bits >> (k - base)) & 1 == 1 for k in range(n_keys)],
                       dtype=torch.bool)
    return (key < base) | own


def attend(b, q, scale, window=0, masks=None, sel=None, block=0):
    """out, lse, and the error bounds' ingredients: sum of p |v| and the largest scale sum |q k| of a row."""
    T, H, hd = q.shape
    G = H // b.KVH
    out, lse = torch.zeros((T, H, hd), dtype=torch.float64), torch.full((T, H), -math.inf, dtype=torch.float64)
    pv, amp = torch.zeros_like(out), torch.zeros_like(lse)
    kv = {s: b.cached(s) for s in range(len(b.rows))}
    for t, s, pos in b.positions():
        k, v, have = kv[s]
        for g in range(b.KVH):
            if sel is None:
                idx = torch.nonzero(see(b, s, t - b.start[s], pos, len(have), window, None if masks is None else masks[t])
                                    & have)[:, 0]
            else:
                idx = [i for e in sel[t, g].tolist() if e >= 0 for i in range(e * block, (e + 1) * block)
                       if i <= pos and i < len(have) and have[i]]
                idx = torch.tensor(idx, dtype=torch.long)
            if len(idx) == 0:
                continue
            for h in range(g * G, (g + 1) * G):
                qq = q[t, h].double().cpu()
                z = k[idx, g] @ qq * scale
                p = torch.softmax(z, 0)
                out[t, h], lse[t, h] = p @ v[idx, g], torch.logsumexp(z, 0)
                pv[t, h] = p @ v[idx, g].abs()
                amp[t, h] = (k[idx, g].abs() @ qq.abs()).max() * scale
    return out, lse, pv, amp


def bounds(dtype, hd, n, ref, lse, pv, amp, p_bits):
    """Error bounds of attention over at most n keys.  A score is a dot product of hd terms and a
    product, in 32 bits: (hd + 4) 2^-24 amp, and an exponential as far off relatively, twice (weight
    and sum).  Weights are held to p_bits bits; sums of n terms in 32 bits; one rounding at the end."""
    d = (hd + 4) * 2.0 ** -24 * amp[..., None] + 2.0 ** -22
    rel = 2 * d + (n + 8) * 2.0 ** -24 + 2.0 ** -p_bits
    out = torch.finfo(dtype).eps / 2 * ref.abs() * (1 + rel) + rel * pv + 1e-30
    z = d[..., 0] + (n + 8) * 2.0 ** -24 + 2.0 ** -22 * lse.abs()
    return out, z


def append(b, qkv, theta, eps, q_gain, k_gain, pos=None):
    """Rotated queries [T, H, hd] of the sequences' rows, pool after the append (both float64), and the
    magnitude of the rotated pair behind every entry."""
    T, H, KVH, hd = b.T, b.H, b.KVH, b.hd
    x = qkv.double().cpu().view(T, H + 2 * KVH, hd)
    half = hd // 2
    q, mag = torch.zeros((T, H, hd), dtype=torch.float64), torch.zeros((T, H, hd), dtype=torch.float64)
    pool, pool_mag = b.pool.double().cpu(), torch.zeros(b.pool.shape, dtype=torch.float64)
    pool_mag = pool_mag.view(2, KVH, b.n_blocks, 2, PAGE * hd)
    freq = torch.tensor([theta ** (-2.0 * i / hd) for i in range(half)], dtype=torch.float64)
    d = torch.arange(hd)
    for t, s, p in b.positions():
        a = freq * float(pos[t] if pos is not None else p)
        c, sn = torch.cos(a), torch.sin(a)

        def turn(y, gain):
            if gain is not None:
                y = y / torch.sqrt((y * y).mean(-1, keepdim=True) + eps) * gain.double().cpu()
            y1, y2 = y[:, :half], y[:, half:]
            m = torch.sqrt(y1 * y1 + y2 * y2)
            return torch.cat([y1 * c - y2 * sn, y2 * c + y1 * sn], -1), torch.cat([m, m], -1)

        q[t], mag[t] = turn(x[t, :H], q_gain)
        page = b.page(s, p)
        if page is not None:
            k, km = turn(x[t, H:H + KVH], k_gain)
            at_k, at_v = (d // 8) * 128 + (p % PAGE) * 8 + d % 8, d * PAGE + p % PAGE
            pool[b.slot, :, page, 0][:, at_k] = k
            pool_mag[b.slot, :, page, 0][:, at_k] = km
            pool[b.slot, :, page, 1][:, at_v] = x[t, H + KVH:]
    return q, mag, pool, pool_mag


def means(b, old, block):
    """Mean keys of completed blocks over ``old`` (float64), and the mean of |k| (0 where untouched)."""
    m, mag = old.double().cpu().clone(), torch.zeros(old.shape, dtype=torch.float64)
    for s, (n, ln) in enumerate(zip(b.rows, b.lens)):
        k, _, have = b.cached(s)
        for i in range(max(ln - n, 0) // block, min(ln, b.max_kv) // block):
            if i < old.shape[2] and bool(have[i * block:(i + 1) * block].all()):
                m[s, :, i] = k[i * block:(i + 1) * block].mean(0)
                mag[s, :, i] = k[i * block:(i + 1) * block].abs().mean(0)
    return m, mag


def select(b, q, means, n_sel, block, n_first, n_last):
    T, H, hd = q.shape
    sel = torch.full((T, b.KVH, n_sel), -1, dtype=torch.int32)
    for t, s, pos in b.positions():
        last = min(pos, b.max_kv - 1) // block
        for g in range(b.KVH):
            if pos < 0:
                continue
            qq = q[t].double().cpu().view(b.KVH, -1, hd)[g].sum(0)
            order = []
            for i in range(last + 1):
                keep = i < n_first or i > last - n_last
                z = float((qq * means[s, g, i].double().cpu()).sum())
                order.append((0 if keep else 1 if z == z else 2, 0.0 if keep or z != z else -z, i))
            pick = sorted(i for _, _, i in sorted(order)[:n_sel])
            sel[t, g, :len(pick)] = torch.tensor(pick, dtype=torch.int32)
    return sel
