"""Attention of new tokens over paged caches, the weights of the slots and eviction, in 64 bits from their definitions, with how far the kernels may be off.

u = 2^-24 is half a step of fp32.  A logit is a sum of d products (fp32 tensors: six products of pieces for one, 5 u) in fp32; it is scaled, and the maximum is taken from it.
A weight below fp32's smallest normal number, 2^-126, may come out as 0.  Weights are rounded to bf16 for bf16 tensors (2^-8 of each) or split into pieces (5 u).  Sums over the slots: eight to a matrix instruction's half, then one after the other."""
import torch

U = 2.0 ** -24


def rows_of(b, q_offset, max_new, T):
    if q_offset is None:
        return b * max_new, (b + 1) * max_new
    lo, hi = (min(max(int(q_offset[i]), 0), T) for i in (b, b + 1))
    return lo, max(lo, hi)


def stored(pages, table, n, h, n_pages):
    """(rows [n, d] in 64 bits, which of them there are) of one sequence and key head."""
    page = pages.shape[2]
    slot = torch.arange(n)
    at = table[slot // page].long() if n else slot
    there = (at >= 0) & (at < n_pages)
    rows = pages[torch.where(there, at, 0), h, slot % page].double() if n_pages and n else torch.zeros((n, pages.shape[3]), dtype=torch.float64)
    return torch.where(there[:, None], rows, 0.0), there


def attention(q, k_pages, v_pages, table, key_len, q_offset, max_new, causal, scale, bf16):
    """{out, lse, weights} with {name}_off, all fp64 on the CPU; rows of no sequence NaN.  weights [B, Hkv, slots] are what this attention gives."""
    q, k_pages, v_pages, table, key_len = (t.cpu() for t in (q, k_pages, v_pages, table, key_len))
    q_offset = None if q_offset is None else q_offset.cpu()
    T, H, d = q.shape
    n_pages, Hkv, page, _ = k_pages.shape
    B, slots = table.shape[0], table.shape[1] * page
    out, lse = torch.full((T, H, d), float("nan"), dtype=torch.float64), torch.full((T, H), float("nan"), dtype=torch.float64)
    out_off, lse_off = torch.zeros_like(out), torch.zeros_like(lse)
    weights = torch.zeros((B, Hkv, slots), dtype=torch.float64)
    weights_off = torch.zeros_like(weights)
    for b in range(B):
        lo, hi = rows_of(b, q_offset, max_new, T)
        n, new = min(max(int(key_len[b]), 0), slots), hi - lo
        hi = min(hi, lo + max_new)
        for h in range(Hkv):
            k, there = stored(k_pages, table[b], n, h, n_pages)
            v, _ = stored(v_pages, table[b], n, h, n_pages)
            heads = range(h * (H // Hkv), (h + 1) * (H // Hkv))
            x = q[lo:hi, heads.start:heads.stop].double()
            s = torch.einsum("ihd,jd->ihj", x, k) * scale
            size = torch.einsum("ihd,jd->ihj", x.abs(), k.abs()) * scale
            see = there.expand(hi - lo, n)
            if causal:
                see = see & (torch.arange(n) <= (n - new + torch.arange(hi - lo))[:, None])
            see = see[:, None].expand(s.shape)
            s = torch.where(see, s, -torch.inf)
            some = see.any(2)
            total = torch.logsumexp(s, 2) if n else torch.full(s.shape[:2], -torch.inf, dtype=torch.float64)
            p = torch.where(see, torch.exp(s - torch.where(some, total, 0.0)[..., None]), 0.0)
            size = torch.where(see, size, 0.0)
            # how far a weight is off, relative to itself
            e = (size.amax(2) if n else torch.zeros_like(total)) * (d + 8 + 5 + 8) * U + 8 * U
            sums = (n / 8 + 64) * U
            out[lo:hi, heads.start:heads.stop] = torch.einsum("ihj,jd->ihd", p, v)
            spread = torch.einsum("ihj,jd->ihd", p, v.abs())
            out_off[lo:hi, heads.start:heads.stop] = spread * (2 * e[..., None] + (2.0 ** -8 if bf16 else 10 * U) + 2 * sums) + out[lo:hi, heads.start:heads.stop].abs() * (2.0 ** -8 if bf16 else U)
            lse[lo:hi, heads.start:heads.stop] = total
            off = e + sums + torch.where(some, total, 0.0).abs() * 4 * U
            lse_off[lo:hi, heads.start:heads.stop] = off
            weights[b, h, :n] = p.sum((0, 1))
            weights_off[b, h, :n] = (p * (2 * e + off + 16 * U)[..., None]).sum((0, 1)) + (p.shape[0] * p.shape[1] / 8 + 64) * U * p.sum((0, 1)) + p.shape[0] * p.shape[1] * 2.0 ** -126
    return dict(out=out, out_off=out_off, lse=lse, lse_off=lse_off, weights=weights, weights_off=weights_off)


def evict(k_pages, v_pages, weights, table, key_len, keep, out_table, first, last):
    """(k_pages, v_pages, key_len, weights, kept) afterwards; the pools as they are, not in 64 bits."""
    k_out, v_out, table, out_table = k_pages.clone(), v_pages.clone(), table.tolist(), out_table.tolist()
    n_pages, Hkv, page, _ = k_pages.shape
    slots = weights.shape[2]
    len_out, kept, w_out = key_len.clone(), torch.full((len(table), Hkv, keep), -1, dtype=torch.int32), torch.zeros_like(weights)
    for b in range(len(table)):
        n = min(max(int(key_len[b]), 0), slots)
        len_out[b] = min(n, keep)
        for h in range(Hkv):
            w = weights[b, h].tolist()
            rank = sorted(range(n), key=lambda j: (0 if j < first or j >= n - last else 1, 0 if w[j] != w[j] else 1, -w[j] if w[j] == w[j] else 0.0, j))
            for i, j in enumerate(sorted(rank[:keep])):
                kept[b, h, i], w_out[b, h, i] = j, weights[b, h, j]
                to, at = out_table[b][i // page], table[b][j // page]
                if 0 <= to < n_pages:
                    for out, pool in ((k_out, k_pages), (v_out, v_pages)):
                        out[to, h, i % page] = pool[at, h, j % page] if 0 <= at < n_pages else 0
    return k_out, v_out, len_out, w_out, kept
