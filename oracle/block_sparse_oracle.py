"""Block-sparse attention in 64 bits on the CPU, from the definition: every query against every key, with how often the key stands in the lists of
the query's tile.  Besides the values, how far a result may be off whose weights (and the terms of the gradients) were rounded to a type of unit
roundoff u: sums of the absolute values of the terms that are rounded."""
from __future__ import annotations

import torch


def positions(B, Nq, Nk, q_start):
    first = torch.full((B,), Nk - Nq) if q_start is None else q_start.long().cpu()
    return first[:, None] + torch.arange(Nq)


def held(B, Nk, key_len):
    return torch.full((B,), Nk) if key_len is None else key_len.long().cpu().clamp(0, Nk)


def key_means(k, kb, key_len=None):
    B, H, Nk, d = k.shape
    n = held(B, Nk, key_len)
    out = torch.zeros(B, H, -(-Nk // kb), d, dtype=torch.float64)
    for b in range(B):
        for j in range(out.shape[2]):
            part = k[b, :, j * kb:min((j + 1) * kb, int(n[b]))].double().cpu()
            if part.shape[1]:
                out[b, :, j] = part.mean(1)
    return out


def select(q, means, Nk, n_select, qb, kb, causal=False, q_start=None, key_len=None, keep_first=0, near=-1):
    """Lists as nested loops: tile by tile, block by block."""
    B, H, Nq, d = q.shape
    Hkv, Tk, T = means.shape[1], means.shape[2], -(-Nq // qb)
    n, pos = held(B, Nk, key_len), positions(B, Nq, Nk, q_start)
    out = torch.full((B, Hkv, T, n_select), -1, dtype=torch.int32)
    qd, md = q.double().cpu(), means.double().cpu()
    for b in range(B):
        for h in range(Hkv):
            for t in range(T):
                rows = qd[b, h * (H // Hkv):(h + 1) * (H // Hkv), t * qb:(t + 1) * qb]
                score = (md[b, h] @ rows.sum((0, 1))).tolist()
                lo, hi = int(pos[b, t * qb]), int(pos[b, min((t + 1) * qb, Nq) - 1])
                order = []
                for j in range(Tk):
                    if j * kb >= n[b] or (causal and j * kb > hi):
                        continue
                    forced = j < keep_first
                    if near >= 0:
                        forced = forced or (j * kb + kb - 1 >= lo - near and j * kb <= hi + (0 if causal else near))
                    order.append((0 if forced else 1, -score[j] if not forced else 0.0, j))
                best = sorted(j for _, _, j in sorted(order)[:n_select])
                out[b, h, t, :len(best)] = torch.tensor(best, dtype=torch.int32)
    return out


def attention(q, k, v, blocks, qb, kb, causal=False, q_start=None, key_len=None, scale=None, dout=None, u=0.0, u_logit=0.0, u_out=0.0):
    """Values and, with rounding units, error bounds: u of a weight or gradient term that enters a product, u_logit of every product behind a logit or
    dP, u_out of what is stored."""
    B, H, Nq, d = q.shape
    Hkv, Nk = k.shape[1], k.shape[2]
    G, Tk = H // Hkv, -(-Nk // kb)
    scale = d ** -0.5 if scale is None else scale
    n, pos = held(B, Nk, key_len), positions(B, Nq, Nk, q_start)
    f64 = dict(dtype=torch.float64)
    r = dict(out=torch.zeros(B, H, Nq, d, **f64), lse=torch.full((B, H, Nq), -torch.inf, **f64), out_tol=torch.zeros(B, H, Nq, d, **f64), lse_tol=torch.zeros(B, H, Nq, **f64))
    if dout is not None:
        for name, like in (("dq", q), ("dk", k), ("dv", v)):
            r[name], r[name + "_tol"] = torch.zeros(like.shape, **f64), torch.zeros(like.shape, **f64)
    for b in range(B):
        for h in range(H):
            hk = h // G
            count = torch.zeros(Nq, Nk, **f64)
            for t in range(blocks.shape[2]):
                for j in blocks[b, hk, t].tolist():
                    if 0 <= j < Tk:
                        count[t * qb:(t + 1) * qb, j * kb:(j + 1) * kb] += 1
            count[:, int(n[b]):] = 0
            if causal:
                count[torch.arange(Nk)[None, :] > pos[b][:, None]] = 0
            used = count > 0
            any_key, any_query = used.any(1), used.any(0)
            qh, kh, vh = q[b, h].double().cpu(), k[b, hk].double().cpu().clone(), v[b, hk].double().cpu().clone()
            kh[~any_query], vh[~any_query] = 0, 0                   # (nothing that no query sees takes part, not as 0 * NaN either)
            s = (qh @ kh.t()) * scale
            s[~used] = -torch.inf
            top = torch.where(any_key, s.amax(1) if Nk else torch.zeros(Nq, **f64), 0.0)
            w = count * torch.exp(s - top[:, None])
            l = w.sum(1)
            p = w / torch.where(any_key, l, 1.0)[:, None]
            r["out"][b, h], r["lse"][b, h] = p @ vh, torch.where(any_key, top + torch.log(l), -torch.inf)
            # a weight is off by the error of its logit (relatively) and by its own rounding
            e_s = u_logit * (qh.abs() @ kh.abs().t()) * scale + 2.0 ** -21 * (1 + torch.where(used, s, 0.0).abs() + top.abs()[:, None])
            e_p = p * (u + e_s)
            e_l = (p * e_s).sum(1, keepdim=True)
            r["lse_tol"][b, h] = e_l[:, 0] * 2 + 2.0 ** -22 * torch.where(any_key, r["lse"][b, h], 0.0).abs() + 2.0 ** -22
            r["out_tol"][b, h] = e_p @ vh.abs() + (e_l + 2.0 ** -20) * (p @ vh.abs()) + u_out * r["out"][b, h].abs() + u * (p @ vh.abs()) * u_logit
            if dout is None:
                continue
            do = dout[b, h].double().cpu().clone()
            do[~any_key] = 0
            dp = do @ vh.t()
            delta = (do * r["out"][b, h]).sum(1, keepdim=True)
            ds = p * (dp - delta)
            mag_dp = do.abs() @ vh.abs().t()
            e_delta = (do.abs() * (r["out_tol"][b, h] + 2.0 ** -20 * r["out"][b, h].abs())).sum(1, keepdim=True)
            e_w = p * (e_s + e_l + r["lse_tol"][b, h][:, None])     # of the recomputed weight, before it is rounded
            e_ds = u * ds.abs() + e_w * (dp - delta).abs() + p * ((u_logit + 2.0 ** -20) * mag_dp + e_delta)
            r["dq"][b, h], r["dq_tol"][b, h] = ds @ kh * scale, e_ds @ kh.abs() * scale * (1 + u_logit) + u_logit * (ds.abs() @ kh.abs()) * scale
            r["dk"][b, hk] += ds.t() @ qh * scale
            r["dk_tol"][b, hk] += (e_ds + (u_logit + 2.0 ** -20) * ds.abs()).t() @ qh.abs() * scale
            r["dv"][b, hk] += p.t() @ do
            r["dv_tol"][b, hk] += (e_w + (u + u_logit + 2.0 ** -20) * p).t() @ do.abs()
    if dout is not None:
        for name in ("dq", "dk", "dv"):
            r[name + "_tol"] += u_out * r[name].abs() + 2.0 ** -20 * r[name].abs()
    return r
