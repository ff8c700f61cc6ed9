"""fp64 oracle of the memory in pages and of the log probabilities of given tokens.

Written from the definitions in include/cover.h, one row at a time; it shares no code with the kernels or the binding.
"""
import math

import numpy as np

from . import memory8_oracle as M8


def appended(pages, table, rows, *, start=None, count=None, pos=None):
    """The pages [n_pages, H, page, D] after rows [B, H, n, D] were written."""
    pages = np.array(pages, dtype=np.float64)
    n_pages, _, page, _ = pages.shape
    B, _, n, _ = rows.shape
    for b in range(B):
        named = set()
        for s in range(n):
            if pos is None:
                if count is not None and s >= count[b]:
                    continue
                p = int(start[b]) + s
            else:
                p = int(pos[b, s])
            if p in named:
                continue
            named.add(p)
            if not 0 <= p < table.shape[1] * page:
                continue
            entry = int(table[b, p // page])
            if 0 <= entry < n_pages:
                pages[entry, :, p % page] = rows[b, :, s]
    return pages


def turned(x, inv_freq, at, *, interleaved, mscale=1.0):
    """x [B, H, n, D] turned by the positions at [B, n]."""
    return M8.rope(x, inv_freq, at, interleaved=interleaved, mscale=mscale)


def sequence(pages, table_row, h, n):
    """(rows [n, D], held [n]) of a KV head's first n positions; rows without a page are zeros and not held."""
    n_pages, _, page, D = pages.shape
    rows, held = np.zeros((n, D)), np.zeros(n, bool)
    for j in range(n):
        entry = int(table_row[j // page])
        if 0 <= entry < n_pages:
            rows[j], held[j] = pages[entry, h, j % page], True
    return rows, held


def attention(q, k_pages, v_pages, table, lens, km, vm, seed_idx, *, q0=None, key_lo=None, key_hi=None, softcap=0.0):
    """out, lse and two bounds for a tolerance, as memory8_oracle.attention: sum_j w_j |v_j| per output element, and per row the
    largest sum_i |q_i k_ji| / sqrt(D) over the keys it sees."""
    B, Hq, Lq, D = q.shape
    Hkv, page = k_pages.shape[1], k_pages.shape[2]
    G = Hq // Hkv
    out, mass = np.zeros((B, Hq, Lq, D)), np.zeros((B, Hq, Lq, D))
    lse, size = np.full((B, Hq, Lq), -math.inf), np.zeros((B, Hq, Lq))
    for b in range(B):
        n = max(0, min(int(lens[b]), table.shape[1] * page))
        slot = {}
        for s, p in enumerate([] if seed_idx is None else seed_idx[b]):
            slot.setdefault(int(p), s)
        for h in range(Hkv):
            k_all, held = sequence(k_pages, table[b], h, n)
            v_all, _ = sequence(v_pages, table[b], h, n)
            for r in range(Lq):
                lo = 0 if key_lo is None else max(0, int(key_lo[b, r]))
                hi = n if key_hi is None else min(n, int(key_hi[b, r]))
                seen = held.copy()
                seen[:min(lo, n)] = False
                seen[max(hi, 0):] = False
                if not seen.any():
                    continue
                kk, vv = k_all, v_all
                p = int(q0[b]) + r if q0 is not None else -1
                if p in slot and 0 <= p < n:
                    kk, vv = kk.copy(), vv.copy()
                    kk[p], vv[p] = km[b, h, slot[p]], vm[b, h, slot[p]]
                kk, vv = kk[seen], vv[seen]
                for g in range(G):
                    hq = h * G + g
                    z = kk @ q[b, hq, r] / math.sqrt(D)
                    size[b, hq, r] = (np.abs(kk) @ np.abs(q[b, hq, r])).max() / math.sqrt(D)
                    if softcap > 0:
                        z = softcap * np.tanh(z / softcap)
                    m = z.max()
                    w = np.exp(z - m)
                    lse[b, hq, r] = m + math.log(w.sum())
                    w /= w.sum()
                    out[b, hq, r], mass[b, hq, r] = w @ vv, w @ np.abs(vv)
    return out, lse, mass, size


def logprob(x, tok, K):
    """logp, entropy, lse [N], top_idx, top_logp [N, K] of rows x [N, V]."""
    N, V = x.shape
    logp, ent, lse = np.zeros(N), np.zeros(N), np.zeros(N)
    idx, top = np.full((N, K), -1, np.int32), np.full((N, K), -math.inf)
    for i in range(N):
        m = x[i].max()
        if m == -math.inf:
            lse[i], ent[i] = -math.inf, math.nan
            logp[i] = math.nan if 0 <= tok[i] < V else 0.0
            best = range(min(K, V))
            idx[i, :len(best)], top[i, :len(best)] = list(best), math.nan
            continue
        e = np.exp(x[i] - m)
        lse[i] = m + math.log(e.sum())
        p = e / e.sum()
        ent[i] = -(p[p > 0] * np.log(p[p > 0])).sum()
        if 0 <= tok[i] < V:
            logp[i] = (x[i, tok[i]] - m) - math.log(e.sum())
        best = sorted(range(V), key=lambda j: (-x[i, j], j))[:K]
        idx[i, :len(best)] = best
        top[i, :len(best)] = (x[i, best] - m) - math.log(e.sum())
    return logp, ent, lse, idx, top


def logprob_grad(x, lse, *, tok=None, d_logp=None, ent=None, d_ent=None, d_lse=None, idx=None, d_top=None):
    """The gradient of sum_i (d_logp log p(tok) + d_ent H + d_lse lse + sum_k d_top_k log p(idx_k)) in x, with the given lse, ent;
    and a bound for its terms: p (|d_lse| + |d_logp| + sum |d_top| + |d_ent| (|ln p| + |H|)) and the named shares."""
    N, V = x.shape
    d, size = np.zeros((N, V)), np.zeros((N, V))
    for i in range(N):
        lp = x[i] - lse[i]
        p = np.exp(lp)
        lp = np.where(p > 0, lp, 0.0)
        terms = [] if d_lse is None else [(None, -d_lse[i])]
        if d_logp is not None and 0 <= tok[i] < V:
            terms.append((int(tok[i]), d_logp[i]))
        if d_top is not None:
            terms += [(int(j), g) for j, g in zip(idx[i], d_top[i]) if 0 <= j < V]
        for j, g in terms:
            d[i] -= p * g
            size[i] += p * abs(g)
            if j is not None:
                d[i, j] += g
                size[i, j] += abs(g)
        if d_ent is not None:
            d[i] -= d_ent[i] * p * (lp + ent[i])
            size[i] += abs(d_ent[i]) * p * (np.abs(lp) + abs(ent[i]))
    return d, size
