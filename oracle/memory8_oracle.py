"""fp64 oracle of the operators around the 8-bit key/value memory: rotary positions, rows quantised to
e4m3 codes with an e8m0 exponent byte each, and the two-view window attention over such a memory.

Written from the definitions in include/cover.h, one row at a time where that is clearer; it shares
no code with the kernels or the binding.
"""
import math

import numpy as np

# the 128 non-negative e4m3 values by code: 2^(e - 7) (1 + m / 8), subnormals m 2^-9; code 127 is NaN
E4M3 = np.array([(m * 2.0 ** -9 if e == 0 else 2.0 ** (e - 7) * (1 + m / 8)) for e in range(16) for m in range(8)])
E4M3[127] = math.nan


def rope(x, inv_freq, pos, *, interleaved, mscale=1.0, inverse=False):
    """x [B, H, L, D], inv_freq [R / 2], pos [B, L]."""
    y = np.array(x, dtype=np.float64)
    R = 2 * len(inv_freq)
    for i, f in enumerate(np.asarray(inv_freq, dtype=np.float64)):
        a, b = (2 * i, 2 * i + 1) if interleaved else (i, i + R // 2)
        # the reduced angle: positions are whole, so turns and radians reduce alike up to fp64 rounding
        angle = np.asarray(pos, dtype=np.float64)[:, None, :] * f * (-1.0 if inverse else 1.0)
        c, s = np.cos(angle), np.sin(angle)
        xa, xb = np.array(x[..., a], dtype=np.float64), np.array(x[..., b], dtype=np.float64)
        y[..., a], y[..., b] = mscale * (xa * c - xb * s), mscale * (xa * s + xb * c)
    return y


def encode_row(row):
    """(codes uint8 [D], byte) of one row."""
    row = np.asarray(row, dtype=np.float64)
    if not np.all(np.isfinite(row)):
        return np.zeros(len(row), np.uint8), 255
    top = np.abs(row).max()
    if top == 0:
        return (np.signbit(row) * 128).astype(np.uint8), 127
    x = 17
    while x < 246 and top > 448 * 2.0 ** (x - 127):
        x += 1
    y = np.minimum(np.abs(row) * 2.0 ** (127 - x), 448.0)
    # the nearest of the values; of two as near, the even code
    hi = np.searchsorted(E4M3[:127], y)
    hi = np.minimum(hi, 126)
    lo = np.maximum(hi - 1, 0)
    dl, dh = y - E4M3[lo], E4M3[hi] - y
    code = np.where(dh < dl, hi, np.where(dl < dh, lo, np.where(hi % 2 == 0, hi, lo)))
    return (code + 128 * np.signbit(row)).astype(np.uint8), x


def encode(x):
    """Codes and bytes of rows x [..., D]."""
    flat = np.asarray(x).reshape(-1, np.shape(x)[-1])
    rows = [encode_row(r) for r in flat]
    return (np.stack([c for c, _ in rows]).reshape(np.shape(x)),
            np.array([b for _, b in rows], np.uint8).reshape(np.shape(x)[:-1]))


def decode(codes, byte):
    """fp64 values of codes [..., D] and bytes [...]."""
    codes = np.asarray(codes)
    v = E4M3[codes & 127] * np.where(codes & 128, -1.0, 1.0)
    scale = np.where(np.asarray(byte) == 255, math.nan, 2.0 ** (np.asarray(byte, dtype=np.float64) - 127))
    return v * scale[..., None]


def written(mem, mem_exp, rows, *, pos=None, pos0=0):
    """The memory (codes [B, H, L, D], bytes [B, H, L]) after rows [B, H, n, D] were written."""
    mem, mem_exp = mem.copy(), mem_exp.copy()
    B, H, n, _ = rows.shape
    L = mem.shape[2]
    for b in range(B):
        named = set()
        for s in range(n):
            p = pos0 + s if pos is None else int(pos[b, s])
            if not 0 <= p < L or p in named:
                continue
            named.add(p)
            for h in range(H):
                mem[b, h, p], mem_exp[b, h, p] = encode_row(rows[b, h, s])
    return mem, mem_exp


def attention(q, k, v, km, vm, seed_idx, *, q0, key_lo=None, key_hi=None, softcap=0.0):
    """out, lse and two bounds for a tolerance: sum_j w_j |v_j| per output element, and per row the largest
    sum_i |q_i k_ji| / sqrt(D) over the keys it sees. q [B, Hq, Lq, D]; k, v [B, Hkv, Lk, D] values."""
    B, Hq, Lq, D = q.shape
    Hkv, Lk = k.shape[1], k.shape[2]
    out, mass = np.zeros((B, Hq, Lq, D)), np.zeros((B, Hq, Lq, D))
    lse, size = np.full((B, Hq, Lq), -math.inf), np.zeros((B, Hq, Lq))
    for b in range(B):
        slot = {}
        for s, p in enumerate([] if seed_idx is None else seed_idx[b]):
            slot.setdefault(int(p), s)
        for r in range(Lq):
            lo = 0 if key_lo is None else max(0, int(key_lo[b, r]))
            hi = Lk if key_hi is None else min(Lk, int(key_hi[b, r]))
            if lo >= hi:
                continue
            for hq in range(Hq):
                h = hq // (Hq // Hkv)
                kk, vv = k[b, h, lo:hi], v[b, h, lo:hi]
                p = q0 + r
                if p in slot and lo <= p < hi:
                    kk, vv = kk.copy(), vv.copy()
                    kk[p - lo], vv[p - lo] = km[b, h, slot[p]], vm[b, h, slot[p]]
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
