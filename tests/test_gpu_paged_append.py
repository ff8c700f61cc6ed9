"""GPU parity of appending to a memory in pages against the fp64 oracle."""
import math

import numpy as np
import pytest
import torch

from oracle import paged_oracle as PO
from paper_2602_06161_gb300 import CoverError, api

pytestmark = pytest.mark.gpu

BF, F32 = torch.bfloat16, torch.float32
EPS = {BF: 2.0 ** -8, F32: 2.0 ** -24}   # half a step
TYPES = pytest.mark.parametrize("dtype", [BF, F32])


def _gen(seed):
    return torch.Generator("cuda").manual_seed(seed)


def _rows(B, H, n, D, dtype, seed=0):
    return torch.randn((B, n, H, D), generator=_gen(seed), device="cuda").to(dtype).transpose(1, 2)


def _pool(lens, H, page, D, seed=9, extra=2):
    need = [-(-n // page) for n in lens]
    n_pages, M = sum(need) + extra, max(max(need), 1)
    order = torch.randperm(n_pages, generator=_gen(seed), device="cuda").to(torch.int32)
    table, at = torch.full((len(lens), M), -1, device="cuda", dtype=torch.int32), 0
    for b, n in enumerate(need):
        table[b, :n] = order[at:at + n]
        at += n
    k, v = (torch.randn((n_pages, H, page, D), generator=_gen(seed + i), device="cuda").to(BF) for i in (1, 2))
    return k, v, table


def _h(t):
    return t.double().cpu().numpy() if t.is_floating_point() else t.cpu().numpy()


def _ints(x):
    return torch.tensor(x, device="cuda", dtype=torch.int32)


def _turn_tolerance(x, R, inter, mscale, dtype):
    """Per element: half a step of the result's type, and the fp32 arithmetic relative to the pair's |a| + |b|: the reduced angle (2^-26
    turns from its conversion, an fp64 frequency's 2^-53 of at most 2^20 turns), sincospif (2 steps), the factor, the two
    products and their sum."""
    pair = np.abs(_h(x))
    i = np.arange(R // 2)
    lo, hi = (2 * i, 2 * i + 1) if inter else (i, i + R // 2)
    if R:
        pair[..., lo] = pair[..., hi] = pair[..., lo] + pair[..., hi]
    fp32 = 2 * math.pi * (2.0 ** -26 + 2.0 ** -33) + 10 * 2.0 ** -24
    tol = mscale * pair * ((1 + EPS[dtype]) * fp32 + EPS[dtype])
    tol[..., R:] = np.abs(_h(x))[..., R:] * EPS[dtype]
    return tol


def _check(k, v, q, kp, vp, table, f, inter, mscale, **where):
    """Appends, and compares the pages, q and k with the oracle's."""
    old_k, old_v = kp.clone(), vp.clone()
    rope_pos = where.get("rope_pos")
    yq, yk = api.cover_paged_append(k, v, kp, vp, table, q=q, inv_freq=f, interleaved=inter, mscale=mscale, want_k=True, **where)
    torch.cuda.synchronize()
    assert api.cover_device_status() == 0
    given = {n: None if where.get(n) is None else _h(where[n]) for n in ("start", "count", "pos")}
    n, R = k.shape[2], 0 if f is None else 2 * len(f)
    at = _h(rope_pos) if rope_pos is not None else given["pos"] if given["pos"] is not None else given["start"][:, None] + np.arange(n)
    turn = lambda x: _h(x) if f is None else PO.turned(_h(x), _h(f), at, interleaved=inter, mscale=mscale)  # noqa: E731
    rk = turn(k)
    # the pages: those written within the rounding, the others as they were
    marks = PO.appended(np.zeros(old_k.shape[:3] + (1,)), _h(table), np.ones(k.shape[:3] + (1,)), **given) != 0
    tol = PO.appended(np.zeros(old_k.shape), _h(table), _turn_tolerance(k, R, inter, mscale, BF), **given)
    ref = PO.appended(_h(old_k), _h(table), rk, **given)
    assert (np.abs(_h(kp) - ref) <= tol).all()
    want_v = PO.appended(_h(old_v), _h(table), _h(v.to(BF)), **given)
    assert np.array_equal(_h(vp), want_v)
    assert torch.equal(kp[~torch.from_numpy(marks[..., 0]).cuda()], old_k[~torch.from_numpy(marks[..., 0]).cuda()])
    assert yk.is_contiguous() and yk.dtype == k.dtype and (np.abs(_h(yk) - rk) <= _turn_tolerance(k, R, inter, mscale, k.dtype)).all()
    if q is None:
        assert yq is None
    else:
        assert yq.is_contiguous() and yq.shape == q.shape
        assert (np.abs(_h(yq) - turn(q)) <= _turn_tolerance(q, R, inter, mscale, q.dtype)).all()


@TYPES
@pytest.mark.parametrize("inter", [False, True])
@pytest.mark.parametrize("B,Hq,Hkv,n,D,R,page", [
    (1, 1, 1, 1, 64, 64, 16), (3, 28, 4, 1, 128, 128, 16), (2, 6, 2, 37, 64, 32, 32), (2, 4, 4, 130, 128, 64, 64), (1, 0, 3, 300, 128, 128, 256),
    (2, 5, 1, 17, 128, 6, 128), (1, 40, 8, 200, 128, 128, 16), (2, 2, 1, 9, 64, 0, 16), (5, 32, 32, 33, 64, 64, 32),
])
def test_against_oracle(B, Hq, Hkv, n, D, R, page, inter, dtype):
    k, v = _rows(B, Hkv, n, D, dtype), _rows(B, Hkv, n, D, dtype, 1)
    q = _rows(B, Hq, n, D, dtype, 2) if Hq else None
    f = api.rope_frequencies(R)[0] if R else None
    start = [(31 * b + 5) % 70 for b in range(B)]
    count = [max(0, n - 3 * b) for b in range(B)]
    for c in (None, count):
        kp, vp, table = _pool([s + n for s in start], Hkv, page, D)
        _check(k, v, q, kp, vp, table, f, inter, 1.25, start=_ints(start), count=None if c is None else _ints(c))
    kp, vp, table = _pool([s + n for s in start], Hkv, page, D)
    pos = torch.randint(-2, table.shape[1] * page + 2, (B, n), generator=_gen(5), device="cuda").int()   # many named twice
    _check(k, v, q, kp, vp, table, f, inter, 1.0, pos=pos)
    _check(k, v, q, kp, vp, table, f, inter, 1.0, pos=pos, rope_pos=pos * 7 - 3)


@TYPES
def test_places_that_do_not_exist(dtype):
    """Positions before the memory and behind the table, entries that are no pages, counts of any value."""
    kp, vp, table = _pool([60, 60, 60, 60], 2, 16, 64)
    table[0, 1], table[1, 0], table[2, 2] = -7, kp.shape[0], 2 ** 31 - 1
    k, v = _rows(4, 2, 40, 64, dtype), _rows(4, 2, 40, 64, dtype, 1)
    f, _ = api.rope_frequencies(64)
    for start, count in (([3, 10, 20, 50], None), ([-5, -39, 63, 64], None), ([0, 0, 0, 0], [-1, 0, 41, 2 ** 31 - 1])):
        _check(k, v, None, kp, vp, table, f, False, 1.0, start=_ints(start), count=None if count is None else _ints(count))
    # the ends of int32 (the angles there are tested with the rotation itself)
    old = kp.clone(), vp.clone()
    api.cover_paged_append(k, v, kp, vp, table, start=_ints([2 ** 31 - 1, -2 ** 31, 2 ** 31 - 20, -2 ** 31 + 30]))
    assert torch.equal(kp, old[0]) and torch.equal(vp, old[1])


@pytest.mark.parametrize("shift", [0, 1, 3])
@pytest.mark.parametrize("inter", [False, True])
def test_unaligned_rows(shift, inter):
    flat = torch.randn(shift + 2 * 3 * 5 * 64, generator=_gen(5), device="cuda").to(BF)
    x = flat[shift:].view(2, 3, 5, 64)
    f, _ = api.rope_frequencies(64)
    got = []
    for k in (x, x.clone()):
        kp, vp, table = _pool([20, 20], 3, 16, 64)
        got.append((kp, vp, *api.cover_paged_append(k, k, kp, vp, table, start=_ints([3, 9]), q=k, inv_freq=f, interleaved=inter, want_k=True)))
    for a, b in zip(*got):
        assert torch.equal(a, b)


def test_rows_of_one_projection_and_as_rope_turns_them():
    """q, k and v are views of one [B, n, (Hq + 2 Hkv) D] projection; the results are cover_rope_fwd's."""
    B, Hq, Hkv, n, D = 2, 6, 2, 19, 128
    qkv = torch.randn((B, n, Hq + 2 * Hkv, D), generator=_gen(4), device="cuda").to(BF)
    q, k, v = (qkv[:, :, a:b].transpose(1, 2) for a, b in ((0, Hq), (Hq, Hq + Hkv), (Hq + Hkv, Hq + 2 * Hkv)))
    f, m = api.rope_frequencies(D, scaling="yarn", factor=8.0)
    kp, vp, table = _pool([64, 64], Hkv, 16, D)
    yq, yk = api.cover_paged_append(k, v, kp, vp, table, start=_ints([7, 7]), q=q, inv_freq=f, mscale=m, want_k=True)
    rq, rk = api.cover_rope_fwd(q, k, f, pos0=7, mscale=m)
    assert torch.equal(yq, rq) and torch.equal(yk, rk)
    at = torch.arange(7, 7 + n, device="cuda")
    for b in range(B):
        pages = table[b, at // 16].long()
        assert torch.equal(kp[pages, :, at % 16], rk[b].transpose(0, 1)) and torch.equal(vp[pages, :, at % 16], v[b].transpose(0, 1))


def test_frequencies_that_are_not_finite():
    f, _ = api.rope_frequencies(64)
    f[3] = math.nan
    f[7] = math.inf
    k = _rows(1, 1, 5, 64, BF)
    kp, vp, table = _pool([16], 1, 16, 64)
    api.cover_paged_append(k, k, kp, vp, table, start=_ints([2]), inv_freq=f)
    rows = kp[int(table[0, 0]), 0, 2:7]
    bad = torch.zeros(64, dtype=torch.bool)
    bad[[3, 35, 7, 39]] = True
    assert rows[:, bad].isnan().all() and not rows[:, ~bad].isnan().any()
    assert torch.equal(vp[int(table[0, 0]), 0, 2:7], k[0, 0])


def test_no_rows_and_refusals():
    kp, vp, table = _pool([20, 20], 2, 16, 64)
    k = _rows(2, 2, 3, 64, BF)
    start = _ints([0, 1])
    empty = k[:, :, :0]
    q, kk = api.cover_paged_append(empty, empty, kp, vp, table, start=start, q=empty, want_k=True)
    assert q.shape == kk.shape == (2, 2, 0, 64)
    a = api.cover_paged_append
    for kw, err in ((dict(), ValueError), (dict(start=start, pos=_ints([[0] * 3] * 2)), ValueError), (dict(pos=_ints([[0] * 3] * 2), count=start), ValueError),
                    (dict(start=start[:1]), ValueError), (dict(start=start.long()), TypeError), (dict(start=start, count=start[:1]), ValueError),
                    (dict(pos=_ints([[0] * 2] * 2)), ValueError), (dict(start=start, q=k.float()), TypeError), (dict(start=start, q=k[:1]), ValueError),
                    (dict(start=start, inv_freq=torch.zeros(33, device="cuda", dtype=torch.float64)), ValueError),
                    (dict(start=start, inv_freq=torch.zeros(3, device="cuda")), TypeError), (dict(start=start, rope_pos=start), ValueError)):
        with pytest.raises(err):
            a(k, k, kp, vp, table, **kw)
    for args in ((k, k[:, :1], kp, vp, table), (k, k.float(), kp, vp, table), (k[:, :1], k[:, :1], kp, vp, table), (k, k, kp, vp[1:], table),
                 (k, k, kp, vp, table[:1]), (k, k, kp.float(), vp.float(), table), (k, k, kp[:, :, ::2], vp[:, :, ::2], table)):
        with pytest.raises((TypeError, ValueError)):
            a(*args, start=start)
    for page in (8, 24, 512):
        kq = torch.zeros((3, 2, page, 64), device="cuda", dtype=BF)
        with pytest.raises(CoverError, match="UNSUPPORTED"):
            a(k, k, kq, kq.clone(), table, start=start)


def test_pool_of_more_than_2_32_elements():
    page, H, D = 256, 8, 128
    n_pages = 2 ** 32 // (page * H * D) + 5
    kp, vp = (torch.empty((n_pages, H, page, D), device="cuda", dtype=BF) for _ in range(2))
    table = _ints([[n_pages - 1, 0, n_pages - 2]])
    for p in table[0].tolist():
        kp[p], vp[p] = 0, 0
    k, v = _rows(1, H, 700, D, BF), _rows(1, H, 700, D, BF, 1)
    api.cover_paged_append(k, v, kp, vp, table, start=_ints([20]))
    got = torch.cat([kp[p] for p in table[0].tolist()], 1), torch.cat([vp[p] for p in table[0].tolist()], 1)
    for g, x in zip(got, (k, v)):
        assert torch.equal(g[:, 20:720], x[0]) and not g[:, :20].any() and not g[:, 720:].any()
