"""Pins of the oracle of the memory in pages and of the log probabilities, on the CPU."""
import math

import numpy as np
import torch

from oracle import memory8_oracle as M8, paged_oracle as PO


def _pool(rng, lens, H, page, D):
    need = [-(-n // page) for n in lens]
    n_pages, M = sum(need) + 2, max(max(need), 1)
    order, table, at = rng.permutation(n_pages), np.full((len(lens), M), -1, np.int32), 0
    for b, n in enumerate(need):
        table[b, :n] = order[at:at + n]
        at += n
    return rng.standard_normal((n_pages, H, page, D)), rng.standard_normal((n_pages, H, page, D)), table


def test_pages_in_any_order_are_the_dense_window():
    rng = np.random.default_rng(0)
    B, Hq, Hkv, Lq, D, S, L = 2, 6, 2, 4, 8, 3, 21
    k, v, table = _pool(rng, [L, L], Hkv, 4, D)
    dense = [np.stack([np.stack([PO.sequence(x, table[b], h, L)[0] for h in range(Hkv)]) for b in range(B)]) for x in (k, v)]
    q, km, vm = rng.standard_normal((B, Hq, Lq, D)), rng.standard_normal((B, Hkv, S, D)), rng.standard_normal((B, Hkv, S, D))
    seeds = np.array([[11, 3, 11], [10, -1, 13]])
    lo, hi = rng.integers(-2, 12, (B, Lq)), rng.integers(8, 30, (B, Lq))
    got = PO.attention(q, k, v, table, [L, L], km, vm, seeds, q0=[10, 10], key_lo=lo, key_hi=hi, softcap=3.0)
    ref = M8.attention(q, *dense, km, vm, seeds, q0=10, key_lo=lo, key_hi=hi, softcap=3.0)
    for a, b in zip(got, ref):
        assert np.allclose(a, b, rtol=0, atol=1e-13) or np.array_equal(a, b)


def test_positions_without_a_page_are_not_seen():
    rng = np.random.default_rng(1)
    k, v, table = _pool(rng, [20], 1, 4, 8)
    q = rng.standard_normal((1, 2, 1, 8))
    holed = table.copy()
    holed[0, 2] = -1
    a = PO.attention(q, k, v, holed, [20], None, None, None)
    left = np.array([0, 1, 3, 4])
    b = PO.attention(q, k, v, table[:, left], [16], None, None, None)
    assert np.allclose(a[0], b[0], atol=1e-14) and np.allclose(a[1], b[1], atol=1e-14)
    none = PO.attention(q, k, v, np.full_like(table, 99), [20], None, None, None)
    assert (none[0] == 0).all() and (none[1] == -math.inf).all()


def test_append_lowest_row_wins_and_the_rest_stays():
    rng = np.random.default_rng(2)
    k, _, table = _pool(rng, [9, 9], 1, 4, 2)
    rows = rng.standard_normal((2, 1, 4, 2))
    pos = np.array([[8, 2, 8, -1], [3, 12, 11, 0]])
    got = PO.appended(k, table, rows, pos=pos)
    want = k.copy()
    want[table[0, 2], :, 0], want[table[0, 0], :, 2] = rows[0, :, 0], rows[0, :, 1]
    want[table[1, 0], :, 3], want[table[1, 2], :, 3], want[table[1, 0], :, 0] = rows[1, :, 0], rows[1, :, 2], rows[1, :, 3]
    assert np.array_equal(got, want)
    got = PO.appended(k, table, rows, start=[7, 10], count=[3, 4])
    want = k.copy()
    want[table[0, 1], :, 3], want[table[0, 2], :, 0], want[table[0, 2], :, 1] = (rows[0, :, i] for i in range(3))
    want[table[1, 2], :, 2], want[table[1, 2], :, 3] = rows[1, :, 0], rows[1, :, 1]
    assert np.array_equal(got, want)


def test_log_probabilities_are_those_of_torch():
    x = torch.randn(5, 37, dtype=torch.float64, generator=torch.Generator().manual_seed(0)) * 3
    x[1, 4:30] = -math.inf
    x[2, 7] = x[2, 3]
    tok = np.array([0, 2, 36, -1, 37])
    logp, ent, lse, idx, top = PO.logprob(x.numpy(), tok, 4)
    ref = torch.log_softmax(x, 1)
    assert np.allclose(logp[:3], ref[range(3), tok[:3]].numpy(), atol=1e-13) and (logp[3:] == 0).all()
    assert np.allclose(ent, torch.distributions.Categorical(logits=x.clamp(min=-1e4)).entropy().numpy(), atol=1e-12)
    assert np.allclose(lse, torch.logsumexp(x, 1).numpy(), atol=1e-13)
    assert np.allclose(top, ref.topk(4).values.numpy(), atol=1e-13)
    assert all((x[i, idx[i]].numpy() == np.sort(x[i].numpy())[::-1][:4]).all() for i in range(5))


def test_ties_go_to_the_lowest_index():
    x = np.zeros((1, 6))
    x[0, 4] = 1
    assert PO.logprob(x, [0], 4)[3].tolist() == [[4, 0, 1, 2]]


def test_gradient_is_that_of_autograd_and_of_differences():
    g = torch.Generator().manual_seed(1)
    x = (torch.randn(3, 11, dtype=torch.float64, generator=g) * 2).requires_grad_()
    tok, idx = np.array([2, 10, -1]), np.array([[2, 0], [5, 5], [1, -1]])
    gl, ge, gs, gt = (torch.randn(*s, dtype=torch.float64, generator=g) for s in ((3,), (3,), (3,), (3, 2)))

    def value(x):
        lp = torch.log_softmax(x, 1)
        ent = -(lp.exp() * lp).sum(1)
        v = (gl[:2] * lp[range(2), tok[:2]]).sum() + (ge * ent).sum() + (gs * torch.logsumexp(x, 1)).sum()
        return v + sum(gt[i, k] * lp[i, idx[i, k]] for i in range(3) for k in range(2) if idx[i, k] >= 0)
    value(x).backward()
    n = lambda t: t.detach().numpy()  # noqa: E731
    _, ent, lse, _, _ = PO.logprob(n(x), tok, 0)
    d, size = PO.logprob_grad(n(x), lse, tok=tok, d_logp=n(gl), ent=ent, d_ent=n(ge), d_lse=n(gs), idx=idx, d_top=n(gt))
    assert np.allclose(d, x.grad.numpy(), atol=1e-13) and (np.abs(d) <= size + 1e-15).all()
    with torch.no_grad():
        for i, j in ((0, 2), (1, 5), (2, 8)):
            e = torch.zeros_like(x)
            e[i, j] = 1e-5
            assert abs((value(x + e) - value(x - e)).item() / 2e-5 - d[i, j]) < 1e-8
