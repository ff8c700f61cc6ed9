"""GPU parity of the log probabilities of given tokens and of their gradient against the fp64 oracle.

Tolerances. A weight e^(x - m) is off by |x - m| 2^-23 (two fp32 operations) and 2^-22 (ex2.approx) of itself; 256 threads and
more add a row up, so that a sum is off by (V / 256 + 24) 2^-24 of its terms' magnitudes at most; with what is rounded behind it
that is step = (V / 256 + 64) 2^-24 of 1 + the mean |x - m|, which is at most 2 + ln V + H + 6 (the reference may lie 6 below the
largest logit). Results are rounded to fp32.
"""
import math

import numpy as np
import pytest
import torch

from oracle import paged_oracle as PO
from paper_2602_06161_gb300 import api

pytestmark = pytest.mark.gpu

BF, F32 = torch.bfloat16, torch.float32
EPS = {BF: 2.0 ** -8, F32: 2.0 ** -24}   # half a step
TYPES = pytest.mark.parametrize("dtype", [BF, F32])


def _gen(seed):
    return torch.Generator("cuda").manual_seed(seed)


def _logits(N, V, dtype, seed=0, scale=2.0):
    return (torch.randn((N, V), generator=_gen(seed), device="cuda") * scale).to(dtype)


def _tok(N, V, seed=1):
    t = torch.randint(0, V, (N,), generator=_gen(seed), device="cuda").int()
    if N > 2:
        t[1], t[2] = -1, V
    return t


def _h(t):
    return t.double().cpu().numpy() if t.is_floating_point() else t.cpu().numpy()


def _check(x, tok, K):
    r = api.cover_logprob_fwd(x, tok, topk=K)
    torch.cuda.synchronize()
    assert api.cover_device_status() == 0
    logp, ent, lse, idx, top = PO.logprob(_h(x), _h(tok), K)
    V = x.shape[1]
    far = 2 + math.log(V) + ent + 6
    step = (V / 256 + 64) * 2.0 ** -24 * far

    def close(got, ref, tol):
        got, fine = _h(got), np.isfinite(ref)
        assert np.array_equal(got[~fine], ref[~fine], equal_nan=True)
        tol = np.broadcast_to(tol, ref.shape)
        assert (np.abs(got - ref)[fine] <= tol[fine]).all(), float((np.abs(got - ref)[fine] / tol[fine]).max())
    close(r["lse"], lse, step + 2.0 ** -23 * np.abs(np.where(np.isfinite(lse), lse, 0)))
    close(r["logp"], logp, step + 2.0 ** -23 * np.abs(np.where(np.isfinite(logp), logp, 0)))
    close(r["entropy"], ent, 2 * step * far)
    if K:
        assert np.array_equal(_h(r["top_idx"]), idx)
        close(r["top_logp"], top, (step + 2.0 ** -23 * far)[:, None] + 2.0 ** -23 * np.abs(np.where(np.isfinite(top), top, 0)))
    else:
        assert set(r) == {"logp", "entropy", "lse"}
    return r


SIZES = [(1, 1), (3, 2), (2, 7), (5, 8), (4, 9), (3, 63), (7, 257), (2, 2047), (5, 4099), (3, 20001), (1, 40000)]


@TYPES
@pytest.mark.parametrize("K", [0, 1, 20, 64])
@pytest.mark.parametrize("N,V", SIZES)
def test_against_oracle(N, V, K, dtype):
    _check(_logits(N, V, dtype), _tok(N, V), K)


@TYPES
def test_ties_and_orders(dtype):
    """Equal logits, rising and falling ones, few values, and the best of a row crowded where one thread looks."""
    V = 9001
    x = torch.zeros((8, V), device="cuda")
    up = torch.linspace(-20, 20, V, device="cuda")
    x[1], x[2] = up, up.flip(0)
    x[3] = torch.randint(0, 4, (V,), generator=_gen(0), device="cuda").float()
    x[4, ::512] = 5
    x[5, 100:100 + 80] = 3
    for s in range(8):
        x[6, s::2048] = 7 - s / 8
        x[7, 4 + s::4096] = 9
    _check(x.to(dtype), _tok(8, V), 64)


@TYPES
def test_the_best_crowd_in_few_threads(dtype):
    """More than the elements that are ranked at once pass the bound: 63 of a row's threads hold nothing but large logits."""
    V = 256 * 8 * 12
    x = torch.full((2, V // 8, 8), -30.0, device="cuda")
    vec = torch.arange(V // 8, device="cuda")
    x[0, vec % 256 < 40] = torch.randn((int((vec % 256 < 40).sum()), 8), generator=_gen(3), device="cuda")
    x[1, vec % 128 < 20] = torch.randn((int((vec % 128 < 20).sum()), 8), generator=_gen(4), device="cuda")
    _check(x.view(2, V).to(dtype), _tok(2, V), 64)


@TYPES
def test_masked_vocabularies(dtype):
    """Logits of -inf: a few left, one left, none left; the lowest numbers of the type; fewer tokens than alternatives."""
    V = 3001
    x = _logits(7, V, dtype)
    x[0, 5:] = -math.inf
    x[1, :] = -math.inf
    x[1, 1777] = -2.5
    x[2, :] = -math.inf
    x[3, ::3] = -math.inf
    x[4, 10:] = torch.finfo(dtype).min
    x[5, :] = torch.finfo(dtype).min
    x[6, 1:] = -math.inf
    tok = torch.tensor([3, 1777, 9, 3, 3, 0, 2000], device="cuda", dtype=torch.int32)
    r = _check(x, tok, 20)
    assert r["logp"][1].item() == 0 and r["entropy"][1].item() == 0 and r["logp"][6].item() == -math.inf
    r = api.cover_logprob_fwd(x[:, :5].contiguous(), tok, topk=8)
    assert (r["top_idx"][:, 5:] == -1).all() and (r["top_logp"][:, 5:] == -math.inf).all()


@pytest.mark.parametrize("value", [math.nan, math.inf])
@TYPES
def test_rows_with_nan_or_infinity(value, dtype):
    V = 5000
    x = _logits(4, V, dtype)
    x[1, 4321] = value
    x[3, :] = value
    tok = torch.tensor([1, 2, 3, -1], device="cuda", dtype=torch.int32)
    r = api.cover_logprob_fwd(x, tok, topk=64)
    ref = api.cover_logprob_fwd(x[::2].contiguous(), tok[::2].contiguous(), topk=64)
    for name in r:
        assert torch.equal(r[name][::2], ref[name])
    assert all(r[n][i].isnan() for n in ("entropy", "lse") for i in (1, 3)) and r["logp"][1].isnan() and r["logp"][3] == 0
    assert ((r["top_idx"] >= -1) & (r["top_idx"] < V)).all()


@TYPES
@pytest.mark.parametrize("offset", [1e4, -3e4])
def test_logits_far_from_zero(offset, dtype):
    """An offset that the type holds exactly changes nothing but lse."""
    x = torch.randint(-20, 20, (3, 4000), generator=_gen(2), device="cuda").to(dtype)
    shift = float(torch.tensor(offset).to(dtype))
    y = (x.float() * 64 + shift).to(dtype)
    _check(y, _tok(3, 4000), 10)


def test_rows_that_start_anywhere():
    """Rows and tensors at any element: a view that starts within 16 bytes gives the aligned one's results."""
    for dtype in (BF, F32):
        flat = _logits(1, 7 * 1003 + 8, dtype)[0]
        for shift in range(8 if dtype == BF else 4):
            x = flat[shift:shift + 7 * 1003].view(7, 1003)
            a, b = (api.cover_logprob_fwd(t, _tok(7, 1003), topk=5) for t in (x, x.clone()))
            for n in ("logp", "entropy", "lse", "top_logp"):
                assert torch.allclose(a[n], b[n], rtol=2.0 ** -20, atol=2.0 ** -20)
            assert torch.equal(a["top_idx"], b["top_idx"])


def test_forms():
    x, tok = _logits(5, 999, BF), _tok(5, 999)
    full = api.cover_logprob_fwd(x, tok, topk=3)
    none = api.cover_logprob_fwd(x, topk=3)
    assert set(none) == {"entropy", "lse", "top_idx", "top_logp"} and all(torch.equal(none[n], full[n]) for n in none)
    s = torch.cuda.Stream()
    torch.cuda.synchronize()
    there = api.cover_logprob_fwd(x, tok, topk=3, stream=s)
    torch.cuda.synchronize()
    assert all(torch.equal(there[n], full[n]) for n in full)
    empty = api.cover_logprob_fwd(x[:0], tok[:0], topk=3)
    assert empty["logp"].shape == (0,) and empty["top_idx"].shape == (0, 3)
    d = api.cover_logprob_bwd(x[:0], full["lse"][:0])
    assert d.shape == (0, 999)
    for bad in (lambda: api.cover_logprob_fwd(x, tok, topk=65), lambda: api.cover_logprob_fwd(x, tok, topk=-1)):
        with pytest.raises(Exception, match="UNSUPPORTED|INVALID"):
            bad()
    for bad in (lambda: api.cover_logprob_fwd(x, tok[:3]), lambda: api.cover_logprob_fwd(x, tok.long()), lambda: api.cover_logprob_fwd(x[:, ::2], tok),
                lambda: api.cover_logprob_bwd(x, full["lse"], d_logp=full["logp"]), lambda: api.cover_logprob_bwd(x, full["lse"][:2]),
                lambda: api.cover_logprob_bwd(x, full["lse"], d_entropy=full["logp"]), lambda: api.cover_logprob_bwd(x, full["lse"], d_top=full["top_logp"]),
                lambda: api.cover_logprob_bwd(x, full["lse"], out=x[:3]), lambda: api.cover_logprob_bwd(x, full["lse"], out=x.float()),
                lambda: api.cover_logprob_bwd(x, full["lse"].half())):
        with pytest.raises((TypeError, ValueError)):
            bad()
    flat = torch.zeros(6 * 999, device="cuda", dtype=BF)
    with pytest.raises(ValueError, match="must not overlap logits"):
        api.cover_logprob_bwd(flat[:5 * 999].view(5, 999), full["lse"], out=flat[999:].view(5, 999))


def _grads(N, V, K, seed=5):
    f = lambda *s: torch.randn(s, generator=_gen(seed + len(s)), device="cuda")  # noqa: E731
    idx = torch.randint(-1, V + 1, (N, K), generator=_gen(seed), device="cuda").int() if K else None
    return dict(d_logp=f(N), d_entropy=f(N), d_lse=f(N) * 0.5, top_idx=idx, d_top=f(N, K) if K else None)


def _check_grad(x, tok, g, **kw):
    r = api.cover_logprob_fwd(x, tok)
    lse, ent = r["lse"], r["entropy"]
    d = api.cover_logprob_bwd(x, lse, tok=tok, entropy=ent, **g, **kw)
    torch.cuda.synchronize()
    n = lambda t: None if t is None else _h(t)  # noqa: E731
    return d, lse, PO.logprob_grad(_h(kw["x0"]) if "x0" in kw else _h(x), n(lse), tok=n(tok), d_logp=n(g["d_logp"]), ent=n(ent),
                                   d_ent=n(g["d_entropy"]), d_lse=n(g["d_lse"]), idx=n(g["top_idx"]), d_top=n(g["d_top"]))


def _assert_grad(d, x, lse, ref, size, K, dtype):
    """A weight is off by |x - lse| 2^-23 and 2^-22 of itself, the sum of the row's shares by K + 4 roundings of its terms."""
    far = np.where(np.isfinite(_h(x)), np.abs(_h(x) - _h(lse)[:, None]), 0)
    tol = size * ((K + 8) * 2.0 ** -24 + 2.0 ** -21 + np.minimum(far, 200) * 2.0 ** -22)
    tol = (tol + EPS[dtype] * np.abs(ref)) * (1 + EPS[dtype]) + 1e-38
    err = np.abs(_h(d) - ref)
    assert (err <= tol).all(), float((err / tol).max())


@TYPES
@pytest.mark.parametrize("K", [0, 1, 5, 64])
@pytest.mark.parametrize("N,V", SIZES)
def test_gradient_against_oracle(N, V, K, dtype):
    x, tok, g = _logits(N, V, dtype), _tok(N, V), _grads(N, V, K)
    d, lse, (ref, size) = _check_grad(x, tok, g)
    assert d.dtype == dtype and d.shape == x.shape
    _assert_grad(d, x, lse, ref, size, K, dtype)


@TYPES
@pytest.mark.parametrize("left", [("d_logp",), ("d_entropy",), ("d_lse",), ("d_top",), ()])
def test_gradient_of_one_result(left, dtype):
    N, V, K = 4, 1003, 3
    x, tok, g = _logits(N, V, dtype), _tok(N, V), _grads(N, V, K)
    g = {n: t if n in left or (n == "top_idx" and "d_top" in left) else None for n, t in g.items()}
    d, lse, (ref, size) = _check_grad(x, tok, g)
    _assert_grad(d, x, lse, ref, size, K, dtype)
    if not left:
        assert not d.any()


@TYPES
def test_gradient_of_masked_rows_and_repeated_tokens(dtype):
    N, V, K = 5, 2001, 6
    x, tok, g = _logits(N, V, dtype), _tok(N, V), _grads(N, V, K)
    x[0, 7:] = -math.inf
    x[3, ::2] = -math.inf
    tok[0], tok[3], tok[4] = 3, 1, 1999
    g["top_idx"][:, 1] = tok
    g["top_idx"][:, 2] = tok
    g["top_idx"][4] = 1999
    d, lse, (ref, size) = _check_grad(x, tok, g)
    _assert_grad(d, x, lse, ref, size, K, dtype)
    assert not d[0, 8:][x[0, 8:] == -math.inf].abs().sum() or (g["top_idx"][0] > 7).any()


@TYPES
@pytest.mark.parametrize("V", [512, 4099])
def test_gradient_in_the_logits_place(V, dtype):
    N, K = 6, 4
    x, tok, g = _logits(N, V, dtype), _tok(N, V), _grads(N, V, K)
    r = api.cover_logprob_fwd(x, tok)
    args = dict(tok=tok, entropy=r["entropy"], **g)
    ref = api.cover_logprob_bwd(x, r["lse"], **args)
    # beside it, at another alignment, and in its place
    flat = torch.zeros(N * V + 9, device="cuda", dtype=dtype)
    for shift in (0, 1, 3):
        out = flat[shift:shift + N * V].view(N, V)
        assert api.cover_logprob_bwd(x, r["lse"], out=out, **args) is out and torch.equal(out, ref)
        assert not flat[shift + N * V:].any() and not flat[:shift].any()
        flat.zero_()
    assert api.cover_logprob_bwd(x, r["lse"], out=x, **args) is x and torch.equal(x, ref)


def test_gradient_against_differences():
    """The kernels' own results at x + e and x - e, in fp32: values up to 12 are off by 2^-20, so differences over 2^-4 by 2^-16, and the
    third derivative's share, at most e^2 times the gradients' sizes."""
    N, V, K = 3, 300, 2
    x, tok = _logits(N, V, F32, scale=1.0), _tok(N, V)
    g = _grads(N, V, K)
    g["top_idx"] = torch.randint(0, V, (N, K), generator=_gen(8), device="cuda").int()
    r = api.cover_logprob_fwd(x, tok)
    d = api.cover_logprob_bwd(x, r["lse"], tok=tok, entropy=r["entropy"], **g)

    def value(x):
        r = api.cover_logprob_fwd(x, tok)
        top = [api.cover_logprob_fwd(x, g["top_idx"][:, k].contiguous())["logp"] for k in range(K)]
        return sum((a * b).double() for a, b in ((g["d_logp"], r["logp"]), (g["d_entropy"], r["entropy"]), (g["d_lse"], r["lse"]),
                                                *((g["d_top"][:, k], top[k]) for k in range(K))))
    e = 2.0 ** -5
    for j in (0, int(tok[0]), 150, 299):
        step = torch.zeros_like(x)
        step[:, j] = e
        diff = (value(x + step) - value(x - step)) / (2 * e)
        assert (diff - d[:, j].double()).abs().max() < 2.0 ** -13 + 4 * e * e


def test_captured_and_replayed():
    x, tok = _logits(40, 5003, BF), _tok(40, 5003)
    r = api.cover_logprob_fwd(x, tok, topk=5)
    g = _grads(40, 5003, 5)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        y = api.cover_logprob_fwd(x, tok, topk=5)
        d = api.cover_logprob_bwd(x, y["lse"], tok=tok, entropy=y["entropy"], d_logp=g["d_logp"], top_idx=y["top_idx"], d_top=g["d_top"])
    for seed in (0, 7):
        x.copy_(_logits(40, 5003, BF, seed=seed))
        graph.replay()
        r = api.cover_logprob_fwd(x, tok, topk=5)
        e = api.cover_logprob_bwd(x, r["lse"], tok=tok, entropy=r["entropy"], d_logp=g["d_logp"], top_idx=r["top_idx"], d_top=g["d_top"])
        assert all(torch.equal(r[n], y[n]) for n in r) and torch.equal(d, e)
