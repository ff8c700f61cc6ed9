"""Rows whose best alternatives crowd where few threads look: more elements than are ranked at once (768) are not behind the bound
that the threads' best vectors give.

A part of a row deals its 16-byte vectors to 192 threads in turn. The indices are exact, against a stable sort; the log probabilities of the
alternatives are theirs less lse, each rounded to fp32 (2^-24 of the value), and lse is off by at most (V / 768 + 64) 2^-24 (2 + ln V)
of its sums (a thread adds V / 192 terms up in four sums) and 2^-24 of itself: 2^-22 (1 + |x|) + that is allowed."""
import math

import pytest
import torch

from paper_2602_06161_gb300 import api

pytestmark = pytest.mark.gpu

BF, F32 = torch.bfloat16, torch.float32
TYPES = pytest.mark.parametrize("dtype", [BF, F32])


def _gen(seed):
    return torch.Generator("cuda").manual_seed(seed)


def _crowd(N, vecs, threads, dtype, order, seed=0, parts=1):
    """Rows whose logits lie at -30, but those of `threads` threads of every part of them."""
    n = 8 if dtype == BF else 4
    x = torch.full((N, vecs, n), -30.0, device="cuda")
    at = torch.arange(vecs, device="cuda") % (vecs // parts) % 192 < threads
    m = int(at.sum()) * n
    some = {"any": lambda: torch.randn((N, m), generator=_gen(seed), device="cuda"),
            "rising": lambda: torch.linspace(-8, 8, m, device="cuda").expand(N, m),
            "falling": lambda: torch.linspace(8, -8, m, device="cuda").expand(N, m),
            "few values": lambda: torch.randint(0, 3, (N, m), generator=_gen(seed), device="cuda").float(),
            "equal": lambda: torch.zeros((N, m), device="cuda")}[order]()
    x[:, at] = some.reshape(N, -1, n)
    return x.view(N, -1).to(dtype)


def _check(x, K):
    N, V = x.shape
    r = api.cover_logprob_fwd(x, torch.zeros(N, device="cuda", dtype=torch.int32), topk=K)
    torch.cuda.synchronize()
    assert api.cover_device_status() == 0
    value, idx = x.float().sort(dim=1, stable=True, descending=True)
    assert torch.equal(r["top_idx"].long(), idx[:, :K])
    lse = torch.logsumexp(x.double(), 1)
    ref = value[:, :K].double() - lse[:, None]
    tol = 2.0 ** -22 * (1 + ref.abs()) + (V / 768 + 64) * 2.0 ** -24 * (2 + math.log(V)) + 2.0 ** -24 * lse.abs()[:, None]
    there = ref.isfinite()
    assert torch.equal(r["top_logp"][~there].double(), ref[~there])
    assert ((r["top_logp"].double() - ref).abs() <= tol)[there].all()


@TYPES
@pytest.mark.parametrize("order", ["any", "rising", "falling", "few values", "equal"])
@pytest.mark.parametrize("K,threads", [(64, 40), (20, 15), (16, 12), (5, 4), (64, 63)])
def test_few_threads_hold_the_best(K, threads, order, dtype):
    vecs = 192 * (-(-900 // (threads * (8 if dtype == BF else 4))) + 3)
    _check(_crowd(3, vecs, threads, dtype, order), K)
    # a row of several parts, of which each crowds
    _check(_crowd(1, 8 * vecs, threads, dtype, order, parts=8), K)


@TYPES
def test_several_rows_of_a_cta_and_rows_that_start_anywhere(dtype):
    """More rows than CTAs are on the GPU, of which every third crowds; V odd, so that the vectors at the rows' ends are shared."""
    n = 8 if dtype == BF else 4
    x = torch.randn((1300, 192 * 8 * n + 5), generator=_gen(1), device="cuda").to(dtype)
    x[::3, 3:-2] = _crowd(1, 192 * 8, 40, dtype, "any")
    _check(x, 64)
    x[:, -100:] = -math.inf
    _check(x, 17)


@TYPES
def test_crowds_beside_nothing(dtype):
    """Few threads have anything but -inf: fewer vectors than alternatives pass, and ties of -inf follow."""
    x = _crowd(2, 192 * 16, 20, dtype, "any")
    x[x == -30] = -math.inf
    _check(x, 64)
    x[:, 5000:] = -math.inf
    _check(x, 64)


@TYPES
def test_crowded_rows_take_a_walk_or_two(dtype):
    """A part's share of 2^22 logits is looked at a few times, not once an alternative (some 0.1 s for 64 of them in these rows, by a walk of
    a dependent load a step; 6 ms so): below 30 ms."""
    n = 8 if dtype == BF else 4
    x = _crowd(1, 2 ** 22 // n // 1536 * 1536, 40, dtype, "rising", parts=8)
    _check(x, 64)
    events = [torch.cuda.Event(enable_timing=True) for _ in range(2)]
    best = math.inf
    for _ in range(3):
        events[0].record()
        api.cover_logprob_fwd(x, topk=64)
        events[1].record()
        torch.cuda.synchronize()
        best = min(best, events[0].elapsed_time(events[1]))
    assert best < 30, best


@pytest.mark.parametrize("value", [math.nan, math.inf])
@TYPES
def test_crowds_with_nan_or_infinity(value, dtype):
    x = _crowd(2, 192 * 16, 40, dtype, "any")
    x[0, 1::3] = value
    r = api.cover_logprob_fwd(x, topk=64)
    torch.cuda.synchronize()
    assert api.cover_device_status() == 0
    assert ((r["top_idx"] >= -1) & (r["top_idx"] < x.shape[1])).all()
    assert torch.equal(r["top_idx"][1].long(), x[1].float().sort(stable=True, descending=True)[1][:64])


def test_a_masked_token_gets_no_gradient():
    """Logits of -inf that nothing names have a gradient of zero, those of a row whose alternatives are all unmasked too."""
    for dtype in (BF, F32):
        x = torch.randn((4, 3001), generator=_gen(5), device="cuda").to(dtype)
        x[:, 1000:2000] = -math.inf
        tok = torch.tensor([3, 7, -1, 2999], device="cuda", dtype=torch.int32)
        r = api.cover_logprob_fwd(x, tok, topk=9)
        g = [torch.randn(s, generator=_gen(6), device="cuda") for s in ((4,), (4,), (4,), (4, 9))]
        d = api.cover_logprob_bwd(x, r["lse"], tok=tok, d_logp=g[0], entropy=r["entropy"], d_entropy=g[1], d_lse=g[2], top_idx=r["top_idx"], d_top=g[3])
        assert not ((r["top_idx"] >= 1000) & (r["top_idx"] < 2000)).any()
        assert (d[:, 1000:2000] == 0).all() and d.isfinite().all() and (d[:, :1000] != 0).any()
