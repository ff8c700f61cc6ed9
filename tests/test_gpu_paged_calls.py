"""How the calls over a memory in pages and the log probabilities are made: other streams, captures, calls at once, both ways of
marshalling; and the sizes at which their kernels change what they do."""
import math

import numpy as np
import pytest
import torch

from paper_2602_06161_gb300 import api
from tests import test_gpu_attn_paged as A
from tests import test_gpu_logprob as L
from tests import test_gpu_paged_append as P

pytestmark = pytest.mark.gpu

BF, F32 = torch.bfloat16, torch.float32


def _span(t):
    return t.data_ptr(), t.data_ptr() + t.numel() * t.element_size()


def _calls():
    """Calls that can be made again: what they write into pages is the same each time."""
    B, n = 2, 40
    k, v, q = P._rows(B, 4, n, 128, BF), P._rows(B, 4, n, 128, BF, 1), P._rows(B, 8, n, 128, BF, 2)
    kp, vp, table = P._pool([200, 130], 4, 16, 128)
    f, start = api.rope_frequencies(128)[0], P._ints([150, 7])
    few, many = A._inputs([777, 300], 8, 2, 1, 2, 16), A._inputs([1500, 40], 8, 2, 100, 4, 64)
    long = A._inputs([5000] * 40, 8, 2, 1, 0, 64)
    x, tok = L._logits(300, 4099, BF), L._tok(300, 4099)
    r = api.cover_logprob_fwd(x, tok, topk=5)
    g = torch.randn(300, device="cuda")
    attn = lambda d: lambda **kw: api.cover_attn_fwd_paged(d["q"], d["kp"], d["vp"], d["table"], d["lens"], d["km"], d["vm"], d["seeds"],  # noqa: E731
                                                           q0=d["q0"], **kw)
    return {
        "append": lambda **kw: api.cover_paged_append(k, v, kp, vp, table, start=start, q=q, inv_freq=f, want_k=True, **kw),
        "attn_few": attn(few), "attn_many": attn(many), "attn_batch": attn(long),
        "logprob": lambda **kw: tuple(api.cover_logprob_fwd(x, tok, topk=20, **kw).values()),
        "logprob_grad": lambda **kw: (api.cover_logprob_bwd(x, r["lse"], tok=tok, entropy=r["entropy"], d_logp=g, d_entropy=g, **kw),),
    }


NAMES = ["append", "attn_few", "attn_many", "attn_batch", "logprob", "logprob_grad"]


@pytest.mark.parametrize("given", ["stream", "handle", "default"])
@pytest.mark.parametrize("name", NAMES)
def test_no_block_of_pending_work_is_taken(name, given):
    call = _calls()[name]
    ref = call()
    torch.cuda.synchronize()
    here = torch.cuda.Stream()
    there = torch.cuda.default_stream() if given == "default" else torch.cuda.Stream()
    with torch.cuda.stream(here):
        blocks = [torch.empty(max(1, t.numel() * t.element_size() * n), dtype=torch.uint8, device="cuda") for t in ref for n in (1, 1, 4)]
        spans = [_span(b) for b in blocks]
        torch.cuda._sleep(20_000_000)
        for b in blocks:
            b.fill_(255)
        del b, blocks
        got = call(stream={"stream": there, "handle": there.cuda_stream, "default": 0}[given])
        for t in got:
            lo, hi = _span(t)
            assert not any(lo < e and b < hi for b, e in spans)
        here.wait_stream(there)
        kept = [t.clone() for t in got]
    torch.cuda.synchronize()
    assert api.cover_device_status() == 0
    for x, y in zip(kept, ref):
        assert torch.equal(x, y)


@pytest.mark.parametrize("name", NAMES)
def test_a_captured_call_on_another_stream(name):
    call = _calls()[name]
    ref = call()
    torch.cuda.synchronize()
    side, g = torch.cuda.Stream(), torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        side.wait_stream(torch.cuda.current_stream())
        got = call(stream=side)
        torch.cuda.current_stream().wait_stream(side)
        kept = [t.clone() for t in got]
    others = [torch.full_like(got[0], 7.0) for _ in range(50)]      # of the allocator's other memory
    for _ in range(2):
        g.replay()
    torch.cuda.synchronize()
    assert api.cover_device_status() == 0
    assert all(torch.equal(a, b) for a, b in zip(kept, ref)) and all((o == 7.0).all() for o in others)


@pytest.mark.parametrize("name", NAMES)
def test_two_graphs_and_eager_calls_at_once(name):
    """Two captured calls replayed at once on two streams, and eager ones beside them: each has its own workspace."""
    call = _calls()[name]
    ref = call()
    torch.cuda.synchronize()
    graphs, outs = [], []
    for _ in range(2):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            outs.append(call())
        graphs.append(g)
    streams = [torch.cuda.Stream() for _ in range(3)]
    for _ in range(10):
        for g, s in zip(graphs, streams):
            with torch.cuda.stream(s):
                g.replay()
        with torch.cuda.stream(streams[2]):
            eager = call()
    torch.cuda.synchronize()
    assert api.cover_device_status() == 0
    for got in (*outs, eager):
        assert all(torch.equal(a, b) for a, b in zip(got, ref))


def test_captured_append_with_places_that_change():
    k, v = P._rows(3, 2, 4, 64, F32), P._rows(3, 2, 4, 64, F32, 1)
    f, _ = api.rope_frequencies(64)
    kp, vp, table = P._pool([90, 90, 90], 2, 16, 64)
    start, count, old = P._ints([0, 0, 0]), P._ints([4, 4, 4]), (kp.clone(), vp.clone())
    api.cover_paged_append(k, v, kp, vp, table, start=start, count=count, inv_freq=f)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        api.cover_paged_append(k, v, kp, vp, table, start=start, count=count, inv_freq=f)
    for at, n in (([3, 15, 80], [4, 1, 0]), ([94, -2, 40], [4, 4, 4])):
        for t, o in zip((kp, vp), old):
            t.copy_(o)
        start.copy_(P._ints(at))
        count.copy_(P._ints(n))
        k.normal_()
        graph.replay()
        want = [o.clone() for o in old]
        api.cover_paged_append(k, v, *want, table, start=start, count=count, inv_freq=f)
        assert torch.equal(kp, want[0]) and torch.equal(vp, want[1])
        assert not torch.equal(kp, old[0])


def test_both_ways_of_marshalling_agree():
    """Arguments that the native call hands back (a Python int for a factor, a stream object's handle) take the other way."""
    k, v, q = P._rows(2, 2, 9, 64, BF), P._rows(2, 2, 9, 64, BF, 1), P._rows(2, 4, 9, 64, BF, 2)
    f, _ = api.rope_frequencies(64)
    got = []
    for mscale in (2.0, 2, np.float32(2)):
        kp, vp, table = P._pool([40, 30], 2, 16, 64)
        got.append((*api.cover_paged_append(k, v, kp, vp, table, start=P._ints([11, 4]), q=q, inv_freq=f, mscale=mscale, want_k=True), kp, vp))
    x, tok = L._logits(20, 777, BF), L._tok(20, 777)
    g = torch.randn(20, device="cuda")
    rows = []
    for topk in (5, np.int64(5)):
        r = api.cover_logprob_fwd(x, tok, topk=topk)
        rows.append((*r.values(), api.cover_logprob_bwd(x, r["lse"], tok=tok, d_logp=g)))
    torch.cuda.synchronize()
    for group in (got, rows):
        for other in group[1:]:
            assert all(torch.equal(a, b) for a, b in zip(group[0], other))


def test_the_same_bits_again():
    for name, call in _calls().items():
        ref = call()
        for _ in range(3):
            assert all(torch.equal(a, b) for a, b in zip(call(), ref)), name


# ---------------- sizes at which a kernel changes what it does ----------------


@pytest.mark.parametrize("cap", [0.0, 30.0])
@pytest.mark.parametrize("kind", [None, "any", "causal"])
@pytest.mark.parametrize("Hq,Hkv,Lq", [(8, 2, 1), (6, 1, 3), (4, 4, 2)])
def test_units_of_one_tile_among_longer_ones(Hq, Hkv, Lq, kind, cap):
    """Sequences of no key, one, a KV tile, one more, and some tiles, in turn: units that one stream does alone, beside units of both."""
    lens = [(0, 1, 128, 50, 129, 7, 500, 100, 256, 128)[(3 * b) % 10] for b in range(61)]
    d = A._inputs(lens, Hq, Hkv, Lq, 3, 16)
    lo, hi = A._ranges(kind, d)
    A._check(d, *A._run(d, key_lo=lo, key_hi=hi, softcap=cap), lo, hi, cap)
    for parts in (1, 3, 152):       # more units a CTA than are laid out ahead, down to less than one
        n = parts * (2 * 32 * 520 + 16)
        out, lse = api.cover_debug_attn_paged(d["q"], d["kp"], d["vp"], d["table"], d["lens"], d["km"], d["vm"], d["seeds"], q0=d["q0"],
                                              mode=0 if Hq // Hkv * Lq <= 16 else 1, parts=parts, key_lo=lo, key_hi=hi, softcap=cap,
                                              workspace=torch.full((n,), 255, device="cuda", dtype=torch.uint8))
        torch.cuda.synchronize()
        assert api.cover_device_status() == 0
        A._check(d, out, lse, lo, hi, cap)


@pytest.mark.parametrize("Lq", [1, 60])
def test_values_that_are_not_finite_in_units_of_one_tile(Lq):
    """A NaN in a value that some rows see and others do not: the others are as without it, these have no finite number in its column."""
    d = A._inputs([100] * 20, 4, 2, Lq, 0, 16)
    lo = A._ints([[(0 if (b + r) % 2 else 60) for r in range(Lq)] for b in range(20)])
    ref, ref_lse = A._run(d, key_lo=lo)
    page = d["table"][7, 3]
    d["vp"][page, 1, 5, 40] = math.nan                   # key 53 of sequence 7
    d["vp"][d["table"][8, 0], 0, 0, 0] = math.nan        # key 0 of sequence 8
    out, lse = A._run(d, key_lo=lo)
    sees = torch.zeros(ref.shape[:3], device="cuda", dtype=torch.bool)
    sees[7, 2:], sees[8, :2] = lo[7] <= 53, lo[8] <= 0
    assert torch.equal(out[~sees], ref[~sees]) and torch.equal(lse[~sees], ref_lse[~sees])
    assert not out[7, 2:][sees[7, 2:]][..., 40].isfinite().any() and not out[8, :2][sees[8, :2]][..., 0].isfinite().any()


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("K", [15, 16, 17, 33])
@pytest.mark.parametrize("N,V", [(1, 16), (3, 40), (2, 1500), (700, 900), (3, 20001), (1, 130000)])
def test_few_and_many_alternatives(N, V, K, dtype):
    L._check(L._logits(N, V, dtype), L._tok(N, V), K)


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("K", [5, 16, 17, 64])
@pytest.mark.parametrize("each", [5, 30])
def test_alternatives_that_few_threads_have(each, K, dtype):
    """Rows whose best are in one, two, three and more vectors of the same threads, alike and in order, and where more pass the bound than
    are ranked at once (a row's vectors go to 192 threads in turn, `each` to a thread; longer rows are split)."""
    n = 16 // torch.tensor([], dtype=dtype).element_size()
    V = 192 * n * each
    vec = torch.arange(V // n, device="cuda")
    x = torch.randn((7, V // n, n), generator=L._gen(2), device="cuda")
    x[0, vec % 192 == 5] += 30
    x[1, (vec % 192 < 3) & (vec // 192 < 2)] += 30
    x[2, (vec % 192 < 9) & (vec // 192 < 3)] = 30.0
    x[3, vec % 192 < 20] += 30
    x[4, vec % 192 < 20] = 30.0
    x[5] = 1.0
    x[6] = -math.inf
    x[6, (vec % 192 == 7) & (vec // 192 < 5), 1] = 2.0
    L._check(x.view(7, V).to(dtype), L._tok(7, V), K)


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("inter,Hq,Hkv,n,D,R", [
    (True, 3, 2, 17, 128, 120), (True, 2, 1, 9, 128, 124), (True, 5, 17, 8, 64, 8), (False, 33, 1, 7, 128, 16), (False, 64, 2, 25, 64, 48),
    (False, 0, 20, 65, 128, 0), (True, 0, 3, 1, 64, 64),
])
def test_rows_with_columns_that_do_not_turn(inter, Hq, Hkv, n, D, R, dtype):
    """An odd and an even number of vectors that do not turn, more heads than a thread has on their way, blocks of tokens that are not full."""
    for B in (1, 3):
        k, v = P._rows(B, Hkv, n, D, dtype), P._rows(B, Hkv, n, D, dtype, 1)
        q = P._rows(B, Hq, n, D, dtype, 2) if Hq else None
        f = api.rope_frequencies(R)[0] if R else None
        kp, vp, table = P._pool([n + 40] * B, Hkv, 32, D)
        P._check(k, v, q, kp, vp, table, f, inter, 1.0, start=P._ints([5 * b + 30 for b in range(B)]))
        pos = torch.randint(-1, n + 3, (B, n), generator=P._gen(4), device="cuda").int()
        P._check(k, v, q, kp, vp, table, f, inter, 1.0, pos=pos)


def test_many_rows_of_a_few_heads():
    """Enough rows for sixteen heads a thread."""
    k, v, q = P._rows(3, 2, 2500, 64, BF), P._rows(3, 2, 2500, 64, BF, 1), P._rows(3, 40, 2500, 64, BF, 2)
    kp, vp, table = P._pool([2600] * 3, 2, 64, 64)
    P._check(k, v, q, kp, vp, table, api.rope_frequencies(32)[0], False, 1.0, start=P._ints([0, 77, 100]), count=P._ints([2500, 1, 2041]))


def test_groups_of_rows_that_cross_heads():
    """Heads' rows at sizes around a group's 256."""
    for Lq, G in ((255, 2), (256, 2), (257, 2), (86, 3), (129, 4)):
        d = A._inputs([Lq + 10, 300], G, 1, Lq, 7, 16, seed=Lq)
        lo, hi = A._ranges("window", d)
        A._check(d, *A._run(d, key_lo=lo, key_hi=hi), lo, hi)
