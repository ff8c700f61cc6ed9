"""GPU parity of the window attention over a memory in pages against the fp64 oracle.

Tolerances. The probabilities and the output are rounded to bf16 (half a step: 2^-8 of the value each); a score
of fp32 accumulation is off by at most d = 2^-20 of sum |q_i k_i| / sqrt(D) (128 terms, each rounded or cut off at
2^-24 .. 2^-23 of the partial sum) and, capped, by 2^-20 of the cap (three fp32 operations on values up to the cap); an
error d of the scores changes every weight by a factor of at most e^{2d}. So with mass = sum_j w_j |v_j|,
|out - ref| <= 2^-8 |ref| + (2^-8 + 4 d) mass (1 + 2^-6), and lse is off by d and by 2^-20 of its sums' rounding.
"""
import math

import numpy as np
import pytest
import torch

from oracle import paged_oracle as PO
from paper_2602_06161_gb300 import CoverError, api

pytestmark = pytest.mark.gpu

BF = torch.bfloat16


def _gen(seed):
    return torch.Generator("cuda").manual_seed(seed)


def _randn(*shape, seed=0, scale=1.0):
    return (torch.randn(shape, generator=_gen(seed), device="cuda") * scale).to(BF)


def _h(t):
    return None if t is None else t.double().cpu().numpy() if t.is_floating_point() else t.cpu().numpy()


def _ints(x):
    return torch.tensor(x, device="cuda", dtype=torch.int32)


def _inputs(lens, Hq, Hkv, Lq, S, page, q0=None, seed=0, scale=1.0, junk=True, M=0):
    """Sequences of so many keys in pages in any order; what lies in the pool beside them is NaN (junk)."""
    B = len(lens)
    need = [-(-n // page) for n in lens]
    n_pages, M = sum(need) + 2, max(max(need), 1, M)
    order = torch.randperm(n_pages, generator=_gen(seed), device="cuda").to(torch.int32)
    table = torch.full((B, M), -1, device="cuda", dtype=torch.int32)
    kp, vp = (torch.full((n_pages, Hkv, page, 128), math.nan if junk else 0.0, device="cuda", dtype=BF) for _ in range(2))
    at = 0
    for b, n in enumerate(need):
        table[b, :n] = order[at:at + n]
        at += n
        if lens[b]:
            j = torch.arange(lens[b], device="cuda")
            pages = table[b, j // page].long()
            kp[pages, :, j % page] = _randn(lens[b], Hkv, 128, seed=seed + 100 + b, scale=scale)
            vp[pages, :, j % page] = _randn(lens[b], Hkv, 128, seed=seed + 500 + b)
    q0 = _ints([max(0, n - Lq) for n in lens] if q0 is None else q0)
    d = dict(q=_randn(B, Hq, Lq, 128, seed=seed + 3), kp=kp, vp=vp, table=table, lens=_ints(lens), km=None, vm=None, seeds=None, q0=q0)
    if S:
        d["seeds"] = (q0[:, None] + torch.randint(-3, Lq + 3, (B, S), generator=_gen(seed + 6), device="cuda")).int().contiguous()
        if S >= 4:
            d["seeds"][:, 2] = 2 ** 31 - 1
        d["km"], d["vm"] = _randn(B, Hkv, S, 128, seed=seed + 4), _randn(B, Hkv, S, 128, seed=seed + 5)
    return d


def _run(d, **kw):
    out, lse = api.cover_attn_fwd_paged(d["q"], d["kp"], d["vp"], d["table"], d["lens"], d["km"], d["vm"], d["seeds"], q0=d["q0"], **kw)
    torch.cuda.synchronize()
    assert api.cover_device_status() == 0
    return out, lse


def _check(d, out, lse, key_lo=None, key_hi=None, softcap=0.0):
    ref, ref_lse, mass, size = PO.attention(_h(d["q"]), _h(d["kp"]), _h(d["vp"]), _h(d["table"]), _h(d["lens"]), _h(d["km"]), _h(d["vm"]),
                                            _h(d["seeds"]), q0=_h(d["q0"]), key_lo=_h(key_lo), key_hi=_h(key_hi), softcap=softcap)
    delta = (2.0 ** -20 * size + 2.0 ** -20 * softcap)[..., None]
    tol = 2.0 ** -8 * np.abs(ref) + (2.0 ** -8 + 4 * delta) * mass * (1 + 2.0 ** -6)
    got, got_lse, nan = _h(out), _h(lse), np.isnan(ref)     # (a row that sees NaN is NaN)
    assert np.array_equal(np.isnan(got), nan)
    ratio = np.abs(got - ref)[~nan] / np.maximum(tol, 1e-30)[~nan]
    assert ratio.size == 0 or ratio.max() <= 1, float(ratio.max())
    none, nan = ref_lse == -math.inf, np.isnan(ref_lse)
    assert np.array_equal(got_lse == -math.inf, none) and np.array_equal(np.isnan(got_lse), nan)
    there = ~none & ~nan
    tol = delta[..., 0] + 2.0 ** -20 * (1 + np.abs(np.where(there, ref_lse, 0)))
    assert (np.abs(got_lse - ref_lse)[there] <= tol[there]).all()


def _ranges(kind, d, seed=0):
    B, Lq = d["q"].shape[0], d["q"].shape[2]
    at = d["q0"][:, None] + torch.arange(Lq, device="cuda", dtype=torch.int32)
    if kind is None:
        return None, None
    if kind == "causal":
        return None, (at + 1).contiguous()
    if kind == "window":
        return (at - 100).contiguous(), (at + 3).contiguous()
    if kind == "blocks":
        return None, (at // 64 * 64 + 64).contiguous()
    top = int(d["lens"].max())
    lo = torch.randint(-5, top + 5, (B, Lq), generator=_gen(seed), device="cuda").int()     # anything, many rows empty
    return lo, lo + torch.randint(-3, 40, (B, Lq), generator=_gen(seed + 1), device="cuda").int()


SHAPES = [   # lens, Hq, Hkv, Lq, S, page
    ([1], 1, 1, 1, 0, 16), ([777], 28, 4, 1, 0, 16), ([129, 0, 40], 4, 4, 1, 1, 32), ([128], 8, 2, 2, 0, 64), ([300, 17], 28, 4, 32, 8, 16),
    ([128], 4, 4, 128, 128, 128), ([257], 2, 1, 129, 5, 32), ([511], 3, 1, 200, 40, 256), ([64, 1, 0, 33, 50], 2, 2, 17, 4, 16),
    ([385], 16, 1, 33, 16, 64), ([300], 1, 1, 300, 0, 128), ([1000, 130], 6, 2, 100, 20, 64), ([90], 64, 1, 7, 3, 16),
    ([400, 3, 260, 1, 128, 129, 127, 256], 16, 2, 1, 2, 64), ([5, 600], 32, 8, 4, 3, 256),
]


@pytest.mark.parametrize("shape", SHAPES)
@pytest.mark.parametrize("kind", [None, "causal", "window", "any"])
def test_against_oracle(shape, kind):
    d = _inputs(*shape)
    lo, hi = _ranges(kind, d)
    _check(d, *_run(d, key_lo=lo, key_hi=hi), lo, hi)


FORCED = [(mode, parts) for mode in range(3) for parts in (1, 2, 7, 60, -1, -2, -3, -8)] + [(0, 152), (1, 700)]


@pytest.mark.parametrize("mode,parts", FORCED)
@pytest.mark.parametrize("shape", [([777], 28, 4, 1, 1, 16), ([300, 0, 129, 1], 12, 2, 5, 6, 32), ([1000, 130], 6, 2, 100, 20, 64), ([513] * 9, 2, 2, 1, 0, 256),
                                   ([70, 640], 5, 1, 60, 9, 128)])
@pytest.mark.parametrize("kind,cap", [(None, 0.0), ("any", 0.0), ("causal", 20.0)])
def test_every_kernel(mode, parts, shape, kind, cap):
    d = _inputs(*shape)
    lo, hi = _ranges(kind, d)
    for fill in (0, 255):      # what the workspace holds does not matter
        B, Hq, Lq = d["q"].shape[:3]
        n = 16 if parts < 0 else B * Hq * Lq * parts * 520 if mode == 2 else parts * (2 * (16 << mode) * 520 + 16)
        out, lse = api.cover_debug_attn_paged(d["q"], d["kp"], d["vp"], d["table"], d["lens"], d["km"], d["vm"], d["seeds"], q0=d["q0"], mode=mode,
                                              parts=parts, key_lo=lo, key_hi=hi, softcap=cap,
                                              workspace=torch.full((n,), fill, device="cuda", dtype=torch.uint8))
        torch.cuda.synchronize()
        assert api.cover_device_status() == 0
    _check(d, out, lse, lo, hi, cap)


@pytest.mark.parametrize("cap", [30.0, 0.5, 1e4, 55.0, 56.0, 3e38, 1e-30])
@pytest.mark.parametrize("Lq", [1, 4, 60])
def test_capped_scores(cap, Lq):
    d = _inputs([700, 520], 14, 2, Lq, 12, 32, scale=4.0)
    lo, hi = _ranges("blocks", d)
    _check(d, *_run(d, key_lo=lo, key_hi=hi, softcap=cap), lo, hi, cap)


@pytest.mark.parametrize("scale", [0.01, 8.0, 60.0])
@pytest.mark.parametrize("Lq", [1, 40])
def test_flat_and_peaked_scores(scale, Lq):
    d = _inputs([900], 8, 2, Lq, 6, 64, scale=scale)
    _check(d, *_run(d))


@pytest.mark.parametrize("Lq", [1, 3, 70])
def test_pages_that_a_sequence_does_not_have(Lq):
    """Holes at the front, inside and at the end of a table, entries of any value: their positions hold no key, a seed's neither."""
    d = _inputs([640, 640, 640, 640], 8, 2, Lq, 5, 16)
    t = d["table"]
    t[0, :9], t[1, 3], t[1, 20:30], t[2, -5:] = -1, t.max() + 1, 2 ** 31 - 1, -2 ** 31
    t[3] = -1
    _check(d, *_run(d))
    lo, hi = _ranges("window", d)
    _check(d, *_run(d, key_lo=lo, key_hi=hi), lo, hi)


@pytest.mark.parametrize("Lq", [1, 5, 80])
def test_lengths_and_positions_of_any_value(Lq):
    d = _inputs([200, 200, 200, 200, 200], 8, 4, Lq, 4, 32, M=9)
    d["lens"] = _ints([-1, -2 ** 31, 2 ** 31 - 1, 201, 199])
    q0 = _ints([0, 5, 2 ** 31 - 1, -2 ** 31, -3])
    d["q0"] = q0
    d["seeds"] = _ints([[0, 1, 2, 3], [5, 5, 6, 7], [2 ** 31 - 1, 0, 1, 2], [-2 ** 31, 0, 1, 2], [-3, -2, 0, 1]])
    _check(d, *_run(d))
    e = _ints([[-2 ** 31] * Lq, [0] * Lq, [5] * Lq, [2 ** 31 - 1] * Lq, [-1] * Lq])
    f = _ints([[2 ** 31 - 1] * Lq, [0] * Lq, [2 ** 31 - 1] * Lq, [-2 ** 31] * Lq, [77] * Lq])
    _check(d, *_run(d, key_lo=e, key_hi=f), e, f)


@pytest.mark.parametrize("Lq,kind", [(1, None), (4, "window"), (50, "causal"), (300, "blocks")])
def test_what_a_row_does_not_see_does_not_reach_it(Lq, kind):
    """NaN and infinities in K and V behind the lengths, outside the ranges and at the seeds' own positions."""
    d = _inputs([600, 333], 8, 2, Lq, 6, 64, junk=False)
    lo, hi = _ranges(kind, d)
    ref = _run(d, key_lo=lo, key_hi=hi)
    j = torch.arange(d["table"].shape[1] * 64, device="cuda")
    r = torch.arange(Lq, device="cuda")
    for b in range(2):
        at = d["q0"][b] + r
        seen = (j < d["lens"][b]).expand(Lq, -1)
        if lo is not None:
            seen = seen & (j >= lo[b][:, None])
        if hi is not None:
            seen = seen & (j < hi[b][:, None])
        seed = torch.isin(at, d["seeds"][b])
        seen = seen & ~((j == at[:, None]) & seed[:, None])
        for x in j[~seen.any(0)].tolist():
            p = int(d["table"][b, x // 64])
            if p >= 0:
                d["kp"][p, :, x % 64] = [math.nan, math.inf, -math.inf, math.nan][x % 4]
                d["vp"][p, :, x % 64] = [math.inf, math.nan, math.nan, -math.inf][x % 4]
    out, lse = _run(d, key_lo=lo, key_hi=hi)
    assert torch.equal(out, ref[0]) and torch.equal(lse, ref[1])


@pytest.mark.parametrize("Lq,Hq", [(1, 8), (3, 8), (40, 2), (300, 2)])
def test_rows_that_see_a_value_that_is_not_finite(Lq, Hq):
    """Some rows see it, some do not: those are as without it, these have no finite number in its column."""
    d = _inputs([400, 400], Hq, 2, Lq, 0, 32, junk=False)
    hi = _ints([[400] * Lq, [150] * Lq])
    if Lq > 1:
        hi[0, ::2] = 100
    ref, _ = _run(d, key_hi=hi)
    for value in (math.nan, math.inf, -math.inf):
        for b in range(2):
            d["vp"][int(d["table"][b, 200 // 32]), :, 200 % 32, 77] = value
        out, _ = _run(d, key_hi=hi)
        sees = hi > 200
        assert torch.equal(out.transpose(1, 2)[~sees], ref.transpose(1, 2)[~sees])
        assert not out.transpose(1, 2)[sees][..., 77].isfinite().any()


def test_keys_that_are_not_numbers_reach_the_rows_that_see_them():
    for Lq in (1, 50):
        d = _inputs([300], 4, 2, Lq, 0, 16, junk=False)
        hi = torch.full((1, Lq), 300, device="cuda", dtype=torch.int32)
        if Lq > 1:
            hi[0, 10:] = 100
        ref, ref_lse = _run(d, key_hi=hi)
        d["kp"][int(d["table"][0, 200 // 16]), :, 200 % 16, 5] = math.nan
        out, lse = _run(d, key_hi=hi)
        sees = (hi > 200)[0]
        assert out[:, :, sees].isnan().all() and lse[:, :, sees].isnan().all()
        assert torch.equal(out[:, :, ~sees], ref[:, :, ~sees]) and torch.equal(lse[:, :, ~sees], ref_lse[:, :, ~sees])


@pytest.mark.parametrize("lens", ["equal", "ragged", "one"])
@pytest.mark.parametrize("B,Lq", [(70, 1), (400, 1), (33, 3), (1000, 2)])
def test_many_sequences(B, Lq, lens):
    """Against the same call sequence by sequence: the parts of the keys differ, the rows agree up to rounding."""
    n = {"equal": [130] * B, "ragged": [(37 * b) % 300 for b in range(B)], "one": [0] * (B - 1) + [3000]}[lens]
    d = _inputs(n, 4, 2, Lq, 2, 16)
    out, lse = _run(d)
    pick = sorted({0, 1, B // 2, B - 2, B - 1})
    for b in pick:
        e = {k: (t if k in ("kp", "vp") or t is None else t[b:b + 1].contiguous()) for k, t in d.items()}
        o, s = _run(e)
        _check(e, o, s)
        _check(e, out[b:b + 1], lse[b:b + 1])


def test_long_memory_and_a_pool_of_more_than_2_32_elements():
    """The pages used lie at both ends of the pool; a row's weights are spread over more than 100000 keys."""
    page, H, L = 256, 8, 131000
    n_pages = 2 ** 32 // (page * H * 128) + 600
    kp, vp = (torch.empty((n_pages, H, page, 128), device="cuda", dtype=BF) for _ in range(2))
    need = -(-L // page)
    table = torch.arange(n_pages - 1, n_pages - 1 - need, -1, device="cuda", dtype=torch.int32)[None].contiguous()
    table[0, ::2] = torch.arange(table[0, ::2].numel(), device="cuda", dtype=torch.int32)
    rows = [_randn(need, H, page, 128, seed=s) for s in (1, 2)]
    kp[table[0].long()], vp[table[0].long()] = rows[0], rows[1]
    for Lq in (1, 40):
        q = _randn(1, 32, Lq, 128, seed=3)
        out, lse = api.cover_attn_fwd_paged(q, kp, vp, table, _ints([L]))
        torch.cuda.synchronize()
        assert api.cover_device_status() == 0
        for h in (0, 5):
            k, v = (x[:, h].reshape(-1, 128)[:L].double() for x in rows)
            z = q[0, 4 * h:4 * h + 4].double() @ k.T / math.sqrt(128)
            ref = torch.softmax(z, -1) @ v
            mass = torch.softmax(z, -1) @ v.abs()
            assert ((out[0, 4 * h:4 * h + 4].double() - ref).abs() <= 2.0 ** -8 * ref.abs() + 2.0 ** -7 * mass).all()
            assert ((lse[0, 4 * h:4 * h + 4].double() - torch.logsumexp(z, -1)).abs() < 2.0 ** -16).all()


def test_the_same_bits_again_and_guarded_outputs():
    d = _inputs([700, 90, 0], 28, 4, 9, 5, 16)
    out, lse = _run(d)
    flat, flat_lse = torch.full((out.numel() + 256,), 7.0, device="cuda", dtype=BF), torch.full((lse.numel() + 64,), 7.0, device="cuda")
    n = api.cover_attn_paged_workspace_bytes(3, 28, 4, 9, d["table"].shape[1], 16)
    for fill in (0, 255):
        ws = torch.full((max(n, 1) + 64,), fill, device="cuda", dtype=torch.uint8)
        o, s = flat[128:128 + out.numel()].view(out.shape), flat_lse[32:32 + lse.numel()].view(lse.shape)
        a, b = _run(d, out=o, lse=s, workspace=ws[:max(n, 1)])
        assert a is o and b is s and torch.equal(o, out) and torch.equal(s, lse)
        assert (ws[max(n, 1):] == fill).all()
        assert (flat[:128] == 7).all() and (flat[128 + out.numel():] == 7).all() and (flat_lse[:32] == 7).all() and (flat_lse[32 + lse.numel():] == 7).all()
    a, none = _run(d, want_lse=False)
    assert none is None and torch.equal(a, out)


def test_captured_with_lengths_that_change():
    d = _inputs([500, 500, 500], 8, 2, 2, 4, 16)
    _run(d)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out, lse = api.cover_attn_fwd_paged(d["q"], d["kp"], d["vp"], d["table"], d["lens"], d["km"], d["vm"], d["seeds"], q0=d["q0"])
    for lens in ([500, 500, 500], [0, 1, 499], [128, 0, 0], [300, 200, 100]):
        d["lens"].copy_(_ints(lens))
        d["q0"].copy_(_ints([max(0, x - 2) for x in lens]))
        graph.replay()
        torch.cuda.synchronize()
        assert api.cover_device_status() == 0
        _check(d, out, lse)


def test_two_calls_at_once():
    ds = [_inputs([900, 200], 28, 4, 3, 4, 16), _inputs([64, 1500], 8, 8, 40, 4, 64, seed=50)]
    refs = [_run(d) for d in ds]
    streams = [torch.cuda.Stream() for _ in ds]
    torch.cuda.synchronize()
    got = [[], []]
    for _ in range(20):
        for d, s, g in zip(ds, streams, got):
            with torch.cuda.stream(s):
                g.append(api.cover_attn_fwd_paged(d["q"], d["kp"], d["vp"], d["table"], d["lens"], d["km"], d["vm"], d["seeds"], q0=d["q0"]))
    torch.cuda.synchronize()
    assert api.cover_device_status() == 0
    for (ro, rl), g in zip(refs, got):
        assert all(torch.equal(o, ro) and torch.equal(s, rl) for o, s in g)


def test_native_and_python_marshalling_agree():
    d = _inputs([300, 40], 8, 2, 5, 4, 32)
    lo, hi = _ranges("window", d)
    a = _run(d, key_lo=lo, key_hi=hi, softcap=20.0)
    b = _run(d, key_lo=lo, key_hi=hi, softcap=20)
    s = torch.cuda.Stream()
    torch.cuda.synchronize()
    c = _run(d, key_lo=lo, key_hi=hi, softcap=20.0, stream=s)
    for x in (b, c):
        assert torch.equal(a[0], x[0]) and torch.equal(a[1], x[1])


def test_refusals():
    d = _inputs([300, 40], 8, 2, 5, 4, 32)
    call = lambda **kw: api.cover_attn_fwd_paged(*[kw.pop(n, d[n]) for n in ("q", "kp", "vp", "table", "lens", "km", "vm", "seeds")],  # noqa: E731
                                                 **{"q0": d["q0"], **kw})
    for kw in (dict(q0=None), dict(lens=None), dict(lens=d["lens"][:1]), dict(lens=d["lens"].long()), dict(table=d["table"][:1]),
               dict(table=d["table"].long()), dict(vp=d["vp"][1:]), dict(kp=d["kp"].float()), dict(km=None), dict(km=d["km"][:, :1].contiguous()),
               dict(seeds=d["seeds"][:1]), dict(key_lo=d["lens"]), dict(q=d["q"].float()), dict(q=d["q"].transpose(1, 2)),
               dict(out=d["q"][:1]), dict(lse=d["q"]), dict(workspace=torch.zeros(0, device="cuda", dtype=torch.int32))):
        with pytest.raises((TypeError, ValueError)):
            call(**kw)
    for kw in (dict(softcap=-1.0), dict(softcap=math.nan)):
        with pytest.raises(CoverError, match="INVALID"):
            call(**kw)
    with pytest.raises(CoverError, match="INVALID"):
        call(q=d["q"][:, :3].contiguous())
    small = torch.zeros((3, 2, 16, 64), device="cuda", dtype=BF)
    with pytest.raises(CoverError, match="UNSUPPORTED"):
        api.cover_attn_fwd_paged(d["q"][..., :64].contiguous(), small, small, d["table"], d["lens"])


def test_append_attend_and_score_as_one_step():
    """A serving step: two rounds of appending rows (rotated) and attending over all that was appended, against the dense window
    call over the same keys; then the logits' log probabilities."""
    B, Hq, Hkv, page = 2, 8, 2, 16
    kp, vp = api.paged_memory(20, Hkv, page)
    table = _ints([[3, 0, 7, 9, 11, 1], [2, 5, 4, 6, 8, 10]])
    f, _ = api.rope_frequencies(128)
    have = [0, 0]
    k_all, v_all = torch.zeros((B, Hkv, 90, 128), device="cuda", dtype=BF), torch.zeros((B, Hkv, 90, 128), device="cuda", dtype=BF)
    for n, count in ((37, [37, 20]), (1, [1, 1]), (4, [4, 4])):
        qkv = _randn(B, n, Hq + 2 * Hkv, 128, seed=n)
        q, k, v = (qkv[:, :, a:b].transpose(1, 2) for a, b in ((0, Hq), (Hq, Hq + Hkv), (Hq + Hkv, Hq + 2 * Hkv)))
        start = _ints(have)
        q, k = api.cover_paged_append(k, v, kp, vp, table, start=start, count=_ints(count), q=q, inv_freq=f, want_k=True)
        for b in range(B):
            k_all[b, :, have[b]:have[b] + count[b]], v_all[b, :, have[b]:have[b] + count[b]] = k[b, :, :count[b]], v[b, :, :count[b]]
            have[b] += count[b]
        seeds = (start[:, None] + torch.tensor([[n - 1, 0]], device="cuda")).int().contiguous()
        km, vm = (x[:, :, [n - 1, 0]].contiguous() * 2 for x in (k, v))
        out, lse = api.cover_attn_fwd_paged(q, kp, vp, table, _ints(have), km, vm, seeds, q0=start)
        for b in range(B):
            ref, ref_lse = api.cover_attn_fwd_prefix(q[b:b + 1, :, :count[b]].contiguous(), k_all[b:b + 1, :, :have[b]].contiguous(),
                                                     v_all[b:b + 1, :, :have[b]].contiguous(), km[b:b + 1], vm[b:b + 1], seeds[b:b + 1],
                                                     q0=have[b] - count[b])
            assert (out[b:b + 1, :, :count[b]].float() - ref.float()).abs().max() < 1e-2 * max(1.0, ref.abs().max().item())
            assert (lse[b:b + 1, :, :count[b]] - ref_lse).abs().max() < 1e-4
        x = (out.transpose(1, 2).reshape(B * n, Hq * 128).float() @ torch.randn((Hq * 128, 777), generator=_gen(9), device="cuda")).to(BF)
        tok = torch.randint(0, 777, (B * n,), generator=_gen(n), device="cuda").int()
        r = api.cover_logprob_fwd(x, tok, topk=4)
        u = api.cover_score_fwd(x, 1, 0, cur_tok=tok)
        assert torch.equal(r["top_idx"][:, 0], u["argmax"]) and (r["logp"] + u["score"]).abs().max() < 1e-3
        assert (r["entropy"] - u["entropy"]).abs().max() < 1e-4
    torch.cuda.synchronize()
    assert api.cover_device_status() == 0
