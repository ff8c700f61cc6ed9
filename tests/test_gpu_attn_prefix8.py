"""GPU parity of the window attention over an 8-bit memory against the fp64 oracle.

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

from oracle import memory8_oracle as M8
from paper_2602_06161_gb300 import CoverError, api

pytestmark = pytest.mark.gpu


def _gen(seed):
    return torch.Generator("cuda").manual_seed(seed)


def _randn(*shape, seed=0, scale=1.0):
    return (torch.randn(shape, generator=_gen(seed), device="cuda") * scale).to(torch.bfloat16)


def _h(t):
    return t.view(torch.uint8).cpu().numpy() if t.dtype == torch.float8_e4m3fn else t.double().cpu().numpy() if t.is_floating_point() else t.cpu().numpy()


def _inputs(B, Hq, Hkv, Lq, Lk, S, q0, seed=0, scale=1.0):
    g = _gen(seed)
    mem = api.kv8_memory(B, Hkv, Lk)
    api.cover_kv8_write(_randn(B, Hkv, Lk, 128, seed=seed + 1, scale=scale), _randn(B, Hkv, Lk, 128, seed=seed + 2), *mem)
    d = dict(q=_randn(B, Hq, Lq, 128, seed=seed + 3), mem=mem, km=None, vm=None, seeds=None, q0=q0)
    if S:
        near = torch.rand((B, Lk), generator=g, device="cuda")
        near[:, q0:q0 + Lq] -= 0.6
        d["seeds"] = near.argsort(1)[:, :S].to(torch.int32).contiguous()
        if S >= 4:
            d["seeds"][:, 3] = d["seeds"][:, 0]    # named twice
            d["seeds"][:, 2] = Lk + 5              # out of range
        d["km"], d["vm"] = _randn(B, Hkv, S, 128, seed=seed + 4), _randn(B, Hkv, S, 128, seed=seed + 5)
    return d


def _run(d, **kw):
    out, lse = api.cover_attn_fwd_prefix8(d["q"], *d["mem"], d["km"], d["vm"], d["seeds"], q0=d["q0"], **kw)
    torch.cuda.synchronize()
    assert api.cover_device_status() == 0
    return out, lse


def _reference(d, key_lo=None, key_hi=None, softcap=0.0):
    n = lambda t: None if t is None else _h(t)  # noqa: E731
    k8, v8, kx, vx = (_h(m) for m in d["mem"])
    return M8.attention(_h(d["q"]), M8.decode(k8, kx), M8.decode(v8, vx), n(d["km"]), n(d["vm"]), n(d["seeds"]),
                        q0=d["q0"], key_lo=n(key_lo), key_hi=n(key_hi), softcap=softcap)


def _check(d, out, lse, key_lo=None, key_hi=None, softcap=0.0, per_score=2.0 ** -20):
    ref, ref_lse, mass, size = _reference(d, key_lo, key_hi, softcap)
    delta = (per_score * size + 2.0 ** -20 * softcap)[..., None]
    tol = 2.0 ** -8 * np.abs(ref) + (2.0 ** -8 + 4 * delta) * mass * (1 + 2.0 ** -6)
    err = np.abs(_h(out) - ref)
    assert (err <= tol).all(), float((err / np.maximum(tol, 1e-30)).max())
    none = ref_lse == -math.inf
    got = _h(lse)
    assert np.array_equal(got == -math.inf, none)
    tol = delta[..., 0] + 2.0 ** -20 * (1 + np.abs(np.where(none, 0, ref_lse)))
    assert (np.abs(got - ref_lse)[~none] <= tol[~none]).all()


def _ranges(kind, B, Lq, Lk, q0, seed=0):
    at = q0 + torch.arange(Lq, device="cuda", dtype=torch.int32).repeat(B, 1)
    lens = torch.randint(0, Lk + 1, (B, 1), generator=_gen(seed), device="cuda").int()
    if kind == "lens":
        lens[0] = 0
        return None, lens.expand(B, Lq).contiguous()
    if kind == "causal":
        return None, at + 1
    if kind == "prefix":
        return torch.zeros_like(at), torch.maximum(at + 1, lens)
    if kind == "window":
        return at - 100, at + 3
    if kind == "docs":
        size = max(1, Lk // 3)
        return at // size * size, at // size * size + size
    lo = torch.randint(-5, Lk + 5, (B, Lq), generator=_gen(seed), device="cuda").int()     # anything, many rows empty
    return lo, lo + torch.randint(-3, 40, (B, Lq), generator=_gen(seed + 1), device="cuda").int()


SHAPES = [   # B, Hq, Hkv, Lq, Lk, S, q0
    (1, 1, 1, 1, 1, 0, 0), (1, 28, 4, 1, 777, 0, 776), (3, 4, 4, 1, 129, 1, 40), (1, 8, 2, 2, 128, 0, 3), (2, 28, 4, 32, 300, 8, 100),
    (1, 4, 4, 128, 128, 128, 0), (1, 2, 1, 129, 257, 5, 128), (1, 3, 1, 200, 511, 40, 300), (5, 2, 2, 17, 64, 4, 30),
    (1, 16, 1, 33, 385, 16, 352), (1, 1, 1, 300, 300, 0, 0), (2, 6, 2, 100, 1000, 20, 450), (1, 64, 1, 7, 90, 3, 50),
]


@pytest.mark.parametrize("shape", SHAPES)
@pytest.mark.parametrize("kind", [None, "lens", "prefix", "any"])
def test_against_oracle(shape, kind):
    B, Hq, Hkv, Lq, Lk, S, q0 = shape
    d = _inputs(*shape[:6], q0)
    lo, hi = (None, None) if kind is None else _ranges(kind, B, Lq, Lk, q0)
    out, lse = _run(d, key_lo=lo, key_hi=hi)
    _check(d, out, lse, lo, hi)


@pytest.mark.parametrize("cap", [30.0, 0.5, 1e4])
@pytest.mark.parametrize("kind", ["causal", "docs", "window"])
def test_capped_scores(cap, kind):
    B, Hq, Hkv, Lq, Lk, S, q0 = 2, 14, 2, 60, 700, 12, 500
    d = _inputs(B, Hq, Hkv, Lq, Lk, S, q0, scale=4.0)
    lo, hi = _ranges(kind, B, Lq, Lk, q0)
    out, lse = _run(d, key_lo=lo, key_hi=hi, softcap=cap)
    _check(d, out, lse, lo, hi, cap)


@pytest.mark.parametrize("cap", [3e5, 1e9, 1e18, 3e38])
@pytest.mark.parametrize("mode", range(4))
def test_caps_far_above_the_scores(cap, mode):
    """They change nothing: c tanh(s / c) is s but for (s / c)^2 / 3 < 2^-30 of it. The polynomial is off by 2^-22 of the score and six
    roundings of 2^-24, which with what an uncapped score is off by is at most 2^-19 of sum |q_i k_i| / sqrt(D)."""
    d = _inputs(2, 8, 2, 30, 500, 6, 400, scale=2.0)
    lo, hi = _ranges("prefix", 2, 30, 500, 400)
    out, lse = api.cover_debug_attn_prefix8(d["q"], *d["mem"], d["km"], d["vm"], d["seeds"], q0=400, mode=mode, key_lo=lo, key_hi=hi,
                                            softcap=cap)
    torch.cuda.synchronize()
    assert api.cover_device_status() == 0
    _check(d, out, lse, lo, hi, per_score=2.0 ** -19)


@pytest.mark.parametrize("scale", [0.01, 8.0, 60.0])
def test_flat_and_peaked_scores(scale):
    d = _inputs(1, 8, 2, 40, 900, 6, 300, scale=scale)
    out, lse = _run(d)
    _check(d, out, lse)


@pytest.mark.parametrize("Lq,Lk", [(1, 40000), (3, 9000), (64, 20000)])
def test_long_memories(Lq, Lk):
    d = _inputs(1, 4, 2, Lq, Lk, 4, Lk - Lq)
    out, lse = _run(d)
    _check(d, out, lse)


def test_rows_grow_late():
    """The largest scores come last, and far above the first ones: every running maximum is outdone."""
    d = _inputs(1, 4, 1, 20, 1500, 0, 0)
    for e in range(4):
        d["mem"][2][:, :, 350 * (e + 1):] += 2          # key rows grow by 4 each time
    out, lse = _run(d)
    _check(d, out, lse)


def test_exponents_of_every_size():
    """Rows of keys and values from 2^-100 to 2^60 (the scores stay finite: queries are as small as keys are large)."""
    d = _inputs(1, 2, 1, 5, 300, 0, 0)
    d["mem"][2].copy_(torch.randint(17, 126, (1, 1, 300), generator=_gen(1), device="cuda").to(torch.uint8))
    d["mem"][3].copy_(torch.randint(17, 187, (1, 1, 300), generator=_gen(2), device="cuda").to(torch.uint8))
    out, lse = _run(d)
    _check(d, out, lse)
    d["mem"][2].add_(60)
    d["q"].mul_(2.0 ** -60)
    out, lse = _run(d)
    _check(d, out, lse)
    d["mem"][2].fill_(246)            # the largest bytes, above those that one bf16 multiplication reaches
    d["q"].mul_(2.0 ** -62)
    out, lse = _run(d)
    _check(d, out, lse)


def test_every_code():
    """Codes of every value but NaN, as keys and as values."""
    d = _inputs(1, 2, 1, 9, 254, 0, 0)
    c = torch.arange(254, device="cuda").to(torch.uint8)
    c = c + (c >= 127).to(torch.uint8)
    for i in range(2):
        d["mem"][i].view(torch.uint8)[0, 0] = torch.stack([c.roll(s * (i + 1)) for s in range(128)], 1)
    d["mem"][2].fill_(117)
    d["mem"][3].fill_(120)
    out, lse = _run(d)
    _check(d, out, lse)


def test_what_is_not_seen_does_not_reach_a_row():
    """NaN rows outside a row's keys change no bit; a row that sees one has NaN."""
    B, Hq, Hkv, Lq, Lk, S, q0 = 2, 8, 2, 70, 600, 10, 200
    d = _inputs(B, Hq, Hkv, Lq, Lk, S, q0)
    lo, hi = _ranges("window", B, Lq, Lk, q0)
    ref, ref_lse = _run(d, key_lo=lo, key_hi=hi)
    unseen = torch.ones(Lk, dtype=torch.bool, device="cuda")
    unseen[max(0, q0 - 100):q0 + Lq + 2] = False
    for i in range(2):
        d["mem"][i].view(torch.uint8)[:, :, unseen] = 0x7f
        d["mem"][2 + i][:, :, unseen] = 255
    out, lse = _run(d, key_lo=lo, key_hi=hi)
    assert torch.equal(out, ref) and torch.equal(lse, ref_lse)
    at = q0 + 10
    for i in range(2):
        d2 = dict(d, mem=tuple(m.clone() for m in d["mem"]))
        d2["mem"][2 + i][1, 0, at] = 255
        out, lse = _run(d2, key_lo=lo, key_hi=hi)
        own_pair = (d["seeds"][1] == at).any()
        sees = (lo[1] <= at) & (at < hi[1])
        if own_pair:
            sees[10] = False
        hit = torch.zeros((B, Hq, Lq), dtype=torch.bool, device="cuda")
        hit[1, :Hq // Hkv] = sees
        assert out.isnan().all(-1)[hit].all() and lse.isnan()[hit].all()
        assert torch.equal(out[~hit], ref[~hit]) and torch.equal(lse[~hit], ref_lse[~hit])


def test_a_seed_row_does_not_read_its_cached_row():
    d = _inputs(1, 4, 2, 30, 200, 6, 90)
    ref, ref_lse = _run(d)
    rows = [int(p) for p in d["seeds"][0] if 90 <= p < 120]
    assert rows
    for p in rows:
        d2 = dict(d, mem=tuple(m.clone() for m in d["mem"]))
        d2["mem"][2][:, :, p] = 255
        out, lse = _run(d2)
        assert torch.equal(out[:, :, p - 90], ref[:, :, p - 90]) and torch.equal(lse[:, :, p - 90], ref_lse[:, :, p - 90])
        assert out[:, :, [r for r in range(30) if r != p - 90]].isnan().all()


def test_a_seed_outside_its_rows_keys():
    """The pair of a seed row is seen where its position is among the row's keys, and only there."""
    d = _inputs(1, 2, 1, 4, 50, 0, 20)
    d["seeds"] = torch.tensor([[21, 22]], device="cuda", dtype=torch.int32)
    d["km"], d["vm"] = _randn(1, 1, 2, 128, seed=11), _randn(1, 1, 2, 128, seed=12)
    lo = torch.tensor([[0, 0, 22, 0]], device="cuda", dtype=torch.int32)
    hi = torch.tensor([[50, 21, 23, 0]], device="cuda", dtype=torch.int32)
    out, lse = _run(d, key_lo=lo, key_hi=hi)
    _check(d, out, lse, lo, hi)
    assert torch.equal(out[0, :, 2], d["vm"][0, 0, 1].expand(2, 128))     # its own pair alone


def test_agrees_with_the_bf16_attention_of_what_is_read_back():
    """Read back, the memory is exact in bf16: both attentions are within rounding of each other."""
    for shape in [(2, 28, 4, 32, 1024, 16, 600), (1, 4, 4, 300, 600, 10, 100), (1, 8, 8, 64, 2048, 0, 1984)]:
        d = _inputs(*shape)
        k, v = api.cover_kv8_read(*d["mem"])
        ref, ref_lse = api.cover_attn_fwd_prefix(d["q"], k, v, d["km"], d["vm"], d["seeds"], q0=d["q0"])
        out, lse = _run(d)
        big = k.float().abs().amax() * d["q"].float().abs().amax() * math.sqrt(128)
        assert (lse - ref_lse).abs().max() <= 2 * 2.0 ** -20 * big + 1e-5
        mass = v.float().abs().amax()
        assert (out.float() - ref.float()).abs().max() <= 2 * (2 * 2.0 ** -8 + 4 * 2.0 ** -20 * big) * mass


KERNELS = [(0, 1), (0, 3), (1, 1), (1, 2), (2, 1), (2, 4), (3, 1), (3, 3), (2, 64), (0, -2), (0, -7), (1, -3), (1, -8), (2, -2), (2, -5), (2, -8)]


@pytest.mark.parametrize("mode,nsplit", KERNELS)
@pytest.mark.parametrize("shape", [(1, 1, 1, 1, 1, 0, 0), (2, 28, 4, 3, 700, 4, 300), (1, 8, 2, 40, 385, 9, 200), (1, 4, 1, 150, 640, 20, 400),
                                   (2, 2, 2, 300, 512, 30, 100)])
def test_every_kernel(shape, mode, nsplit):
    """Every kernel on every kind of call, whichever the call itself would take: seeds, key ranges, capped scores, parts of the
    keys that see nothing."""
    B, Hq, Hkv, Lq, Lk, S, q0 = shape
    d = _inputs(*shape[:6], q0, scale=2.0)
    for kind, cap in ((None, 0.0), ("docs", 0.0), ("any", 30.0), (None, 2.0), ("window", 1e4)):
        lo, hi = (None, None) if kind is None else _ranges(kind, B, Lq, Lk, q0)
        out, lse = api.cover_debug_attn_prefix8(d["q"], *d["mem"], d["km"], d["vm"], d["seeds"], q0=q0, mode=mode, nsplit=nsplit,
                                                key_lo=lo, key_hi=hi, softcap=cap)
        torch.cuda.synchronize()
        assert api.cover_device_status() == 0
        _check(d, out, lse, lo, hi, cap)


@pytest.mark.parametrize("mode,more", [(0, 0), (0, 1), (0, 70), (1, 5)])
@pytest.mark.parametrize("B,Lq,lens", [(5, 2, [900, 0, 130, 1, 511]), (32, 1, [900] + [0] * 30 + [3]), (3, 4, [0, 0, 0]), (2, 9, [900, 900])])
def test_parts_of_uneven_sequences(B, Lq, lens, mode, more):
    """A batch's parts go to its sequences by their lengths: long ones among empty ones, all empty, all alike; as many parts as
    sequences, and more than there are KV tiles."""
    d = _inputs(B, 8, 2, Lq, 900, 3, 500)
    hi = torch.tensor([[n] * Lq for n in lens], device="cuda", dtype=torch.int32)
    lo = (hi // 3).contiguous()
    lo[:, 0] = 0
    for kw in (dict(key_hi=hi), dict(key_lo=lo, key_hi=hi), dict(key_lo=lo)):
        out, lse = api.cover_debug_attn_prefix8(d["q"], *d["mem"], d["km"], d["vm"], d["seeds"], q0=500, mode=mode, nsplit=100 + B + more, **kw)
        torch.cuda.synchronize()
        assert api.cover_device_status() == 0
        _check(d, out, lse, kw.get("key_lo"), kw.get("key_hi"))


@pytest.mark.parametrize("mode,nsplit", [(0, 8), (1, 5), (2, 7)])
def test_parts_joined_in_a_cluster(mode, nsplit):
    """The same parts added up by the cluster and by the second kernel: their terms differ by a rounding of the weights at most,
    and rows without a key, parts without a key, NaN and masked-input scores are the same."""
    B, Hq, Hkv, Lq, Lk, S, q0 = 2, 28, 4, 19, 1500, 9, 1400
    d = _inputs(B, Hq, Hkv, Lq, Lk, S, q0)
    d["mem"][2][1, 2, 1100] = 255
    for kind in (None, "any", "lens", "window"):
        lo, hi = (None, None) if kind is None else _ranges(kind, B, Lq, Lk, q0)
        a, b = (api.cover_debug_attn_prefix8(d["q"], *d["mem"], d["km"], d["vm"], d["seeds"], q0=q0, mode=mode, nsplit=n, key_lo=lo,
                                             key_hi=hi, softcap=20.0) for n in (-nsplit, nsplit))
        assert torch.equal(a[0].isnan(), b[0].isnan()) and torch.equal(a[1].isnan(), b[1].isnan())
        assert kind is not None or a[1].isnan().any()
        assert torch.equal(a[1] == -math.inf, b[1] == -math.inf)
        x, y = (t.float().nan_to_num(0.0) for t in (a[0], b[0]))
        assert ((x - y).abs() <= 2.0 ** -7 * y.abs() + 2.0 ** -18).all()
        x, y = (t.nan_to_num(0.0, neginf=0.0) for t in (a[1], b[1]))
        assert ((x - y).abs() <= 2.0 ** -20 * (1 + y.abs())).all()
    torch.cuda.synchronize()
    assert api.cover_device_status() == 0


@pytest.mark.parametrize("mode", range(5))
def test_every_kernel_and_what_is_not_seen(mode):
    """Codes and bytes of NaN behind the keys that rows see change no bit, whatever the kernel; seen, they are NaN."""
    B, Hq, Hkv, Lq, Lk, S, q0 = 1, 8, 2, 40, 600, 6, 200
    d = _inputs(B, Hq, Hkv, Lq, Lk, S, q0)
    hi = torch.full((B, Lq), 450, device="cuda", dtype=torch.int32)
    kw = dict(q0=q0, mode=mode) if mode == 4 else dict(q0=q0, mode=mode, key_hi=hi, nsplit=2)
    call = lambda m: api.cover_debug_attn_prefix8(d["q"], *m, d["km"], d["vm"], d["seeds"], **kw)  # noqa: E731
    if mode < 4:
        ref = call(d["mem"])
        for codes, byte in ((0x7f, 255), (0xff, 120), (0x7e, 250)):
            m = tuple(x.clone() for x in d["mem"])
            for i in range(2):
                m[i].view(torch.uint8)[:, :, 450:] = codes
                m[2 + i][:, :, 450:] = byte
            out = call(m)
            assert torch.equal(out[0], ref[0]) and torch.equal(out[1], ref[1])
    for i in range(2):
        m = tuple(x.clone() for x in d["mem"])
        m[2 + i][0, 1, 30] = 255
        out, lse = call(m)
        assert out[:, 4:].isnan().all() and lse[:, 4:].isnan().all() and not out[:, :4].isnan().any()
    torch.cuda.synchronize()
    assert api.cover_device_status() == 0


@pytest.mark.parametrize("shape", [(2, 28, 4, 32, 700, 4, 300), (1, 8, 8, 40, 385, 9, 345), (1, 2, 1, 300, 300, 7, 0)])
def test_read_back_kernel(shape):
    d = _inputs(*shape)
    out, lse = api.cover_debug_attn_prefix8(d["q"], *d["mem"], d["km"], d["vm"], d["seeds"], q0=shape[6], mode=4)
    torch.cuda.synchronize()
    assert api.cover_device_status() == 0
    _check(d, out, lse)


@pytest.mark.parametrize("mode", [0, 1])
def test_weights_of_every_size(mode):
    """Few rows: the weights of a key whose V row is far smaller or larger than the others' count as they are, and tails of
    weights far below the largest do not vanish."""
    d = _inputs(1, 2, 1, 5, 300, 0, 0)
    d["mem"][3].copy_(torch.randint(17, 187, (1, 1, 300), generator=_gen(2), device="cuda").to(torch.uint8))
    out, lse = api.cover_debug_attn_prefix8(d["q"], *d["mem"], q0=0, mode=mode)
    _check(d, out, lse)
    # one key with nearly all of the weight and a V row of zeros; the others share 2^-12 of it
    d = _inputs(1, 1, 1, 1, 4000, 0, 0)
    d["q"].fill_(0.25)
    d["mem"][0].view(torch.uint8).fill_(0)
    d["mem"][0].view(torch.uint8)[0, 0, 77] = 0x70            # 128: a score of 128 * 128 * 2^x * 0.25 / sqrt(128)
    d["mem"][2].fill_(127)
    d["mem"][2][0, 0, 77] = 127 - 4                           # about 22.6, against zero
    d["mem"][1].view(torch.uint8)[0, 0, 77] = 0
    out, lse = api.cover_debug_attn_prefix8(d["q"], *d["mem"], q0=0, mode=mode)
    _check(d, out, lse)


def test_outputs_given_and_repeated():
    d = _inputs(2, 8, 2, 50, 3000, 8, 100)
    ref, ref_lse = _run(d)
    out, lse = torch.empty_like(ref), torch.empty_like(ref_lse)
    ws = torch.empty(api.cover_attn_prefix8_workspace_bytes(2, 8, 2, 50, 3000) + 64, dtype=torch.uint8, device="cuda")
    for fill in (0, 255):
        ws.fill_(fill)
        a, b = _run(d, out=out, lse=lse, workspace=ws)
        assert a is out and b is lse and torch.equal(out, ref) and torch.equal(lse, ref_lse)
    _, none = _run(d, want_lse=False)
    assert none is None


def test_streams_and_graphs():
    d = _inputs(2, 8, 2, 40, 2500, 8, 100)
    e = _inputs(2, 8, 2, 40, 2500, 8, 100, seed=40)
    ref, ref2 = _run(d)[0], _run(e)[0]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    for _ in range(3):
        got, _ = api.cover_attn_fwd_prefix8(d["q"], *d["mem"], d["km"], d["vm"], d["seeds"], q0=100, stream=side)
        got2, _ = api.cover_attn_fwd_prefix8(e["q"], *e["mem"], e["km"], e["vm"], e["seeds"], q0=100)
        torch.cuda.synchronize()
        assert torch.equal(got, ref) and torch.equal(got2, ref2)
    ws = torch.empty(max(16, api.cover_attn_prefix8_workspace_bytes(2, 8, 2, 40, 2500)), dtype=torch.uint8, device="cuda")
    graphs, outs = [], []
    for x in (d, e):          # two graphs with one workspace, replayed one after the other
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            outs.append(api.cover_attn_fwd_prefix8(x["q"], *x["mem"], x["km"], x["vm"], x["seeds"], q0=100, workspace=ws)[0])
        graphs.append(g)
    for _ in range(3):
        for g in graphs:
            g.replay()
    torch.cuda.synchronize()
    assert torch.equal(outs[0], ref) and torch.equal(outs[1], ref2)


def test_refusals():
    d = _inputs(1, 4, 2, 8, 64, 2, 10)
    a = (d["q"], *d["mem"])
    for kw in (dict(q0=-1), dict(q0=57), dict(q0=0, softcap=-1.0), dict(q0=0, softcap=math.nan), dict(q0=0, softcap=math.inf)):
        with pytest.raises(CoverError):
            api.cover_attn_fwd_prefix8(*a, **kw)
    with pytest.raises(TypeError, match="q must be"):
        api.cover_attn_fwd_prefix8(d["q"].float(), *d["mem"], q0=0)
    with pytest.raises(ValueError, match="matching q"):
        api.cover_attn_fwd_prefix8(d["q"][..., :64].contiguous(), *d["mem"], q0=0)
    with pytest.raises(ValueError, match="key_hi"):
        api.cover_attn_fwd_prefix8(*a, q0=0, key_hi=torch.zeros((1, 7), device="cuda", dtype=torch.int32))
    with pytest.raises(TypeError, match="key_lo"):
        api.cover_attn_fwd_prefix8(*a, q0=0, key_lo=torch.zeros((1, 8), device="cuda", dtype=torch.int64))
    with pytest.raises(ValueError, match="k_seedmask"):
        api.cover_attn_fwd_prefix8(*a, d["km"][:, :1].contiguous(), d["vm"], d["seeds"], q0=0)
    with pytest.raises(ValueError, match="contiguous"):
        api.cover_attn_fwd_prefix8(d["q"].transpose(1, 2), *d["mem"], q0=0)
    with pytest.raises(ValueError, match="out must match"):
        api.cover_attn_fwd_prefix8(*a, q0=0, out=torch.empty((1, 4, 7, 128), device="cuda", dtype=torch.bfloat16))
    for kw in (dict(mode=5), dict(mode=-1), dict(mode=0, nsplit=0), dict(mode=2, nsplit=65), dict(mode=4, nsplit=2), dict(mode=4, softcap=1.0),
               dict(mode=0, nsplit=-1), dict(mode=2, nsplit=-9), dict(mode=3, nsplit=-2), dict(mode=4, nsplit=-2), dict(mode=0, nsplit=100), dict(mode=0, nsplit=110),
               dict(mode=0, nsplit=4197)):
        with pytest.raises(CoverError):
            api.cover_debug_attn_prefix8(*a, q0=0, **kw)
    small = api.kv8_memory(1, 2, 64, 64)
    with pytest.raises(CoverError):
        api.cover_attn_fwd_prefix8(d["q"][..., :64].contiguous(), *small, q0=0)
    big = api.cover_attn_prefix8_workspace_bytes(1, 4, 2, 8, 5000)
    if big:
        e = _inputs(1, 4, 2, 8, 5000, 0, 10)
        with pytest.raises(ValueError, match="workspace"):
            api.cover_attn_fwd_prefix8(e["q"], *e["mem"], q0=0, workspace=torch.empty(big - 1, dtype=torch.uint8, device="cuda"))


def test_a_layers_step():
    """A step of one layer as it is used: rotate, write the block, override the seeds with their cached rows, attend; then
    cache the next seeds' rows. Against the same steps of the oracle."""
    B, Hq, Hkv, L, n, S, q0 = 2, 14, 2, 400, 32, 6, 320
    proj = _randn(B, n, Hq + 2 * Hkv, 128, seed=20)
    q, k, v = (x.transpose(1, 2) for x in proj.split([Hq, Hkv, Hkv], 2))
    mem = api.kv8_memory(B, Hkv, L)
    old_k, old_v = _randn(B, Hkv, L, 128, seed=21), _randn(B, Hkv, L, 128, seed=22)
    api.cover_kv8_write(old_k, old_v, *mem)
    seeds = (q0 + torch.stack([torch.randperm(n)[:S] for _ in range(B)])).to(torch.int32).cuda()
    f, m = api.rope_frequencies(128)
    # the previous step's states of the seeds, cached
    ck, cv = api.cover_kv8_read(*mem, pos=seeds)
    rq, rk = api.cover_rope_fwd(q, k, f, pos0=q0, mscale=m)
    km, vm = api.cover_seed_kv_gather(rk, v.contiguous(), seeds - q0)
    before = tuple(x.clone() for x in mem)
    api.cover_kv8_write(rk, v, *mem, pos0=q0)
    api.cover_kv8_write(ck, cv, *mem, pos=seeds)
    d = dict(q=rq, mem=mem, km=km, vm=vm, seeds=seeds, q0=q0)
    out, lse = _run(d)
    want = [None] * 4
    for i, (rows, cached) in enumerate(((rk, ck), (v, cv))):
        c, x = M8.written(_h(before[i]), _h(before[2 + i]), _h(rows), pos0=q0)
        want[i], want[2 + i] = M8.written(c, x, _h(cached), pos=_h(seeds))
    for got, w in zip(mem, want):
        assert np.array_equal(_h(got), w)
    # the seeds' cached rows came from the memory itself: written again they are the same values
    again, _ = api.cover_kv8_read(*mem, pos=seeds)
    assert torch.equal(again, ck)
    _check(d, out, lse)
