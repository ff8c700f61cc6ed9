"""The rotary and 8-bit memory calls at the ends of what their documentation allows: rows and bounds of every kind, values and bytes
of every size, tensors of another stream. Against the fp64 oracle, with the tolerances of the operators' own tests."""
import math

import numpy as np
import pytest
import torch

from oracle import memory8_oracle as M8
from paper_2602_06161_gb300 import api

pytestmark = pytest.mark.gpu


def _r(*shape, seed=0, scale=1.0, dtype=torch.bfloat16):
    return (torch.randn(shape, generator=torch.Generator("cuda").manual_seed(seed), device="cuda") * scale).to(dtype)


def _h(t):
    return t.view(torch.uint8).cpu().numpy() if t.dtype == torch.float8_e4m3fn else t.double().cpu().numpy() if t.is_floating_point() else t.cpu().numpy()


def _mem(B, H, L, seed=1, scale=1.0):
    m = api.kv8_memory(B, H, L)
    api.cover_kv8_write(_r(B, H, L, 128, seed=seed, scale=scale), _r(B, H, L, 128, seed=seed + 1), *m)
    return m


def _i32(x):
    return torch.tensor(x, device="cuda", dtype=torch.int32)


def _attn(q, mem, mode=None, seeds=(None, None, None), **kw):
    """The call itself, or the kernel ``mode``."""
    r = api.cover_attn_fwd_prefix8(q, *mem, *seeds, **kw) if mode is None else api.cover_debug_attn_prefix8(q, *mem, *seeds, mode=mode, **kw)
    torch.cuda.synchronize()
    assert api.cover_device_status() == 0
    return r


def _check(got, q, mem, seeds=(None, None, None), *, q0, key_lo=None, key_hi=None, softcap=0.0):
    """The weights and the output are rounded to bf16 (half a step each, 2^-8); scores are off by at most 2^-20 of
    sum |q_i k_i| / sqrt(D) and, capped, of the cap; that is at most a factor e^{2d} of a weight. lse is off by d and 2^-20 of its
    sums' rounding."""
    n = lambda t: None if t is None else _h(t)  # noqa: E731
    k, v = (M8.decode(_h(mem[i]), _h(mem[2 + i])) for i in range(2))
    ref, ref_lse, mass, size = M8.attention(_h(q), k, v, *(n(t) for t in seeds), q0=q0, key_lo=n(key_lo), key_hi=n(key_hi), softcap=softcap)
    out, lse = (_h(t) for t in got)
    d = 2.0 ** -20 * (size + softcap)
    tol = 2.0 ** -8 * np.abs(ref) + (2.0 ** -8 + 4 * d[..., None]) * mass * (1 + 2.0 ** -6)
    assert (np.abs(out - ref) <= tol).all()
    none = ref_lse == -math.inf
    assert np.array_equal(lse == -math.inf, none)
    assert (np.abs(np.where(none, 0, lse) - np.where(none, 0, ref_lse)) <= d + 2.0 ** -20 * (1 + np.abs(np.where(none, 0, ref_lse)))).all()


@pytest.mark.parametrize("mode", [2, 3])
@pytest.mark.parametrize("softcap", [0.0, 30.0, 100.0])
def test_warps_that_see_no_key_of_a_tile(mode, softcap):
    """Neighbouring groups of 32 rows see different KV tiles, or half of one, in turns: in every tile some warps store zeros while
    others read their scores."""
    Lq, Lk = 256, 1000
    mem, q = _mem(1, 2, Lk), _r(1, 2, Lq, 128, seed=3)
    group = torch.arange(Lq, device="cuda") // 32
    lo = ((group * 5) % 8 * 128 + (group % 2) * 64).int()[None].contiguous()
    hi = torch.where(group % 3 == 0, lo + 64, lo + 300).int().contiguous()
    for kw in (dict(), dict(nsplit=3)):
        got = _attn(q, mem, mode, q0=100, key_lo=lo, key_hi=hi, softcap=softcap, **kw)
        _check(got, q, mem, q0=100, key_lo=lo, key_hi=hi, softcap=softcap)


def test_rotation_beside_other_tensors():
    """Outputs in one buffer, rows of q between rows of k, are written as they are apart; an output that overlaps another tensor is
    refused, in place too."""
    B, L, D = 2, 37, 64
    qkv, out = _r(B, L, 10, D, seed=20), torch.zeros((B, L, 10, D), device="cuda", dtype=torch.bfloat16)
    parts = lambda t: (t[:, :, :6].transpose(1, 2), t[:, :, 6:8].transpose(1, 2))  # noqa: E731
    (q, k), (oq, ok) = parts(qkv), parts(out)
    f, _ = api.rope_frequencies(D)
    ref = api.cover_rope_fwd(q, k, f, pos0=5)
    got = api.cover_rope_fwd(q, k, f, pos0=5, out_q=oq, out_k=ok)
    assert got[0] is oq and torch.equal(oq, ref[0]) and torch.equal(ok, ref[1]) and not out[:, :, 8:].any()
    for kw in (dict(out_q=q), dict(out_k=q), dict(out_q=q, out_k=q)):
        with pytest.raises(ValueError, match="overlap"):
            api.cover_rope_fwd(q, q, f, **kw)
    shifted = qkv[:, :, 4:8].transpose(1, 2)          # shares two heads with q
    with pytest.raises(ValueError, match="overlap"):
        api.cover_rope_fwd(q, shifted, f, out_q=q)
    with pytest.raises(ValueError, match="overlap"):
        api.cover_rope_fwd(q, shifted, f, out_k=shifted)


def test_the_debug_call_checks_its_tensors():
    q, mem = _r(1, 4, 8, 128), api.kv8_memory(1, 2, 64)
    seeds = (_r(1, 2, 2, 128), _r(1, 2, 2, 128), _i32([[3, 4]]))
    for kw, what in ((dict(key_hi=torch.zeros((1, 8), device="cuda", dtype=torch.int64)), "key_hi"), (dict(key_lo=_i32([[0] * 7])), "key_lo")):
        with pytest.raises((TypeError, ValueError), match=what):
            api.cover_debug_attn_prefix8(q, *mem, q0=0, mode=0, **kw)
    for args in ((seeds[0][:, :1].contiguous(), *seeds[1:]), (*seeds[:2], seeds[2].expand(2, 2).contiguous()), (None, None, seeds[2])):
        with pytest.raises((TypeError, ValueError), match="seed"):
            api.cover_debug_attn_prefix8(q, *mem, *args, q0=0, mode=0)
    with pytest.raises(ValueError, match="k_exp"):
        api.cover_debug_attn_prefix8(q, *mem[:2], mem[2][:, :, :32].contiguous(), mem[3], q0=0, mode=0)


PARTS = [(0, 1), (0, 2), (0, 4), (0, -2), (0, -4), (0, 102), (0, 107), (1, 1), (1, 4), (1, -4), (1, 105), (2, 1), (2, 4), (2, -4), (3, 1), (3, 4)]


@pytest.mark.parametrize("mode,parts", PARTS)
@pytest.mark.parametrize("order", ["small first", "large first", "in turns", "in pairs"])
@pytest.mark.parametrize("large", [2, 36, 60, 90])
def test_values_of_whole_tiles(mode, parts, order, large):
    """KV tiles of zero value rows before, behind and between tiles of rows around 2^(large + 8): the keys of both count alike, in lse
    and in the weights."""
    L, B = 1024, 2
    big = {"small first": [0] * 4 + [1] * 4, "large first": [1] * 4 + [0] * 4, "in turns": [0, 1] * 4, "in pairs": [0, 0, 1, 1, 0, 0, 0, 1]}[order]
    mem, q = _mem(B, 1, L, scale=0.5), _r(B, 2, 3, 128, seed=3, scale=0.5)
    rows = torch.tensor(big, device="cuda", dtype=torch.bool).repeat_interleave(128)
    mem[3][:, :, rows] += large
    mem[1].view(torch.uint8)[:, :, ~rows] = 0
    mem[3][:, :, ~rows] = 127
    kw = dict(key_hi=_i32([[L] * 3, [L - 200] * 3])) if parts > 100 else {}
    got = _attn(q, mem, mode, nsplit=parts, q0=0, **kw)
    _check(got, q, mem, q0=0, **kw)
    # and where the first rows are small, not zero
    mem[1].view(torch.uint8)[:, :, ~rows] = 0x3a
    mem[3][:, :, ~rows] = 20
    got = _attn(q, mem, mode, nsplit=parts, q0=0, **kw)
    _check(got, q, mem, q0=0, **kw)


@pytest.mark.parametrize("mode", [None, 0, 1, 2, 3])
def test_bounds_of_every_size(mode):
    """Rows whose bounds are the ends of int32, or say nothing in another way, among rows that see keys beyond the first KV tile: each
    is held to the memory, whatever its neighbours see."""
    Lq, Lk, q0 = 300, 700, 50
    mem, q = _mem(1, 1, Lk), _r(1, 2, Lq, 128, seed=3)
    seeds = (_r(1, 1, 4, 128, seed=4), _r(1, 1, 4, 128, seed=5), _i32([[60, 61, 62, 349]]))
    ends = [-2 ** 31, -2 ** 31 + 1, -5, 0, 1, 300, Lk, Lk + 1, 2 ** 31 - 1, 2 ** 31 - 128]
    pairs = [(a, b) for a in ends for b in ends] + [(300, 600), (0, 130), (500, Lk)] * 67
    lo, hi = (_i32([[p[i] for p in pairs[:Lq]]]) for i in range(2))
    at = torch.randperm(Lq, generator=torch.Generator().manual_seed(0)).cuda()
    lo, hi = lo[:, at].contiguous(), hi[:, at].contiguous()
    for kw in (dict(key_hi=hi), dict(key_lo=lo), dict(key_lo=lo, key_hi=hi), dict(key_lo=lo, key_hi=hi, softcap=20.0)):
        got = _attn(q, mem, mode, seeds, q0=q0, **kw)
        _check(got, q, mem, seeds, q0=q0, **kw)


@pytest.mark.parametrize("mode,parts", [(0, 1), (0, 3), (1, 1), (2, 1), (2, 3), (2, -2), (3, 1), (3, 3), (4, 1), (None, None)])
@pytest.mark.parametrize("code", [0x7f, 0xff])
@pytest.mark.parametrize("which", [0, 1])
def test_nan_codes(mode, parts, code, which):
    """A code of NaN in a key or value row is a NaN row of the keys' readers, whichever kernel runs; to others it is nothing."""
    Lq, L = 200, 700
    mem, q = _mem(1, 2, L), _r(1, 4, Lq, 128, seed=3)
    kw = dict(q0=0) if mode is None else dict(q0=0, nsplit=parts)
    hi = None
    if mode != 4:
        hi = _i32([[400] * 40 + [L] * (Lq - 40)])
        kw["key_hi"] = hi
    ref = _attn(q, mem, mode, **kw)
    for at, column in ((450, 0), (600, 127), (511, 77)):
        m = tuple(x.clone() for x in mem)
        m[which].view(torch.uint8)[0, 1, at, column] = code
        out, lse = _attn(q, m, mode, **kw)
        sees = torch.ones((1, 4, Lq), dtype=torch.bool, device="cuda") if hi is None else (hi > at)[:, None].repeat(1, 4, 1)
        sees[:, :2] = False
        assert out.isnan().all(-1)[sees].all() and lse.isnan()[sees].all()
        assert torch.equal(out[~sees], ref[0][~sees]) and torch.equal(lse[~sees], ref[1][~sees])


@pytest.mark.parametrize("mode", [None, 0, 1, 2, 3])
@pytest.mark.parametrize("cap", [5.0, 30.0, 50.0, 51.9])
@pytest.mark.parametrize("byte", [20, 60, 95, 119, 160, 184, 200, 218])
def test_capped_values_of_every_size(mode, cap, byte):
    """Scores at both ends of the cap with value rows of every size: sums neither overflow nor vanish."""
    B, Lq, L = 2, 40, 900
    mem, q = _mem(B, 2, L, scale=0.3), _r(B, 4, Lq, 128, seed=3, scale=0.3)
    mem[3].fill_(byte)
    mem[3][:, :, ::3] -= 2
    for shift in (0.0, 30.0, -30.0):       # all scores alike, near the cap, near its opposite
        k = (_r(B, 2, L, 128, seed=8, scale=0.3) + shift * torch.sign(q[:, ::2, :1].float())).bfloat16()
        v = api.kv8_memory(B, 2, L)
        api.cover_kv8_write(k, k, *v)
        m = (v[0], mem[1], v[2], mem[3])
        got = _attn((q + 0.1 * torch.sign(q[:, :, :1])).bfloat16() if shift else q, m, mode, q0=0, softcap=cap)
        _check(got, (q + 0.1 * torch.sign(q[:, :, :1])).bfloat16() if shift else q, m, q0=0, softcap=cap)


@pytest.mark.parametrize("mode", [2, 3])
@pytest.mark.parametrize("L,H", [(900, 3), (1025, 2), (129, 1)])
@pytest.mark.parametrize("byte", [30, 210, 255])
def test_one_value_row_outside_the_others_range(mode, L, H, byte):
    """Wherever it lies in the memory, of which a head may start at any byte: its CTA's sums hold, and so do the others'."""
    mem, q = _mem(1, H, L), _r(1, H, 60, 128, seed=3)
    at = _i32([[L - 60 + i for i in range(60)]])
    for row in (0, 1, 15, 16, 17, 127, 128, L // 2, L - 17, L - 2, L - 1):
        m = tuple(x.clone() for x in mem)
        m[3][0, H - 1, row] = byte
        for kw in (dict(), dict(nsplit=2, key_hi=(at + 1).contiguous())):
            got = _attn(q, m, mode, q0=L - 60, softcap=50.0, **kw)
            if byte < 255:
                _check(got, q, m, q0=L - 60, softcap=50.0, key_hi=kw.get("key_hi"))
            else:
                sees = torch.ones((1, 1, 60), dtype=torch.bool, device="cuda") if "key_hi" not in kw else (kw["key_hi"] > row)[:, None]
                assert torch.equal(got[1][:, -1:].isnan(), sees) and not got[1][:, :-1].isnan().any()


@pytest.mark.parametrize("mode", [None, 0, 1, 2, 3])
@pytest.mark.parametrize("cap", [1e-3, 1e-9, 1e-20, 1e-38, 1e-45])
def test_small_caps(mode, cap):
    """Scores that are all capped to nothing weigh alike, a score of 0 among them."""
    mem, q = _mem(1, 2, 300), _r(1, 4, 40, 128, seed=3)
    q[:, :, ::3] = 0
    mem[0].view(torch.uint8)[:, :, ::2] = 0
    got = _attn(q, mem, mode, q0=0, softcap=cap)
    _check(got, q, mem, q0=0, softcap=cap)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("inter", [False, True])
@pytest.mark.parametrize("D", [64, 6])
def test_frequencies_that_are_not_finite(dtype, inter, D):
    """Their columns are NaN, as the formula's are; the others are as without them."""
    x = _r(1, 2, 5, D, seed=3, dtype=dtype)
    f, _ = api.rope_frequencies(D)
    ref, _ = api.cover_rope_fwd(x, None, f, pos0=3, interleaved=inter)
    g = f.clone()
    g[0], g[2] = math.inf, math.nan
    y, _ = api.cover_rope_fwd(x, None, g, pos0=3, interleaved=inter)
    cols = torch.zeros(D, dtype=torch.bool, device="cuda")
    for i in (0, 2):
        cols[[2 * i, 2 * i + 1] if inter else [i, i + D // 2]] = True
    assert y[..., cols].isnan().all() and torch.equal(y[..., ~cols], ref[..., ~cols])


@pytest.mark.parametrize("inter", [False, True])
@pytest.mark.parametrize("inverse", [False, True])
def test_columns_that_do_not_turn_are_copied(inter, inverse):
    """By the rotation and by its gradient alike, bit for bit, NaN and infinities too."""
    x = _r(2, 3, 5, 16, seed=3, dtype=torch.float32)
    x[0, 0, 0, 12], x[1, 2, 3, 15], x[0, 1, 1, 14] = math.nan, math.inf, -0.0
    f, _ = api.rope_frequencies(12)
    y, _ = api.cover_rope_fwd(x, None, f, pos0=5, interleaved=inter, mscale=1.5, inverse=inverse)
    assert torch.equal(y[..., 12:].contiguous().view(torch.int32), x[..., 12:].contiguous().view(torch.int32))
    assert not torch.equal(y[..., :12], x[..., :12])


@pytest.mark.parametrize("mode", [2, 3, 4])
def test_more_sequences_than_a_grid_is_deep(mode):
    """70000 sequences of three positions, also where the memory is decoded first."""
    B = 70000
    heads = _mem(1, B, 3)
    mem, q = tuple(m.view(B, 1, *m.shape[2:]) for m in heads), _r(B, 2, 1, 128, seed=3)
    ref, ref_lse = _attn(q, mem, 0, q0=1)
    out, lse = _attn(q, mem, mode, q0=1)
    v = api.cover_kv8_read(*heads, dtype=torch.float32)[1].abs().amax()
    assert (out.float() - ref.float()).abs().max() <= 2 * 2.0 ** -7 * v    # each rounds weights and output by 2^-8
    assert (lse - ref_lse).abs().max() <= 2.0 ** -12
    for b in (0, 65535, 65536, B - 1):
        one = tuple(m[b:b + 1].contiguous() for m in mem)
        _check((out[b:b + 1], lse[b:b + 1]), q[b:b + 1], one, q0=1)


@pytest.mark.parametrize("mode,parts", [(0, 3), (0, -3), (1, 3), (2, 1), (2, 3), (2, -3), (3, 1), (3, 3)])
@pytest.mark.parametrize("cap", [30.0, 50.0])
def test_capped_parts_of_different_values(mode, parts, cap):
    """Parts of the keys without a key, with values of other sizes than the others', and masked-input values of every size: what a part's
    reference is changes nothing."""
    q = _r(1, 4, 20, 128, seed=3)
    for L, byte in ((5, 23), (5, 119), (300, 23), (300, 119), (700, 119)):
        mem = _mem(1, 2, L)
        if L == 5:                            # scores near the cap's opposite
            api.cover_kv8_write((_r(1, 2, L, 128, seed=9) - 16 * torch.sign(q[:, ::2, :1])).bfloat16(), _r(1, 2, L, 128, seed=8), *mem)
        mem[3].fill_(byte)
        if L == 700:
            mem[3][:, :, :256] = 60           # the first part's: far smaller, with nearly all of the weight
            api.cover_kv8_write((_r(1, 2, 256, 128, seed=9, scale=0.2) + 4 * torch.sign(q[:, ::2, :1])).bfloat16(), _r(1, 2, 256, 128, seed=8), *mem)
            mem[3][:, :, :256] = 60
        kw = dict(q0=0, softcap=cap)
        if L < 20:
            qq = q[:, :, :L].contiguous()
        else:
            qq = q
        got = _attn(qq, mem, mode, nsplit=parts, **kw)
        _check(got, qq, mem, **kw)
        n = min(L, 4)
        for e in (-90.0, 0.0, 60.0, 90.0):
            for shift in (0.0, 16.0, -16.0):    # the masked-input keys: any, near the cap, near its opposite
                km = (_r(1, 2, n, 128, seed=11) + shift * torch.sign(qq[:, ::2, :n])).bfloat16()
                seeds = (km, (_r(1, 2, n, 128, seed=12) * 2.0 ** e).bfloat16(), torch.arange(n, device="cuda", dtype=torch.int32)[None].contiguous())
                got = _attn(qq, mem, mode, seeds, nsplit=parts, **kw)
                _check(got, qq, mem, seeds, **kw)


@pytest.mark.parametrize("mode,parts", [(0, 1), (0, 3), (1, 1), (2, 1), (2, 2), (2, -2), (3, 1), (3, 2)])
@pytest.mark.parametrize("cap", [30.0, 50.0])
def test_what_is_not_seen_under_a_cap(mode, parts, cap):
    """Rows behind, before and between the keys that a call's rows see change no bit, whatever their bytes and codes; nor do rows of NaN
    that other rows see."""
    Lq, L = 150, 600
    mem, q = _mem(1, 2, L), _r(1, 4, Lq, 128, seed=3)
    lo, hi = _i32([[70] * Lq]), _i32([[300] * 75 + [530] * 75])
    call = lambda m: _attn(q, m, mode, q0=0, nsplit=parts, key_lo=lo, key_hi=hi, softcap=cap)  # noqa: E731
    ref = call(mem)
    for code, byte in ((0x7f, 119), (0x38, 255), (0x7e, 246), (0x7e, 250), (0x01, 0), (0x7e, 20)):
        m = tuple(x.clone() for x in mem)
        for i in range(2):
            for rows in (slice(0, 70), slice(530, L)):
                m[i].view(torch.uint8)[:, :, rows] = code
                m[2 + i][:, :, rows] = byte
        out = call(m)
        assert torch.equal(out[0], ref[0]) and torch.equal(out[1], ref[1])
    for i in range(2):
        m = tuple(x.clone() for x in mem)
        m[2 + i][0, 1, 400] = 255
        out, lse = call(m)
        assert torch.equal(out[:, :, :75], ref[0][:, :, :75]) and torch.equal(lse[:, :, :75], ref[1][:, :, :75])
        assert out[:, 2:, 75:].isnan().all() and torch.equal(out[:, :2], ref[0][:, :2])
