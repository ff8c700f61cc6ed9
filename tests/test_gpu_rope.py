"""GPU parity of the rotary positions against the fp64 oracle."""
import math

import numpy as np
import pytest
import torch

from oracle import memory8_oracle as M8
from paper_2602_06161_gb300 import CoverError, api

pytestmark = pytest.mark.gpu

EPS = {torch.bfloat16: 2.0 ** -8, torch.float32: 2.0 ** -24}   # half a step


def _gen(seed):
    return torch.Generator("cuda").manual_seed(seed)


def _rows(B, H, L, D, dtype, seed=0, layout="tokens"):
    if layout == "tokens":
        return torch.randn((B, L, H, D), generator=_gen(seed), device="cuda").to(dtype).transpose(1, 2)
    return torch.randn((B, H, L, D), generator=_gen(seed), device="cuda").to(dtype)


def _host(t):
    return t.double().cpu().numpy()


def _tolerance(x, f, inter, mscale, dtype):
    """Per element: half a step of the result, and in fp32 the reduced angle (2^-26 turns from its conversion, an fp64
    frequency's 2^-53 of at most 2^20 turns), sincospif (2 steps), the factor and the two products and their sum (3 steps),
    all relative to the pair's |a| + |b|."""
    a = np.abs(_host(x))
    pair = a.copy()
    R = 2 * len(f)
    i = np.arange(R // 2)
    lo, hi = (2 * i, 2 * i + 1) if inter else (i, i + R // 2)
    pair[..., lo] = pair[..., hi] = a[..., lo] + a[..., hi]
    fp32 = 2 * math.pi * (2.0 ** -26 + 2.0 ** -33) + 10 * 2.0 ** -24
    return mscale * pair * ((1 + EPS[dtype]) * fp32 + EPS[dtype])


def _check(x, y, f, pos, inter, mscale, inverse):
    ref = M8.rope(_host(x), f.cpu().numpy(), pos, interleaved=inter, mscale=mscale, inverse=inverse)
    d = np.abs(_host(y) - ref)
    tol = _tolerance(x, f, inter, mscale, x.dtype) + 1e-30
    assert (d <= tol).all(), (d / tol).max()
    R = 2 * len(f)
    assert torch.equal(y[..., R:], x[..., R:])


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("inter", [False, True])
@pytest.mark.parametrize("B,Hq,Hkv,L,D,R", [
    (1, 1, 1, 1, 2, 2), (1, 28, 4, 1, 128, 128), (3, 5, 2, 7, 64, 32), (2, 4, 4, 33, 128, 64), (1, 3, 1, 9, 24, 24),
    (2, 2, 1, 5, 20, 12), (1, 2, 2, 3, 7, 4), (2, 32, 8, 130, 128, 128), (1, 9, 3, 40, 128, 16),
])
def test_against_oracle(B, Hq, Hkv, L, D, R, inter, dtype):
    q, k = _rows(B, Hq, L, D, dtype), _rows(B, Hkv, L, D, dtype, 1, "heads")
    pos = torch.randint(-5, 200000, (B, L), generator=_gen(2), device="cuda", dtype=torch.int32)
    f, _ = api.rope_frequencies(R)
    for inverse in (False, True):
        yq, yk = api.cover_rope_fwd(q, k, f, pos=pos, interleaved=inter, mscale=1.25, inverse=inverse)
        assert yq.is_contiguous() and yk.is_contiguous() and yq.shape == q.shape and yk.dtype == dtype
        _check(q, yq, f, pos.cpu().numpy(), inter, 1.25, inverse)
        _check(k, yk, f, pos.cpu().numpy(), inter, 1.25, inverse)


def test_run_of_positions_and_no_k():
    q = _rows(2, 3, 11, 64, torch.float32)
    f, m = api.rope_frequencies(64, scaling="yarn", factor=8.0)
    y, none = api.cover_rope_fwd(q, None, f, pos0=1000, mscale=m)
    assert none is None
    _check(q, y, f, np.arange(1000, 1011)[None].repeat(2, 0), False, m, False)


@pytest.mark.parametrize("at", [2 ** 31 - 1, -2 ** 31, 2 ** 30 + 7, 0])
def test_positions_at_the_ends_of_their_range(at):
    """The oracle's fp64 product is off by 2^-53 of the angle, up to 2^31 * 2^-53 radians: counted twice."""
    x = _rows(1, 2, 1, 64, torch.float32)
    f, _ = api.rope_frequencies(64)
    y, _ = api.cover_rope_fwd(x, None, f, pos=torch.full((1, 1), at, device="cuda", dtype=torch.int32))
    ref = M8.rope(_host(x), f.cpu().numpy(), np.array([[at]]), interleaved=False)
    tol = _tolerance(x, f, False, 1.0, torch.float32) + 2 * 2.0 ** -22 * 2 * np.abs(_host(x)).max()
    assert (np.abs(_host(y) - ref) <= tol).all()


@pytest.mark.parametrize("inter", [False, True])
@pytest.mark.parametrize("D,R,dtype", [(64, 64, torch.bfloat16), (64, 32, torch.float32), (6, 4, torch.bfloat16)])
def test_in_place_of_one_projection(inter, D, R, dtype):
    """q and k are views of one [B, L, (Hq + 2 Hkv) D] projection; its v columns stay as they were."""
    B, Hq, Hkv, L = 2, 6, 2, 19
    qkv = torch.randn((B, L, Hq + 2 * Hkv, D), generator=_gen(4), device="cuda").to(dtype)
    old = qkv.clone()
    q, k = qkv[:, :, :Hq].transpose(1, 2), qkv[:, :, Hq:Hq + Hkv].transpose(1, 2)
    f, _ = api.rope_frequencies(R)
    ref = api.cover_rope_fwd(q, k, f, pos0=3, interleaved=inter)
    oq, ok = api.cover_rope_fwd(q, k, f, pos0=3, interleaved=inter, out_q=q, out_k=k)
    assert oq is q and ok is k and torch.equal(q, ref[0]) and torch.equal(k, ref[1])
    assert torch.equal(qkv[:, :, Hq + Hkv:], old[:, :, Hq + Hkv:])


@pytest.mark.parametrize("shift", [0, 1, 3])
def test_unaligned_rows(shift):
    flat = torch.randn(shift + 2 * 3 * 5 * 64, generator=_gen(5), device="cuda").to(torch.bfloat16)
    x = flat[shift:].view(2, 3, 5, 64)
    f, _ = api.rope_frequencies(64)
    a, _ = api.cover_rope_fwd(x, None, f, pos0=9)
    b, _ = api.cover_rope_fwd(x.clone(), None, f, pos0=9)
    assert torch.equal(a, b)


def test_empty():
    f, _ = api.rope_frequencies(64)
    q = torch.empty((2, 3, 0, 64), device="cuda")
    y, _ = api.cover_rope_fwd(q, None, f)
    assert y.shape == q.shape
    x = _rows(1, 2, 3, 64, torch.float32)
    y, _ = api.cover_rope_fwd(x, x[:, :0], f[:0])
    assert torch.equal(y, x)


@pytest.mark.parametrize("inter", [False, True])
def test_gradient(inter):
    """The inverse is the gradient: of the formula, by autograd in fp64, and of differences of the kernel itself."""
    B, H, L, D, R, m = 1, 2, 3, 16, 12, 1.5
    x = _rows(B, H, L, D, torch.float32)
    w = _rows(B, H, L, D, torch.float32, 7)
    f, _ = api.rope_frequencies(R)
    grad, _ = api.cover_rope_fwd(w, None, f, pos0=5, interleaved=inter, mscale=m, inverse=True)
    grad[..., R:] = w[..., R:]
    xd = x.double().cpu().requires_grad_()
    i = torch.arange(R // 2)
    a, b = (2 * i, 2 * i + 1) if inter else (i, i + R // 2)
    t = (5 + torch.arange(L, dtype=torch.float64))[:, None] * f.cpu()
    y = xd.clone()
    y[..., a] = m * (xd[..., a] * t.cos() - xd[..., b] * t.sin())
    y[..., b] = m * (xd[..., a] * t.sin() + xd[..., b] * t.cos())
    (y * w.double().cpu()).sum().backward()
    tol = _tolerance(w, f, inter, m, torch.float32)
    assert (np.abs(_host(grad) - xd.grad.numpy()) <= tol).all()
    # a linear map: the difference over a step of 1 is the derivative, up to the roundings of both values
    for at in [(0, 0, 0, 0), (0, 1, 2, R - 1), (0, 1, 1, D - 1), (0, 0, 2, R // 2)]:
        step = x.clone()
        step[at] += 1.0
        up, _ = api.cover_rope_fwd(step, None, f, pos0=5, interleaved=inter, mscale=m)
        down, _ = api.cover_rope_fwd(x, None, f, pos0=5, interleaved=inter, mscale=m)
        slope = ((up.double() - down.double()) * w.double()).sum().item()
        assert abs(slope - grad[at].item()) <= 64 * 2.0 ** -24 * 16


def test_refusals():
    q, k = _rows(1, 2, 4, 64, torch.bfloat16), _rows(1, 2, 4, 64, torch.bfloat16)
    f, _ = api.rope_frequencies(64)
    with pytest.raises(TypeError, match="k must be"):
        api.cover_rope_fwd(q, k.float(), f)
    with pytest.raises(TypeError, match="inv_freq"):
        api.cover_rope_fwd(q, k, f.float())
    with pytest.raises(ValueError, match="D / 2"):
        api.cover_rope_fwd(q[..., :32], None, f)
    with pytest.raises(ValueError, match="k must be"):
        api.cover_rope_fwd(q, k[:, :, :3], f)
    with pytest.raises(ValueError, match="dense"):
        api.cover_rope_fwd(q.transpose(2, 3), None, f[:1])
    with pytest.raises(ValueError, match="pos must be"):
        api.cover_rope_fwd(q, k, f, pos=torch.zeros((1, 3), device="cuda", dtype=torch.int32))
    with pytest.raises(ValueError, match="overlap"):
        api.cover_rope_fwd(q, k, f, out_q=k)
    with pytest.raises(ValueError, match="expanded"):
        api.cover_rope_fwd(q, None, f, out_q=q[:, :1].expand_as(q))
    with pytest.raises(CoverError):
        api.cover_rope_fwd(torch.zeros((1, 1, 1, 5000), device="cuda"), None, f)


def test_frequencies():
    f, m = api.rope_frequencies(8, 100.0)
    assert m == 1.0 and np.allclose(f.cpu().numpy(), [1, 100 ** -0.25, 0.1, 100 ** -0.75])
    g, _ = api.rope_frequencies(8, 100.0, scaling="linear", factor=4.0)
    assert torch.allclose(g * 4, f)
    g, _ = api.rope_frequencies(8, 100.0, scaling="ntk", factor=4.0)
    assert g[0] == 1 and abs(g[-1].item() * 4 / f[-1].item() - 1) < 1e-12
    g, m = api.rope_frequencies(128, scaling="yarn", factor=4.0)
    f, _ = api.rope_frequencies(128)
    assert torch.equal(g[:10], f[:10]) and torch.allclose(g[-10:] * 4, f[-10:]) and abs(m - (0.1 * math.log(4) + 1)) < 1e-15
    for kw in (dict(R=7), dict(R=0), dict(R=8, scaling="x"), dict(R=8, factor=0.5)):
        with pytest.raises(ValueError):
            api.rope_frequencies(**kw)


def test_streams_and_graph():
    q, k = _rows(2, 4, 37, 128, torch.bfloat16), _rows(2, 2, 37, 128, torch.bfloat16, 1)
    f, _ = api.rope_frequencies(128)
    ref = api.cover_rope_fwd(q, k, f, pos0=2)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    got = api.cover_rope_fwd(q, k, f, pos0=2, stream=side)
    torch.cuda.current_stream().wait_stream(side)
    assert torch.equal(got[0], ref[0]) and torch.equal(got[1], ref[1])
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        out = api.cover_rope_fwd(q, k, f, pos0=2)
    q.mul_(2)
    k.mul_(2)
    g.replay()
    assert torch.equal(out[0], ref[0] * 2) and torch.equal(out[1], ref[1] * 2)
