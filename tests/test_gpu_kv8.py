"""GPU parity of rows written into and read from an 8-bit memory: bit for bit against the oracle."""
import math

import numpy as np
import pytest
import torch

from oracle import memory8_oracle as M8
from paper_2602_06161_gb300 import CoverError, api

pytestmark = pytest.mark.gpu


def _gen(seed):
    return torch.Generator("cuda").manual_seed(seed)


def _rows(B, H, n, D, dtype, seed=0, layout="tokens"):
    shape = (B, n, H, D) if layout == "tokens" else (B, H, n, D)
    x = torch.randn(shape, generator=_gen(seed), device="cuda")
    x = x * torch.exp2(torch.randint(-20, 20, shape[:3], generator=_gen(seed + 50), device="cuda").float())[..., None]
    x = x.to(dtype)
    return x.transpose(1, 2) if layout == "tokens" else x


def _memory(B, H, L, D, seed=9):
    """A memory of random codes (no NaN codes) and bytes."""
    mem = api.kv8_memory(B, H, L, D)
    for i in range(2):
        c = torch.randint(0, 254, mem[i].shape, generator=_gen(seed + i), device="cuda").to(torch.uint8)
        mem[i].view(torch.uint8).copy_(c + (c >= 127).to(torch.uint8))
        mem[2 + i].copy_(torch.randint(100, 150, mem[2 + i].shape, generator=_gen(seed + 5 + i), device="cuda").to(torch.uint8))
    return mem


def _h(t):
    return t.view(torch.uint8).cpu().numpy() if t.dtype == torch.float8_e4m3fn else t.double().cpu().numpy() if t.is_floating_point() else t.cpu().numpy()


def _list(B, n, L, seed=3):
    pos = torch.rand((B, max(L, n)), generator=_gen(seed), device="cuda").argsort(1)[:, :n].to(torch.int32)
    if n >= 6:
        pos[:, n - 1] = pos[:, 0]      # named twice
        pos[:, n - 2] = pos[:, n // 2]
        pos[:, 1] = -1                 # padding
        pos[:, 2] = L                  # out of range
        pos[:, 3] = -2 ** 31
    return pos.contiguous()


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("listed", [False, True])
@pytest.mark.parametrize("B,H,n,L,D", [(1, 1, 1, 1, 64), (1, 4, 32, 100, 128), (2, 3, 7, 9, 64), (3, 2, 65, 70, 128),
                                       (1, 2, 129, 129, 64), (2, 5, 300, 311, 128)])
def test_write_and_read(B, H, n, L, D, listed, dtype):
    k, v = _rows(B, H, n, D, dtype), _rows(B, H, n, D, dtype, 1, "heads")
    mem = _memory(B, H, L, D)
    pos = _list(B, n, L) if listed else None
    pos0 = 0 if listed else L - n
    want_k, want_kx = M8.written(_h(mem[0]), _h(mem[2]), _h(k), pos=None if pos is None else pos.cpu().numpy(), pos0=pos0)
    want_v, want_vx = M8.written(_h(mem[1]), _h(mem[3]), _h(v), pos=None if pos is None else pos.cpu().numpy(), pos0=pos0)
    assert api.cover_kv8_write(k, v, *mem, pos=pos, pos0=pos0) is None
    torch.cuda.synchronize()
    for got, want in zip(mem, (want_k, want_v, want_kx, want_vx)):
        assert np.array_equal(_h(got), want)
    rk, rv = api.cover_kv8_read(*mem, pos=pos, pos0=pos0, n=n, dtype=dtype)
    assert rk.dtype == dtype and rk.shape == (B, H, n, D) and rk.is_contiguous()
    for got, c, x in ((rk, want_k, want_kx), (rv, want_v, want_vx)):
        rows = M8.decode(c, x)
        for b in range(B):
            for s in range(n):
                p = pos0 + s if pos is None else int(pos[b, s])
                want = rows[b, :, p] if 0 <= p < L else np.zeros((H, D))
                assert np.array_equal(_h(got)[b, :, s], want)


def test_every_code_and_byte_reads_back_exactly():
    """All 256 codes under all 256 bytes, in both types: the value where the type holds it (bf16 and fp32 hold every one of
    bytes 17 .. 246 without rounding), NaN for the NaN codes and for byte 255."""
    mem = api.kv8_memory(1, 1, 1024, 64)
    codes = torch.arange(256, device="cuda", dtype=torch.uint8).view(4, 64).repeat(256, 1).view(1, 1, 1024, 64)
    byte = torch.arange(256, device="cuda", dtype=torch.uint8).repeat_interleave(4).view(1, 1, 1024)
    for i in range(2):
        mem[i].view(torch.uint8).copy_(codes)
        mem[2 + i].copy_(byte)
    ref = torch.from_numpy(M8.decode(_h(codes), _h(byte)))
    for dtype in (torch.bfloat16, torch.float32):
        k, v = api.cover_kv8_read(*mem, dtype=dtype)
        want = ref.to(dtype).double().numpy()
        held = slice(17 * 4, 247 * 4)
        assert np.array_equal(_h(k)[0, 0, held], ref.numpy()[0, 0, held], equal_nan=True)
        assert np.array_equal(_h(k), want, equal_nan=True) and np.array_equal(_h(v), want, equal_nan=True)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_rows_that_are_not_ordinary(dtype):
    """Zeros, infinities, NaN, the type's ends, and magnitudes on both sides of each border of the exponent."""
    big = torch.finfo(dtype).max
    rows = [[0.0], [-0.0, 0.0], [math.inf, 1.0], [-math.inf], [math.nan], [big, -big, 1.0], [torch.finfo(dtype).tiny], [2.0 ** -133],
            [448.0, 0.4375], [450.0 if dtype == torch.bfloat16 else 448.00003], [1e-30, 1e-38], [240.0, -17.0, 0.001953125, 0.0009765625]]
    rows += [[1.75 * 2.0 ** e, 1.0] for e in range(-120, 120, 13)] + [[1.7578125 * 2.0 ** e, 1.0] for e in range(-120, 120, 13)]
    x = torch.zeros((1, 1, len(rows), 64), dtype=dtype)
    for i, r in enumerate(rows):
        x[0, 0, i, 7:7 + len(r)] = torch.tensor(r)
    x = x.cuda()
    mem = _memory(1, 1, len(rows), 64)
    want, want_x = M8.encode(_h(x))
    api.cover_kv8_write(x, x, *mem)
    for i in range(2):
        assert np.array_equal(_h(mem[i]), want) and np.array_equal(_h(mem[2 + i]), want_x)
    k, _ = api.cover_kv8_read(*mem, dtype=dtype)
    assert np.array_equal(_h(k), M8.decode(want, want_x), equal_nan=True)


def test_quantisation_error():
    """Each element within 2^-4 of itself, or half the smallest code's step of its row."""
    x = _rows(2, 3, 40, 128, torch.float32)
    mem = api.kv8_memory(2, 3, 40, 128)
    api.cover_kv8_write(x, x, *mem)
    k, _ = api.cover_kv8_read(*mem, dtype=torch.float32)
    step = torch.exp2(mem[2].double() - 127)[..., None] * 2.0 ** -10
    assert ((k.double() - x.double()).abs() <= torch.maximum(x.double().abs() * 2.0 ** -4, step)).all()


def test_strided_and_broadcast_rows():
    B, H, n, D = 2, 4, 21, 64
    big = torch.randn((B, n, 3 * H, D), generator=_gen(2), device="cuda").to(torch.bfloat16)
    k, v = big[:, :, :H].transpose(1, 2), big[:, :, H:2 * H].transpose(1, 2)
    one = k[:, :1].expand(B, H, n, D)
    for a, b in ((k, v), (one, v)):
        m1, m2 = _memory(B, H, 30, D), _memory(B, H, 30, D)
        api.cover_kv8_write(a, b, *m1, pos0=4)
        api.cover_kv8_write(a.contiguous(), b.contiguous(), *m2, pos0=4)
        for x, y in zip(m1, m2):
            assert np.array_equal(_h(x), _h(y))


def test_long_lists_with_repeats():
    """More slots than a CTA holds, every position named several times: the lowest slot is taken."""
    B, H, n, L, D = 2, 2, 700, 97, 64
    x = _rows(B, H, n, D, torch.bfloat16)
    pos = torch.randint(-3, L + 3, (B, n), generator=_gen(8), device="cuda", dtype=torch.int32)
    mem = _memory(B, H, L, D)
    want, want_x = M8.written(_h(mem[0]), _h(mem[2]), _h(x), pos=pos.cpu().numpy())
    api.cover_kv8_write(x, x, *mem, pos=pos)
    assert np.array_equal(_h(mem[0]), want) and np.array_equal(_h(mem[2]), want_x)


def test_nothing_to_write_or_read():
    mem = _memory(1, 2, 5, 64)
    old = [m.clone() for m in mem]
    x = torch.empty((1, 2, 0, 64), device="cuda")
    api.cover_kv8_write(x, x, *mem)
    api.cover_kv8_write(x, x, *mem, pos=torch.empty((1, 0), device="cuda", dtype=torch.int32))
    k, v = api.cover_kv8_read(*mem, pos0=5)
    assert k.shape == v.shape == (1, 2, 0, 64)
    for a, b in zip(mem, old):
        assert np.array_equal(_h(a), _h(b))


def test_refusals():
    mem = api.kv8_memory(1, 2, 16, 64)
    x = torch.zeros((1, 2, 4, 64), device="cuda")
    with pytest.raises(CoverError):
        api.cover_kv8_write(x, x, *mem, pos0=13)
    with pytest.raises(CoverError):
        api.cover_kv8_write(x, x, *mem, pos0=-1)
    with pytest.raises(CoverError):
        api.cover_kv8_read(*mem, pos0=10, n=7)
    with pytest.raises(TypeError, match="v must be"):
        api.cover_kv8_write(x, x.bfloat16(), *mem)
    with pytest.raises(TypeError, match="k must be"):
        api.cover_kv8_write(x.half(), x.half(), *mem)
    with pytest.raises(ValueError, match="matching the memory"):
        api.cover_kv8_write(x[:, :1], x[:, :1], *mem)
    with pytest.raises(ValueError, match="dense"):
        api.cover_kv8_write(x.transpose(2, 3), x, *mem)
    with pytest.raises(ValueError, match="pos must be"):
        api.cover_kv8_write(x, x, *mem, pos=torch.zeros((1, 3), device="cuda", dtype=torch.int32))
    with pytest.raises(TypeError, match="dtype must be"):
        api.cover_kv8_read(*mem, dtype=torch.float16)
    with pytest.raises(ValueError, match="k_exp"):
        api.cover_kv8_read(mem[0], mem[1], mem[2][:, :1].contiguous(), mem[3])
    flat = torch.zeros(1 + 2 * 4 * 64, device="cuda")[1:].view(1, 2, 4, 64)
    with pytest.raises(CoverError):
        api.cover_kv8_write(flat, flat, *mem)                         # rows that are not 16-byte aligned
    odd = torch.zeros((1, 2, 4, 65), device="cuda")[..., :64]
    with pytest.raises(CoverError):
        api.cover_kv8_write(odd, odd, *mem)
    small = api.kv8_memory(1, 2, 16, 32)
    with pytest.raises(CoverError):
        api.cover_kv8_read(*small)


def test_streams_and_graph():
    mem = _memory(2, 2, 50, 128)
    k, v = _rows(2, 2, 10, 128, torch.bfloat16), _rows(2, 2, 10, 128, torch.bfloat16, 1)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    api.cover_kv8_write(k, v, *mem, pos0=7, stream=side)
    a = api.cover_kv8_read(*mem, pos0=7, n=10, stream=side)
    torch.cuda.current_stream().wait_stream(side)
    b = api.cover_kv8_read(*mem, pos0=7, n=10)
    assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1])
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        api.cover_kv8_write(k, v, *mem, pos0=30)
        out = api.cover_kv8_read(*mem, pos0=30, n=10)
    k.copy_(-k)
    g.replay()
    assert torch.equal(out[0], -b[0]) and torch.equal(out[1], b[1])


def test_offsets_beyond_32_bits():
    """A memory of more than 2^32 codes: its last rows are written and read, the rows that a 32-bit offset would name stay."""
    B, H, L, D = 1, 9, 4000000, 128
    mem = api.kv8_memory(B, H, L, D)
    x = _rows(B, H, 3, D, torch.bfloat16)
    api.cover_kv8_write(x, x, *mem, pos0=L - 3)
    k, v = api.cover_kv8_read(*mem, pos0=L - 4, n=4, dtype=torch.float32)
    want = M8.decode(*M8.encode(_h(x)))
    assert np.array_equal(_h(k)[:, :, 1:], want) and np.array_equal(_h(v)[:, :, 1:], want)
    assert not k[:, :, 0].any()
    assert int((mem[0].view(torch.uint8) != 0).any(-1).sum()) <= 3 * H
