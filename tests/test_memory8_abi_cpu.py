"""CPU checks of the 8-bit memory's entry points: invalid arguments are refused before anything is launched."""
import ctypes

import pytest
import torch

from paper_2602_06161_gb300 import _lib, api, build

P = 0x10000   # aligned, never dereferenced


@pytest.fixture(scope="module")
def lib():
    build.build()
    return _lib.load()


def _st(*v):
    a = (ctypes.c_int64 * len(v))(*v)
    return ctypes.addressof(a), a


def rope(lib, **kw):
    st, keep = _st(*[64] * 12)
    a = dict(q=P, k=P, qo=P, ko=P, st=st, B=1, Hq=2, Hkv=1, L=4, D=64, R=64, f=P, pos=P, pos0=0, e=2)
    a.update(kw)
    return lib.cover_rope_fwd(a["q"], a["k"], a["qo"], a["ko"], a["st"], a["B"], a["Hq"], a["Hkv"], a["L"], a["D"], a["R"], a["f"],
                              a["pos"], a["pos0"], 0, 1.0, 0, a["e"], None)


@pytest.mark.parametrize("kw", [
    dict(q=None), dict(qo=None), dict(k=None), dict(ko=None), dict(st=None), dict(f=None), dict(B=0), dict(Hq=0), dict(Hkv=-1),
    dict(L=-1), dict(D=0), dict(R=3), dict(R=-2), dict(R=66), dict(e=1), dict(e=8), dict(q=P + 1), dict(qo=P + 1), dict(k=P + 1),
    dict(e=4, ko=P + 2), dict(f=P + 4), dict(pos=P + 2),
])
def test_rope_invalid(lib, kw):
    assert rope(lib, **kw) == -1


def test_rope_bounds(lib):
    assert rope(lib, D=4098, R=64) == -2
    assert rope(lib, L=0) == 0 and rope(lib, L=0, q=None, f=None) == 0


def write(lib, **kw):
    a = dict(k=P, v=P, st=(64, 64, 64, 64, 64, 64), pos=None, pos0=0, n=4, B=2, H=2, L=16, D=64, e=2, k8=P, v8=P, kx=P, vx=P)
    a.update(kw)
    st, keep = (None, None) if a["st"] is None else _st(*a["st"])
    return lib.cover_kv8_write(a["k"], a["v"], st, a["pos"], a["pos0"], a["n"], a["B"], a["H"], a["L"], a["D"], a["e"], a["k8"],
                               a["v8"], a["kx"], a["vx"], None)


def read(lib, **kw):
    a = dict(k=P, v=P, pos=None, pos0=0, n=4, B=2, H=2, L=16, D=64, e=2, k8=P, v8=P, kx=P, vx=P)
    a.update(kw)
    return lib.cover_kv8_read(a["k8"], a["v8"], a["kx"], a["vx"], a["pos"], a["pos0"], a["n"], a["B"], a["H"], a["L"], a["D"], a["e"],
                              a["k"], a["v"], None)


COMMON = [dict(k=None), dict(v=None), dict(k8=None), dict(v8=None), dict(kx=None), dict(vx=None), dict(B=0), dict(H=0), dict(L=0),
          dict(D=0), dict(n=-1), dict(e=1), dict(pos0=-1), dict(pos0=13), dict(pos0=2 ** 31 - 1), dict(k=P + 8), dict(v=P + 8),
          dict(k8=P + 8), dict(v8=P + 8), dict(pos=P + 2)]


@pytest.mark.parametrize("kw", COMMON + [dict(st=None), dict(st=(64, 64, 65, 64, 64, 64)), dict(st=(64, 64, 64, 64, 4, 64))])
def test_write_invalid(lib, kw):
    assert write(lib, **kw) == -1


@pytest.mark.parametrize("kw", COMMON)
def test_read_invalid(lib, kw):
    assert read(lib, **kw) == -1


def test_memory_bounds(lib):
    for fn in (write, read):
        assert fn(lib, D=96) == -2 and fn(lib, B=70000) == -2
        assert fn(lib, n=0) == 0 and fn(lib, n=0, k=None, v=None) == 0


def attn(lib, **kw):
    a = dict(q=P, k8=P, v8=P, kx=P, vx=P, km=P, vm=P, seeds=P, S=2, B=1, Hq=2, Hkv=1, Lq=8, Lk=128, q0=0, D=128, lo=None, hi=None,
             cap=0.0, out=P, lse=P, ws=P)
    a.update(kw)
    return lib.cover_attn_fwd_prefix8(a["q"], a["k8"], a["v8"], a["kx"], a["vx"], a["km"], a["vm"], a["seeds"], a["S"], a["B"], a["Hq"],
                                      a["Hkv"], a["Lq"], a["Lk"], a["q0"], a["D"], a["lo"], a["hi"], a["cap"], a["out"], a["lse"],
                                      a["ws"], None)


@pytest.mark.parametrize("kw", [
    dict(q=None), dict(k8=None), dict(v8=None), dict(kx=None), dict(vx=None), dict(out=None), dict(km=None), dict(seeds=None),
    dict(S=-1), dict(S=129), dict(B=0), dict(Hq=3, Hkv=2), dict(Hkv=0), dict(Lq=0), dict(Lk=0), dict(q0=-1), dict(q0=121),
    dict(cap=-1.0), dict(cap=float("nan")), dict(cap=float("inf")), dict(q=P + 8), dict(k8=P + 8), dict(out=P + 8), dict(lse=P + 2),
    dict(lo=P + 2), dict(hi=P + 1), dict(ws=P + 8),
])
def test_attention_invalid(lib, kw):
    assert attn(lib, **kw) == -1


def test_attention_unsupported(lib):
    assert attn(lib, D=64) == -2


def test_workspace_bytes_of_invalid_sizes(lib):
    for a in ((0, 1, 1, 1, 1), (1, 0, 1, 1, 1), (1, 1, 0, 1, 1), (1, 3, 2, 1, 1), (1, 1, 1, 0, 1), (1, 1, 1, 1, 0)):
        assert lib.cover_attn_prefix8_workspace_bytes(*a) == 0


def test_cpu_tensors_are_handed_back_and_refused():
    x, f = torch.zeros(1, 2, 4, 64), torch.zeros(32, dtype=torch.float64)
    mem = api.kv8_memory(1, 2, 16, 64, device="cpu")
    n = _lib.native()
    assert n.rope(x, x, f, None, 0, False, 1.0, False) is None
    assert n.kv8_write(x, x, *mem, None, 0) is None
    assert n.kv8_read(*mem, None, 0, None, False) is None
    assert n.attn8(x, *mem, None, None, None, 0, None, None, 0.0, None, None, True, None) is None
    with pytest.raises(ValueError, match="q must be a CUDA tensor"):
        api.cover_rope_fwd(x, x, f)
    with pytest.raises(ValueError, match="k8 must be a CUDA tensor"):
        api.cover_kv8_write(x, x, *mem)
    with pytest.raises(ValueError, match="k8 must be a CUDA tensor"):
        api.cover_kv8_read(*mem)
    with pytest.raises(ValueError, match="q must be a CUDA tensor"):
        api.cover_attn_fwd_prefix8(x.bfloat16(), *mem, q0=0)
    for fn in ("rope", "kv8_write", "kv8_read", "attn8"):
        with pytest.raises(TypeError):
            getattr(n, fn)(1, 2)
        assert getattr(n, fn)(*[None] * {"attn8": 16}.get(fn, 8)) is None
