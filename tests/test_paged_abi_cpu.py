"""CPU checks of the paged memory's and the log probabilities' entry points: invalid arguments are refused before anything is
launched, and the Python calls raise their errors."""
import ctypes

import pytest
import torch

from paper_2602_06161_gb300 import _lib, api, build

P = 0x10000   # aligned, never dereferenced


@pytest.fixture(scope="module")
def lib():
    build.build()
    return _lib.load()


_ST = (ctypes.c_int64 * 9)(*[64] * 9)


def append(lib, **kw):
    a = dict(k=P, v=P, q=P, qo=P, ko=P, st=ctypes.addressof(_ST), table=P, n_pages=4, M=3, page=16, start=P, count=P, pos=None, rope=None,
             n=4, B=2, Hq=4, Hkv=2, D=64, R=64, f=P, inter=0, mscale=1.0, e=2, kp=P, vp=P, stream=None)
    a.update(kw)
    return lib.cover_paged_append(*a.values())


@pytest.mark.parametrize("kw", [
    dict(k=None), dict(v=None), dict(q=None), dict(qo=None), dict(st=None), dict(table=None), dict(kp=None), dict(vp=None), dict(f=None),
    dict(start=None), dict(pos=P), dict(start=None, pos=P), dict(n_pages=0), dict(M=0), dict(n=-1), dict(B=0), dict(Hq=-1), dict(Hkv=0),
    dict(D=0), dict(R=3), dict(R=-2), dict(R=66), dict(e=1), dict(e=8), dict(k=P + 1), dict(e=4, v=P + 2), dict(q=P + 1), dict(qo=P + 1),
    dict(ko=P + 1), dict(kp=P + 8), dict(vp=P + 8), dict(table=P + 2), dict(start=P + 2), dict(count=P + 2), dict(rope=P + 2),
    dict(f=P + 4),
])
def test_append_invalid(lib, kw):
    assert append(lib, **kw) == -1


def test_append_bounds(lib):
    assert append(lib, D=96, R=64) == -2 and append(lib, page=8) == -2 and append(lib, page=48) == -2 and append(lib, page=512) == -2
    assert append(lib, M=2 ** 27, page=16) == -2 and append(lib, M=2 ** 30, page=256) == -2
    assert append(lib, n=0) == 0 and append(lib, n=0, k=None, v=None, start=None, count=None) == 0


def attn(lib, **kw):
    a = dict(q=P, kp=P, vp=P, table=P, n_pages=4, M=3, page=16, lens=P, km=P, vm=P, seeds=P, S=2, q0=P, B=2, Hq=4, Hkv=2, Lq=3, D=128, lo=P,
             hi=P, cap=0.0, out=P, lse=P, ws=P, stream=None)
    a.update(kw)
    return lib.cover_attn_fwd_paged(*a.values())


@pytest.mark.parametrize("kw", [
    dict(q=None), dict(kp=None), dict(vp=None), dict(table=None), dict(lens=None), dict(km=None), dict(vm=None), dict(seeds=None),
    dict(q0=None), dict(out=None), dict(n_pages=0), dict(M=0), dict(S=-1), dict(B=0), dict(Hq=0), dict(Hkv=0), dict(Hq=3), dict(Lq=0),
    dict(D=0), dict(cap=-1.0), dict(cap=float("nan")), dict(cap=float("inf")), dict(q=P + 8), dict(kp=P + 8), dict(vp=P + 8),
    dict(out=P + 8), dict(ws=P + 8), dict(table=P + 2), dict(lens=P + 2), dict(lo=P + 2), dict(hi=P + 2), dict(lse=P + 2), dict(q0=P + 2),
    dict(seeds=P + 2), dict(km=P + 8), dict(vm=P + 8),
])
def test_attn_invalid(lib, kw):
    assert attn(lib, **kw) == -1


def test_attn_bounds(lib):
    assert attn(lib, D=64) == -2 and attn(lib, page=24) == -2 and attn(lib, M=2 ** 28, page=128) == -2
    assert attn(lib, B=2 ** 20, Hq=64, Lq=64) == -2 and attn(lib, B=2 ** 30, Hq=2 ** 30, Lq=2 ** 30) == -2


def test_workspace_sizes(lib):
    for bad in ((0, 4, 2, 1, 3, 16), (1, 3, 2, 1, 3, 16), (1, 4, 0, 1, 3, 16), (1, 4, 2, 0, 3, 16), (1, 4, 2, 1, 0, 16)):
        assert lib.cover_attn_paged_workspace_bytes(*bad) == 0
    with pytest.raises(ValueError, match="32 bits"):
        api.cover_attn_paged_workspace_bytes(2 ** 31, 1, 1, 1, 1, 16)


def fwd(lib, **kw):
    a = dict(x=P, N=4, V=10, e=2, tok=P, K=3, logp=P, ent=P, lse=P, idx=P, top=P, stream=None)
    a.update(kw)
    return lib.cover_logprob_fwd(*a.values())


@pytest.mark.parametrize("kw", [
    dict(x=None), dict(N=-1), dict(V=0), dict(e=1), dict(K=-1), dict(logp=None), dict(ent=None), dict(lse=None), dict(idx=None),
    dict(top=None), dict(x=P + 1), dict(e=4, x=P + 2), dict(tok=P + 2), dict(logp=P + 2), dict(ent=P + 2), dict(lse=P + 2), dict(idx=P + 2),
    dict(top=P + 2),
])
def test_logprob_invalid(lib, kw):
    assert fwd(lib, **kw) == -1


def bwd(lib, **kw):
    a = dict(x=P, N=4, V=10, e=2, lse=P, tok=P, g=P, ent=P, ge=P, gs=P, idx=P, gt=P, K=3, out=P, stream=None)
    a.update(kw)
    return lib.cover_logprob_bwd(*a.values())


@pytest.mark.parametrize("kw", [
    dict(x=None), dict(N=-1), dict(V=0), dict(e=3), dict(K=-1), dict(lse=None), dict(tok=None), dict(ent=None), dict(idx=None),
    dict(gt=None), dict(out=None), dict(x=P + 1), dict(out=P + 1), dict(e=4, out=P + 2), dict(lse=P + 1), dict(tok=P + 2), dict(g=P + 2),
    dict(ent=P + 2), dict(ge=P + 2), dict(gs=P + 2), dict(idx=P + 2), dict(gt=P + 2),
])
def test_logprob_grad_invalid(lib, kw):
    assert bwd(lib, **kw) == -1


def test_logprob_bounds(lib):
    assert fwd(lib, K=65) == -2 and bwd(lib, K=65) == -2
    assert fwd(lib, N=0, x=None) == 0 and bwd(lib, N=0, x=None, out=None) == 0


def test_cpu_tensors_are_refused():
    z, i = torch.zeros, lambda *s: torch.zeros(s, dtype=torch.int32)
    kp = z(3, 2, 16, 64, dtype=torch.bfloat16)
    k = z(1, 2, 4, 64, dtype=torch.bfloat16)
    with pytest.raises(ValueError, match="k_pages must be a CUDA tensor"):
        api.cover_paged_append(k, k, kp, kp, i(1, 2), start=i(1))
    with pytest.raises(ValueError, match="q must be a CUDA tensor"):
        api.cover_attn_fwd_paged(z(1, 2, 4, 128, dtype=torch.bfloat16), kp, kp, i(1, 2), i(1))
    with pytest.raises(ValueError, match="logits must be a CUDA tensor"):
        api.cover_logprob_fwd(z(2, 8), i(2))
    with pytest.raises(TypeError, match="logits must be torch.bfloat16 or torch.float32"):
        api.cover_logprob_fwd(z(2, 8, dtype=torch.float16), i(2))
    with pytest.raises(TypeError, match="logits must be a torch.Tensor"):
        api.cover_logprob_fwd([1.0], i(2))
    with pytest.raises(ValueError, match="logits must be a CUDA tensor"):
        api.cover_logprob_bwd(z(2, 8), z(2))


def test_other_forms_are_handed_back():
    n = _lib.native()
    k = torch.zeros(1, 2, 4, 64, dtype=torch.bfloat16)
    assert n.paged_append(k, k, k, k, None, None, None, None, None, None, None, False, 1.0, False) is None
    assert n.attn_paged(*[k] * 5, *[None] * 6, 0.0, None, None, True, None) is None
    assert n.logprob(k, None, 0) is None and n.logprob_grad(k, *[None] * 8) is None
    for fn in ("paged_append", "attn_paged", "logprob", "logprob_grad"):
        with pytest.raises(TypeError):
            getattr(n, fn)(1)
