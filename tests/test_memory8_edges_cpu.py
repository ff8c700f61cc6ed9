"""CPU checks of the host logic around the rotary and 8-bit memory calls."""
import itertools
import random

import pytest
import torch

from paper_2602_06161_gb300 import api


def _bytes(t):
    return {t.data_ptr() + t.element_size() * sum(i * s for i, s in zip(at, t.stride())) + e
            for at in itertools.product(*(range(n) for n in t.shape)) for e in range(t.element_size())}


def test_overlap_is_that_of_the_bytes():
    rng = random.Random(1)
    flat = torch.zeros(4000, dtype=torch.uint8)
    met = 0
    for _ in range(3000):
        a, b = (torch.as_strided(flat.view(rng.choice([torch.bfloat16, torch.float32])), [rng.choice([1, 1, 2, 3, 4]) for _ in range(4)],
                                 rng.choice([[64, 16, 4, 1], [64, 4, 16, 1], [48, 12, 24, 1], [rng.randint(0, 60) for _ in range(3)] + [1]]),
                                 rng.randint(0, 200)) for _ in range(2))
        want = bool(_bytes(a) & _bytes(b))
        assert api._overlap(a, b) == want
        met += want
    assert 300 < met < 2700


def test_rotated_rows_lie_apart_or_in_place():
    """In place, an output is still held against the other tensors; rows that only lie between another's are no overlap."""
    qkv = torch.zeros((2, 5, 8, 16), dtype=torch.bfloat16)
    q, k = qkv[:, :, :4].transpose(1, 2), qkv[:, :, 4:6].transpose(1, 2)
    f, pos = torch.zeros(8, dtype=torch.float64), torch.zeros((2, 5), dtype=torch.int32)
    out = torch.zeros_like(qkv)
    oq, ok = out[:, :, :4].transpose(1, 2), out[:, :, 4:6].transpose(1, 2)
    check = lambda pairs: api._rope_aliases(pairs, [f, pos])  # noqa: E731
    check([("out_q", q, q), ("out_k", k, k)])
    check([("out_q", q, oq), ("out_k", k, ok)])
    check([("out_q", q, None), ("out_k", k, k)])
    check([("out_q", q, oq)])
    one = q[:1]      # a dimension of one entry has any stride
    check([("out_q", one, one.as_strided(one.shape, (7, *one.stride()[1:])))])
    for pairs in ([("out_q", q, q), ("out_k", q, None)], [("out_q", q, q), ("out_k", q, q)], [("out_q", q, None), ("out_k", q, q)],
                  [("out_q", q, k.expand_as(k)), ("out_k", k, None)], [("out_q", q, oq), ("out_k", k, oq[:, :2])],
                  [("out_q", q, qkv[:, :, 1:5].transpose(1, 2)), ("out_k", k, None)],
                  [("out_q", q, None), ("out_k", k, qkv[:, :, 3:5].transpose(1, 2))],
                  [("out_q", pos[:, None, :, None], pos[:, None, :, None]), ("out_k", k, None)]):
        with pytest.raises(ValueError, match="overlap"):
            check(pairs)


def test_the_debug_call_checks_its_tensors():
    mem = api.kv8_memory(1, 2, 16, device="cpu")
    q = torch.zeros(1, 2, 4, 128, dtype=torch.bfloat16)
    with pytest.raises(ValueError, match="q must be a CUDA tensor"):
        api.cover_debug_attn_prefix8(q, *mem, q0=0, mode=0)
    with pytest.raises(TypeError, match="q must be"):
        api.cover_debug_attn_prefix8(q.float(), *mem, q0=0, mode=0)


def test_numbers_above_32_bits_are_refused(monkeypatch):
    """ctypes cuts them: row 2^32 of a memory would be row 0. (On tensors that pass for CUDA ones; nothing is launched.)"""
    def launch(*a):
        raise AssertionError("launched")

    class Hands:
        def __getattr__(self, name):
            return lambda *a: None

    monkeypatch.setattr(api, "_launch", launch)
    monkeypatch.setattr(api, "_nat", Hands())
    monkeypatch.setattr(api, "_need", lambda *a: None)
    monkeypatch.setattr(api, "_rows_need", lambda *a: None)
    mem, x = api.kv8_memory(1, 2, 16, device="cpu"), torch.zeros(1, 2, 4, 128, dtype=torch.bfloat16)
    f = torch.zeros(64, dtype=torch.float64)
    for big in (2 ** 32, 2 ** 31, -2 ** 31 - 1, 2 ** 63, 2 ** 64 + 1):
        for call in (lambda: api.cover_rope_fwd(x, x, f, pos0=big), lambda: api.cover_kv8_write(x, x, *mem, pos0=big),
                     lambda: api.cover_kv8_read(*mem, pos0=big, n=1), lambda: api.cover_kv8_read(*mem, pos0=big),
                     lambda: api.cover_attn_fwd_prefix8(x, *mem, q0=big), lambda: api.cover_debug_attn_prefix8(x, *mem, q0=0, mode=big),
                     lambda: api.cover_attn_fwd_prefix(x, x, x, q0=big), lambda: api.cover_attn_prefix8_workspace_bytes(1, 2, 2, 4, big)):
            with pytest.raises(ValueError, match="32 bits"):
                call()
    with pytest.raises(ValueError, match="32 bits"):
        api.cover_kv8_read(*mem, n=2 ** 32 + 1)
    with pytest.raises(ValueError, match="longer than"):
        api._sizes_fit(torch.empty(1, device="meta").expand(2 ** 31, 1), "q")
    api._sizes_fit(torch.empty(1, device="meta").expand(2 ** 31 - 1, 7), "q")


def test_outputs_of_another_shape_are_refused(monkeypatch):
    """By every attention call, before anything is launched: the kernels write what q's shape says."""
    class Lib:
        def __getattr__(self, name):
            raise AssertionError("launched")

    class Hands:
        def __getattr__(self, name):
            return lambda *a: None

    monkeypatch.setattr(api._lib, "load", lambda: Lib())
    monkeypatch.setattr(api, "_launch", lambda *a: Lib().launch)
    monkeypatch.setattr(api, "_nat", Hands())
    monkeypatch.setattr(api, "_need", lambda *a: None)
    monkeypatch.setattr(api, "cover_attn_prefix8_workspace_bytes", lambda *a: 0)
    q, lse = torch.zeros(1, 2, 4, 128, dtype=torch.bfloat16), torch.zeros(1, 2, 4)
    mem = api.kv8_memory(1, 2, 4, device="cpu")
    for call in (lambda **kw: api.cover_attn_fwd(q, q, q, **kw), lambda **kw: api.cover_attn_fwd_prefix(q, q, q, q0=0, **kw),
                 lambda **kw: api.cover_attn_fwd_prefix8(q, *mem, q0=0, **kw)):
        for kw in (dict(out=q[:, :, :3]), dict(out=q[:, :1]), dict(lse=lse[:, :, :3]), dict(out=q, lse=lse[:, :1])):
            with pytest.raises(ValueError, match="must"):
                call(**kw)
        with pytest.raises(AssertionError, match="launched"):
            call(out=q, lse=lse)
