"""The rotary and 8-bit memory calls as programs make them: through the native marshalling and the Python path, two at once
on two streams, as one captured step, and at the sizes where a grid's dimensions end."""
import numpy as np
import pytest
import torch

from oracle import memory8_oracle as M8
from paper_2602_06161_gb300 import api

pytestmark = pytest.mark.gpu


def _r(*shape, dtype=torch.bfloat16, seed=0):
    return torch.randn(shape, generator=torch.Generator("cuda").manual_seed(seed), device="cuda").to(dtype)


def _h(t):
    return t.view(torch.uint8).cpu().numpy() if t.dtype == torch.float8_e4m3fn else t.double().cpu().numpy() if t.is_floating_point() else t.cpu().numpy()


def _mem(B, H, L, seed=30):
    m = api.kv8_memory(B, H, L)
    api.cover_kv8_write(_r(B, H, L, 128, seed=seed), _r(B, H, L, 128, seed=seed + 1), *m)
    return m


def _bits(t):
    return t.view(torch.uint8) if t.dtype == torch.float8_e4m3fn else t


def _calls():
    q, k, v = _r(2, 4, 9, 128), _r(2, 2, 9, 128, seed=1), _r(2, 2, 9, 128, seed=2)
    f, _ = api.rope_frequencies(128)
    at = torch.randint(0, 9000, (2, 9), device="cuda", dtype=torch.int32)
    pos = torch.stack([torch.randperm(70)[:9] for _ in range(2)]).to(torch.int32).cuda()
    mem = _mem(2, 2, 70)

    def write(**kw):
        m = tuple(x.clone() for x in mem)
        assert api.cover_kv8_write(k, v, *m, **kw) is None
        return m
    km, vm = _r(2, 2, 3, 128, seed=3), _r(2, 2, 3, 128, seed=4)
    lo, hi = torch.zeros((2, 9), device="cuda", dtype=torch.int32), torch.full((2, 9), 50, device="cuda", dtype=torch.int32)
    return {
        "rope": lambda **kw: api.cover_rope_fwd(q, k, f, pos0=33, **kw),
        "rope_listed_back": lambda **kw: api.cover_rope_fwd(q.transpose(1, 2).contiguous().transpose(1, 2), k, f, pos=at, inverse=True,
                                                            mscale=1.25, **kw),
        "rope_q": lambda **kw: api.cover_rope_fwd(q, None, f, pos0=33, **kw),
        "write": lambda **kw: write(pos0=7, **kw),
        "write_listed": lambda **kw: write(pos=pos, **kw),
        "read": lambda **kw: api.cover_kv8_read(*mem, pos0=7, n=9, **kw),
        "read_listed": lambda **kw: api.cover_kv8_read(*mem, pos=pos, dtype=torch.float32, **kw),
        "attn": lambda **kw: api.cover_attn_fwd_prefix8(q, *mem, q0=20, **kw),
        "attn_all": lambda **kw: api.cover_attn_fwd_prefix8(q, *mem, km, vm, pos[:, :3].contiguous(), q0=20, key_lo=lo, key_hi=hi,
                                                            softcap=9.0, **kw),
        "attn_no_lse": lambda **kw: api.cover_attn_fwd_prefix8(q, *mem, q0=20, want_lse=False, **kw),
    }


NAMES = ["rope", "rope_listed_back", "rope_q", "write", "write_listed", "read", "read_listed", "attn", "attn_all", "attn_no_lse"]


class _Counting:
    """The native marshalling, counting the calls that it took."""

    def __init__(self, native):
        self.native, self.took = native, 0

    def __getattr__(self, name):
        def call(*args):
            r = getattr(self.native, name)(*args)
            self.took += r is not None
            return r
        return call


@pytest.mark.parametrize("name", NAMES)
def test_native_call_equals_the_python_path(name, monkeypatch):
    torch.manual_seed(0)
    call = _calls()[name]
    counting = _Counting(api._native())
    monkeypatch.setattr(api, "_nat", counting)
    a = call()
    assert counting.took == 1
    b = call(stream=torch.cuda.current_stream())
    assert counting.took == 1
    torch.cuda.synchronize()
    assert type(a) is type(b) and len(a) == len(b)
    for x, y in zip(a, b):
        if x is None or y is None:
            assert x is y
            continue
        assert (x.shape, x.dtype, x.device, x.stride()) == (y.shape, y.dtype, y.device, y.stride())
        assert torch.equal(_bits(x), _bits(y))
    assert api.cover_device_status() == 0


def test_more_heads_than_a_grid_is_high():
    """70000 KV heads of one token."""
    H = 70000
    x = _r(1, H, 1, 64, seed=5)
    mem = api.kv8_memory(1, H, 1, 64)
    api.cover_kv8_write(x, -x, *mem)
    want = M8.decode(*M8.encode(_h(x)))
    for pos in (None, torch.zeros((1, 1), device="cuda", dtype=torch.int32)):
        k, v = api.cover_kv8_read(*mem, pos=pos)
        assert np.array_equal(_h(k), want) and np.array_equal(_h(v), -want)
    again = api.kv8_memory(1, H, 1, 64)
    api.cover_kv8_write(x, -x, *again, pos=torch.zeros((1, 1), device="cuda", dtype=torch.int32))
    for a, b in zip(mem, again):
        assert torch.equal(_bits(a), _bits(b))


def test_more_rows_at_once_than_a_grid_is_high():
    """2.2 million rows in one call (more than 65535 tiles of rows)."""
    n = 2200003
    x = _r(1, 1, n, 128, seed=6)
    mem = api.kv8_memory(1, 1, n)
    api.cover_kv8_write(x, x, *mem)
    k, v = api.cover_kv8_read(*mem)
    assert torch.equal(k, v)
    for at in (0, 65535 * 32 - 16, 65536 * 32 - 16, n - 40):
        rows = slice(at, at + 40)
        assert np.array_equal(_h(k[:, :, rows]), M8.decode(*M8.encode(_h(x[:, :, rows]))))
    assert ((k.float() - x.float()).abs() <= torch.maximum(x.float().abs() / 16, torch.exp2(mem[2].float() - 127)[..., None] / 1024)).all()


def _step(p):
    """Rotate a block, write it, override its seeds, attend: one layer's step."""
    q, k = api.cover_rope_fwd(p["q"], p["k"], p["f"], pos0=p["q0"])
    km, vm = api.cover_seed_kv_gather(k, p["v"], p["seeds"] - p["q0"])
    api.cover_kv8_write(k, p["v"], *p["mem"], pos0=p["q0"])
    api.cover_kv8_write(p["ck"], p["cv"], *p["mem"], pos=p["seeds"])
    return api.cover_attn_fwd_prefix8(q, *p["mem"], km, vm, p["seeds"], q0=p["q0"], key_hi=p["hi"])


def _program(seed, B=2, Hq=8, Hkv=2, n=32, L=3000, q0=2400, S=5):
    g = torch.Generator().manual_seed(seed)
    at = torch.stack([torch.randperm(n, generator=g)[:S] for _ in range(B)]).to(torch.int32).cuda() + q0
    hi = torch.full((B, n), q0 + n, device="cuda", dtype=torch.int32)
    hi[1] = 700          # a shorter sequence of a padded batch
    return dict(q=_r(B, Hq, n, 128, seed=seed), k=_r(B, Hkv, n, 128, seed=seed + 1), v=_r(B, Hkv, n, 128, seed=seed + 2),
                ck=_r(B, Hkv, S, 128, seed=seed + 3), cv=_r(B, Hkv, S, 128, seed=seed + 4), seeds=at, q0=q0, hi=hi,
                f=api.rope_frequencies(128)[0], mem=_mem(B, Hkv, L, seed + 5))


def test_two_steps_at_once_on_two_streams():
    ps = [_program(40), _program(60)]
    refs = [tuple(x.clone() for x in _step(p)) for p in ps]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in ps]
    for _ in range(5):
        outs = []
        for p, s in zip(ps, streams):
            with torch.cuda.stream(s):
                outs.append(_step(p))
        torch.cuda.synchronize()
        for o, r in zip(outs, refs):
            assert torch.equal(o[0], r[0]) and torch.equal(o[1], r[1])
    assert api.cover_device_status() == 0


def test_a_captured_step_beside_an_eager_one():
    p, e = _program(80), _program(100)
    ref, eager = _step(p)[0].clone(), _step(e)[0].clone()
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        out, lse = _step(p)
    side = torch.cuda.Stream()
    for _ in range(4):
        p["mem"][0].view(torch.uint8)[:, :, p["q0"]:p["q0"] + 32] = 0x38
        out.zero_()
        torch.cuda.synchronize()
        g.replay()
        with torch.cuda.stream(side):
            got = _step(e)[0]
        torch.cuda.synchronize()
        assert torch.equal(out, ref) and torch.equal(got, eager)


def test_a_padded_batch_ends_where_its_sequences_end():
    """Rows behind a sequence's last are neither written nor read: padding slots of the list, key_hi of the lengths."""
    B, Hkv, L, n = 3, 2, 900, 16
    lens = [5, 16, 0]
    mem = _mem(B, Hkv, L, 120)
    old = [x.clone() for x in mem]
    pos = torch.full((B, n), -1, device="cuda", dtype=torch.int32)
    for b, m in enumerate(lens):
        pos[b, :m] = 100 + torch.arange(m, device="cuda", dtype=torch.int32)
    k = _r(B, Hkv, n, 128, seed=130)
    for b, m in enumerate(lens):
        k[b, :, m:] = float("nan")
    api.cover_kv8_write(k, k, *mem, pos=pos)
    for a, b in zip(mem, old):
        for i, m in enumerate(lens):
            assert torch.equal(_bits(a)[i, :, 100 + m:], _bits(b)[i, :, 100 + m:]) and torch.equal(_bits(a)[i, :, :100], _bits(b)[i, :, :100])
    hi = torch.tensor([[100 + m if m else 0] * n for m in lens], device="cuda", dtype=torch.int32)
    q = _r(B, 4, n, 128, seed=131)
    out, lse = api.cover_attn_fwd_prefix8(q, *mem, q0=100, key_hi=hi)
    assert not out.isnan().any() and not out[2].any() and (lse[2] == -float("inf")).all()
    for x in mem[2:]:
        for b, m in enumerate(lens):
            x[b, :, 100 + m if m else 0:] = 255
    again, lse2 = api.cover_attn_fwd_prefix8(q, *mem, q0=100, key_hi=hi)
    assert torch.equal(again, out) and torch.equal(lse2, lse)


def test_lengths_that_change_between_replays():
    """A captured call follows the lengths that its key ranges hold when it is replayed (parts are shared out on the device)."""
    B, Hq, Hkv, L = 3, 32, 8, 20000
    assert api.cover_debug_attn_prefix8_plan(B, Hq, Hkv, 1, L, False, True)[2] > 100
    mem, q = _mem(B, Hkv, L, 140), _r(B, Hq, 1, 128, seed=141)
    hi = torch.full((B, 1), L, device="cuda", dtype=torch.int32)
    api.cover_attn_fwd_prefix8(q, *mem, q0=0, key_hi=hi)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        out, lse = api.cover_attn_fwd_prefix8(q, *mem, q0=0, key_hi=hi)
    k, v = (t.double() for t in api.cover_kv8_read(*mem, dtype=torch.float32))
    for lens in ([20000, 20000, 20000], [1, 19999, 0], [0, 0, 0], [0, 0, 12345], [4000, 8000, 20000]):
        hi.copy_(torch.tensor(lens, dtype=torch.int32)[:, None])
        g.replay()
        torch.cuda.synchronize()
        assert api.cover_device_status() == 0
        for b, n in enumerate(lens):
            if n == 0:
                assert not out[b].any() and (lse[b] == -float("inf")).all()
                continue
            s = torch.einsum("hgd,hnd->hgn", q[b, :, 0].double().view(Hkv, Hq // Hkv, 128), k[b, :, :n]) / 128 ** 0.5
            w = torch.softmax(s, -1)
            want, mass = torch.einsum("hgn,hnd->hgd", w, v[b, :, :n]), torch.einsum("hgn,hnd->hgd", w, v[b, :, :n].abs())
            # weights rounded to 9 bits or bf16 (2^-8), scores off by 2^-20 of sum |q_i k_i| / sqrt(D) <= 2^7, the output to bf16
            err = (out[b, :, 0].double().view_as(want) - want).abs()
            assert (err <= 2.0 ** -8 * want.abs() + (2.0 ** -8 + 4 * 2.0 ** -13) * mass).all()
            assert (lse[b, :, 0].double().view(Hkv, -1) - torch.logsumexp(s, -1)).abs().max() <= 2.0 ** -13 + 2.0 ** -15


@pytest.mark.parametrize("mode,parts", [(0, 16), (0, -8), (1, 16), (2, 16), (3, 16), (4, 1)])
def test_attention_over_more_than_32_bits_of_codes(mode, parts):
    """4.6e9 codes: zeros but for the last rows of every head, which have scores of their own; the rows before count exp(0)."""
    H, L, n = 9, 4000000, 700
    mem = api.kv8_memory(1, H, L)
    rows = _r(1, H, n, 128, seed=150)
    api.cover_kv8_write(rows, -rows, *mem, pos0=L - n)
    k, _ = api.cover_kv8_read(*mem, pos0=L - n, dtype=torch.float32)
    q = (k[:, :, [5, n - 1]] * 1.5).bfloat16()
    out, lse = api.cover_debug_attn_prefix8(q, *mem, q0=100, mode=mode, nsplit=parts)
    torch.cuda.synchronize()
    assert api.cover_device_status() == 0
    s = torch.einsum("bhrd,bhnd->bhrn", q.double(), k.double()) / 128 ** 0.5
    z = torch.logaddexp(torch.logsumexp(s, -1), torch.full_like(s[..., 0], L - n).log())
    w = torch.exp(s - z[..., None])
    want, mass = -torch.einsum("bhrn,bhnd->bhrd", w, k.double()), torch.einsum("bhrn,bhnd->bhrd", w, k.double().abs())
    # weights and output rounded to bf16; scores off by 2^-20 of sum |q_i k_i| / sqrt(D) <= 2^6; sums of up to 2^22 equal terms in
    # fp32, 128 and more threads or 32 columns at a time, off by 2^-24 for each of at most 2^15 additions
    rel = 4 * 2.0 ** -14 + 2.0 ** -9
    assert ((out.double() - want).abs() <= 2.0 ** -8 * want.abs() + (2.0 ** -8 + rel) * mass * (1 + 2.0 ** -6)).all()
    assert (lse.double() - z).abs().max() <= rel


def test_more_sequences_than_share_their_parts():
    """33 sequences of uneven lengths, some empty."""
    B, Hq, Hkv, L = 33, 8, 2, 700
    mem, q = _mem(B, Hkv, L, 160), _r(B, Hq, 1, 128, seed=161)
    hi = torch.tensor([[(37 * b) % (L + 1)] for b in range(B)], device="cuda", dtype=torch.int32)
    out, lse = api.cover_attn_fwd_prefix8(q, *mem, q0=0, key_hi=hi)
    for b in (0, 1, 15, 18, 32):
        n = int(hi[b])
        if n == 0:
            assert not out[b].any() and (lse[b] == -float("inf")).all()
            continue
        one = tuple(m[b:b + 1].contiguous() for m in mem)
        ref, ref_lse = api.cover_attn_fwd_prefix8(q[b:b + 1].contiguous(), *one, q0=0, key_hi=hi[b:b + 1].contiguous())
        v = api.cover_kv8_read(*one, dtype=torch.float32)[1].abs().max()
        assert (out[b:b + 1].float() - ref.float()).abs().max() <= 2 * 2.0 ** -7 * v    # each rounds weights and output by 2^-8
        assert (lse[b:b + 1] - ref_lse).abs().max() <= 2.0 ** -12
