"""Calls whose kernels run on a stream that is not the current one: what a call makes for itself (results, workspaces) is not
taken from blocks that the current stream's pending work still uses."""
import pytest
import torch

from paper_2602_06161_gb300 import api

pytestmark = pytest.mark.gpu


def _r(*shape, dtype=torch.bfloat16, seed=0):
    return torch.randn(shape, generator=torch.Generator("cuda").manual_seed(seed), device="cuda").to(dtype)


def _calls():
    B, Hq, Hkv, L, Lq = 2, 8, 2, 3000, 40
    q, k, v = _r(B, Hq, L, 128), _r(B, Hkv, L, 128, seed=1), _r(B, Hkv, L, 128, seed=2)
    qw = q[:, :, :Lq].contiguous()
    f, _ = api.rope_frequencies(128)
    mem = api.kv8_memory(B, Hkv, L)
    api.cover_kv8_write(k, v, *mem)
    seeds = torch.arange(4, device="cuda", dtype=torch.int32).repeat(B, 1)
    x = _r(64, 5000, seed=3)
    lse = _r(B, Hq, L, dtype=torch.float32, seed=4) + 8
    tok = torch.randint(0, 9, (B * 64,), device="cuda", dtype=torch.int32)
    flags = torch.full((B * 64,), 2, device="cuda", dtype=torch.uint8)
    hi = torch.tensor([[L], [200]], device="cuda", dtype=torch.int32)
    q1 = q[:, :, :1].contiguous()
    # a decision step changes its state: one for each call, made before
    a = [[torch.zeros(64, device="cuda", dtype=t) for t in (torch.int32, torch.uint8, torch.uint8)] for _ in range(2)]
    return {
        "rope": lambda **kw: api.cover_rope_fwd(q, k, f, **kw),
        "read": lambda **kw: api.cover_kv8_read(*mem, **kw),
        "attn8": lambda **kw: api.cover_attn_fwd_prefix8(qw, *mem, q0=0, **kw),
        "attn8_shared": lambda **kw: api.cover_attn_fwd_prefix8(q1, *mem, q0=0, key_hi=hi, **kw),
        "attn": lambda **kw: api.cover_attn_fwd(q, k, v, **kw),
        "prefix": lambda **kw: api.cover_attn_fwd_prefix(qw, k, v, q0=0, **kw),
        "score": lambda **kw: tuple(api.cover_score_fwd(x, 2, 3, **kw).values()),
        "decide": lambda **kw: tuple(api.cover_score_decide_fwd(x, 2, *a.pop(), tau_draft=0.5, draft_budget=2,
                                                                remask_budget=2, mask_id=0, max_seeds=4, **kw).values()),
        "mass": lambda **kw: api.cover_attn_mass_fwd(q, k, lse, tok, flags, mask_id=3, pos0=0, per=64, **kw),
        "gather": lambda **kw: api.cover_seed_kv_gather(k, v, seeds, **kw),
        "route": lambda **kw: api.cover_seed_route(seeds, B, L, **kw),
    }


def _span(t):
    return t.data_ptr(), t.data_ptr() + t.numel() * t.element_size()


@pytest.mark.parametrize("given", ["stream", "handle", "default"])
@pytest.mark.parametrize("name", ["rope", "read", "attn8", "attn8_shared", "attn", "prefix", "score", "decide", "mass", "gather", "route"])
def test_no_block_of_pending_work_is_taken(name, given):
    call = _calls()[name]
    ref = call()
    torch.cuda.synchronize()
    # the current stream frees blocks of the results' sizes, and of workspaces', that its pending work is still to write
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


def test_a_result_is_kept_until_the_current_stream_is_done_with_it():
    """A result that is freed while the caller's stream still reads it is not handed out again by the other stream's memory."""
    q, f = _r(1, 8, 1000, 128), api.rope_frequencies(128)[0]
    here, there = torch.cuda.Stream(), torch.cuda.Stream()
    torch.cuda.synchronize()
    with torch.cuda.stream(here):
        y, _ = api.cover_rope_fwd(q, None, f, stream=there)
        here.wait_stream(there)
        torch.cuda._sleep(20_000_000)
        kept, (lo, hi) = y.clone(), _span(y)
        del y
        with torch.cuda.stream(there):
            other = torch.full_like(q, 9.0)
        assert not (_span(other)[0] < hi and lo < _span(other)[1])
    torch.cuda.synchronize()
    assert torch.equal(kept, api.cover_rope_fwd(q, None, f)[0])


def test_a_captured_call_on_another_stream():
    """A call on a stream that a capture has forked to makes its tensors in the graph's memory."""
    call = _calls()["attn8"]
    ref = call()
    torch.cuda.synchronize()
    side, g = torch.cuda.Stream(), torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        side.wait_stream(torch.cuda.current_stream())
        out, lse = call(stream=side)
        torch.cuda.current_stream().wait_stream(side)
        kept = out.clone(), lse.clone()
    others = [torch.full_like(out, 7.0) for _ in range(50)]      # of the allocator's other memory
    for _ in range(2):
        g.replay()
    torch.cuda.synchronize()
    assert api.cover_device_status() == 0
    assert torch.equal(kept[0], ref[0]) and torch.equal(kept[1], ref[1]) and all((o == 7.0).all() for o in others)
