"""Refusals of the calls over a memory in pages, on both ways of marshalling."""
import pytest
import torch

from paper_2602_06161_gb300 import api
from tests.test_gpu_paged_append import BF, _ints, _pool, _rows

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("mscale", [1.0, 1])   # (an integer goes through the checks in Python)
def test_rows_in_the_pages_are_refused(mscale):
    kp, vp, table = _pool([64, 64], 2, 16, 64)
    start, f = _ints([3, 9]), api.rope_frequencies(64)[0]
    k, v, q = _rows(2, 2, 5, 64, BF), _rows(2, 2, 5, 64, BF, 1), _rows(2, 4, 5, 64, BF, 2)
    old = kp.clone(), vp.clone()
    inside = kp[:2, :, :5], vp[2:4, :, 3:8]
    for args in ((inside[0], v, kp, vp, q), (k, inside[1], kp, vp, q), (k, v, kp, vp, kp[:4].view(2, 4, 16, 64)[:, :, :5]), (k, v, kp, kp, q)):
        with pytest.raises(ValueError, match="must not overlap"):
            api.cover_paged_append(*args[:4], table, start=start, q=args[4], inv_freq=f, mscale=mscale)
    torch.cuda.synchronize()
    assert torch.equal(kp, old[0]) and torch.equal(vp, old[1])
    # pages and rows that are neighbours in one buffer
    flat = torch.zeros(2 * kp.numel() + k.numel(), device="cuda", dtype=BF)
    mine = flat[:kp.numel()].view(kp.shape), flat[kp.numel():2 * kp.numel()].view(kp.shape)
    rows = flat[2 * kp.numel():].view(k.shape)
    for a, b in zip(mine, (kp, vp)):
        a.copy_(b)
    rows.copy_(k)
    yq, _ = api.cover_paged_append(rows, rows, *mine, table, start=start, q=q, inv_freq=f, mscale=mscale)
    zq, _ = api.cover_paged_append(k, k, kp, vp, table, start=start, q=q, inv_freq=f, mscale=mscale)
    assert torch.equal(yq, zq) and torch.equal(mine[0], kp) and torch.equal(mine[1], vp) and torch.equal(rows, k)


def test_the_debug_attention_call_checks_its_tensors():
    kp, vp = api.paged_memory(5, 2, 16)
    q, table, lens = torch.zeros((1, 4, 8, 128), device="cuda", dtype=BF), _ints([[0, 1]]), _ints([20])
    pair, seeds, q0 = torch.zeros((1, 2, 2, 128), device="cuda", dtype=BF), _ints([[3, 4]]), _ints([2])
    call = lambda *a, mode=0, **kw: api.cover_debug_attn_paged(*a, mode=mode, **kw)  # noqa: E731
    for args, kw, what in (((q, kp, vp, table, lens), dict(key_hi=torch.zeros((1, 8), device="cuda", dtype=torch.int64)), "key_hi"),
                           ((q, kp, vp, table, lens), dict(key_lo=_ints([[0] * 7])), "key_lo"), ((q, kp, vp, table, lens), dict(q0=_ints([0, 0])), "q0"),
                           ((q, kp, vp, table.expand(2, 2).contiguous(), lens), {}, "table"), ((q, kp, vp, table, _ints([20, 3])), {}, "lens"),
                           ((q, kp, vp[1:], table, lens), {}, "v_pages"), ((q[..., :64].contiguous(), kp, vp, table, lens), {}, "pages"),
                           ((q, kp, vp, table, lens, pair[:, :1].contiguous(), pair, seeds), dict(q0=q0), "k_seedmask"),
                           ((q, kp, vp, table, lens, pair, pair, seeds.expand(2, 2).contiguous()), dict(q0=q0), "seed_idx"),
                           ((q, kp, vp, table, lens, pair, pair, seeds), {}, "q0"),
                           ((q, kp, vp, table, lens), dict(workspace=torch.zeros(4096, device="cuda")), "workspace")):
        for mode in (0, 1, 2):
            with pytest.raises((TypeError, ValueError), match=what):
                call(*args, mode=mode, **kw)
