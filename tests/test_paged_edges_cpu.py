"""What the calls over a memory in pages refuse before anything is launched, on CPU tensors."""
import pytest
import torch

from paper_2602_06161_gb300 import api

BF = torch.bfloat16


def test_pages_that_are_written_lie_apart_from_everything():
    flat = torch.zeros(4 * 2 * 16 * 64 * 3, dtype=BF)
    pool = flat.view(3, 4, 2, 16, 64)
    kp, vp, rest = pool[0], pool[1], pool[2]
    k = rest[:2]
    api._pages_apart(kp, vp, k=k, v=k.transpose(1, 2), q=None, table=torch.zeros(4, 4, dtype=torch.int32))
    api._pages_apart(kp, vp, k=kp[:0], q=k)                                   # nothing lies anywhere
    for args, match in (((kp, vp, dict(k=kp[:1])), "k_pages must not overlap k"), ((kp, vp, dict(q=k, v=vp[3:, :, :1])), "v_pages must not overlap v"),
                        ((kp, kp, {}), "k_pages must not overlap v_pages"), ((kp, vp, dict(table=vp.view(torch.int32)[0, 0])), "v_pages must not overlap table"),
                        ((flat[:8192].view(4, 2, 16, 64), flat[8191:8191 + 8192].view(4, 2, 16, 64), {}), "k_pages must not overlap v_pages"),
                        # rows of which one element lies in the pages
                        ((kp, vp, dict(q=flat[2 * 8192 - 1:][:128 * 8].view(1, 2, 8, 64))), "v_pages must not overlap q")):
        with pytest.raises(ValueError, match=match):
            api._pages_apart(*args[:2], **args[2])


def test_the_debug_attention_call_checks_its_tensors():
    kp, vp = api.paged_memory(3, 2, 16, device="cpu")
    q, i = torch.zeros(1, 4, 2, 128, dtype=BF), lambda *s: torch.zeros(s, dtype=torch.int32)
    with pytest.raises(ValueError, match="q must be a CUDA tensor"):
        api.cover_debug_attn_paged(q, kp, vp, i(1, 2), i(1), mode=0)
    with pytest.raises(TypeError, match="q must be"):
        api.cover_debug_attn_paged(q.float(), kp, vp, i(1, 2), i(1), mode=0)
