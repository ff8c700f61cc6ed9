"""Values that are not finite in a memory in pages, and in the seeds' own pairs: wherever the keys' parts are cut and whatever the weight of
the element is in fp32, the rows that see it have no finite number in its column; the others are as without it."""
import math

import pytest
import torch

from paper_2602_06161_gb300 import api
from tests.test_gpu_attn_paged import _inputs, _ints, _run

pytestmark = pytest.mark.gpu

COLUMN = 77
# the kernels with their parts of the keys: streams of a CTA, CTAs joined by a second kernel, and in a cluster
WAYS = [(mode, parts) for mode in range(3) for parts in (1, 2, 5, -1, -2, -3, -8)]


def _peaked(Lq, S=0, tiles=6, Hq=2, Hkv=1, page=32):
    """One sequence: the scores are 0 in its second-last KV tile and -180 elsewhere (11.3 x 16 units), a weight of e^-180 = 0 in fp32."""
    d = _inputs([128 * tiles], Hq, Hkv, Lq, S, page, q0=[128 * tiles - Lq], junk=False)
    sign = torch.where(torch.arange(128, device="cuda") % 3 == 0, 1.0, -1.0)
    d["q"][:] = sign
    pages = d["table"][0].long().view(tiles, -1)
    d["kp"][:] = -16 * sign
    d["kp"][pages[tiles - 2]] = 0.01 * d["kp"][pages[tiles - 2]]
    return d, sign


def _forced(d, mode, parts, **kw):
    out, lse = api.cover_debug_attn_paged(d["q"], d["kp"], d["vp"], d["table"], d["lens"], d["km"], d["vm"], d["seeds"], q0=d["q0"], mode=mode,
                                          parts=parts, **kw)
    torch.cuda.synchronize()
    assert api.cover_device_status() == 0
    return out, lse


@pytest.mark.parametrize("mode,parts", WAYS)
@pytest.mark.parametrize("Lq", [1, 5])
@pytest.mark.parametrize("cap", [0.0, 200.0])
def test_a_value_of_no_weight(mode, parts, Lq, cap):
    d, _ = _peaked(Lq)
    ref, ref_lse = _forced(d, mode, parts, softcap=cap)
    assert ref.isfinite().all()
    for tile in range(6):
        page = int(d["table"][0, 4 * tile + 1])
        for value in (math.inf, math.nan):
            kept = d["vp"][page, 0, 3, COLUMN].item()
            d["vp"][page, 0, 3, COLUMN] = value
            out, lse = _forced(d, mode, parts, softcap=cap)
            d["vp"][page, 0, 3, COLUMN] = kept
            assert not out[..., COLUMN].isfinite().any(), tile
            rest = [c for c in range(128) if c != COLUMN]
            assert torch.equal(out[..., rest], ref[..., rest]) and torch.equal(lse, ref_lse)


@pytest.mark.parametrize("mode,parts", WAYS)
def test_pairs_of_no_weight(mode, parts):
    """A seed row whose own pair has all the weight sees the memory's values too, and its own value where the memory has all the weight."""
    for own, which in ((400.0, "memory"), (-400.0, "own")):
        d, sign = _peaked(4, S=1)
        d["seeds"] = _ints([[128 * 6 - 2]])          # row 2
        d["km"][:], d["vm"][:] = own / 128 ** 0.5 * sign, 1.0
        ref, _ = _forced(d, mode, parts)
        assert ref.isfinite().all()
        if which == "own":
            d["vm"][..., COLUMN] = math.inf
        else:
            d["vp"][int(d["table"][0, 5]), 0, 3, COLUMN] = math.inf
        out, _ = _forced(d, mode, parts)
        assert not out[:, :, 2, COLUMN].isfinite().any()
        if which == "own":
            assert torch.equal(out[:, :, [0, 1, 3]], ref[:, :, [0, 1, 3]])


@pytest.mark.parametrize("mode,parts", WAYS)
def test_rows_without_keys_and_parts_without_keys(mode, parts):
    """Every value that a row sees nothing of is infinite: a row without keys has zeros still, and parts without tiles add nothing."""
    d, _ = _peaked(3)
    d["vp"][:] = math.inf
    lo, hi = _ints([[0, 5, 700]]), _ints([[0, 5, 100]])
    out, lse = _forced(d, mode, parts, key_lo=lo, key_hi=hi)
    assert (out == 0).all() and (lse == -math.inf).all()
    d["vp"][:] = 2.0
    d["vp"][int(d["table"][0, 0]), 0, 9:] = math.inf
    hi = _ints([[7, 0, 9]])
    out, lse = _forced(d, mode, parts, key_hi=hi)
    assert (out[:, :, 1] == 0).all() and (out[:, :, [0, 2]] == 2).all()


def test_the_call_itself():
    for lens, Lq in (([5000], 1), ([700] * 30, 1), ([3000], 40), ([900, 900], 300)):
        d = _inputs(lens, 4, 2, Lq, 0, 64, junk=False)
        ref, ref_lse = _run(d)
        for b in range(len(lens)):
            d["vp"][int(d["table"][b, 2]), :, 1, COLUMN] = math.inf
        out, lse = _run(d)
        rest = [c for c in range(128) if c != COLUMN]
        assert not out[..., COLUMN].isfinite().any() and torch.equal(out[..., rest], ref[..., rest]) and torch.equal(lse, ref_lse)


@pytest.mark.parametrize("mode,parts", WAYS)
@pytest.mark.parametrize("Lq,cap", [(1, 0.0), (5, 0.0), (5, 30.0), (40, 0.0)])
def test_lse_is_of_queries_and_keys_alone(mode, parts, Lq, cap):
    """Values that are not finite in KV tiles which some row does not see whole, beside which others are seen: lse stays what it is."""
    d = _inputs([700, 300], 4, 2, Lq, 3, 32, junk=False)
    hi = _ints([[650 - 3 * r for r in range(Lq)], [290 - r if r % 2 == 0 else 60 for r in range(Lq)]])
    ref, ref_lse = _forced(d, mode, parts, key_hi=hi, softcap=cap)
    assert ref_lse.isfinite().all()
    for value in (math.nan, math.inf, -math.inf):
        for b, key in ((0, 520), (0, 3), (1, 257)):
            d["vp"][int(d["table"][b, key // 32]), :, key % 32, COLUMN] = value
        out, lse = _forced(d, mode, parts, key_hi=hi, softcap=cap)
        assert torch.equal(lse, ref_lse)
        sees = torch.stack([hi[0] > 3, hi[1] > 257])
        assert not out.transpose(1, 2)[sees][..., COLUMN].isfinite().any()
        assert torch.equal(out.transpose(1, 2)[~sees], ref.transpose(1, 2)[~sees])
