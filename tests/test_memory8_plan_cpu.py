"""The 8-bit attention's choice of a kernel and of the keys' parts, and the workspace that goes with it: host arithmetic."""
import itertools

import pytest

from paper_2602_06161_gb300 import api

ROWS, WIDE, TILE, PAIRS, READ_BACK = range(5)


def plan(*a, plain=False, ranges=False):
    return api.cover_debug_attn_prefix8_plan(*a, plain, ranges)


def bytes_of(mode, nsplit, B, Hq, Hkv, Lq, Lk):
    decoded = 2 * B * Hkv * Lk * 128 * 2 if mode in (PAIRS, READ_BACK) else 0
    if nsplit > 100:
        return decoded + (nsplit - 100 + B) * Hq * Lq * 520 + 256
    parts = (B * Hq * Lq * nsplit * 520 + 15) // 16 * 16 if nsplit > 1 else 0
    return decoded + parts


@pytest.mark.parametrize("B,heads,Lq,Lk", list(itertools.product(
    [1, 5, 16], [(28, 4), (32, 8), (32, 32), (16, 1)], [1, 2, 17, 64, 300, 2048], [2048, 8191, 70000])))
def test_parts_and_workspace(B, heads, Lq, Lk):
    Hq, Hkv = heads
    need = 0
    for plain, ranges in ((False, False), (False, True), (True, False)):
        mode, groups, nsplit, us = plan(B, Hq, Hkv, Lq, Lk, plain=plain, ranges=ranges)
        assert us > 0
        if nsplit > 100:     # shared out to a batch's sequences
            assert ranges and mode <= WIDE and 2 <= B <= 32 and B * Lq <= 2048 and B <= nsplit - 100 <= 64 * B
        else:
            assert (1 <= nsplit <= 64 or -8 <= nsplit <= -2 and mode <= TILE) and abs(nsplit) <= (Lk + 127) // 128
        assert plain or mode != READ_BACK
        if mode != READ_BACK:
            size = (16, 32, 128, 256)[mode]
            assert groups == -(-(Hq // Hkv) * Lq // size)
        need = max(need, bytes_of(mode, nsplit, B, Hq, Hkv, Lq, Lk))
    assert api.cover_attn_prefix8_workspace_bytes(B, Hq, Hkv, Lq, Lk) == need


def test_choices():
    assert plan(4, 32, 8, 1, 131072)[0] == ROWS                       # tokens over long memories read the codes
    assert plan(4, 32, 8, 8, 131072)[0] == WIDE                       # 32 packed rows
    assert plan(8, 32, 32, 64, 2048)[0] == TILE                       # blocks of a batch
    assert plan(1, 32, 8, 2048, 8192)[0] == PAIRS                     # a prompt's last part
    assert plan(1, 32, 8, 2048, 8192, plain=True)[0] == READ_BACK
    assert plan(1, 28, 4, 32, 1024, plain=True)[0] == READ_BACK       # an active block
    assert plan(1, 28, 4, 1, 100)[2] == 1                             # one KV tile has no parts
    assert plan(4, 32, 8, 1, 131072)[2] > 1
    assert plan(4, 32, 8, 1, 131072, ranges=True)[2] > 100            # a padded batch
    assert plan(1, 32, 8, 1, 131072, ranges=True)[2] < 100            # one sequence has nothing to share


def test_invalid_sizes():
    for a in ((0, 1, 1, 1, 1), (1, 3, 2, 1, 1), (1, 1, 1, 2, 1), (1, 1, 1, 0, 1), (1, 1, 0, 1, 1)):
        with pytest.raises(api._lib.CoverError):
            plan(*a)
    with pytest.raises(api._lib.CoverError):
        plan(1, 1, 1, 1, 1, plain=True, ranges=True)
