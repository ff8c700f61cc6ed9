"""Pins of the 8-bit memory's oracle: known codes, known angles, and the two-view attention's oracle."""
import math

import numpy as np
import pytest
import torch

import oracle
from oracle import memory8_oracle as M8


def test_code_values_are_torchs():
    codes = torch.arange(256, dtype=torch.uint8)
    ref = codes.view(torch.float8_e4m3fn).double().numpy()
    got = M8.decode(codes.numpy()[:, None], np.full(256, 127))[:, 0]
    assert np.array_equal(got, ref, equal_nan=True)


def test_rows_round_as_torch_rounds():
    rng = np.random.default_rng(0)
    rows = rng.standard_normal((64, 64)) * 2.0 ** rng.integers(-9, 9, (64, 1))
    rows = torch.from_numpy(rows).to(torch.bfloat16).double().numpy()   # many ties
    codes, byte = M8.encode(rows)
    scaled = rows * 2.0 ** (127 - byte.astype(np.float64))[:, None]
    assert np.all(np.abs(scaled).max(1) <= 448) and np.all(np.abs(scaled).max(1) > 224)
    ref = torch.from_numpy(scaled).float().to(torch.float8_e4m3fn).view(torch.uint8).numpy()
    assert np.array_equal(codes, ref)


@pytest.mark.parametrize("row,codes,byte", [
    ([0.0, -0.0], [0, 128], 127), ([448.0, 1.0], [126, 56], 127), ([449.0, 0.0], [118, 0], 128), ([1.0, -1.0], [120, 248], 119),
    ([math.inf, 1.0], [0, 0], 255), ([math.nan, 0.0], [0, 0], 255), ([2.0 ** -140, 0.0], [0, 0], 17),
    ([3.4e38, -3.4e38], [126, 254], 246),
])
def test_known_rows(row, codes, byte):
    got, b = M8.encode_row(row)
    assert got.tolist() == codes and b == byte


def test_rope_of_a_quarter_turn_and_back():
    x = np.arange(8.0).reshape(1, 1, 1, 8)
    f = np.array([math.pi / 2, 0.0])
    half = M8.rope(x, f, np.array([[1]]), interleaved=False)
    assert np.allclose(half[0, 0, 0], [-2, 1, 0, 3, 4, 5, 6, 7], atol=1e-15)
    inter = M8.rope(x, f, np.array([[1]]), interleaved=True)
    assert np.allclose(inter[0, 0, 0], [-1, 0, 2, 3, 4, 5, 6, 7], atol=1e-15)
    assert np.allclose(M8.rope(inter, f, np.array([[1]]), interleaved=True, inverse=True), x, atol=1e-15)


def test_attention_is_the_two_view_oracles():
    rng = np.random.default_rng(1)
    q, k, v = rng.standard_normal((2, 4, 9, 16)), rng.standard_normal((2, 2, 9, 16)), rng.standard_normal((2, 2, 9, 16))
    km, vm = rng.standard_normal((2, 2, 3, 16)), rng.standard_normal((2, 2, 3, 16))
    seeds = np.array([[4, 0, 4], [8, -1, 20]], np.int32)
    out, lse, _, _ = M8.attention(q, k, v, km, vm, seeds, q0=0)
    ref, ref_lse = oracle.override_attention(q, k, v, km, vm, seeds)
    assert np.abs(out - ref).max() < 1e-12 and np.abs(lse - ref_lse).max() < 1e-12


def test_attention_ranges_are_a_shorter_memory():
    rng = np.random.default_rng(2)
    q, k, v = rng.standard_normal((1, 2, 3, 16)), rng.standard_normal((1, 2, 12, 16)), rng.standard_normal((1, 2, 12, 16))
    lo, hi = np.array([[2, 2, 7]]), np.array([[9, 9, 7]])
    out, lse, _, _ = M8.attention(q, k, v, None, None, None, q0=0, key_lo=lo, key_hi=hi, softcap=2.0)
    ref, ref_lse, _, _ = M8.attention(q[:, :, :2], k[:, :, 2:9], v[:, :, 2:9], None, None, None, q0=0, softcap=2.0)
    assert np.allclose(out[:, :, :2], ref) and np.allclose(lse[:, :, :2], ref_lse)
    assert np.all(out[:, :, 2] == 0) and np.all(lse[:, :, 2] == -math.inf)
