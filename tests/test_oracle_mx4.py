"""Pins of the microscaled 4-bit oracle: none of the expected values comes from the oracle itself."""
import numpy as np
import pytest
import torch

from oracle import mx4


def test_grids_are_the_types():
    f8 = torch.arange(127, dtype=torch.uint8).view(torch.float8_e4m3fn).double().numpy()
    assert np.array_equal(mx4.E4M3, f8)
    # e2m1 by its definition: two exponent bits with bias one, one mantissa bit, no infinities
    want = [(c & 1) * 0.5 if c < 2 else 2.0 ** ((c >> 1) - 1) * (1 + (c & 1) / 2) for c in range(8)]
    assert np.array_equal(mx4.GRID, want)


def test_ties_and_ends():
    x = np.array([0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0, 100.0, 0.2500001, 4.9999])
    assert mx4.GRID[mx4.nearest_even(x, mx4.GRID)].tolist() == [0, 1, 1, 2, 2, 4, 4, 6, 0.5, 4]
    r = np.random.default_rng(0).uniform(0, 460, 5000).astype(np.float32)
    r = r[r < 448]
    want = torch.tensor(r).to(torch.float8_e4m3fn).double().numpy()
    assert np.array_equal(mx4.E4M3[mx4.nearest_even(r.astype(np.float64), mx4.E4M3)], want)


def test_block_scales_worked_by_hand():
    X = np.zeros((1, 96))
    X[0, 3], X[0, 40], X[0, 70] = 6.0, -6.0001, 0.75
    _, byte, _ = mx4.quantize(X, "mxfp4")
    assert byte.tolist() == [[127, 128, 124]]            # 1, 2, 1/8: the smallest power of two with at most six of it
    X = np.zeros((2, 16))
    X[0, 0], X[1, 3] = 2688.0, 3.0
    _, byte, whole = mx4.quantize(X, "nvfp4")
    assert whole == 1.0 and mx4.E4M3[byte].tolist() == [[448.0, 0.0], [0.5, 0.0]]
    assert mx4.whole_scale(np.array([[2688.5]]), "nvfp4") == 2.0
    assert mx4.whole_scale(np.array([[2688.0 / 2 ** 20, np.inf]]), "nvfp4") == 2.0 ** -20


@pytest.mark.parametrize("fmt", ["mxfp4", "nvfp4"])
def test_error_of_a_round_trip(fmt):
    """The spacing of e2m1 is at most a third of the value (between 4 and 6) or half a unit: |error| <= max(|x| / 5, scale / 4), and
    nothing is clipped by more than the scale's own rounding (1/16, nvfp4)."""
    rng = np.random.default_rng(1)
    X = rng.standard_normal((40, 100)) * np.exp(2 * rng.standard_normal((40, 1)))
    index, byte, whole = mx4.quantize(X, fmt)
    back = mx4.values(index, byte, whole, fmt, 100)
    s = np.repeat(mx4.decode_scale(byte, fmt, whole), mx4.BLOCK[fmt], axis=1)[:, :100]
    assert np.all(np.abs(back - X) <= np.maximum(np.abs(X) / 5, s / 4) * (1 + 1e-12))
    assert np.array_equal(mx4.round_trip(back, fmt), back) or fmt == "nvfp4"


def test_bad_values_stay_in_their_block():
    X = np.full((3, 64), 6.0)          # a scale of one in either format
    X[1, 5], X[2, 60] = np.nan, -np.inf
    for fmt, blk in mx4.BLOCK.items():
        back = mx4.round_trip(X, fmt)
        want = np.zeros((3, 64), dtype=bool)
        want[1, 5 // blk * blk:(5 // blk + 1) * blk] = True
        want[2, 60 // blk * blk:(60 // blk + 1) * blk] = True
        assert np.array_equal(np.isnan(back), want) and np.all(back[~want] == 6.0)


def test_layout():
    byte = np.arange(130 * 5).reshape(130, 5).astype(np.uint8)
    t = mx4.tiles(byte)
    assert t.shape == (2, 2, 512)
    assert t[0, 0, 0] == byte[0, 0] and t[0, 0, 3] == byte[0, 3] and t[0, 0, 4] == byte[32, 0] and t[0, 0, 16] == byte[1, 0]
    assert t[1, 1, 16] == byte[129, 4] and t[1, 1, 17] == 0
    assert mx4.pack(np.array([[1, 2, 15, 0]], dtype=np.uint8)).tolist() == [[0x21, 0x0F]]
