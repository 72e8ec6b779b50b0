"""Pins of the 8-bit cache's oracle: its code tables against torch's, rounding against a search over all codes, scales and
writes against the definition."""
import numpy as np
import pytest
import torch

from oracle import quant as oq


def test_tables_are_the_types():
    c = torch.arange(256, dtype=torch.uint8)
    assert np.array_equal(oq.TABLE["e4m3"], c.view(torch.float8_e4m3fn).double().numpy(), equal_nan=True)
    i = c.view(torch.int8).double().numpy()
    i[128] = np.nan
    assert np.array_equal(oq.TABLE["int8"], i, equal_nan=True)


@pytest.mark.parametrize("fmt", ["e4m3", "int8"])
def test_encode_rounds_to_the_nearest_code(fmt):
    rng = np.random.default_rng(1)
    top = oq.LARGEST[fmt]
    t = oq.TABLE[fmt]
    grid = np.sort(t[np.isfinite(t)])
    x = np.concatenate([rng.uniform(-top, top, 2000), top * 2.0 ** -rng.uniform(0, 20, 2000), grid, (grid[1:] + grid[:-1]) / 2])
    got = t[oq.encode(x, fmt)]
    best = np.abs(x[:, None] - grid).min(1)
    assert np.array_equal(np.abs(x - got), best)
    ref = torch.from_numpy(x.astype(np.float32))                     # (the grid's midpoints are fp32 numbers)
    x32 = x.astype(np.float32).astype(np.float64)
    want = ref.to(torch.float8_e4m3fn).double().numpy() if fmt == "e4m3" else torch.round(ref).double().numpy()
    assert np.array_equal(t[oq.encode(x32, fmt)], want)


@pytest.mark.parametrize("fmt", ["e4m3", "int8"])
def test_scale_is_the_smallest_that_holds(fmt):
    c = oq.LARGEST[fmt]
    for e in (-140, -126, -100, -3, 0, 5, 100, 119):
        for f in (1.0, 1 + 2.0 ** -23, 1 - 2.0 ** -24, 1.5):
            top = c * 2.0 ** e * f
            s = oq.need(top, fmt)
            assert 1 <= s <= 249 and top <= c * 2.0 ** (s - 127) and (s == 1 or top > c * 2.0 ** (s - 128))
    assert oq.need(0.0, fmt) == 0


@pytest.mark.parametrize("fmt", ["e4m3", "int8"])
def test_writes_in_pieces(fmt):
    """Whole blocks do not depend on the calls' borders; a block written in pieces is within a step of its final scale of
    the rows, and a NaN row stays alone."""
    rng = np.random.default_rng(2)
    x = rng.standard_normal((70, 8)).astype(np.float32) * np.exp(rng.uniform(-3, 3, (70, 1)))
    x[37, 3], x[41, 0] = np.nan, np.inf
    one, s1 = np.full((80, 8), 9, np.uint8), np.full(5, 7, np.uint8)
    oq.write(one, s1, x, 0, 70, 16, fmt)
    two, s2 = one.copy(), s1.copy()
    two[:], s2[:] = 9, 7
    for a, b in ((0, 32), (32, 33), (33, 48), (48, 70)):
        oq.write(two, s2, x[a:b], a, b - a, 16, fmt)
    blocks = [0, 1, 3]
    assert np.array_equal(s1[blocks], s2[blocks]) and (one[70:] == 9).all() and np.array_equal(one[:32], two[:32])
    assert np.array_equal(s1, s2)                                    # (the last piece's need covers the first one's)
    v = oq.values(two[:70], s2, 16, fmt)
    bad = np.isnan(v)
    assert bad[37].all() and bad[41].all() and bad.sum() == 16
    step = 2.0 ** (s2[np.arange(70) // 16].astype(float) - 127)[:, None]
    # twice a half step: of the codes' distance, 1 for int8 and at most 32 for e4m3
    assert (np.abs(v - x)[~bad] <= (np.broadcast_to(step, x.shape) * (1 if fmt == "int8" else 32))[~bad]).all()


def test_attend_of_one_and_no_keys():
    rng = np.random.default_rng(3)
    q, k, v = rng.standard_normal(8), rng.standard_normal((4, 8)), rng.standard_normal((4, 8))
    O, lse, A, Z = oq.attend(q, k, v, np.array([2]))
    assert np.allclose(O, v[2]) and np.isclose(lse, q @ k[2] / np.sqrt(8)) and np.allclose(A, np.abs(v[2])) and Z >= abs(lse)
    O, lse, _, _ = oq.attend(q, k, v, np.array([], int))
    assert (O == 0).all() and lse == -np.inf
