"""The tests' own model of the 8-bit cache: its conversions against another library's, its growth rule on cases worked out by hand."""
import numpy as np
import pytest
import torch

import kv_reference as R


def test_e4m3_table_and_rounding_agree_with_the_library_type():
    codes = torch.arange(256, dtype=torch.uint8)
    theirs = codes.view(torch.float8_e4m3fn).float().numpy()
    assert np.array_equal(theirs, R.E4M3, equal_nan=True)
    rng = np.random.default_rng(0)
    x = np.concatenate([rng.normal(0, 100, 20000), rng.normal(0, 0.01, 20000), R._MID, -R._MID, [0.0, -0.0, 448, -448]]).astype(np.float32)
    x = np.clip(x, -448, 448)
    assert np.array_equal(R.encode(x, "e4m3"), torch.from_numpy(x).to(torch.float8_e4m3fn).view(torch.uint8).numpy())


def test_v_places_are_a_permutation_in_which_eight_tokens_are_neighbours():
    for P, D in ((32, 64), (64, 128), (128, 192)):
        assert sorted(R.v_index(P, D).ravel()) == list(range(P * D))
    assert [R.v_place(t, 0, 64) for t in (0, 1, 2, 3, 16, 17, 18, 19)] == list(range(8))
    assert R.v_place(0, 1, 64) == 8 and R.v_place(4, 0, 64) == 16 and R.v_place(0, 2, 64) == 64 and R.v_place(32, 0, 64) == 32 * 64


@pytest.mark.parametrize("fmt,first,second,scale,older", [
    ("int8", 127.0, 126.0, 1.0, 127),          # fits
    ("int8", 127.0, 128.0, 2.0, 64),           # 127 / 2 = 63.5: to even
    ("int8", 127.0, 254.0, 2.0, 64),           # exactly twice
    ("int8", 127.0, 255.0, 4.0, 32),           # 31.75
    ("e4m3", 448.0, 449.0, 2.0, 224.0),
])
def test_growth_by_powers_of_two(fmt, first, second, scale, older):
    m = R.Model(1, 1, 64, 32, fmt)
    row = np.zeros((1, 1, 64), np.float32)
    m.append(0, row + np.float32(first), 0, [0])
    assert m.scale[0][0, 0] == 1.0
    m.append(0, row + np.float32(second), 1, [0])
    assert m.scale[0][0, 0] == scale and R.decode(m.codes[0][0, 0, 0, :1], fmt)[0] == older
