"""The oracle's keys against values that can be read off."""
import numpy as np

from oracle import efim_kv4_oracle as orc


def _rounded(x):
    return orc.key(np.array([x]), None)[0]


def test_norm_and_rotation():
    table = np.array([0.6, 1.0, 0.8, 0.0], np.float32)
    c, s = np.float64(table[0]), np.float64(table[2])
    x = np.array([3.0, 5.0, 4.0, 7.0])
    assert orc.key(x, table).tolist() == [_rounded(3 * c - 4 * s), 5.0, _rounded(4 * c + 3 * s), 7.0]
    assert orc.key(x, table, True).tolist() == [_rounded(3 * c - 5 * s), _rounded(5 * c + 3 * s), 4.0, 7.0]
    # 3 / sqrt(12.5) 5 = 4.2426, 4 / sqrt(12.5) 10 = 11.3137
    assert orc.key(np.array([3.0, 4.0]), None, weight=np.array([5.0, 10.0])).tolist() == [4.25, 11.3125]


def test_roundings():
    """fp32 first, then bf16, ties to even."""
    half = 1 + 2.0 ** -8                                                  # halfway between two bf16 numbers
    x = np.array([half, half + 2.0 ** -7, half + 2.0 ** -23, half + 2.0 ** -26, -half - 2.0 ** -23])
    assert orc.key(x, None).tolist() == [1.0, 1 + 2.0 ** -6, 1 + 2.0 ** -7, 1.0, -1 - 2.0 ** -7]
    assert np.isnan(_rounded(np.nan)) and _rounded(1e39) == np.inf and _rounded(-3.4e38) == -np.inf and np.signbit(_rounded(-0.0))
