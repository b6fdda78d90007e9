"""The oracle of a step over a 4-bit cache against values that can be read off."""
import numpy as np

from oracle import efim_kv4_oracle as orc


def test_values():
    assert orc.E4M3[1] == 2.0 ** -9 and orc.E4M3[8] == 2.0 ** -6 and orc.E4M3[126] == 448 and (np.diff(orc.E4M3) > 0).all()
    x = np.array([0, 0.25, 0.26, 0.5, 0.75, -1.25, 1.75, 2.5, 3.5, 5, -5.01, 6, -0.2, 1, 2, 4])
    codes, scales = orc.quantize(x[None], 1.0)
    assert scales.tolist() == [[0x38]]                                       # 1.0
    assert orc.held(codes, scales, 1.0)[0].tolist() == [0, 0, 0.5, 0.5, 1, -1, 2, 2, 4, 4, -6, 6, 0, 1, 2, 4]
    assert codes[0, 0] == 0 and codes[0, 1] == 1 | 1 << 4


def test_ends():
    huge = np.full((1, 16), 1e30)
    assert orc.held(*orc.quantize(huge, 1.0), 1.0).max() == 2688
    assert orc.held(*orc.quantize(np.full((1, 16), -np.inf), 0.5), 0.5).min() == -1344
    assert (orc.quantize(np.zeros((1, 16)), 1.0)[1] == 1).all()
    block = np.zeros((1, 32))
    block[0, 3] = np.nan
    got = orc.held(*orc.quantize(block, 1.0), 1.0)
    assert np.isnan(got[0, :16]).all() and (got[0, 16:] == 0).all()


def test_steps():
    indptr, table, free, pos, slots, seqs, out = orc.step_tables([15, 32, 0], [2, 0, 33], [[7, -1, -1], [5, 6, -1], [-1, 9, -1]], [1, 2, 3], 40)
    assert indptr == [0, 2, 2, 35] and table == [[7, 3, -1], [5, 6, -1], [2, 9, 1]] and free == [] and not out
    assert pos[:3] == [15, 16, 0] and slots[:3] == [127, 48, 32] and slots[34] == 16 and pos[35:] == slots[35:] == seqs[35:] == [-1] * 5


def test_adjusted():
    x, _ = orc.adjust([2.0, -2.0, 1.0, 0.0, 5.0], [0], [1, 1, 2], 2.0, 0.5, 0.25, [(3, 1.0), (3, 4.0)], np.array([1, 1, 1, 1, 0], bool))
    assert x.tolist() == [1.0, -5.25, -0.25, 4.0, -np.inf]


def test_attention_of_equal_keys():
    k, v = np.zeros((5, 4)), np.arange(20.0).reshape(5, 4)
    out, lse, _, _ = orc.attend(np.ones((3, 4)), k, v, [0, 1, 5], 0.5)
    assert out[0].tolist() == [0] * 4 and lse[0] == -np.inf and (out[1] == v[0]).all() and (out[2] == v.mean(0)).all() and np.isclose(lse[2], np.log(5))
