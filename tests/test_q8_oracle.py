"""The 64-bit oracle of the 8-bit cache against what its definition says by hand."""
import numpy as np

import q8_oracle as Q


def test_table_is_e4m3():
    assert Q.TABLE[0] == 0 and Q.TABLE[1] == 2.0 ** -9 and Q.TABLE[7] == 7 * 2.0 ** -9 and Q.TABLE[8] == 2.0 ** -6
    assert Q.TABLE[126] == 448 and Q.TABLE[0x38] == 1 and Q.TABLE[0xB8] == -1 and np.isnan(Q.TABLE[[127, 255]]).all()
    assert (np.diff(Q.TABLE[:127]) > 0).all()


def row(*x):
    return np.array(x + (0.0,) * (16 - len(x)), np.float32)


def test_exponents_and_roundings():
    for most, e in [(448.0, 0), (448.5, 1), (224.0, -1), (225.0, 0), (1.0, -8), (1.75, -8), (1.7501, -7), (0.0, -110), (1e-38, -110), (3e38, 119)]:
        assert Q.quantise(row(most))[1] == e, most
    byte, e = Q.quantise(row(448.0, 17.0, 19.0, 18.0, -17.0, 2.0 ** -10, 3 * 2.0 ** -10, 2.0 ** -10 * 1.001))
    assert e == 0
    # ties to even: 17 lies between 16 and 18, 19 between 18 and 20; halves of the least subnormal
    assert Q.values(byte, e)[:8].tolist() == [448, 16, 20, 18, -16, 0, 2.0 ** -8, 2.0 ** -9]


def test_what_is_not_finite_is_nan_and_leaves_the_power_alone():
    byte, e = Q.quantise(row(np.inf, -np.inf, np.nan, 3.0))
    assert np.isnan(Q.values(byte, e)[:3]).all() and Q.values(byte, e)[3] == 3 and e == -7
    top = np.float32(3.4e38)
    byte, e = Q.quantise(row(top, -top, 1.0))
    assert Q.values(byte, e)[:2].tolist() == [448 * 2.0 ** 119, -448 * 2.0 ** 119]


def test_error_and_reading_back_what_was_read():
    rng = np.random.default_rng(3)
    x = (rng.standard_normal((500, 64)) * np.exp2(rng.integers(-30, 30, (500, 1)))).astype(np.float32)
    byte, e = Q.quantise(x)
    y = Q.values(byte, e)
    assert (np.abs(y - x) <= np.maximum(2.0 ** -4 * np.abs(x), np.ldexp(2.0 ** -10, e)[:, None])).all()
    byte2, e2 = Q.quantise(y)
    assert np.array_equal(Q.values(byte2, e2), y)


def test_attention_of_one_key_and_of_equal_keys():
    rng = np.random.default_rng(4)
    q, v = rng.standard_normal((3, 4, 16)), rng.standard_normal((8, 2, 16))
    out, size, _ = Q.attend(q, np.zeros((8, 2, 16)), v, 5, 0.25)
    for i in range(3):
        for h in range(4):
            assert np.allclose(out[i, h], v[:6 + i, h // 2].mean(0)) and np.allclose(size[i, h], np.abs(v[:6 + i, h // 2]).mean(0))
    out, _, _ = Q.attend(q[:1], rng.standard_normal((1, 2, 16)), v[:1], 0, 0.25)
    assert np.allclose(out[0], np.repeat(v[0], 2, 0))
