"""Pins of the oracle's 4-bit cache: values by hand, and the rules by another road."""
import numpy as np

import oracle as O

R = O.kv_ref


def _block(*head):
    x = np.zeros(32)
    x[:len(head)] = head
    return x


def test_codes_by_hand():
    # the greatest magnitude 6: s = 1; ties go to the even code
    codes, exps = R.to_mxfp4(_block(6, 5, 3.5, 2.5, 1.75, 1.25, 0.75, 0.25, -0.26, -5.01))
    assert exps.tolist() == [127]
    assert codes[:10].tolist() == [7, 6, 6, 4, 4, 2, 2, 0, 9, 15]
    assert R.mxfp4_values(codes, exps)[:10].tolist() == [6, 4, 4, 2, 2, 1, 1, 0, -0.5, -6]


def test_the_power_of_two():
    # 7 still belongs to s = 1 (6, half a step off), the next value to s = 2
    assert R.to_mxfp4(_block(7.0))[1] == 127 and R.to_mxfp4(_block(7.03125))[1] == 128
    assert R.to_mxfp4(_block(3.5))[1] == 126 and R.to_mxfp4(_block(3.515625))[1] == 127
    assert R.to_mxfp4(np.zeros(32))[1] == 2 and R.to_mxfp4(_block(1e-38))[1] == 2
    big = _block(3.3895314e38)
    codes, exps = R.to_mxfp4(big)
    assert exps == 252 and codes[0] == 7 and np.isfinite(R.mxfp4_values(codes, exps)).all()
    for odd in (np.inf, -np.inf, np.nan):
        codes, exps = R.to_mxfp4(np.concatenate([_block(1, odd), _block(1)]))
        assert exps.tolist() == [255, 125]
        assert np.isnan(R.mxfp4_values(codes, exps)[:32]).all()
        assert R.mxfp4_values(codes, exps)[32] == 1


def test_no_value_is_off_by_more_than_half_a_step_of_the_greatest():
    x = np.random.default_rng(1).normal(size=(500, 128)) * 2.0 ** np.linspace(-160, 120, 500)[:, None]
    codes, exps = R.to_mxfp4(x)
    s = 2.0 ** (exps.astype(float) - 127)
    err = np.abs(R.mxfp4_values(codes, exps) - x).reshape(500, 4, 32)
    assert (err <= s[..., None]).all()               # steps up to 2 s, for magnitudes 4 s .. 7 s
    top = np.abs(x).reshape(500, 4, 32).max(-1)
    assert ((top <= 7 * s) & ((top > 3.5 * s) | (exps == 2))).all()


def test_pages_pack_and_unpack():
    rng = np.random.default_rng(2)
    codes = rng.integers(0, 16, size=(3, 2, 16, 64)).astype(np.uint8)
    exps = rng.integers(0, 256, size=(3, 2, 16, 2)).astype(np.uint8)
    b = R.pack_mxfp4(codes, exps)
    assert b.shape == (3, 2, 16 * 34)
    # dim 2 i in the low half of byte i of the row, exponents behind the rows' codes
    assert b[1, 1, 5 * 32 + 3] == codes[1, 1, 5, 6] + 16 * codes[1, 1, 5, 7]
    assert b[1, 1, 16 * 32 + 5 * 2 + 1] == exps[1, 1, 5, 1]
    c, e = R.unpack_mxfp4(b, 16, 64)
    assert np.array_equal(c, codes) and np.array_equal(e, exps)
