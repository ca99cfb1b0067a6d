"""Pins of the paged-cache oracle: cases with answers by hand or by another road."""
import numpy as np
import pytest

import oracle as O

R = O.kv_ref


def test_pages_by_hand():
    # pages of 4: request 0 grows from 3 to 9 tokens (two more), 1 shrinks from 9
    # to 4 (two back), 2 stays
    p = R.Pool(4, [10, 11], [[0], [1, 2, 3], [4]])
    cu, kv, slots, lost, bad = p.step([3, 4, 1], [6, 0, 2], 16)
    assert p.tables == [[0, 2, 3], [1], [4]] and p.free == [10, 11]
    assert cu == [0, 6, 6, 8] and kv == [9, 4, 3] and not lost and not bad
    assert slots == [3, 8, 9, 10, 11, 12, 17, 18]
    # taking back what was just given restores stack and order
    p.step([3, 4, 1], [0, 5, 2], 16)
    assert p.tables == [[0], [1, 2, 3], [4]] and p.free == [10, 11]


def test_first_come_first_served():
    p = R.Pool(16, [7, 8], [[], [], [1], []])
    cu, kv, slots, lost, _ = p.step([0, 0, 5, 0], [16, 40, 3, 1], 16)
    assert lost == [1, 3] and p.tables == [[8], [], [1], []] and p.free == [7]
    assert kv == [16, 0, 8, 0] and cu == [0, 16, 56, 59, 60]
    assert slots[16:56] == [-1] * 40 and slots[56:] == [21, 22, 23, -1]


def test_e4m3_rounding():
    v = R.e4m3_values()
    assert v[0x7e] == 448 and v[0x08] == 2.0 ** -6 and v[0x01] == 2.0 ** -9 and np.isnan(v[0x7f])
    ok = ~np.isnan(v)
    assert np.array_equal(R.to_e4m3(v[ok]), v[ok])
    # ties: 17 and 19 lie halfway between 16, 18 and 20 (step 2): to even codes
    assert R.to_e4m3([17.0, 19.0, 1e9, -np.inf, 2.0 ** -10, 3 * 2.0 ** -10]).tolist() == \
        [16.0, 20.0, 448.0, -448.0, 0.0, 2.0 ** -8]
    import torch
    x = np.random.default_rng(0).normal(size=4096).astype(np.float32) * 60
    want = torch.from_numpy(x).to(torch.float8_e4m3fn).float().numpy()
    assert np.array_equal(R.to_e4m3(x), want)


def test_visible_by_hand():
    see = R.visible(6, 2, True, 2, 1)               # positions 4 and 5
    assert see.astype(int).tolist() == [[1, 0, 0, 1, 1, 0], [1, 0, 0, 0, 1, 1]]
    assert R.visible(3, 2, False, 0, 5).all()       # without a window sinks do nothing
    assert not R.visible(1, 3, True, 0, 0)[:2].any()   # positions -2 and -1 see nothing


@pytest.mark.parametrize("causal,window,sinks", [(True, 0, 0), (False, 0, 0), (True, 3, 2)])
def test_attend_is_a_masked_softmax(causal, window, sinks):
    import torch
    rng = np.random.default_rng(3)
    q, k, v = rng.normal(size=(5, 4, 8)), rng.normal(size=(9, 2, 8)), rng.normal(size=(9, 2, 8))
    out, lse, spread, score = R.attend(q, k, v, causal, window, sinks, scale=0.7)
    s = torch.einsum("mhd,nhd->hmn", *(torch.from_numpy(x) for x in (q, k.repeat(2, 1)))) * 0.7
    s = s.masked_fill(~torch.from_numpy(R.visible(9, 5, causal, window, sinks)), -torch.inf)
    o = torch.einsum("hmn,nhd->mhd", s.softmax(-1), torch.from_numpy(v.repeat(2, 1)))
    assert np.abs(out - o.numpy()).max() < 1e-12
    assert np.abs(lse.T - s.logsumexp(-1).numpy()).max() < 1e-12
    assert (spread >= np.abs(out) - 1e-12).all()
    top = s.masked_fill(torch.isinf(s), 0).abs().amax(-1).numpy()
    assert (score.T >= top - 1e-12).all()


def test_one_visible_key_gives_its_value():
    v = np.arange(12.0).reshape(3, 1, 4)
    out, lse, _, _ = R.attend(np.ones((1, 2, 4)), np.ones((3, 1, 4)), v, True, 1, 0)
    assert np.array_equal(out[0], [v[2, 0]] * 2) and np.allclose(lse, 2.0)


def test_gather_follows_the_table():
    cache = np.arange(4 * 1 * 2 * 1).reshape(4, 1, 2, 1)
    assert R.gather(cache, [3, 0, 2], 5).ravel().tolist() == [6, 7, 0, 1, 4]
