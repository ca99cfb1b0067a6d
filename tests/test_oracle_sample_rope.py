"""Pins of the sampler's and the rotary oracles, and the refusals of their C ABI on the
host, before any GPU work."""
import ctypes

import numpy as np
import pytest

from oracle import rope_ref, sample_ref
from paper_2608_02438_amd import xpress as X

S = sample_ref.sample_row


def test_sample_by_hand():
    l = np.log([0.1, 0.4, 0.2, 0.3])
    assert [S(l, True, u=u)[0] for u in (0.0, 0.0999, 0.1001, 0.499, 0.501, 0.71, 0.999)] == \
        [0, 0, 1, 1, 2, 3, 3]
    assert S(l, False)[0] == 1
    assert S(l, True, k=2)[2] == [1, 3] and S(l, True, p=0.65)[2] == [1, 3]
    assert S(l, True, p=0.75)[2] == [1, 2, 3] and S(l, True, min_p=0.7)[2] == [1, 3]
    # top-p of what top-k left: 0.4 of 0.9 is less than half of it
    assert S(l, True, k=3, p=0.5)[2] == [1, 3]
    y, lp, _ = S(l, True, k=2, u=0.6)
    assert y == 3 and abs(lp - np.log(3 / 7)) < 1e-12
    # T = 0.5 squares the weights
    assert abs(S(l, True, T=0.5, u=0.9)[1] - np.log(0.09 / 0.3)) < 1e-12


def test_sample_ties_and_rows_with_few_tokens():
    z = np.zeros(4)
    assert S(z, True, u=0.25)[0] == 1                    # strictly more than u of the mass
    assert S(z, True, k=2)[2] == [0, 1, 2, 3]            # ties with the k-th stay
    assert S(z, True, p=0.5)[2] == [0, 1] and S(z, True, p=0.51)[2] == [0, 1, 2]
    bad = np.array([-np.inf, np.nan, -np.inf])
    assert S(bad, True)[0] == -1 and S(bad, False)[0] == -1
    assert S([-np.inf, 3, np.nan], True, u=0.99)[0] == 1
    assert S([np.inf, 0, np.inf], True, u=0.6)[0] == 2
    assert S(z, True, u=1.0)[0] == 3 and S(z, True, u=np.nan)[0] == 3


def test_axes_by_hand():
    assert rope_ref.axis_of([2, 1, 1], False) == [0, 0, 1, 2]
    assert rope_ref.axis_of([4, 2, 2], True) == [0, 1, 2, 0, 1, 2, 0, 0]
    assert rope_ref.axis_of([3, 3], True) == [0, 1, 0, 1, 0, 1]


def test_rope_rotates_planes():
    x = np.zeros((1, 1, 6))
    x[0, 0, 0] = x[0, 0, 5] = 1
    y, _ = rope_ref.rope(x, [[np.pi / 2]], [2], 1.0)     # theta 1: every pair the same angle
    assert np.allclose(y[0, 0], [0, 0, 1, 0, 0, 1])
    rng = np.random.default_rng(0)
    x = rng.normal(size=(4, 2, 16))
    pos = rng.integers(-50, 50, size=(2, 4))
    a, _ = rope_ref.rope(x, pos, [5, 3], 1e4)
    b, _ = rope_ref.rope(a, 7 - pos, [5, 3], 1e4)        # angles add
    assert np.allclose(b, rope_ref.rope(x, 7 + 0 * pos, [5, 3], 1e4)[0])
    n, _ = rope_ref.rope(3 * x, pos, [5, 3], 1e4, g=np.ones(16), eps=0)
    assert np.allclose((n * n).mean(-1), 1)


def _shape(**kw):
    s = dict(head_dim=128, rot_dim=128, axes=1, sections=(64, 0, 0, 0), interleaved=0,
             dtype=X.XP_BF16, theta=1e6, eps=1e-6)
    s.update(kw)
    s["sections"] = (ctypes.c_int32 * 4)(*s["sections"])
    return X._RopeShape(**s)


P = 0x10000                                              # never dereferenced


def _rope(shape=None, **kw):
    a = dict(tokens=1, pos=P, pos_ld=1, q=P, q_ld=4096, nh=32, gq=None, qo=P, qo_ld=4096, k=P,
             k_ld=1024, nkv=8, gk=None, ko=P, ko_ld=1024)
    a.update(kw)
    s = _shape() if shape is None else shape
    return X.load_library().xp_rope(None if s is False else ctypes.byref(s), *a.values(), None)


@pytest.mark.parametrize("change", [
    dict(head_dim=0), dict(rot_dim=8), dict(rot_dim=136), dict(rot_dim=24), dict(axes=0), dict(axes=5),
    dict(interleaved=2), dict(dtype=X.XP_E4M3), dict(theta=0.5), dict(theta=float("nan")),
    dict(theta=float("inf")), dict(eps=-1.0), dict(eps=float("nan")), dict(sections=(63, 0, 0, 0)),
    dict(sections=(-1, 65, 0, 0), axes=2), dict(sections=(65, -1, 0, 0), axes=2),
    dict(axes=2, sections=(31, 33, 0, 0), interleaved=1),    # pair 1 + 2 * 32 is none
    dict(axes=3, sections=(20, 22, 22, 0), interleaved=1)])
def test_rope_rejects_shapes(change):
    assert _rope(_shape(**change)) == X.XP_EINVAL


@pytest.mark.parametrize("kw", [
    dict(tokens=-1), dict(pos=None), dict(pos_ld=0), dict(q=None), dict(qo=None), dict(q_ld=4095),
    dict(q_ld=4100), dict(q=P + 8), dict(qo=P + 4, q=P + 16), dict(gq=P + 2), dict(k=None), dict(ko=None),
    dict(k_ld=1000), dict(ko_ld=1016), dict(nh=-1), dict(nh=0, nkv=0), dict(nkv=70000),
    dict(qo_ld=8192)])                                   # in place with another distance
def test_rope_rejects_arguments(kw):
    assert _rope(**kw) == X.XP_EINVAL


def test_rope_unbuilt_shapes_and_empty_calls():
    assert _rope(False) == X.XP_EINVAL
    assert _rope(_shape(head_dim=96, rot_dim=96, sections=(48, 0, 0, 0))) == X.XP_EUNSUPPORTED
    assert _rope(tokens=0, pos_ld=0) == X.XP_OK


@pytest.mark.parametrize("V,rows,status", [
    (0, 1, X.XP_EINVAL), (-5, 1, X.XP_EINVAL), (10, 0, X.XP_EINVAL), (10, 65537, X.XP_EINVAL),
    ((1 << 18) + 1, 1, X.XP_EUNSUPPORTED)])
def test_sampler_rejects_sizes(V, rows, status):
    L = X.load_library()
    h = ctypes.c_void_p(0)
    assert L.xp_sampler_create(V, rows, ctypes.byref(h)) == status
    assert not h.value and L.xp_sampler_last_error(None)
    assert L.xp_sampler_create(10, 1, None) == X.XP_EINVAL


def test_null_samplers_are_rejected():
    L = X.load_library()
    assert L.xp_sample(None, 1, X.XP_F32, P, 10, None, None, None, None, None, None, P, None,
                       None) == X.XP_EINVAL
    assert L.xp_sampler_device_errors(None, None, None) == X.XP_EINVAL
    assert L.xp_kv_read(None, 1, P, P, P, None, None, P, 8, P, 8, None) == X.XP_EINVAL
    L.xp_sampler_destroy(None)
