"""Edges of the paged context cache on the device (needs an MI355X): arrays used
in place, requests that end while others share their prefix, groups out of order,
scores that are all infinite, quotients next to the middles of e4m3, contexts past
2^20 keys, the ends of the scales' and sizes' ranges."""
import numpy as np
import pytest

import oracle as O
from _kv import Call, R, bf16, parts_of
from test_gpu_kv import Pages, _i32, _paged_layer

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("n,slots", [(3, 40), (3, 5120), (3, 5121), (40, 9000)])
def test_map_advances_lengths_in_place(n, slots):
    """kv_len given as the array of lens, and as that of add, in calls of one launch
    and of two: what separate arrays give."""
    import torch
    print(f"map in place: n={n} slots={slots}", flush=True)
    rng = np.random.default_rng(n + slots)
    for alias in ("lens", "add"):
        a, b = (Pages(16, 4000, n, 90, seed=5) for _ in range(2))
        for s in (a, b):
            s.step([0] * n, [300 + 17 * (i % 40) for i in range(n)])
        lens, add = rng.integers(0, 300, size=n), rng.integers(0, min(slots // n, 400), size=n)
        want = [torch.zeros(m, dtype=torch.int32, device="cuda") for m in (n, slots)]
        a.kv.map(_i32(lens), _i32(add), a.table, a.held, a.pool, a.pool_n, kv_len=want[0],
                 slots=want[1])
        t = dict(lens=_i32(lens), add=_i32(add))
        got = torch.zeros(slots, dtype=torch.int32, device="cuda")
        b.kv.map(t["lens"], t["add"], b.table, b.held, b.pool, b.pool_n, kv_len=t[alias], slots=got)
        assert got.equal(want[1]) and t[alias].equal(want[0])
        assert b.table.equal(a.table) and b.pool_n.equal(a.pool_n)
        assert a.kv.device_errors() == 0 and b.kv.device_errors() == 0
        for s in (a, b):
            s.kv.close()


def test_map_of_two_launches_returns_and_takes():
    """Requests that shrink and end beside ones that grow, with more slots than one
    launch fills."""
    n = 50
    s = Pages(16, 5000, n, 700, seed=6)
    rng = np.random.default_rng(6)
    lens = np.zeros(n, dtype=int)
    for step in range(4):
        add = np.where(rng.random(n) < 0.3, rng.integers(1000, 3000, size=n), rng.integers(0, 20, size=n))
        add[0] = 5200                                         # two launches
        add = np.minimum(add, 700 * 16 - lens)
        cu, kv, _, lost, bad = s.step(lens, add)
        assert cu[-1] > 5120
        lens = np.where(rng.random(n) < 0.4, rng.integers(0, 40, size=n).clip(max=np.array(kv)), kv)
        lens[0] = 100
        lens[rng.integers(1, n)] = 0
    s.kv.close()
