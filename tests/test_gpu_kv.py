"""The paged context cache on the device against the fp64 oracle (needs an
MI355X): pages and slots, writes, attention over the pages with windows, first
keys that stay and shared prefixes, at the sizes, masks, orders and values where
they can go wrong; refusals; captured calls; and the calls together as a serving
loop makes them."""
import ctypes

import numpy as np
import pytest

import oracle as O
from _kv import Call, R, bf16, parts_of

pytestmark = pytest.mark.gpu


def _i32(x):
    import torch
    return torch.tensor(np.asarray(x, dtype=np.int32), device="cuda")


# ---------------------------------------------------------------------------
# pages and slots
# ---------------------------------------------------------------------------
class Pages:
    """A device pool beside the oracle's."""

    def __init__(self, P, n_pages, n, width, max_len=None, seed=0):
        import torch
        from paper_2608_02438_amd.xpress import PagedKV
        free = list(np.random.default_rng(seed).permutation(n_pages))
        self.P, self.n, self.width, self.n_pages = P, n, width, n_pages
        self.max_pages = min(width, R.pages_of(max_len or width * P, P))
        self.kv = PagedKV(1, 1, P, n_pages, max_batch=max(n, 1), max_tokens=64,
                          max_len=max_len or width * P)
        self.ref = R.Pool(P, free, [[] for _ in range(n)])
        self.table = torch.full((n, width), -1, dtype=torch.int32, device="cuda")
        self.held, self.pool, self.pool_n = _i32([0] * n), _i32(free), _i32([n_pages])

    def step(self, lens, add, slots=True, pad=5):
        import torch
        want = self.ref.step(list(lens), list(add), self.max_pages)
        cu, kv_len, w, lost, bad = want
        sl = torch.full((max(cu[-1] + pad, 1),), 77, dtype=torch.int32, device="cuda") if slots \
            else None
        c, k = torch.full((self.n + 1,), 99, dtype=torch.int32, device="cuda"), _i32([99] * self.n)
        self.kv.map(_i32(lens), _i32(add), self.table, self.held, self.pool, self.pool_n, cu=c,
                    kv_len=k, slots=sl)
        assert c.tolist() == cu and k.tolist() == kv_len
        if slots:
            assert sl.tolist() == w + [-1] * (sl.numel() - len(w))
        assert self.held.tolist() == [len(t) for t in self.ref.tables]
        assert self.table.tolist() == [t + [-1] * (self.width - len(t)) for t in self.ref.tables]
        assert self.pool_n.item() == len(self.ref.free)
        assert self.pool[:len(self.ref.free)].tolist() == [int(x) for x in self.ref.free]
        from paper_2608_02438_amd import xpress as X
        assert self.kv.device_errors() == (X.XP_DEVERR_POOL if lost else 0) | \
            (X.XP_DEVERR_LENGTH if bad else 0)
        return want


@pytest.mark.parametrize("P,n,width,add_hi,short", [
    (16, 1, 9, 40, False), (16, 7, 30, 90, False), (256, 5, 3, 300, False),
    (32, 65, 20, 60, True), (16, 300, 12, 50, True), (64, 1500, 4, 70, False),
    (16, 4096, 3, 20, True)])
def test_map_over_steps(P, n, width, add_hi, short):
    print(f"map: P={P} n={n} width={width}", flush=True)
    rng = np.random.default_rng(P + n)
    cap = width * P
    s = Pages(P, max(n * width // (3 if short else 1), 1), n, width, seed=n)
    lens = np.zeros(n, dtype=int)
    for step in range(6):
        add = np.minimum(rng.integers(0, add_hi + 1, size=n), cap - lens)
        cu, kv, _, lost, _ = s.step(lens, add)
        kept = np.array(kv) - np.floor(rng.random(n) * (np.array(kv) - lens + 1)).astype(int)
        lens = np.where(rng.random(n) < 0.15, 0, kept)      # some requests end
        if step % 2:
            s.step(lens, np.zeros(n, dtype=int), slots=False)
    s.kv.close()


def test_map_prompts_take_the_large_path():
    s = Pages(16, 9000, 40, 1300, seed=1)
    lens = [0] * 20 + [37] * 20
    s.step([0] * 40, [0] * 20 + [37] * 20)
    s.step(lens, [20000, 1, 0, 16, 17, 9999, 500] + [600] * 13 + [1] * 20)
    s.step([0] * 40, [0] * 40)
    assert sorted(s.ref.free) == list(range(9000))
    s.kv.close()


def test_map_leaves_bad_requests_alone():
    from paper_2608_02438_amd import xpress as X
    s = Pages(16, 50, 6, 8, max_len=100, seed=2)           # 7 pages each at most
    s.step([0, 0, 0, 0, 0, 0], [20, 20, 20, 20, 20, 20])
    s.step([-1, 20, 2 ** 31 - 1, 20, 113, 20], [5, -3, 2 ** 31 - 1, 92, 0, 10])
    # a page count that cannot be
    s.held[1] = 9
    before = s.table.clone()
    s.kv.map(_i32([20] * 6), _i32([0] * 6), s.table, s.held, s.pool, s.pool_n)
    assert s.kv.device_errors() == X.XP_DEVERR_LENGTH
    assert s.table[1].equal(before[1]) and s.held[1].item() == 9
    s.kv.close()


def test_map_slots_beyond_the_buffer_and_bad_pages():
    import torch
    from paper_2608_02438_amd import xpress as X
    s = Pages(16, 50, 3, 8, seed=3)
    s.step([0, 0, 0], [20, 20, 20])
    sl = torch.zeros(4, dtype=torch.int32, device="cuda")
    s.kv.map(_i32([20] * 3), _i32([2, 2, 2]), s.table, s.held, s.pool, s.pool_n, slots=sl)
    assert s.kv.device_errors() == X.XP_DEVERR_SLOT and (sl >= 0).all()
    s.table[0, 1] = 5000                                     # no such page
    s.kv.map(_i32([20] * 3), _i32([1, 1, 1]), s.table, s.held, s.pool, s.pool_n, slots=sl)
    assert s.kv.device_errors() == X.XP_DEVERR_PAGE
    assert sl[0] == -1 and (sl[1:3] >= 0).all() and sl[3] == -1
    s.pool_n[0] = 51
    s.kv.map(_i32([20] * 3), _i32([1, 1, 1]), s.table, s.held, s.pool, s.pool_n)
    assert s.kv.device_errors() == X.XP_DEVERR_POOL
    s.kv.close()


# ---------------------------------------------------------------------------
# the write
# ---------------------------------------------------------------------------
@pytest.mark.parametrize("cache,hd,n_kv,P,tokens", [
    ("bf16", 128, 8, 16, 33), ("bf16", 64, 1, 256, 1), ("bf16", 64, 5, 32, 700),
    ("e4m3", 128, 8, 64, 65), ("e4m3", 64, 3, 16, 259), ("e4m3", 128, 1, 128, 1)])
def test_write(cache, hd, n_kv, P, tokens):
    import torch
    from paper_2608_02438_amd import xpress as X
    print(f"write: {cache} hd={hd} n_kv={n_kv} P={P} tokens={tokens}", flush=True)
    rng = np.random.default_rng(tokens)
    n_pages = R.pages_of(tokens, P) + 2
    dt = torch.bfloat16 if cache == "bf16" else torch.float8_e4m3fn
    kv = X.PagedKV(n_kv, n_kv, P, n_pages, 1, tokens, P, head_dim=hd, cache_dtype=dt)
    fused = bf16(rng.normal(size=(tokens, 2 * n_kv * hd + 24)) * 30)
    fused[0, :6] = [np.inf, -np.inf, np.nan, 1e30, -0.0, 1e-38]
    dev = torch.tensor(fused).to(torch.bfloat16).cuda()
    fused = dev.double().cpu().numpy()                        # what the device holds
    cut = lambda x, o: x[:, o:o + n_kv * hd].reshape(tokens, n_kv, hd)  # noqa: E731
    view = lambda o: dev[:, o:o + n_kv * hd].view(tokens, n_kv, hd)     # noqa: E731
    slots = rng.permutation(n_pages * P)[:tokens].astype(np.int32)
    if tokens > 2:
        slots[1::7] = -1
    old = [torch.tensor(R.to_e4m3(rng.normal(size=kv.cache_shape) * 50)).to(dt).cuda()
           for _ in range(2)]
    want = [o.double().cpu().numpy() for o in old]
    scales = [None, None] if cache == "bf16" else \
        [rng.uniform(0.05, 0.4, size=n_kv).astype(np.float32) for _ in range(2)]
    ds = [None if s is None else torch.tensor(s).cuda() for s in scales]
    kv.write(view(0), view(n_kv * hd + 8), _i32(slots), *old, k_scale=ds[0], v_scale=ds[1])
    for w, off, s in zip(want, (0, n_kv * hd + 8), scales):
        with np.errstate(invalid="ignore", over="ignore"):
            x = cut(fused, off)
            x = x if s is None else R.to_e4m3(x / s.astype(np.float64)[:, None])
        for t, sl in enumerate(slots):
            if sl >= 0:
                w[sl // P, :, sl % P] = x[t]
    for got, w in zip(old, want):
        np.testing.assert_array_equal(got.double().cpu().numpy(), w)
    # slots outside the cache: skipped and reported
    slots[0] = n_pages * P
    if tokens > 2:
        slots[2] = -2
    kv.write(view(0), view(n_kv * hd + 8), _i32(slots), *old, k_scale=ds[0], v_scale=ds[1])
    assert kv.device_errors() == X.XP_DEVERR_SLOT
    for got, w in zip(old, want):
        np.testing.assert_array_equal(got.double().cpu().numpy(), w)
    kv.close()


def test_write_rounds_every_quotient_once():
    """Quotients next to the middles between e4m3 values, where rounding to fp32 first
    would move them onto the middle."""
    import torch
    from paper_2608_02438_amd import xpress as X
    rng = np.random.default_rng(5)
    tokens, hd, P = 4096, 64, 16
    grid = R.e4m3_values()[8:127]
    mid = (grid[1:] + grid[:-1]) / 2
    s = np.float32(rng.uniform(0.3, 0.9))
    x = bf16(rng.choice(mid, size=(tokens, 1, hd)) * s * rng.choice([-1, 1], size=(tokens, 1, hd)))
    kv = X.PagedKV(1, 1, P, tokens // P, 1, tokens, P, head_dim=hd, cache_dtype=torch.float8_e4m3fn)
    c = [torch.zeros(kv.cache_shape, device="cuda").to(torch.float8_e4m3fn) for _ in range(2)]
    d, sc = torch.tensor(x).to(torch.bfloat16).cuda(), torch.tensor([s]).cuda()
    kv.write(d, d, _i32(np.arange(tokens)), *c, k_scale=sc, v_scale=sc)
    got = c[0].double().cpu().numpy().reshape(tokens, 1, hd)
    np.testing.assert_array_equal(got, R.to_e4m3(x / np.float64(s)))
    kv.close()


# ---------------------------------------------------------------------------
# attention
# ---------------------------------------------------------------------------
# (kv, ql, kwargs of Call)
LENGTHS = {
    "one": ([1], [1], {}),
    "token": ([1, 63, 64, 65, 127, 128, 129, 300], [1] * 8, dict(heads=8, n_kv=2)),
    "block": ([16, 80, 17, 400], [16] * 4, dict(heads=8, n_kv=2)),
    "block32": ([32, 200, 95], [32] * 3, dict(heads=4, n_kv=1)),
    "ragged": ([5, 0, 70, 33, 1, 200], [5, 0, 3, 33, 0, 70], dict(heads=4, n_kv=2)),
    "prompt": ([150, 1, 90], [150, 1, 37], dict(heads=4, n_kv=2)),
    "short": ([3, 0, 10], [7, 2, 10], dict(heads=2, n_kv=2)),      # more tokens than keys
    "odd group": ([70, 100], [9, 20], dict(heads=7, n_kv=1)),
    "wide group": ([130], [3], dict(heads=64, n_kv=1)),
    "many": ([20 + i % 90 for i in range(130)], [1 + i % 2 for i in range(130)], {}),
}
MASKS = [dict(causal=True), dict(causal=False), dict(causal=True, window=19, sinks=3),
         dict(causal=True, window=64), dict(causal=False, window=30, sinks=70),
         dict(causal=True, window=1), dict(causal=True, window=1 << 22, sinks=1 << 22)]


@pytest.mark.parametrize("name", LENGTHS)
@pytest.mark.parametrize("hd,cache,P", [(128, "bf16", 16), (64, "bf16", 64), (128, "e4m3", 32),
                                        (64, "e4m3", 256), (128, "bf16", 128)])
def test_attend(name, hd, cache, P):
    import torch
    kv_len, ql, kw = LENGTHS[name]
    c = Call(len(name) + hd + P, kv_len, ql, hd=hd, cache=cache, P=P, **kw)
    kv = c.device()
    masks = MASKS if len(kv_len) < 20 else MASKS[:3]
    for m in masks:
        print(f"attend: {name} hd={hd} {cache} P={P} {m}", flush=True)
        out = torch.full((c.total, c.heads, hd), float("nan"), dtype=torch.bfloat16, device="cuda")
        lse = torch.full((c.total, c.heads), float("nan"), device="cuda")
        c.run(kv, out=out, lse=lse, **m)
        c.check(out, lse, parts=parts_of(c.rows(), c.cache), **m)
        assert kv.device_errors() == 0
    kv.close()


@pytest.mark.parametrize("rows", [32, 64, 128, 256])
def test_attend_max_q_costs_time_only(rows):
    """Every size of row tile gives every length's result."""
    c = Call(rows, [40, 300, 71], [40, 2, 71], heads=4, n_kv=2, P=32)
    kv = c.device(max_tokens=512)
    m = dict(causal=True, window=50, sinks=10)
    print(f"attend: tiles of {rows} rows", flush=True)
    c.check(c.run(kv, max_q=rows // 2, **m), parts=parts_of(rows), **m)
    kv.close()


@pytest.mark.parametrize("hd,cache", [(128, "bf16"), (64, "e4m3")])
def test_attend_more_sequences_than_lanes(hd, cache):
    """Prompts, blocks and single tokens of more sequences than a wave's lanes, and
    the same ones in calls of few."""
    ql = [(150, 1, 16, 33, 0, 2)[i % 6] for i in range(70)]
    kv_len = [x + (0, 200, 90, 7, 30, 1)[i % 5] for i, x in enumerate(ql)]
    c = Call(44, kv_len, ql, heads=4, n_kv=2, hd=hd, cache=cache)
    kv = c.device()
    for m in (dict(causal=True), dict(causal=False, window=70, sinks=5)):
        print(f"many sequences: hd={hd} {cache} {m}", flush=True)
        out = c.run(kv, **m)
        assert kv.device_errors() == 0
        c.check(out, parts=1, **m)
        few = c.run(kv, **m).fill_(7)
        for b in range(0, 70, 14):
            t = slice(c.cu[b], c.cu[b + 14])
            kv.attend(c.dq[t], c.dk, c.dv, c.dtable[b:b + 14], c.dkv[b:b + 14],
                      cu_q=(c.dcu[b:b + 15] - c.dcu[b]).contiguous(), max_q=150, k_scale=c.dks,
                      v_scale=c.dvs, out=few[t], **m)
        c.check(few, parts=1, **m)
    kv.close()


def test_attend_takes_any_upper_bound_of_the_tokens():
    """A bound above the handle's own (a configuration's longest prompt)."""
    c = Call(43, [90, 30], [20, 7], heads=4, n_kv=2)
    kv = c.device()
    assert c.run(kv, max_q=100000).equal(c.run(kv, max_q=c.total))
    kv.close()


def test_attend_uniform_lengths_without_cu_q():
    c = Call(11, [40, 300, 71, 16], [16] * 4, heads=4, n_kv=2)
    kv = c.device()
    a = c.run(kv)
    b = c.run(kv, cu_q=None, max_q=None)
    assert a.equal(b)
    c.check(b, causal=True, parts=2)
    kv.close()


def test_attend_scale_strides_and_untouched_rows():
    import torch
    c = Call(12, [70, 33], [5, 4], heads=4, n_kv=2, hd=64)
    kv = c.device(max_tokens=32)
    # rows of a fused projection, four tokens more than the sequences have
    wide = torch.zeros((13, 4 * 64 + 136), dtype=torch.bfloat16, device="cuda")
    q = wide[:, 8:8 + 256].unflatten(1, (4, 64))
    q[:9] = c.dq
    out = torch.full((13, 4 * 64 + 64), 3.0, dtype=torch.bfloat16, device="cuda")
    o = out[:, 64:].unflatten(1, (4, 64))
    lse = torch.full((13, 4), 5.0, device="cuda")
    c.run(kv, q=q, out=o, lse=lse, scale=0.3)
    c.check(o[:9], lse[:9], causal=True, parts=2, scale=0.3)
    assert (out[:, :64] == 3).all() and (o[9:] == 3).all() and (lse[9:] == 5).all()
    kv.close()


def _poison(c, hidden_keys):
    """NaN and infinities at the given (request, key)s, K and V."""
    for n, (b, key) in enumerate(hidden_keys):
        bad = [np.nan, np.inf, -np.inf][n % 3]
        page, row = c.table[b, key // c.P], key % c.P
        c.k[page, :, row] = bad if c.cache == "bf16" else np.nan
        c.v[page, :, row] = bad if c.cache == "bf16" else np.nan


@pytest.mark.parametrize("cache,hd", [("bf16", 128), ("e4m3", 64), ("bf16", 64), ("e4m3", 128)])
@pytest.mark.parametrize("ql", [[1, 1], [5, 16], [40, 90], [90, 70]])
def test_values_that_no_row_or_not_every_row_sees(cache, hd, ql):
    """Rows behind the last key of a page, in front of the window, and the later
    tokens of a causal block hold NaN and infinities: whoever does not see them is
    not touched, whoever does gets what the formula gives."""
    import torch
    kv_len = [150, 203]
    c = Call(20 + sum(ql), kv_len, ql, heads=4, n_kv=2, hd=hd, cache=cache, P=64)
    W = 100
    unseen = [(b, j) for b in range(2) for j in range(5, kv_len[b] - ql[b] - W + 1)]
    late = [(0, kv_len[0] - 1), (1, kv_len[1] - 2)]          # seen by the last tokens only
    assert ql == [90, 70] or unseen
    _poison(c, unseen + late)
    for b in range(2):                                        # and behind the last key
        page = c.table[b, (kv_len[b] - 1) // 64]
        c.k[page, :, kv_len[b] % 64:] = np.nan
        c.v[page, :, kv_len[b] % 64:] = np.nan
    kv = c.device()
    print(f"masked values: {cache} hd={hd} ql={ql}", flush=True)
    out = c.run(kv, window=W, sinks=5).double().cpu().numpy()
    want = c.oracle(causal=True, window=W, sinks=5, parts=parts_of(c.rows(), c.cache))
    for b in want:
        o, _, eb, _ = want[b]
        m = ql[b]
        sees_late = np.arange(m) >= (m - 1 if b == 0 else m - 2)
        got = out[c.cu[b]:c.cu[b + 1]]
        assert not np.isfinite(got[sees_late]).any()
        assert np.isfinite(got[~sees_late]).all()
        assert (np.abs(got - o) <= eb)[~sees_late].all()
    kv.close()


@pytest.mark.parametrize("cache", ["bf16", "e4m3"])
@pytest.mark.parametrize("ql", [[4, 7], [60, 90]])
def test_infinite_values_of_later_tokens(cache, ql):
    """V alone holds an infinity (NaN in 8 bits) at a key that later tokens see: the
    earlier ones are the oracle's, the later ones infinite or NaN in that column only."""
    c = Call(31, [100, 130], ql, heads=2, n_kv=1, hd=64, cache=cache, P=16)
    for b, n in enumerate((100, 130)):
        c.v[c.table[b, (n - 2) // 16], 0, (n - 2) % 16, 7] = np.inf if cache == "bf16" else np.nan
    kv = c.device()
    out = c.run(kv).double().cpu().numpy()
    with np.errstate(invalid="ignore"):
        want = c.oracle(causal=True, parts=parts_of(c.rows(), c.cache))
    for b in want:
        o, _, eb, _ = want[b]
        got = out[c.cu[b]:c.cu[b + 1]]
        ok = np.isfinite(o)
        assert ok[:-2].all() and not ok[-2:, :, 7].any() and ok[-2:, :, :7].all()
        assert (np.abs(got - o) <= eb)[ok].all()
        if cache == "bf16":
            assert (got[~ok] == o[~ok]).all()
        else:
            assert np.isnan(got[~ok]).all()
    kv.close()


def test_equal_bits_every_time_and_on_another_stream():
    import torch
    c = Call(41, [3000, 40, 700, 0, 5], [1, 9, 16, 0, 5], heads=8, n_kv=2, P=16)
    kv = c.device()
    a = c.run(kv, window=500, sinks=20)
    s = torch.cuda.Stream()
    torch.cuda.synchronize()
    b = c.run(kv, window=500, sinks=20, stream=s, out=torch.empty_like(a))
    s.synchronize()
    assert a.equal(b)
    c.check(a, causal=True, window=500, sinks=20, parts=parts_of(c.rows(), c.cache))
    kv.close()


def test_two_handles_at_once():
    """Calls of two handles on two streams, and two captured graphs of one handle
    replayed in turn."""
    import torch
    calls = [Call(45, [700, 90, 300], [3, 16, 40], heads=8, n_kv=2),
             Call(46, [1, 2500], [1, 2], heads=4, n_kv=2, cache="e4m3", P=64)]
    handles = [c.device() for c in calls]
    alone = [c.run(kv) for c, kv in zip(calls, handles)]
    streams = [torch.cuda.Stream() for _ in calls]
    torch.cuda.synchronize()
    outs = [[], []]
    for _ in range(10):
        for i, (c, kv) in enumerate(zip(calls, handles)):
            with torch.cuda.stream(streams[i]):
                outs[i].append(c.run(kv))
    torch.cuda.synchronize()
    for i in range(2):
        assert all(o.equal(alone[i]) for o in outs[i])
    c, kv = calls[0], handles[0]
    masks = [dict(causal=True), dict(causal=False, window=50)]
    eager = [c.run(kv, **m) for m in masks]
    graphs, res = [torch.cuda.CUDAGraph() for _ in masks], [torch.empty_like(c.dq) for _ in masks]
    for g, m, o in zip(graphs, masks, res):
        torch.cuda.synchronize()
        with torch.cuda.graph(g):
            c.run(kv, out=o, **m)
    for k in (0, 1, 1, 0, 1):
        res[k].zero_()
        graphs[k].replay()
        torch.cuda.synchronize()
        assert res[k].equal(eager[k])
    for kv in handles:
        kv.close()


@pytest.mark.parametrize("shared", [False, True])
def test_captured_calls_replay_with_new_lengths(shared):
    import torch
    c = Call(42, [500, 140, 700, 90], [3, 3, 3, 3], heads=8, n_kv=2, P=16,
             groups=[(0, 2, 128), (2, 4, 64)] if shared else ())
    kv = c.device(shared=shared)
    out = torch.empty_like(c.dq)
    c.run(kv, shared=shared, out=out)
    g = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(g):
        c.run(kv, shared=shared, out=out)
    for lens in ([500, 140, 700, 90], [480, 133, 650, 70], [500, 140, 90, 80]):
        c.dkv.copy_(_i32(lens))
        c.kv = lens
        out.zero_()
        g.replay()
        torch.cuda.synchronize()
        c.check(out, causal=True, parts=2)
        eager = c.run(kv, shared=shared)
        assert eager.equal(out)
    kv.close()


def test_bad_pages_and_lengths_are_reported_and_read_nothing_else():
    import torch
    from paper_2608_02438_amd import xpress as X
    c = Call(43, [100, 60], [2, 2], heads=4, n_kv=2, P=16)
    kv = c.device()
    good = c.run(kv)
    c.dtable[0, 3] = 10 ** 9                                  # replaced by page 0
    out = c.run(kv)
    assert kv.device_errors() == X.XP_DEVERR_PAGE
    assert out[2:].equal(good[2:]) and torch.isfinite(out.float()).all()
    c.dtable[0, 3] = -1                                       # outside the window: not read
    a = c.run(kv, window=20)
    assert kv.device_errors() == 0
    c.check(a, causal=True, window=20, parts=2)
    c.dkv[0] = 10 ** 6
    c.run(kv, window=20)
    assert kv.device_errors() & X.XP_DEVERR_LENGTH
    c.dkv[0] = -5
    out = c.run(kv)
    assert kv.device_errors() & X.XP_DEVERR_LENGTH
    assert (out[:2] == 0).all() and out[2:].equal(good[2:])
    # token ranges that run backwards or past the end, overlapping ones
    c.dkv.copy_(_i32([100, 60]))
    for cu in ([0, 4, 2], [-7, 2, 900], [3, 1, 4], [0, 4, 4]):
        c.run(kv, cu_q=_i32(cu))
    torch.cuda.synchronize()
    kv.close()


def test_pages_past_four_gigabytes():
    """K and V rows whose byte offsets need more than 32 bits."""
    import torch
    P, n_kv = 256, 8
    c = Call(44, [700, 300], [2, 5], heads=16, n_kv=n_kv, P=P)
    kv = c.device()
    kv.close()
    from paper_2608_02438_amd.xpress import PagedKV
    far = 12000                                               # 524288 bytes a page
    kv = PagedKV(16, n_kv, P, far + c.n_pages, 2, 16, 1024)
    big = [torch.empty(kv.cache_shape, dtype=torch.bfloat16, device="cuda") for _ in range(2)]
    assert big[0].numel() * 2 > 1 << 32
    for b, small in zip(big, (c.dk, c.dv)):
        b[far:] = small
        b[:8] = float("nan")
    c.dk, c.dv = big
    c.dtable = torch.where(c.dtable >= 0, c.dtable + far, c.dtable).contiguous()
    c.check(c.run(kv), causal=True, parts=2)
    # and a write there
    rows = torch.randn(3, n_kv, 128, device="cuda").to(torch.bfloat16)
    slots = (torch.tensor([far + 1, far + 2, far + 3]) * P + 17).to(torch.int32).cuda()
    kv.write(rows, rows, slots, *big)
    for t in range(3):
        assert big[1][far + 1 + t, :, 17].equal(rows[t])
    kv.close()


# ---------------------------------------------------------------------------
# shared prefixes
# ---------------------------------------------------------------------------
SHARED = {
    # (kv, ql, groups, kwargs)
    "one group": ([200, 210, 195, 260], [1] * 4, [(0, 4, 192)], {}),
    "inside a page": ([200, 210, 195], [2, 1, 3], [(0, 3, 150)], {}),
    "groups and a loner": ([100, 90, 70, 300, 310], [5, 4, 3, 2, 1],
                           [(0, 2, 64), (2, 3, 0), (3, 5, 256)], {}),
    "outside": ([50, 100, 120, 70], [1, 2, 2, 1], [(1, 3, 96)], {}),
    "into the new tokens": ([80, 80, 80], [16, 16, 16], [(0, 3, 72)], {}),
    "empty members": ([130, 0, 140, 0], [3, 0, 2, 0], [(0, 3, 128), (3, 4, 0)], {}),
    "many": ([130 + i % 40 for i in range(90)], [1] * 90, [(0, 40, 128), (40, 90, 112)], {}),
    "prompts": ([150, 170], [80, 90], [(0, 2, 48)], {}),
    "long": ([3000, 2900, 2950], [2, 2, 2], [(0, 3, 2880)], dict(heads=16, n_kv=1)),
}


@pytest.mark.parametrize("name", SHARED)
@pytest.mark.parametrize("hd,cache", [(128, "bf16"), (64, "e4m3")])
def test_attend_shared(name, hd, cache):
    import torch
    kv_len, ql, groups, kw = SHARED[name]
    kw = dict(dict(heads=4, n_kv=2), **kw)
    c = Call(60 + len(name), kv_len, ql, hd=hd, cache=cache, P=16, groups=groups, **kw)
    if name == "into the new tokens":                         # the same pages: the same tokens
        c.q[16:32], c.q[32:] = c.q[:16], c.q[:16]
    kv = c.device(shared=True)
    rows = max(max(ql), c.total // len(groups)) * (c.heads // c.n_kv)
    for m in (dict(causal=True), dict(causal=False), dict(causal=True, window=40, sinks=20),
              dict(causal=True, window=150)):
        print(f"shared: {name} hd={hd} {cache} {m}", flush=True)
        out = torch.full((c.total, c.heads, hd), float("nan"), dtype=torch.bfloat16, device="cuda")
        lse = torch.full((c.total, c.heads), float("nan"), device="cuda")
        c.run(kv, shared=True, out=out, lse=lse, **m)
        assert kv.device_errors() == 0
        c.check(out, lse, parts=parts_of(rows, cache), **m)
        again = c.run(kv, shared=True, **m)
        assert again.equal(out)
    kv.close()


def test_shared_prefix_longer_than_a_member_is_cut():
    from paper_2608_02438_amd import xpress as X
    c = Call(70, [100, 64, 120], [1, 1, 1], heads=4, n_kv=2, groups=[(0, 3, 64)])
    kv = c.device(shared=True)
    c.dgl[0] = 90
    out = c.run(kv, shared=True)
    assert kv.device_errors() == X.XP_DEVERR_LENGTH
    c.check(out, causal=True, parts=2)
    kv.close()


def test_shared_tokens_behind_the_last_sequence_stay():
    import torch
    c = Call(71, [100, 110], [2, 2], heads=4, n_kv=2, groups=[(0, 2, 96)])
    kv = c.device(shared=True, max_tokens=16)
    q = torch.cat([c.dq, c.dq])
    out = torch.full_like(q, 7.0)
    c.run(kv, shared=True, q=q, out=out)
    c.check(out[:4], causal=True, parts=2)
    assert (out[4:] == 7).all()
    kv.close()


@pytest.mark.parametrize("hd,cache", [(128, "bf16"), (64, "bf16"), (128, "e4m3"), (64, "e4m3")])
def test_shared_prefixes_of_many_rows(hd, cache):
    """Blocks whose groups fill the largest row tiles and whose own rows do not:
    prefixes and own keys in work lists of their own; captured, replayed with new
    lengths, a request outside the groups."""
    import torch
    ql = [16, 9, 16, 16, 1, 16, 16, 0, 16, 16, 16, 16, 5]
    own = [40, 3, 0, 700, 20, 16, 90, 0, 17, 130, 64, 5, 333]
    pre = [900] * 7 + [640] * 5 + [0]
    kv_len = [max(p + o, q) for p, o, q in zip(pre, own, ql)]
    c = Call(72 + hd, kv_len, ql, heads=8, n_kv=2, hd=hd, cache=cache, P=16,
             groups=[(0, 7, 896), (7, 12, 640)])
    kv = c.device(shared=True)
    rows = c.total // 2 * 4
    assert rows > 256 and max(ql) * 4 <= 64                   # tiles of both sizes
    out = torch.empty_like(c.dq)
    for m in (dict(causal=True), dict(causal=False), dict(causal=True, window=100, sinks=20),
              dict(causal=True, window=800)):
        print(f"shared, many rows: hd={hd} {cache} {m}", flush=True)
        c.run(kv, shared=True, out=out, **m)
        assert kv.device_errors() == 0
        c.check(out, parts=parts_of(rows, cache), **m)
    g = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(g):
        c.run(kv, shared=True, out=out)
    for cut in (0, 7, 0):
        c.kv = [max(x - cut, 0) if p == 0 or x - cut >= p else x for x, p in zip(kv_len, pre)]
        c.dkv.copy_(_i32(c.kv))
        out.zero_()
        g.replay()
        torch.cuda.synchronize()
        c.check(out, causal=True, parts=parts_of(rows, cache))
        assert c.run(kv, shared=True).equal(out)
    kv.close()


@pytest.mark.parametrize("hd", [64, 128])
def test_token_ranges_that_overlap_many_times(hd):
    """Ranges that count far more rows than there are tokens are cut to what the work
    lists hold, reported, and leave the handle as it was."""
    import torch
    from paper_2608_02438_amd import xpress as X
    n, tokens = 600, 512
    c = Call(75 + hd, [40] * n, [1] * tokens + [0] * (n - tokens), heads=8, n_kv=1, hd=hd, P=16,
             groups=[(0, 300, 16), (300, 600, 32)], spare=5)
    kv = c.device(shared=True)
    good, alone = c.run(kv, shared=True), c.run(kv)
    assert kv.device_errors() == 0
    back = _i32([tokens if b % 2 else 0 for b in range(n + 1)])
    down = _i32([tokens - tokens * b // n for b in range(n + 1)])
    for cu, max_q in ((back, 1), (back, tokens), (down, 1)):
        for shared in (False, True):
            print(f"overlapping ranges: hd={hd} max_q={max_q} shared={shared}", flush=True)
            c.run(kv, shared=shared, cu_q=cu, max_q=max_q)
            torch.cuda.synchronize()
        assert (kv.device_errors() & X.XP_DEVERR_LENGTH) == (X.XP_DEVERR_LENGTH if cu is back else 0)
    assert c.run(kv, shared=True).equal(good) and c.run(kv).equal(alone)
    assert kv.device_errors() == 0
    kv.close()


# ---------------------------------------------------------------------------
# refusals
# ---------------------------------------------------------------------------
def test_calls_reject_bad_arguments():
    import torch
    from paper_2608_02438_amd import xpress as X
    L = X.load_library()
    c = Call(80, [40, 50], [1, 1], heads=4, n_kv=2)
    kv = c.device(max_tokens=8)
    p = lambda t: t.data_ptr()                                # noqa: E731
    out = torch.empty_like(c.dq)
    base = dict(n=2, tokens=2, max_q=1, q=p(c.dq), q_ld=512, cu=p(c.dcu), kv=p(c.dkv),
                table=p(c.dtable), ld=c.width, kc=p(c.dk), vc=p(c.dv), ks=None, vs=None, causal=1,
                window=0, sinks=0, scale=0.0, out=p(out), out_ld=512, lse=None)

    def attn(**kw):
        a = dict(base, **kw)
        return L.xp_kv_attn(kv._h, *(a[x] for x in base), None)
    assert attn() == X.XP_OK
    for kw in (dict(n=3), dict(n=-1), dict(tokens=9), dict(tokens=-1), dict(max_q=9), dict(max_q=-1),
               dict(q=None), dict(q=p(c.dq) + 2), dict(q_ld=511), dict(q_ld=516), dict(kv=None),
               dict(table=None), dict(ld=0), dict(kc=None), dict(vc=p(c.dv) + 8),
               dict(ks=p(c.dkv)), dict(causal=2), dict(window=-1), dict(sinks=-1),
               dict(window=(1 << 22) + 1), dict(scale=-1.0), dict(scale=float("nan")),
               dict(scale=float("inf")), dict(out=None), dict(out=p(out) + 4), dict(out_ld=256),
               dict(cu=None, tokens=3)):
        assert attn(**kw) == X.XP_EINVAL, kw
        assert L.xp_kv_last_error(kv._h)
    assert attn(n=0) == X.XP_OK and attn(tokens=0) == X.XP_OK
    a = dict(base)
    rest = [a[x] for x in list(base)[3:]]
    assert L.xp_kv_attn_shared(kv._h, 2, 2, 1, 1, p(c.dcu), p(c.dkv), *rest, None) == X.XP_EINVAL
    w = lambda **k: L.xp_kv_write(kv._h, *dict(dict(  # noqa: E731
        t=1, k=p(c.dq), kl=256, v=p(c.dq), vl=256, s=p(c.dkv), kc=p(c.dk), vc=p(c.dv), ks=None,
        vs=None), **k).values(), None)
    for kw in (dict(t=9), dict(t=-1), dict(k=None), dict(v=p(c.dq) + 2), dict(kl=255), dict(vl=260),
               dict(s=None), dict(kc=None), dict(vs=p(c.dkv))):
        assert w(**kw) == X.XP_EINVAL, kw
    assert w(t=0) == X.XP_OK
    d = p(c.dkv)
    m = lambda **k: L.xp_kv_map(kv._h, *dict(dict(  # noqa: E731
        n=2, lens=d, add=d, table=d, ld=3, held=d, pool=d, pn=d, cu=None, kv=None, s=None, ms=0),
        **k).values(), None)
    for kw in (dict(n=3), dict(n=-1), dict(lens=None), dict(add=None), dict(table=None), dict(ld=0),
               dict(held=None), dict(pool=None), dict(pn=None), dict(ms=-1)):
        assert m(**kw) == X.XP_EINVAL, kw
    # the binding's own checks
    bad = [lambda: kv.attend(c.dq.float(), c.dk, c.dv, c.dtable, c.dkv),
           lambda: kv.attend(c.dq.transpose(0, 1), c.dk, c.dv, c.dtable, c.dkv),
           lambda: kv.attend(c.dq, c.dk[1:], c.dv, c.dtable, c.dkv),
           lambda: kv.attend(c.dq, c.dk, c.dv, c.dtable.t(), c.dkv),
           lambda: kv.attend(c.dq, c.dk, c.dv, c.dtable, c.dkv.long()),
           lambda: kv.attend(c.dq, c.dk, c.dv, c.dtable, c.dkv, cu_q=c.dcu),
           lambda: kv.attend(c.dq, c.dk, c.dv, c.dtable, c.dkv, cu_q=c.dcu[1:], max_q=1),
           lambda: kv.attend(c.dq.cpu(), c.dk, c.dv, c.dtable, c.dkv),
           lambda: kv.attend(c.dq, c.dk, c.dv, c.dtable, c.dkv, lse=torch.empty(2, 4).cuda().t()),
           lambda: kv.write(c.dq[:, :2], c.dq[:1, :2], c.dkv, c.dk, c.dv),
           lambda: kv.map(c.dkv, c.dkv[:1], c.dtable, c.dkv, c.dkv, c.dkv),
           lambda: X.PagedKV(4, 2, 16, 10, 1, 1, 1, cache_dtype=torch.float16)]
    for f in bad:
        with pytest.raises(ValueError):
            f()
    with pytest.raises(X.XpError):
        kv.attend(c.dq, c.dk, c.dv, c.dtable, c.dkv, window=-1)
    kv.close()


# ---------------------------------------------------------------------------
# together
# ---------------------------------------------------------------------------
@pytest.mark.parametrize("cache,window,sinks", [("bf16", 0, 0), ("e4m3", 0, 0), ("bf16", 70, 4)])
def test_prompts_then_blocks_as_a_serving_loop(cache, window, sinks):
    """Prompts are mapped, written and attended to; then blocks are reserved,
    written, attended to and partly accepted, a request ends and its pages serve
    another.  The oracle keeps every request's keys in plain lists."""
    import torch
    from paper_2608_02438_amd.xpress import PagedKV
    rng = np.random.default_rng(90 + window)
    n, heads, n_kv, hd, P, B = 5, 8, 2, 128, 16, 7
    dt = torch.bfloat16 if cache == "bf16" else torch.float8_e4m3fn
    kv = PagedKV(heads, n_kv, P, 64, n, 256, 320, cache_dtype=dt)
    kc, vc = (torch.full(kv.cache_shape, float("nan"), device="cuda").to(dt) for _ in range(2))
    sc = None if cache == "bf16" else np.array([0.011, 0.009], dtype=np.float32)
    dsc = None if sc is None else torch.tensor(sc).cuda()
    table = torch.full((n, 20), -1, dtype=torch.int32, device="cuda")
    held, pool, pool_n = _i32([0] * n), _i32(rng.permutation(64)), _i32([64])
    past = [[np.zeros((0, n_kv, hd))] * 2 for _ in range(n)]
    lens = np.zeros(n, dtype=int)
    adds = [np.array([40, 1, 63, 0, 17])] + [np.array([B, B, B, 0, B])] * 2 + \
        [np.array([B, B, 33, 90, B])] + [np.array([B] * 5)]
    for step, add in enumerate(adds):
        T = int(add.sum())
        cap = T + 3                                           # padded tokens
        cu, kvl = (torch.empty(m, dtype=torch.int32, device="cuda") for m in (n + 1, n))
        slots = torch.empty(cap, dtype=torch.int32, device="cuda")
        kv.map(_i32(lens), _i32(add), table, held, pool, pool_n, cu=cu, kv_len=kvl, slots=slots)
        q, k, v = (bf16(rng.normal(size=(cap, h, hd)) * s) for h, s in
                   ((heads, 2), (n_kv, 1), (n_kv, 1)))
        dq, dk, dv = (torch.tensor(x).to(torch.bfloat16).cuda() for x in (q, k, v))
        kv.write(dk, dv, slots, kc, vc, k_scale=dsc, v_scale=dsc)
        out = kv.attend(dq, kc, vc, table, kvl, cu_q=cu, max_q=int(add.max()), window=window,
                        sinks=sinks, k_scale=dsc, v_scale=dsc)
        assert kv.device_errors() == 0
        call = Call.__new__(Call)
        call.hd, call.kv, call.ql, call.total = hd, [], [], T
        got = out.double().cpu().numpy()
        at = 0
        for b in range(n):
            new = slice(at, at + add[b])
            at += add[b]
            if cache == "bf16":
                rows = [x[new] for x in (k, v)]
            else:
                w = sc.astype(np.float64)[None, :, None]
                rows = [R.to_e4m3(x[new] / w) * w for x in (k, v)]
            keys = [np.concatenate([p, r]) for p, r in zip(past[b], rows)]
            parts = parts_of(int(add.max()) * heads // n_kv, cache)
            if add[b]:
                o, lse, spread, score = R.attend(q[new], *keys, window=window, sinks=sinks)
                m = keys[0].shape[0]
                d = 2 * ((hd + 12) * 2.0 ** -23 * score + 2.0 ** -22) + m * 2.0 ** -23 + 2.0 ** -20
                c = d[..., None] + (2.0 ** -8 if parts == 1 else 2.0 ** -16)
                bound = 2.0 ** -8 * (np.abs(o) + c * spread) + c * spread
                r = (np.abs(got[new] - o) / bound).max()
                print(f"loop: {cache} step {step} request {b}: {r:.3f} of the bound", flush=True)
                assert r <= 1
            # some of the new tokens stay; request 2 ends after the third step
            keep = add[b] if step == 0 else int(rng.integers(0, add[b] + 1))
            lens[b] += keep
            past[b] = [x[:lens[b]] for x in keys]
            if step == 2 and b == 2:
                lens[b], past[b] = 0, [x[:0] for x in keys]
    kv.close()


def _paged_layer(nkv, grp, B, ctx, cache, ffn=256, H=256, P=16, seed=7):
    import synth
    import torch
    from paper_2608_02438_amd.xpress import LAYER_WEIGHT_NAMES, Layer, PagedKV, device_tensor
    nh, batch, cmax = nkv * grp, len(ctx), max(max(ctx), 1)
    w = synth.scaled(synth.configs.QWEN_B1, index=940 + seed, H=H, B=B, batch=batch, n_heads=nh,
                     n_kv_heads=nkv, ffn=ffn, ctx_len=None, ctx_len_range=None)
    weights = synth.make_layer_weights(w)
    inp = synth.make_layer_inputs(w, c_max=cmax)
    inp.ctx_len = np.array(ctx, dtype=np.int32)
    dw = {k: device_tensor(weights[k]) for k in LAYER_WEIGHT_NAMES}
    layer = Layer(dw, H, nh, nkv, ffn, max_batch=batch, max_B=B, max_ctx=cmax)
    x, kc, vc, cl = (device_tensor(a) for a in (inp.x, inp.k_cache, inp.v_cache, inp.ctx_len))
    width = R.pages_of(cmax + B, P)
    dt = torch.bfloat16 if cache == "bf16" else torch.float8_e4m3fn
    kv = PagedKV(nh, nkv, P, batch * width + 1, batch, batch * B, width * P, cache_dtype=dt)
    table = torch.full((batch, width), -1, dtype=torch.int32, device="cuda")
    held, pool, pn = _i32([0] * batch), _i32(np.random.default_rng(seed).permutation(kv.n_pages)), \
        _i32([kv.n_pages])
    # the context as an earlier call wrote it
    kv2 = PagedKV(nh, nkv, P, kv.n_pages, batch, max(sum(ctx), 1), width * P, cache_dtype=dt)
    slots = torch.empty(max(sum(ctx), 1), dtype=torch.int32, device="cuda")
    kv2.map(_i32([0] * batch), cl, table, held, pool, pn, slots=slots)
    pk, pv = (torch.full(kv.cache_shape, float("nan"), device="cuda").to(dt) for _ in range(2))
    one = None if cache == "bf16" else torch.full((nkv,), 0.02, device="cuda")
    if sum(ctx):
        rows = [torch.cat([c[b, :ctx[b]] for b in range(batch)]) for c in (kc, vc)]
        kv2.write(rows[0], rows[1], slots, pk, pv, k_scale=one, v_scale=one)
    kv2.close()
    kv.map(cl, _i32([B] * batch), table, held, pool, pn)
    return layer, kv, dict(w=w, weights=weights, inp=inp, x=x, kc=kc, vc=vc, cl=cl, pk=pk, pv=pv,
                           table=table, one=one, nh=nh)


@pytest.mark.parametrize("nkv,grp,B,ctx", [
    (2, 4, 16, [70, 0, 300]), (2, 8, 7, [900, 1]), (4, 1, 1, [33, 64, 65]), (2, 2, 32, [500, 20]),
    (2, 8, 32, [130, 70])])
@pytest.mark.parametrize("causal", [True, False])
def test_layer_over_pages(nkv, grp, B, ctx, causal):
    """The layer over pages gives what the layer over a contiguous cache gives, and
    its block's keys lie in the pages for the next call."""
    layer, kv, d = _paged_layer(nkv, grp, B, ctx, "bf16")
    print(f"layer: nkv={nkv} grp={grp} B={B} ctx={ctx} causal={causal}", flush=True)
    h, hb = layer.forward_paged(d["x"], kv, d["pk"], d["pv"], d["table"], d["cl"], causal=causal)
    assert kv.device_errors() == 0
    again, _ = layer.forward_paged(d["x"], kv, d["pk"], d["pv"], d["table"], d["cl"], causal=causal)
    assert h.equal(again)
    LP = O.layer_ref.LayerParams.from_arrays(d["weights"], d["nh"], nkv, 128)
    i = d["inp"]
    ref = O.layer_ref.layer_forward(LP, i.x, i.k_cache, i.v_cache, i.ctx_len, causal=causal)
    # the layer parity tests' bar: one bf16 unit at the output's scale
    bar = max(2e-2, 2.0 ** -8 * np.abs(ref).max())
    assert np.abs(h.cpu().numpy() - ref).max() <= bar
    flat, _ = layer.forward(d["x"], d["kc"], d["vc"], d["cl"], causal=causal)
    assert (h - flat).abs().max().item() <= bar
    # the block's own keys: the layer's, after norm and rotation
    u = O.xpress_ref.round_bf16(O.layer_ref.rmsnorm(O.xpress_ref.to_f64(i.x[0]), LP.g_attn, LP.eps))
    k = O.layer_ref.rmsnorm((u @ LP.Wk.T).reshape(B, nkv, 128), LP.g_k, LP.eps)
    k = O.layer_ref.rope(k, ctx[0] + np.arange(B), LP.theta)
    got = R.gather(d["pk"].double().cpu().numpy(), d["table"][0].cpu().numpy(), ctx[0] + B)[ctx[0]:]
    # half a bf16 step and what a differently rounded u moves
    assert np.abs(got - k).max() <= 2.0 ** -7 * np.abs(k).max()
    layer.close()
    kv.close()


def test_layer_over_windowed_and_8bit_pages():
    """Against the oracle's attention inside the oracle's layer, on the pages' values."""
    import torch
    for cache, window, sinks in (("bf16", 40, 4), ("e4m3", 0, 0), ("e4m3", 64, 16)):
        layer, kv, d = _paged_layer(2, 4, 16, [150, 33], cache, seed=9)
        print(f"layer: {cache} window={window} sinks={sinks}", flush=True)
        h, _ = layer.forward_paged(d["x"], kv, d["pk"], d["pv"], d["table"], d["cl"], window=window,
                                   sinks=sinks, k_scale=d["one"], v_scale=d["one"])
        assert kv.device_errors() == 0
        LP = O.layer_ref.LayerParams.from_arrays(d["weights"], 8, 2, 128)
        r16, rms = O.xpress_ref.round_bf16, O.layer_ref.rmsnorm
        s = 1.0 if cache == "bf16" else np.float64(np.float32(0.02))
        for b, C in enumerate((150, 33)):
            x = O.xpress_ref.to_f64(d["inp"].x[b])
            u = r16(rms(x, LP.g_attn, LP.eps))
            q = rms((u @ LP.Wq.T).reshape(16, 8, 128), LP.g_q, LP.eps)
            q = r16(O.layer_ref.rope(q, C + np.arange(16), LP.theta))
            # the pages as the call left them (the block's rows among them)
            k, v = (R.gather(p.double().cpu().numpy(), d["table"][b].cpu().numpy(), C + 16) * s
                    for p in (d["pk"], d["pv"]))
            a = R.attend(q, k, v, True, window, sinks)[0]
            x1 = x + r16(a.reshape(16, -1)) @ LP.Wo.T
            u2 = r16(rms(x1, LP.g_mlp, LP.eps))
            act = r16(O.xpress_ref.silu(u2 @ LP.Wg.T) * (u2 @ LP.Wu.T))
            ref = x1 + act @ LP.Wd.T
            bar = max(2e-2, 2.0 ** -8 * np.abs(ref).max())
            assert np.abs(h[b].cpu().numpy() - ref).max() <= bar
        layer.close()
        kv.close()


def test_layer_over_pages_captured():
    """Replayed with shorter contexts, eager calls in between."""
    import torch
    layer, kv, d = _paged_layer(2, 4, 16, [150, 0, 65], "bf16", seed=12)
    h = torch.empty(3, 16, 256, device="cuda")
    hb = torch.empty(3, 16, 256, dtype=torch.bfloat16, device="cuda")

    def call():
        return layer.forward_paged(d["x"], kv, d["pk"], d["pv"], d["table"], d["cl"], window=90,
                                   sinks=3, h_f32=h, h_bf16=hb)
    call()
    g = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(g):
        call()
    for ctx in ([150, 0, 65], [140, 0, 50], [131, 0, 49], [150, 0, 65]):
        d["cl"].copy_(_i32(ctx))
        h.zero_()
        g.replay()
        torch.cuda.synchronize()
        got, bits = h.clone(), hb.clone()
        call()
        assert got.equal(h) and bits.equal(hb) and got.abs().max() > 0
    assert kv.device_errors() == 0
    layer.close()
    kv.close()


def test_layer_over_pages_rejects_bad_calls():
    import torch
    from paper_2608_02438_amd import xpress as X
    L = X.load_library()
    layer, kv, d = _paged_layer(2, 2, 8, [20, 5], "bf16", seed=11)
    p = lambda t: t.data_ptr()                                # noqa: E731
    h = torch.empty(2, 8, 256, device="cuda")
    base = dict(kv=kv._h, batch=2, B=8, causal=1, window=0, sinks=0, x=p(d["x"]), kc=p(d["pk"]),
                vc=p(d["pv"]), ks=None, vs=None, table=p(d["table"]), ld=d["table"].shape[1],
                ctx=p(d["cl"]), h32=p(h), hb=None)

    def call(**kw):
        return L.xp_layer_forward_paged(layer._h, *dict(base, **kw).values(), None)
    assert call() == X.XP_OK
    other = X.PagedKV(2, 2, 16, 4, 2, 16, 64)
    for kw in (dict(kv=None), dict(kv=other._h), dict(batch=3), dict(batch=0), dict(B=9), dict(B=0),
               dict(causal=2), dict(window=-1), dict(sinks=-1), dict(x=None), dict(x=p(d["x"]) + 8),
               dict(kc=None), dict(vc=p(d["pv"]) + 8), dict(ks=p(h)), dict(table=None), dict(ld=0),
               dict(ctx=None)):
        assert call(**kw) == X.XP_EINVAL, kw
        assert L.xp_layer_last_error(layer._h)
    other.close()
    layer.close()
    kv.close()
