"""The 4-bit context cache on the device: writes and reads bit for bit, attention
within a bound derived from its roundings (tests/_kv.py)."""
import numpy as np
import pytest

import oracle as O
from _kv import bf16
from _kv4 import Call4, parts_of4

R = O.kv_ref
pytestmark = pytest.mark.gpu


def _i32(x):
    import torch
    return torch.tensor(np.asarray(x), dtype=torch.int32, device="cuda")


def _bf(x):
    import torch
    return torch.tensor(np.ascontiguousarray(x)).to(torch.bfloat16).cuda()


def _handle(n_kv=2, P=16, n_pages=8, hd=128, dt="mxfp4", max_tokens=4096, **kw):
    from paper_2608_02438_amd.xpress import PagedKV
    return PagedKV(n_kv, n_kv, P, n_pages, 1, max_tokens, P, head_dim=hd, cache_dtype=dt, **kw)


def _values(cache, P, hd):
    return R.mxfp4_values(*R.unpack_mxfp4(cache.cpu().numpy(), P, hd))


# ---------------------------------------------------------------------------
# writes and reads
# ---------------------------------------------------------------------------
@pytest.mark.parametrize("hd,n_kv,P,tokens", [
    (128, 1, 16, 1), (128, 8, 16, 17), (64, 2, 32, 33), (128, 5, 64, 300), (64, 1, 256, 1),
    (64, 7, 16, 129), (128, 2, 256, 511), (128, 3, 128, 64)])
def test_write_and_read_back(hd, n_kv, P, tokens):
    """Strided rows to scattered slots; every other byte of the cache stays."""
    import torch
    rng = np.random.default_rng(tokens)
    pages = -(-tokens // P) + 3
    kv = _handle(n_kv, P, pages, hd)
    slots = rng.permutation(pages * P)[:tokens].astype(np.int32)
    slots[2::5] = -1
    row = n_kv * hd
    fused = bf16(rng.normal(size=(tokens, 3 * row + 8)) *
                 2.0 ** rng.integers(-30, 30, size=(tokens, 1)))
    d = _bf(fused)
    k, v = (d[:, 8 + i * row:8 + (i + 1) * row].unflatten(1, (n_kv, hd)) for i in (0, 2))
    before = [rng.integers(0, 256, size=tuple(kv.cache_shape)).astype(np.uint8) for _ in range(2)]
    kc, vc = (torch.tensor(b).cuda() for b in before)
    print(f"write: hd={hd} n_kv={n_kv} P={P} tokens={tokens}", flush=True)
    kv.write(k, v, _i32(slots), kc, vc)
    assert kv.device_errors() == 0
    for b, got, at in ((before[0], kc, 0), (before[1], vc, 2)):
        codes, exps = R.unpack_mxfp4(b, P, hd)
        x = fused[:, 8 + at * row:8 + (at + 1) * row].reshape(tokens, n_kv, hd)
        new_c, new_e = R.to_mxfp4(x)
        for t in np.flatnonzero(slots >= 0):
            codes[slots[t] // P, :, slots[t] % P] = new_c[t]
            exps[slots[t] // P, :, slots[t] % P] = new_e[t]
        assert np.array_equal(got.cpu().numpy(), R.pack_mxfp4(codes, exps))
    # all rows, in an order of their own, beside some without a place
    order = rng.permutation(pages * P)[:4000].astype(np.int32)
    order[1::7] = -1
    wide = torch.full((order.size, row + 24), 9.0, dtype=torch.bfloat16, device="cuda")
    gk, gv = kv.read(_i32(order), kc, vc, k=wide[:, 16:16 + row].unflatten(1, (n_kv, hd)))
    assert kv.device_errors() == 0
    for got, cache in ((gk, kc), (gv, vc)):
        want = _values(cache, P, hd).transpose(0, 2, 1, 3).reshape(-1, n_kv, hd)[order]
        want[order < 0] = 0
        assert np.array_equal(got.double().cpu().numpy(), want, equal_nan=True)
    assert (wide[:, :16] == 9).all() and (wide[:, 16 + row:] == 9).all()
    only, none = kv.read(_i32(order), kc, vc, v=False)
    assert none is None and torch.equal(only.view(torch.int16), gk.contiguous().view(torch.int16))
    kv.close()


def test_write_blocks_of_every_magnitude_and_every_tie():
    """Every bf16 magnitude as a block's greatest one, and beside it the values on and
    next to the middles of its codes."""
    import torch
    bits = np.arange(0, 0x8000, dtype=np.uint32)
    top = (bits << 16).view(np.float32).astype(np.float64)
    x = np.zeros((bits.size, 32))
    x[:, 3] = top
    mid = np.array([0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0])
    with np.errstate(over="ignore", invalid="ignore"):
        s = 2.0 ** np.floor(np.log2(np.where(np.isfinite(top) & (top > 0), top, 1)))
        for i, f in enumerate((0.25, 0.5)):                   # the two powers of two in question
            x[:, 4 + 14 * i:4 + 14 * i + 7] = mid * s[:, None] * f
            y = mid * s[:, None] * f * (1 + 2.0 ** -7)
            x[:, 11 + 14 * i:11 + 14 * i + 7] = -y
        x = np.where(np.abs(x) <= np.abs(top)[:, None], x, 0)
        x[:, 3] = top
    x = torch.tensor(x).to(torch.bfloat16)
    rows = x.view(-1, 2, 64).contiguous()
    n = rows.shape[0]
    kv = _handle(2, 64, n // 64, 64, max_tokens=n)
    kc, vc = (torch.zeros(kv.cache_shape, dtype=torch.uint8, device="cuda") for _ in range(2))
    kv.write(rows.cuda(), (-rows).cuda(), _i32(np.arange(n)), kc, vc)
    for got, src in ((kc, rows), (vc, -rows)):
        codes, exps = R.to_mxfp4(src.double().numpy().reshape(n // 64, 64, 2, 64).transpose(0, 2, 1, 3))
        assert np.array_equal(got.cpu().numpy(), R.pack_mxfp4(codes, exps))
    k, _ = kv.read(_i32(np.arange(n)), kc, vc)
    want = R.mxfp4_values(*R.to_mxfp4(rows.double().numpy()))
    assert np.array_equal(k.double().cpu().numpy(), want, equal_nan=True)
    kv.close()


def test_read_of_every_code_and_exponent():
    import torch
    kv = _handle(1, 256, 16, 128)
    codes = np.tile(np.arange(16, dtype=np.uint8), (16, 1, 256, 8))
    exps = np.arange(16 * 256 * 4).reshape(16, 1, 256, 4).astype(np.uint8)
    c = torch.tensor(R.pack_mxfp4(codes, exps)).cuda()
    k, v = kv.read(_i32(np.arange(4096)), c, c)
    want = R.mxfp4_values(codes, exps).reshape(4096, 1, 128)
    assert np.array_equal(k.double().cpu().numpy(), want, equal_nan=True)
    assert torch.equal(k.view(torch.int16), v.view(torch.int16))
    kv.close()


def test_read_of_16_and_8_bit_caches():
    """8-bit values times their scales are rounded once, also where fp32 would move the
    product onto the middle between two bf16 values."""
    import torch
    rng = np.random.default_rng(5)
    n_kv, P, hd, pages = 64, 16, 64, 16
    kv = _handle(n_kv, P, pages, hd, dt=torch.float8_e4m3fn)
    scales = (rng.integers(1 << 23, 1 << 24, size=n_kv) * 2.0 ** rng.integers(-40, 20, size=n_kv))
    # products that end next to a middle: m s = (odd) 2^k + a little, m odd of 4 bits
    for i, m in enumerate((9, 11, 13, 15) * 8):
        mids = (2 * rng.integers(128, 256) + 1) * 2.0 ** 30
        scales[i] = np.float32(mids / m) if i % 2 else np.nextafter(np.float32(mids / m), np.float32(0))
    scales = scales.astype(np.float32)
    vals = R.e4m3_values()
    code = np.resize(np.arange(256, dtype=np.uint8), (pages, n_kv, P, hd))
    c = torch.tensor(code).cuda().view(torch.float8_e4m3fn)
    sc = torch.tensor(scales).cuda()
    k, v = kv.read(_i32(np.arange(pages * P)), c, c, k_scale=sc)
    x = vals[code].transpose(0, 2, 1, 3).reshape(-1, n_kv, hd)
    want = O.xpress_ref.round_bf16(np.nan_to_num(x * scales.astype(np.float64)[None, :, None]))
    ok = ~np.isnan(x)
    g = k.double().cpu().numpy()
    assert np.isnan(g[~ok]).all() and np.array_equal(g[ok], want[ok])
    assert np.array_equal(v.double().cpu().numpy(), x, equal_nan=True)
    kv.close()
    kv = _handle(3, 32, 5, 128, dt=torch.bfloat16)
    c = _bf(rng.normal(size=tuple(kv.cache_shape)))
    slots = rng.permutation(160)
    k, v = kv.read(_i32(slots), c, -c)
    want = c.transpose(1, 2).reshape(160, 3, 128)[torch.tensor(slots).cuda()]
    assert k.equal(want) and v.equal(-want)
    kv.close()


def test_slots_outside_the_cache():
    import torch
    from paper_2608_02438_amd import xpress as X
    kv = _handle(2, 16, 4, 128)
    kc, vc = (torch.full(kv.cache_shape, 0x35, dtype=torch.uint8, device="cuda") for _ in range(2))
    x = torch.ones((4, 2, 128), dtype=torch.bfloat16, device="cuda")
    slots = _i32([64, -2, 2 ** 31 - 1, 63])
    kv.write(x, x, slots, kc, vc)
    assert kv.device_errors() == X.XP_DEVERR_SLOT
    k, v = kv.read(slots, kc, vc)
    assert kv.device_errors() == X.XP_DEVERR_SLOT
    assert (k[:3] == 0).all() and (k[3] == 1).all() and (v[:3] == 0).all() and (v[3] == 1).all()
    assert (kc[:3] == 0x35).all() and (kc[3, :, :15 * 64] == 0x35).all()
    kv.read(_i32([-1]), kc, vc)
    assert kv.device_errors() == 0
    e = _i32([])
    k, v = kv.read(e, kc, vc)
    assert k.shape == (0, 2, 128)
    kv.close()


# ---------------------------------------------------------------------------
# attention
# ---------------------------------------------------------------------------
LENGTHS = {
    "one": ([1], [1], dict(heads=4, n_kv=1)),
    "tokens": ([1, 2, 63, 64, 65, 700, 0, 129], [1, 1, 1, 1, 1, 1, 0, 1], dict(heads=8, n_kv=2)),
    "short": ([5, 0, 17, 31, 16], [1, 0, 1, 1, 1], dict(heads=2, n_kv=2)),
    "long": ([3000, 40, 2049], [1, 1, 1], dict(heads=14, n_kv=2)),
    "group16": ([130, 511, 1000], [1, 1, 1], dict(heads=16, n_kv=1)),
    "group32": ([300, 64], [1, 1], dict(heads=32, n_kv=1)),
    "blocks": ([16, 333, 64, 90], [16, 16, 16, 16], dict(heads=4, n_kv=2)),
    "blocks5": ([5, 37, 260], [5, 5, 3], dict(heads=12, n_kv=4)),
    "rows128": ([200, 77, 33], [32, 32, 30], dict(heads=4, n_kv=1)),
    "prompts": ([190, 1, 64, 260], [190, 1, 64, 70], dict(heads=2, n_kv=1)),
    "mixed": ([400, 300, 50, 129, 7], [1, 150, 33, 129, 2], dict(heads=4, n_kv=2)),
}
MASKS = (dict(causal=True), dict(causal=False), dict(causal=True, window=50, sinks=3),
         dict(causal=False, window=17), dict(causal=True, window=1), dict(causal=True, window=9, sinks=200))


@pytest.mark.parametrize("name", LENGTHS)
@pytest.mark.parametrize("hd,P", [(128, 16), (64, 64), (128, 256), (64, 16)])
def test_attend4(name, hd, P):
    import torch
    kv_len, ql, kw = LENGTHS[name]
    c = Call4(sum(kv_len) + hd, kv_len, ql, hd=hd, P=P, spread=3, **kw)
    kv = c.device()
    for m in MASKS:
        print(f"attend4: {name} hd={hd} P={P} {m}", flush=True)
        lse = torch.zeros((c.total, c.heads), device="cuda")
        out = c.run(kv, lse=lse, **m)
        assert kv.device_errors() == 0
        c.check(out, lse, parts=parts_of4(c.rows()), **m)
    kv.close()


@pytest.mark.parametrize("hd", [64, 128])
@pytest.mark.parametrize("ql", [[1, 1], [5, 16], [40, 90], [90, 70]])
def test_unseen_keys_hold_nan(hd, ql):
    """Keys in front of the window, behind the last one and later than a token are NaN
    (exponents above 252)."""
    kv_len, W = [150, 203], 100
    c = Call4(20 + sum(ql), kv_len, ql, heads=4, n_kv=2, hd=hd, P=64)
    for i, (b, j) in enumerate([(b, j) for b in range(2)
                                for j in range(5, kv_len[b] - ql[b] - W + 1)]):
        for x in (0, 1):
            c.exponent(x, c.table[b, j // 64], j % 64, (255, 254, 253)[i % 3])
    late = [(0, kv_len[0] - 1), (1, kv_len[1] - 2)]           # seen by the last tokens only
    for b, j in late:
        c.exponent(0, c.table[b, j // 64], j % 64, 255)
        c.exponent(1, c.table[b, j // 64], j % 64, 255)
    for b in range(2):
        for j in range(kv_len[b], -(-kv_len[b] // 64) * 64):
            c.exponent(0, c.table[b, j // 64], j % 64, 255)
            c.exponent(1, c.table[b, j // 64], j % 64, 254)
    kv = c.device()
    print(f"masked exponents: hd={hd} ql={ql}", flush=True)
    out = c.run(kv, window=W, sinks=5).double().cpu().numpy()
    with np.errstate(invalid="ignore"):
        want = c.oracle(causal=True, window=W, sinks=5, parts=parts_of4(c.rows()))
    for b in want:
        o, _, eb, _ = want[b]
        m = ql[b]
        sees = np.arange(m) >= (m - 1 if b == 0 else m - 2)
        got = out[c.cu[b]:c.cu[b + 1]]
        assert not np.isfinite(got[sees]).any()
        assert np.isfinite(got[~sees]).all()
        assert (np.abs(got - o) <= eb)[~sees].all()
    kv.close()


@pytest.mark.parametrize("ql", [[4, 7], [60, 90]])
def test_nan_values_of_later_tokens(ql):
    """One block of V is NaN at a key that later tokens see: they are NaN in its 32
    dims alone, the earlier ones the oracle's."""
    c = Call4(31, [100, 130], ql, heads=2, n_kv=1, hd=64, P=16)
    for b, n in enumerate((100, 130)):
        e = c.bits[1][1]
        e[c.table[b, (n - 2) // 16], 0, (n - 2) % 16, 1] = 255
    c.v = R.mxfp4_values(*c.bits[1])
    kv = c.device()
    out = c.run(kv).double().cpu().numpy()
    want = c.oracle(causal=True, parts=parts_of4(c.rows()))
    for b in want:
        o, _, eb, _ = want[b]
        got = out[c.cu[b]:c.cu[b + 1]]
        ok = np.isfinite(o)
        assert ok[:-2].all() and not ok[-2:, :, 32:].any() and ok[-2:, :, :32].all()
        assert (np.abs(got - o) <= eb)[ok].all() and np.isnan(got[~ok]).all()
    kv.close()


@pytest.mark.parametrize("far", [14, 20, 27, 60, 100])
@pytest.mark.parametrize("hd,heads,n_kv,ql", [(128, 8, 2, [1, 1, 2]), (64, 8, 2, [1, 1, 2]),
                                              (128, 16, 1, [1, 1, 1]), (64, 12, 3, [1, 4, 3]),
                                              (128, 8, 1, [4, 2, 3]), (64, 4, 2, [16, 7, 16])])
def test_queries_of_far_apart_magnitudes(hd, heads, n_kv, ql, far):
    """Queries with 32 elements 2^far above the others and keys as far below there: all of
    them count for the scores, as where they are alike."""
    import torch
    c = Call4(far + hd, [130, 64, 333], ql, heads=heads, n_kv=n_kv, hd=hd, P=16)
    c.q[:, ::2, 32:64] *= 2.0 ** far                          # the others' rows beside them
    codes, exps = c.bits[0]
    exps[..., 1] -= far
    c.k = R.mxfp4_values(codes, exps)
    assert np.isfinite(c.k).all() and np.array_equal(bf16(c.q), c.q)
    kv = c.device()
    for m in (dict(causal=True), dict(causal=False, window=90, sinks=7)):
        print(f"far-apart queries: hd={hd} heads={heads}/{n_kv} ql={ql} 2^{far} {m}", flush=True)
        lse = torch.zeros((c.total, c.heads), device="cuda")
        out = c.run(kv, lse=lse, **m)
        assert kv.device_errors() == 0
        c.check(out, lse, parts=parts_of4(c.rows()), **m)
    kv.close()


@pytest.mark.parametrize("tiny", [0.0, 2.0 ** -40])
@pytest.mark.parametrize("hd,heads,n_kv", [(128, 8, 2), (64, 8, 2), (128, 16, 1), (64, 12, 1)])
def test_infinite_queries_and_nan_keys_beside_tiny_elements(hd, heads, n_kv, tiny):
    """A row with an infinity, NaN in keys behind the last one and before the window: with
    and without elements far below their row's greatest, the other rows are the oracle's."""
    c = Call4(hd + heads, [130, 77], [1, 1], heads=heads, n_kv=n_kv, hd=hd, P=16)
    if tiny:
        c.q[..., 3] = tiny
    for x in (0, 1):
        for b, n in enumerate(c.kv):
            for j in [*range(3, n - 50), *range(n, -(-n // 16) * 16)]:
                c.exponent(x, c.table[b, j // 16], j % 16, 255)
    bad = [(0, 1, np.inf), (1, heads - 1, -np.inf), (1, 0, np.nan)]
    want = c.oracle(causal=True, window=50, sinks=3, parts=parts_of4(c.rows()))
    for t, h, v in bad:
        c.q[t, h, 7] = v
    kv = c.device()
    print(f"infinite queries: hd={hd} heads={heads}/{n_kv} tiny={tiny}", flush=True)
    out = c.run(kv, window=50, sinks=3).double().cpu().numpy()
    assert kv.device_errors() == 0
    for b in want:
        o, _, eb, _ = want[b]
        ok = np.array([(b, h) not in [x[:2] for x in bad] for h in range(heads)])
        got = out[c.cu[b]:c.cu[b + 1]]
        assert (np.abs(got - o) <= eb)[:, ok].all()
        assert np.isnan(got[:, ~ok]).all()
    kv.close()


SHARED4 = {
    "one group": ([700, 650, 900], [1, 1, 1], [(0, 3, 512)], dict(heads=8, n_kv=2)),
    "blocks": ([300, 280, 90, 400, 330], [16, 16, 16, 16, 16], [(0, 2, 256), (2, 3, 0), (3, 5, 320)],
               dict(heads=4, n_kv=2)),
    "odd prefix": ([300, 301, 299], [1, 3, 2], [(0, 3, 203)], dict(heads=4, n_kv=1)),
    "prompts": ([500, 450, 620], [200, 150, 300], [(0, 3, 128)], dict(heads=2, n_kv=1)),
}


@pytest.mark.parametrize("name", SHARED4)
@pytest.mark.parametrize("hd", [64, 128])
def test_attend4_shared(name, hd):
    import torch
    kv_len, ql, groups, kw = SHARED4[name]
    c = Call4(len(name), kv_len, ql, groups=groups, hd=hd, P=16, **kw)
    for s0, s1, shared in groups:                             # the members' tables begin alike
        for b in range(s0 + 1, s1):
            assert (c.table[b, :shared // 16] == c.table[s0, :shared // 16]).all()
    kv = c.device(shared=True)
    for m in (dict(causal=True), dict(causal=True, window=150, sinks=20), dict(causal=False)):
        print(f"shared4: {name} hd={hd} {m}", flush=True)
        lse = torch.zeros((c.total, c.heads), device="cuda")
        out = c.run(kv, shared=True, lse=lse, **m)
        assert kv.device_errors() == 0
        c.check(out, lse, parts=1, **m)
    kv.close()


def _behind_prefixes(groups, each, shared, own):
    """Single tokens of `each` requests behind every one of so many prefixes."""
    kv = [shared + 16 * g + 1 + (own * (i + 1)) % 97 for g in range(groups) for i in range(each)]
    return kv, [1] * len(kv), [(g * each, (g + 1) * each, shared + 16 * g) for g in range(groups)]


SHARED4_TWO = {                      # both lists' tiles have up to 32 rows
    "one group": SHARED4["one group"], "odd prefix": SHARED4["odd prefix"],
    "16 prefixes": (*_behind_prefixes(16, 4, 48, 31), dict(heads=8, n_kv=2)),
    "2 prefixes": (*_behind_prefixes(2, 8, 400, 17), dict(heads=4, n_kv=1)),
    "a head each": (*_behind_prefixes(5, 8, 160, 23), dict(heads=2, n_kv=2)),
    "blocks": ([300, 340, 220], [5, 4, 3], [(0, 2, 192), (2, 3, 64)], dict(heads=4, n_kv=2)),
}


@pytest.mark.parametrize("name", SHARED4_TWO)
@pytest.mark.parametrize("hd", [64, 128])
def test_attend4_shared_numerators_of_two_parts(name, hd):
    """Calls whose rows a prefix are 32 at most keep both parts of every numerator."""
    import torch
    kv_len, ql, groups, kw = SHARED4_TWO[name]
    c = Call4(len(name) + 60, kv_len, ql, groups=groups, hd=hd, P=16, spread=2,
              sigma_q=0.5, **kw)
    rows = max(max(ql), sum(ql) // len(groups)) * (c.heads // c.n_kv)
    assert parts_of4(rows) == 2
    kv = c.device(shared=True)
    for m in (dict(causal=True), dict(causal=True, window=150, sinks=20), dict(causal=False)):
        print(f"shared4, two parts: {name} hd={hd} {m}", flush=True)
        lse = torch.full((c.total, c.heads), 777.0, device="cuda")
        out = c.run(kv, shared=True, lse=lse, **m)
        assert kv.device_errors() == 0
        c.check(out, lse, parts=2, **m)
    kv.close()


def _slots_call(seed, n, active, ql=1, **kw):
    """n request slots of which `active` have ql new tokens; some of the idle ones keep keys."""
    rng = np.random.default_rng(seed)
    keys = rng.integers(1, 300, size=n)
    q = [ql if b in active else 0 for b in range(n)]
    kv_len = [int(keys[b]) + q[b] if q[b] else int(keys[b]) * (b % 3 == 0 and n <= 300)
              for b in range(n)]
    return Call4(seed, kv_len, q, **kw)


SLOTS = {                            # slots, those with tokens, tokens of each
    "64 of 65": (65, [b for b in range(65) if b != 3], 1),
    "the last of 65": (65, [64], 1),
    "35 of 96": (96, [5, 20, 63] + list(range(64, 96)), 1),
    "40 of 200": (200, [0, 62] + list(range(64, 200, 4))[:34] + [190, 194, 198, 199], 1),
    "blocks, 30 of 100": (100, [3, 40] + list(range(66, 94)), 2),
    "blocks, 12 of 300": (300, [64, 65, 100, 128, 191, 192, 255, 256, 257, 290, 298, 299], 4),
    "64 of 64": (64, list(range(64)), 1),
    "100 of 100": (100, list(range(100)), 1),
    "64 of 4096": (4096, list(range(63, 4096, 64)), 1),
}


@pytest.mark.parametrize("name", SLOTS)
@pytest.mark.parametrize("hd,heads,n_kv", [(128, 8, 2), (64, 4, 1), (128, 16, 1), (64, 32, 2)])
def test_request_slots_without_tokens(name, hd, heads, n_kv):
    """Few tokens of many request slots, most of them behind the 64th: every token's row is
    written, the rows behind the last one are not."""
    import torch
    n, active, ql = SLOTS[name]
    c = _slots_call(n + hd + heads, n, active, ql, heads=heads, n_kv=n_kv, hd=hd, P=32)
    kv = c.device(max_tokens=c.total + 3)
    q = torch.cat([c.dq, torch.ones((3, heads, hd), dtype=torch.bfloat16, device="cuda")])
    for m in (dict(causal=True), dict(causal=True, window=40, sinks=2)):
        for tokens in ((c.total, c.total + 3) if m == dict(causal=True) else (c.total,)):
            print(f"slots: {name} hd={hd} heads={heads}/{n_kv} tokens={tokens} {m}", flush=True)
            out = torch.full((c.total + 3, heads, hd), 777.0, dtype=torch.bfloat16, device="cuda")
            lse = torch.full((c.total + 3, heads), 777.0, device="cuda")
            c.run(kv, q=q[:tokens], out=out[:tokens], lse=lse[:tokens], **m)
            assert kv.device_errors() == 0
            c.check(out, lse, parts=parts_of4(c.rows()), **m)
            assert (out[c.total:] == 777).all() and (lse[c.total:] == 777).all()
    kv.close()


@pytest.mark.parametrize("heads,n_kv", [(8, 2), (16, 1)])
def test_a_captured_step_over_slots(heads, n_kv):
    """A step captured for 96 request slots is replayed as other slots become active."""
    import torch
    n = 96
    sets = [list(range(40)), list(range(56, 96)), list(range(1, 80, 2)), [95] + list(range(39))]
    calls = [_slots_call(7, n, s, heads=heads, n_kv=n_kv, P=16) for s in sets]
    need = max(c.width for c in calls)
    kv = calls[0].device(max_len=need * 16)
    tokens = calls[0].total
    table = torch.zeros((n, need), dtype=torch.int32, device="cuda")
    pages = max(c.n_pages for c in calls)
    handle = Call4(1, [16 * (pages - 3)], [1], heads=heads, n_kv=n_kv, P=16).device(
        max_batch=n, max_tokens=tokens, max_len=need * 16)
    kv.close()
    kc, vc = (torch.zeros(handle.cache_shape, dtype=torch.uint8, device="cuda") for _ in range(2))
    q, cu, lens = torch.empty_like(calls[0].dq), _i32(np.zeros(n + 1)), _i32(np.zeros(n))
    out, lse = torch.empty_like(q), torch.empty((tokens, heads), device="cuda")
    step = lambda: handle.attend(q, kc, vc, table, lens, cu_q=cu, max_q=1, out=out, lse=lse)  # noqa: E731

    def load(c):
        c.device().close()
        assert c.total == tokens
        kc[:c.n_pages], vc[:c.n_pages] = c.dk, c.dv
        table[:, :c.width] = c.dtable
        q.copy_(c.dq), cu.copy_(c.dcu), lens.copy_(c.dkv)
        out.fill_(777.0), lse.fill_(777.0)
    load(calls[0])
    step()
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        step()
    for i in (0, 1, 2, 3, 1, 0):
        load(calls[i])
        g.replay()
        torch.cuda.synchronize()
        assert handle.device_errors() == 0
        calls[i].check(out, lse, causal=True, parts=parts_of4(calls[i].rows()))
        got = out.clone()
        step()
        assert out.equal(got)
    handle.close()


def test_many_sequences_and_strided_rows():
    import torch
    ql = [(150, 1, 16, 33, 0, 2)[i % 6] for i in range(70)]
    kv_len = [x + (0, 200, 90, 7, 30, 1)[i % 5] for i, x in enumerate(ql)]
    c = Call4(44, kv_len, ql, heads=4, n_kv=2, hd=128)
    kv = c.device()
    out = c.run(kv, window=70, sinks=5)
    c.check(out, parts=1, causal=True, window=70, sinks=5)
    kv.close()
    c = Call4(12, [70, 33], [5, 4], heads=4, n_kv=2, hd=64)
    kv = c.device(max_tokens=32)
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


@pytest.mark.parametrize("ql", [[3, 3, 3, 3], [1, 1, 1, 1], [40, 33, 20, 40]])
def test_captured_calls_replay_with_new_lengths(ql):
    import torch
    c = Call4(42, [500, 140, 700, 90], ql, heads=8, n_kv=2, P=16)
    kv = c.device()
    out = torch.empty_like(c.dq)
    c.run(kv, out=out)
    g = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(g):
        c.run(kv, out=out)
    for lens in ([500, 140, 700, 90], [480, 133, 650, 70], [500, 140, 90, 80]):
        c.dkv.copy_(_i32(lens))
        c.kv = lens
        out.zero_()
        g.replay()
        torch.cuda.synchronize()
        c.check(out, causal=True, parts=parts_of4(c.rows()))
        assert c.run(kv).equal(out)
    kv.close()


def test_equal_bits_on_another_stream():
    import torch
    c = Call4(41, [3000, 40, 700, 0, 5], [1, 1, 1, 0, 1], heads=8, n_kv=2, P=16)
    kv = c.device()
    a = c.run(kv, window=500, sinks=20)
    s = torch.cuda.Stream()
    torch.cuda.synchronize()
    b = c.run(kv, window=500, sinks=20, stream=s, out=torch.empty_like(a))
    s.synchronize()
    assert a.equal(b)
    kv.close()


def test_bad_pages_and_lengths():
    import torch
    from paper_2608_02438_amd import xpress as X
    c = Call4(43, [100, 60], [2, 2], heads=4, n_kv=2, P=16)
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
    kv.close()


def test_pages_past_four_gigabytes():
    """Rows, codes and exponents of the last pages of 4.6 GB caches."""
    import torch
    n_pages, P, n_kv, hd = 66000, 256, 4, 128
    c = Call4(3, [600, 300], [1, 5], heads=8, n_kv=n_kv, hd=hd, P=P, spare=0)
    from paper_2608_02438_amd.xpress import PagedKV
    kv = PagedKV(8, n_kv, P, n_pages, 2, 16, 4 * P, head_dim=hd, cache_dtype="mxfp4")
    kc, vc = (torch.zeros(kv.cache_shape, dtype=torch.uint8, device="cuda") for _ in range(2))
    assert kc.numel() > 4 << 30
    base = n_pages - c.n_pages
    c.device()
    kc[base:], vc[base:] = c.dk, c.dv
    slot = (n_pages - 1) * P + P - 1                          # one row by the device itself
    x = _bf(np.random.default_rng(0).normal(size=(1, n_kv, hd)))
    kv.write(x, x, _i32([slot]), kc, vc)
    k, v = kv.read(_i32([slot]), kc, vc)
    want = R.mxfp4_values(*R.to_mxfp4(x.double().cpu().numpy()))
    assert np.array_equal(k.double().cpu().numpy(), want) and k.equal(v)
    out = kv.attend(c.dq, kc, vc, c.dtable + base, c.dkv, cu_q=c.dcu, max_q=5)
    for which in (0, 1):
        codes, exps = R.to_mxfp4(x[0].double().cpu().numpy())
        c.bits[which][0][-1, :, -1], c.bits[which][1][-1, :, -1] = codes, exps
    c.k, c.v = (R.mxfp4_values(*b) for b in c.bits)
    c.check(out, causal=True, parts=2)
    kv.close()


def test_more_than_2_30_chunks_of_rows():
    """Rows of 1024 heads: 17 GB of them, more workgroups than one dimension of a grid has."""
    import torch
    n_kv, P, tokens = 1024, 16, 2 ** 16 + 40
    kv = _handle(n_kv, P, 8, max_tokens=tokens)
    c = [torch.full(kv.cache_shape, 255, dtype=torch.uint8, device="cuda") for _ in range(2)]
    slots = torch.full((tokens,), -1, dtype=torch.int32, device="cuda")
    at = [0, 5, 2 ** 16 - 1, 2 ** 16, tokens - 1]
    to = [3, 17, 127, 64, 40]
    slots[at] = _i32(to)
    k = torch.zeros((tokens, n_kv, 128), dtype=torch.bfloat16, device="cuda")
    rng = np.random.default_rng(3)
    k[at] = _bf(rng.normal(size=(len(at), n_kv, 128)))
    kv.write(k, k, slots, *c)
    want = R.mxfp4_values(*R.to_mxfp4(k[at].double().cpu().numpy()))
    for cache in c:
        got = _values(cache, P, 128)[np.array(to) // P, :, np.array(to) % P]
        assert np.array_equal(got, want)
    k.fill_(7.0)
    kv.read(slots, *c, k=k, v=False)
    assert np.array_equal(k[at].double().cpu().numpy(), want)
    assert int((k != 0).any(-1).any(-1).sum()) == len(at)
    assert kv.device_errors() == 0
    kv.close()


def test_a_long_prompt_in_a_handle_of_long_contexts():
    """65536 new tokens where contexts may reach 2^20 keys: as over the other caches (whose
    row tiles have 32 rows at least) the call is made, not refused."""
    import torch
    from paper_2608_02438_amd.xpress import PagedKV, XpError
    T, P, hd, nh, n_kv, W = 65536, 256, 128, 32, 8, 40
    kv = PagedKV(nh, n_kv, P, T // P, 1, T, 1 << 20, cache_dtype="mxfp4")
    g = torch.Generator(device="cuda").manual_seed(2)
    q = torch.randn((T, nh, hd), generator=g, device="cuda").bfloat16()
    k, v = (torch.randn((T, n_kv, hd), generator=g, device="cuda").bfloat16() for _ in range(2))
    c = [torch.zeros(kv.cache_shape, dtype=torch.uint8, device="cuda") for _ in range(2)]
    table = torch.full((1, (1 << 20) // P), -1, dtype=torch.int32, device="cuda")
    table[0, :T // P] = torch.arange(T // P, device="cuda")
    slots = torch.arange(T, dtype=torch.int32, device="cuda")
    kv.write(k, v, slots, *c)
    kc, vc = (x.double().cpu().numpy() for x in kv.read(slots, *c))
    out = kv.attend(q, *c, table, _i32([T]), cu_q=_i32([0, T]), max_q=T, window=W)
    assert kv.device_errors() == 0
    for t in (0, 1, 63, 64, 40000, T - 1):
        a = max(t - W + 1, 0)
        o, _, spread, score = R.attend(q[t:t + 1].double().cpu().numpy(), kc[a:t + 1], vc[a:t + 1])
        # tests/_kv.py's bound, one bf16 part
        d = 2 * ((hd + 12) * 2.0 ** -23 * score + 2.0 ** -22) + W * 2.0 ** -23 + 2.0 ** -20
        e = d[..., None] + 2.0 ** -8
        err = np.abs(out[t:t + 1].double().cpu().numpy() - o)
        assert (err <= 2.0 ** -8 * (np.abs(o) + e * spread) + e * spread + 1e-30).all()
    # tiles of 8 rows: their list would not fit 32 bits
    with pytest.raises(XpError):
        kv.attend(q, *c, table, _i32([T]), cu_q=_i32([0, T]), max_q=2, window=W)
    kv.close()


@pytest.mark.parametrize("window,sinks", [(0, 0), (64, 16)])
def test_layer_over_4_bit_pages(window, sinks):
    """The context layer writes its block's rows in 4 bits and attends to them: against
    the oracle's attention inside the oracle's layer, on the pages' values."""
    import synth
    import torch
    from paper_2608_02438_amd.xpress import LAYER_WEIGHT_NAMES, Layer, PagedKV, device_tensor
    ctx, B, P, width = (150, 33), 16, 16, 11
    w = synth.scaled(synth.configs.QWEN_B1, index=951, H=256, B=B, batch=2, n_heads=8,
                     n_kv_heads=2, ffn=256, ctx_len=None, ctx_len_range=None)
    weights = synth.make_layer_weights(w)
    inp = synth.make_layer_inputs(w, c_max=150)
    layer = Layer({k: device_tensor(weights[k]) for k in LAYER_WEIGHT_NAMES}, 256, 8, 2, 256,
                  max_batch=2, max_B=B, max_ctx=150)
    kv = PagedKV(8, 2, P, 2 * width, 2, 150, width * P, cache_dtype="mxfp4")
    order = np.random.default_rng(3).permutation(2 * width).reshape(2, width)
    caches = [torch.full(kv.cache_shape, 255, dtype=torch.uint8, device="cuda") for _ in range(2)]
    kc, vc = (device_tensor(x) for x in (inp.k_cache, inp.v_cache))
    for b, C in enumerate(ctx):
        at = np.arange(C)
        kv.write(kc[b, :C], vc[b, :C], _i32(order[b, at // P] * P + at % P), *caches)
    x, table = device_tensor(inp.x), _i32(order)
    h, _ = layer.forward_paged(x, kv, *caches, table, _i32(ctx), window=window, sinks=sinks)
    again, _ = layer.forward_paged(x, kv, *caches, table, _i32(ctx), window=window, sinks=sinks)
    assert kv.device_errors() == 0 and h.equal(again)
    LP = O.layer_ref.LayerParams.from_arrays(weights, 8, 2, 128)
    r16, rms = O.xpress_ref.round_bf16, O.layer_ref.rmsnorm
    for b, C in enumerate(ctx):
        xb = O.xpress_ref.to_f64(inp.x[b])
        u = r16(rms(xb, LP.g_attn, LP.eps))
        q = rms((u @ LP.Wq.T).reshape(B, 8, 128), LP.g_q, LP.eps)
        q = r16(O.layer_ref.rope(q, C + np.arange(B), LP.theta))
        k, v = (R.gather(_values(c, P, 128), order[b], C + B) for c in caches)
        a = R.attend(q, k, v, True, window, sinks)[0]
        x1 = xb + r16(a.reshape(B, -1)) @ LP.Wo.T
        u2 = r16(rms(x1, LP.g_mlp, LP.eps))
        act = r16(O.xpress_ref.silu(u2 @ LP.Wg.T) * (u2 @ LP.Wu.T))
        ref = x1 + act @ LP.Wd.T
        # the layer parity tests' bar: one bf16 unit at the output's scale
        bar = max(2e-2, 2.0 ** -8 * np.abs(ref).max())
        assert np.abs(h[b].cpu().numpy() - ref).max() <= bar
        # the block's own keys: the layer's, after norm and rotation, within a step of
        # 4 bits (a differently rounded key may take the next code: 2 s) and half of one
        key = rms((u @ LP.Wk.T).reshape(B, 2, 128), LP.g_k, LP.eps)
        key = O.layer_ref.rope(key, C + np.arange(B), LP.theta)
        s = np.repeat(np.abs(key).reshape(B, 2, 4, 32).max(-1) / 3.5, 32, axis=-1)
        assert (np.abs(k[C:] - key) <= 2 * s + 2.0 ** -7 * np.abs(key).max()).all()
    layer.close()
    kv.close()


def test_calls_reject_bad_arguments():
    import torch
    from paper_2608_02438_amd import xpress as X
    c = Call4(1, [20], [1], heads=4, n_kv=2, P=16)
    kv = c.device()
    L = X.load_library()
    p = lambda t: t.data_ptr()  # noqa: E731
    out = torch.zeros((8, 2, 128), dtype=torch.bfloat16, device="cuda")
    base = dict(t=1, s=p(c.dkv), kc=p(c.dk), vc=p(c.dv), ks=None, vs=None, k=p(out), kl=256,
                v=p(out), vl=256)
    r = lambda **k: L.xp_kv_read(kv._h, *dict(base, **k).values(), None)  # noqa: E731
    for kw in (dict(t=-1), dict(t=9), dict(s=None), dict(kc=None), dict(vc=None), dict(kc=p(c.dk) + 8),
               dict(ks=p(c.dkv)), dict(vs=p(c.dkv)), dict(k=None, v=None), dict(k=p(out) + 2),
               dict(v=p(out) + 8), dict(kl=255), dict(vl=260), dict(kl=248)):
        assert r(**kw) == X.XP_EINVAL, kw
        assert L.xp_kv_last_error(kv._h)
    assert r(t=0) == X.XP_OK and r() == X.XP_OK and r(k=None) == X.XP_OK and r(v=None) == X.XP_OK
    s = torch.ones(2, device="cuda")
    bad = [lambda: kv.read(c.dkv.long(), c.dk, c.dv),
           lambda: kv.read(c.dkv, c.dk[:1], c.dv),
           lambda: kv.read(c.dkv, c.dk, c.dv, k=False, v=False),
           lambda: kv.read(c.dkv, c.dk, c.dv, k=out),
           lambda: kv.attend(c.dq, c.dk.view(torch.int8), c.dv, c.dtable, c.dkv),
           lambda: X.PagedKV(4, 2, 16, 10, 1, 1, 1, cache_dtype="mxfp8")]
    for f in bad:
        with pytest.raises(ValueError):
            f()
    for f in (lambda: kv.attend(c.dq, c.dk, c.dv, c.dtable, c.dkv, k_scale=s),
              lambda: kv.write(out[:1], out[:1], c.dkv, c.dk, c.dv, v_scale=s),
              lambda: kv.read(c.dkv, c.dk, c.dv, k_scale=s)):
        with pytest.raises(X.XpError):
            f()
    kv.close()
