"""A serving step over a 4-bit cache as a program runs it: rows are rotated, written to
their pages, attended to, and a token is drawn from logits; each against the oracle on what
the step before it left on the device."""
import numpy as np
import pytest

import oracle as O
from _kv import bf16
from _kv4 import parts_of4
from oracle import rope_ref, sample_ref

R = O.kv_ref
pytestmark = pytest.mark.gpu


def _i32(x):
    import torch
    return torch.tensor(np.asarray(x), dtype=torch.int32, device="cuda")


def _bf(x):
    import torch
    return torch.tensor(np.ascontiguousarray(x)).to(torch.bfloat16).cuda()


def _f64(x):
    return x.double().cpu().numpy()


def _attend_bound(o, spread, score, hd, n, parts):
    # as tests/_kv.py derives it
    d = 2 * ((hd + 12) * 2.0 ** -23 * score + 2.0 ** -22) + n * 2.0 ** -23 + 2.0 ** -20
    c = d[..., None] + (2.0 ** -8 if parts == 1 else 2.0 ** -16)
    return 2.0 ** -8 * (np.abs(o) + c * spread) + c * spread + 1e-30


@pytest.mark.parametrize("hd,heads,n_kv,window", [(128, 8, 2, 0), (64, 6, 3, 40)])
def test_prompts_then_tokens(hd, heads, n_kv, window):
    """Prompts with image patches (three axes), then single tokens and blocks; a request
    ends and its pages serve another; the vocabulary is a fixed projection of the rows."""
    import torch
    from paper_2608_02438_amd.xpress import PagedKV, Sampler, rope
    rng = np.random.default_rng(hd)
    n, P, V = 4, 16, 3001
    sections = [hd // 4, hd // 8, hd // 8]
    kv = PagedKV(heads, n_kv, P, 40, n, 256, 320, head_dim=hd, cache_dtype="mxfp4")
    sampler = Sampler(V, max_rows=n)
    kc, vc = (torch.full(kv.cache_shape, 255, dtype=torch.uint8, device="cuda") for _ in range(2))
    table = torch.full((n, 20), -1, dtype=torch.int32, device="cuda")
    held, pool, pool_n = _i32([0] * n), _i32(rng.permutation(40)), _i32([40])
    gq, gk = (_bf(1 + 0.1 * rng.normal(size=hd)) for _ in range(2))
    W = _bf(rng.normal(size=(heads * hd, V)) / 8)
    lens = np.zeros(n, dtype=int)
    adds = [np.array([50, 1, 37, 0]), np.ones(n, dtype=int), np.array([1, 1, 1, 90]),
            np.array([5, 5, 5, 5]), np.ones(n, dtype=int)]
    for step, add in enumerate(adds):
        T = int(add.sum())
        cap = T + 3                                           # padded tokens
        cu, kvl = (torch.empty(m, dtype=torch.int32, device="cuda") for m in (n + 1, n))
        slots = torch.empty(cap, dtype=torch.int32, device="cuda")
        kv.map(_i32(lens), _i32(add), table, held, pool, pool_n, cu=cu, kv_len=kvl, slots=slots)
        fused = _bf(rng.normal(size=(cap, (heads + 2 * n_kv) * hd)))
        q, k, v = (fused[:, a * hd:b * hd].unflatten(1, (b - a, hd)) for a, b in
                   ((0, heads), (heads, heads + n_kv), (heads + n_kv, heads + 2 * n_kv)))
        pos = rng.integers(0, 4000, size=(3, cap))
        rq, rk = rope(q, _i32(pos), sections, 1e6, k=k, g_q=gq, g_k=gk, interleaved=True)
        kv.write(rk, v, slots, kc, vc)
        out = kv.attend(rq, kc, vc, table, kvl, cu_q=cu, max_q=int(add.max()), window=window, sinks=3)
        assert kv.device_errors() == 0
        # rotation: half a bf16 step, and 2^-17 of the pair (tests/test_gpu_rope.py's bound)
        for got, x, g in ((rq, q, gq), (rk, k, gk)):
            want, size = rope_ref.rope(_f64(x), pos, sections, 1e6, g=_f64(g),
                                       eps=float(np.float32(1e-6)), interleaved=True)
            assert (np.abs(_f64(got) - want) <= 2.0 ** -8 * np.abs(want) + 2.0 ** -17 * size).all()
        # the cache: every written row is the quantised one
        sl = slots.cpu().numpy()
        back_k, back_v = kv.read(slots, kc, vc)
        for got, x in ((back_k, rk), (back_v, v)):
            want = R.mxfp4_values(*R.to_mxfp4(_f64(x)))
            want[sl < 0] = 0
            assert np.array_equal(_f64(got), want)
        # attention over what the pages hold
        vals = [R.mxfp4_values(*R.unpack_mxfp4(c.cpu().numpy(), P, hd)) for c in (kc, vc)]
        tb, c0 = table.cpu().numpy(), cu.cpu().numpy()
        parts = parts_of4(int(add.max()) * heads // n_kv)
        for b in range(n):
            if add[b]:
                m = lens[b] + add[b]
                o, _, spread, score = R.attend(_f64(rq[c0[b]:c0[b + 1]]), *(
                    R.gather(x, tb[b], m) for x in vals), window=window, sinks=3)
                err = np.abs(_f64(out[c0[b]:c0[b + 1]]) - o)
                assert (err <= _attend_bound(o, spread, score, hd, m, parts)).all()
        # tokens from the last row of every request that has new ones
        last = [c0[b + 1] - 1 for b in range(n) if add[b]]
        logits = torch.matmul(out[last].reshape(len(last), -1), W)
        u = rng.random(len(last)).astype(np.float32)
        kind = rng.integers(0, 2, size=len(last))
        dev = dict(device="cuda")
        ids = sampler.sample(logits, temp=torch.tensor(kind, dtype=torch.uint8, **dev),
                             temperature=torch.full((len(last),), 0.8, **dev),
                             top_k=_i32([50] * len(last)), top_p=torch.full((len(last),), 0.9, **dev),
                             min_p=torch.full((len(last),), 0.02, **dev), u=torch.tensor(u, **dev))
        assert sampler.device_errors() == 0
        T32 = float(np.float32(0.8))
        for r, l in enumerate(_f64(logits)):
            want = sample_ref.sample_row(l, bool(kind[r]), T=T32, k=50, p=float(np.float32(0.9)),
                                         min_p=float(np.float32(0.02)), u=float(u[r]))
            assert int(ids[r]) == want[0]
        lens += add
        if step == 1:
            lens[1] = 0                                       # a request ends
    kv.close()
    sampler.close()


def test_context_moves_on_and_to_another_cache():
    """Keys are read back, rotated to new positions and written to a cache of 16 bits:
    rotated again by d they are those of p + d, up to their 4 bits."""
    import torch
    from paper_2608_02438_amd.xpress import PagedKV, rope
    rng = np.random.default_rng(5)
    n_kv, hd, P, T, d = 2, 128, 32, 77, 1000
    kv4 = PagedKV(4, n_kv, P, 8, 1, 128, 96, cache_dtype="mxfp4")
    kv16 = PagedKV(4, n_kv, P, 8, 1, 128, 96)
    c4 = [torch.zeros(kv4.cache_shape, dtype=torch.uint8, device="cuda") for _ in range(2)]
    c16 = [torch.zeros(kv16.cache_shape, dtype=torch.bfloat16, device="cuda") for _ in range(2)]
    slots, to = (_i32(rng.permutation(8 * P)[:T]) for _ in range(2))
    x = _bf(rng.normal(size=(T, n_kv, hd)))
    pos = _i32(np.arange(T)[None])
    k, _ = rope(x, pos, [hd // 2], 1e6)
    kv4.write(k, x, slots, *c4)
    old, vals = kv4.read(slots, *c4)
    new, _ = rope(old, 0 * pos + d, [hd // 2], 1e6)
    kv16.write(new, vals, to, *c16)
    got, got_v = kv16.read(to, *c16)
    assert got.equal(new) and got_v.equal(vals)
    want, size = rope_ref.rope(_f64(old), np.full((1, T), d), [hd // 2], 1e6)
    assert (np.abs(_f64(got) - want) <= 2.0 ** -8 * np.abs(want) + 2.0 ** -17 * size).all()
    # against the keys rotated for p + d at once: the 4 bits' half step (the greatest of a
    # block over 3.5) of both of a pair's, and two bf16 roundings
    far, _ = rope(x, pos + d, [hd // 2], 1e6)
    half = np.abs(_f64(k)).reshape(T, n_kv, 4, 32).max(-1).repeat(32, axis=-1) / 3.5
    pair = half + np.roll(half, hd // 2, axis=-1)
    assert (np.abs(_f64(got) - _f64(far)) <= pair + 2.0 ** -6 * size).all()
    kv4.close()
    kv16.close()


def test_a_captured_step():
    """Rotation, write, attention and draw in one graph, replayed with other positions,
    lengths and uniforms, eager calls of the same objects in between."""
    import torch
    from paper_2608_02438_amd.xpress import PagedKV, Sampler, rope
    rng = np.random.default_rng(9)
    n, heads, n_kv, hd, P, V = 3, 8, 2, 128, 16, 5000
    kv = PagedKV(heads, n_kv, P, 30, n, n, 160, cache_dtype="mxfp4")
    sampler = Sampler(V, max_rows=n)
    caches = [torch.full(kv.cache_shape, 127, dtype=torch.uint8, device="cuda") for _ in range(2)]
    table = _i32(rng.permutation(30).reshape(3, 10))
    q, k, v = (_bf(rng.normal(size=(n, h, hd))) for h in (heads, n_kv, n_kv))
    W = _bf(rng.normal(size=(heads * hd, V)) / 16)
    lens, pos, slots = _i32([0] * n), _i32([[0] * n]), _i32([0] * n)
    u = torch.zeros(n, device="cuda")
    logits = torch.zeros((n, V), dtype=torch.bfloat16, device="cuda")
    one = torch.ones(n, device="cuda")
    bufs = [torch.zeros_like(q), torch.zeros_like(k), torch.zeros_like(q),
            torch.zeros(n, dtype=torch.int32, device="cuda")]

    def step(b):
        rope(q, pos, [hd // 2], 1e6, k=k, q_out=b[0], k_out=b[1])
        kv.write(b[1], v, slots, *caches)
        kv.attend(b[0], *caches, table, lens, out=b[2])
        torch.matmul(b[2].view(n, -1), W, out=logits)
        sampler.sample(logits, temp=one.to(torch.uint8), top_p=0.8 * one, u=u, out=b[3])

    def put(at, seed):
        lens.copy_(_i32(np.array(at) + 1))
        pos.copy_(_i32([at]))
        slots.copy_(_i32([int(table[b, x // P]) * P + x % P for b, x in enumerate(at)]))
        u.copy_(torch.tensor(np.random.default_rng(seed).random(n).astype(np.float32)))

    put([10, 20, 30], 0)
    step(bufs)
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        step(bufs)
    for i, at in enumerate(([10, 20, 30], [11, 140, 31], [0, 0, 0], [63, 64, 65], [159, 1, 100])):
        put(at, i)
        for b in bufs:
            b.zero_()
        g.replay()
        torch.cuda.synchronize()
        got = [b.clone() for b in bufs]
        eager = [torch.zeros_like(b) for b in bufs]
        step(eager)
        for x, y in zip(got, eager):
            assert x.equal(y)
        assert kv.device_errors() == 0 and sampler.device_errors() == 0
    kv.close()
    sampler.close()
