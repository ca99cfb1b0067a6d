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


@pytest.mark.parametrize("ql,kv_len", [([0, 2, 1, 3], [0, 130, 140, 200]),
                                       ([0, 0, 1, 1], [0, 40, 128, 129]),
                                       ([0, 16, 16, 16, 16, 16, 16, 16], [0] + [300] * 7)])
@pytest.mark.parametrize("hd,cache", [(128, "bf16"), (64, "e4m3")])
def test_shared_prefix_of_a_group_whose_first_requests_have_no_tokens(ql, kv_len, hd, cache):
    """The first request has ended: no keys, no pages in its row of the table."""
    import torch
    n = len(ql)
    # the pages come from a call in which every member holds them
    c = Call(140 + n, [max(x, 128) for x in kv_len], ql, heads=8, n_kv=2, hd=hd, cache=cache, P=16,
             groups=[(0, n, 128)])
    kv = c.device(shared=True)
    c.kv = kv_len
    for b, x in enumerate(kv_len):
        c.dtable[b, R.pages_of(x, 16):] = -1
    c.dkv = _i32(kv_len)
    rows = max(max(ql), c.total) * 4
    for m in (dict(causal=True), dict(causal=False), dict(causal=True, window=40, sinks=20)):
        print(f"first member empty: {ql} hd={hd} {cache} {m}", flush=True)
        out = c.run(kv, shared=True, **m)
        assert kv.device_errors() == 0
        c.check(out, parts=parts_of(rows, cache), **m)
    kv.close()


@pytest.mark.parametrize("starts,lens", [([0, 3, 2, 5], [64, 0, 128]), ([5, 0], [128]),
                                         ([0, 2, 9], [64, 128]), ([-3, 2, 5], [64, 128])])
def test_groups_out_of_order_are_reported_and_attended_alone(starts, lens):
    from paper_2608_02438_amd import xpress as X
    c = Call(150, [200, 210, 195, 260, 300], [1, 2, 3, 1, 2], heads=4, n_kv=2,
             groups=[(0, 2, 128), (2, 5, 128)])
    kv = c.device(shared=True)
    for m in (dict(causal=True), dict(causal=True, window=100, sinks=20)):
        print(f"groups {starts} {m}", flush=True)
        c.dgs, c.dgl = _i32(starts), _i32(lens)
        out = c.run(kv, shared=True, **m)
        assert kv.device_errors() == X.XP_DEVERR_LENGTH
        c.check(out, parts=2, **m)
    kv.close()


@pytest.mark.parametrize("shared", [False, True])
@pytest.mark.parametrize("hd", [64, 128])
@pytest.mark.parametrize("ql", [[1, 2], [40, 70]])
def test_rows_whose_every_score_is_minus_infinity(shared, hd, ql):
    """0 / 0 by the formula: NaN, with a log sum of -inf; not the zeros of a row that
    sees no key.  Rows that see one finite score are not touched by the others."""
    import torch
    c = Call(160 + hd, [ql[0] + 700, ql[1] - 1], ql, heads=4, n_kv=2, hd=hd, P=16,
             groups=[(0, 1, 64), (1, 2, 0)] if shared else ())
    first = 3                                                 # key 3 of request 0 is finite
    c.q[:, :, 0] = np.abs(c.q[:, :, 0]) + 1
    for b in range(2):
        for j in range(c.kv[b]):
            if (b, j) != (0, first):
                c.k[c.table[b, j // 16], :, j % 16, 0] = -np.inf
    kv = c.device(shared=shared)
    lse = torch.empty((c.total, 4), device="cuda")
    for m, some in ((dict(causal=True), True), (dict(causal=True, window=90), False),
                    (dict(causal=True, window=90, sinks=2), False)):
        print(f"infinite scores: hd={hd} ql={ql} shared={shared} {m}", flush=True)
        out = c.run(kv, shared=shared, lse=lse, **m).double().cpu().numpy()
        sums = lse.cpu().numpy()
        a, b = out[:ql[0]], out[ql[0]:]
        if some:                                              # key 3 alone has a weight
            want = c.v[c.table[0, 0], :, first][np.repeat(np.arange(2), 2)]
            np.testing.assert_array_equal(a, np.broadcast_to(want, a.shape))
            assert np.isfinite(sums[:ql[0]]).all()
        else:
            assert np.isnan(a).all() and (sums[:ql[0]] == -np.inf).all()
        # request 1 has a token more than keys: its first one sees none
        assert (b[0] == 0).all() and np.isnan(b[1:]).all()
        assert (sums[ql[0]:] == -np.inf).all()
    kv.close()


@pytest.mark.parametrize("ctx", [[(1 << 20) - 17, 20], [(1 << 20) - 16, 1 << 20], [(1 << 20) + 5, 0],
                                 [(1 << 21) - 16, (1 << 21) - 40]])
def test_layer_over_pages_past_2_to_the_20_keys(ctx):
    """The block's keys are rotated for their own positions.  Pages are used many
    times over, so that a long context takes little memory; the window keeps the
    attention to the last of them."""
    import torch
    import synth
    from paper_2608_02438_amd.xpress import LAYER_WEIGHT_NAMES, Layer, PagedKV, device_tensor
    B, nkv, nh, H, P, batch, width = 16, 2, 4, 256, 256, 2, 1 << 13
    w = synth.scaled(synth.configs.QWEN_B1, index=971, H=H, B=B, batch=batch, n_heads=nh,
                     n_kv_heads=nkv, ffn=256, ctx_len=None, ctx_len_range=None)
    weights, inp = synth.make_layer_weights(w), synth.make_layer_inputs(w, c_max=64)
    layer = Layer({k: device_tensor(weights[k]) for k in LAYER_WEIGHT_NAMES}, H, nh, nkv, 256,
                  max_batch=batch, max_B=B, max_ctx=64)
    x = device_tensor(inp.x)
    kv = PagedKV(nh, nkv, P, 8, batch, batch * B, width * P)
    table = torch.zeros((batch, width), dtype=torch.int32, device="cuda")
    for b in range(batch):                                    # the block's pages: their own
        for j in (ctx[b] // P, (ctx[b] + B - 1) // P):
            table[b, j] = 1 + 3 * b + j % 3
    kc, vc = (torch.randn(kv.cache_shape, device="cuda").to(torch.bfloat16) for _ in range(2))
    print(f"layer: contexts {ctx}", flush=True)
    h, _ = layer.forward_paged(x, kv, kc, vc, table, _i32(ctx), window=64)
    assert kv.device_errors() == 0
    LP = O.layer_ref.LayerParams.from_arrays(weights, nh, nkv, 128)
    r16, rms = O.xpress_ref.round_bf16, O.layer_ref.rmsnorm
    for b in range(batch):
        xb = O.xpress_ref.to_f64(inp.x[b])
        u = r16(rms(xb, LP.g_attn, LP.eps))
        pos = ctx[b] + np.arange(B)
        k = O.layer_ref.rope(rms((u @ LP.Wk.T).reshape(B, nkv, 128), LP.g_k, LP.eps), pos, LP.theta)
        n, lo = ctx[b] + B, max(ctx[b] - 64, 0)
        j = np.arange(lo, n)
        rows = table[b].cpu().numpy()[j // P]
        gk, gv = (a.double().cpu().numpy()[rows, :, j % P] for a in (kc, vc))
        # half a bf16 step and what a differently rounded u moves
        assert np.abs(gk[-B:] - k).max() <= 2.0 ** -7 * np.abs(k).max()
        q = r16(O.layer_ref.rope(rms((u @ LP.Wq.T).reshape(B, nh, 128), LP.g_q, LP.eps), pos, LP.theta))
        a = R.attend(q, gk, gv, True, 64, 0)[0]
        x1 = xb + r16(a.reshape(B, -1)) @ LP.Wo.T
        u2 = r16(rms(x1, LP.g_mlp, LP.eps))
        ref = x1 + r16(O.xpress_ref.silu(u2 @ LP.Wg.T) * (u2 @ LP.Wu.T)) @ LP.Wd.T
        bar = max(2e-2, 2.0 ** -8 * np.abs(ref).max())
        assert np.abs(h[b].cpu().numpy() - ref).max() <= bar
    layer.close()
    kv.close()


def test_scales_out_of_range_are_refused():
    """scale=0 is the C ABI's default, not a scale; others beyond 2^-60 .. 2^60 would
    leave fp32's normal range."""
    import torch
    from paper_2608_02438_amd import xpress as X
    c = Call(170, [40, 50], [1, 1], heads=4, n_kv=2)
    kv = c.device(max_tokens=8)
    out = torch.full_like(c.dq, 7)
    for bad in (0.0, 0, -0.0):
        with pytest.raises(ValueError):
            c.run(kv, scale=bad, out=out)
    for bad in (2.0 ** -61, 2.0 ** 61, 1e-45, 3e38, -1.0, float("nan")):
        with pytest.raises((X.XpError, OverflowError)):
            c.run(kv, scale=bad, out=out)
    torch.cuda.synchronize()
    assert (out == 7).all()
    # scores of next to nothing: the mean of V
    got = c.run(kv, scale=2.0 ** -60).double().cpu().numpy()
    for b, n in enumerate(c.kv):
        v = R.gather(c.v, c.table[b], n)
        mean, spread = (np.repeat(x.mean(0), 2, axis=0) for x in (v, np.abs(v)))
        # the numerators' and the sums' roundings, then half a bf16 step
        assert (np.abs(got[b] - mean) <= 2.0 ** -8 * np.abs(mean) + 2.0 ** -15 * spread).all()
    kv.close()


@pytest.mark.parametrize("hd", [64, 128])
def test_scales_of_8_bit_caches_at_the_ends_of_their_range(hd):
    """2^-60 and 2^60 for each of K and V: writes bit for bit, and attention."""
    import torch
    from paper_2608_02438_amd import xpress as X
    rng = np.random.default_rng(hd)
    ends = np.array([2.0 ** -60, 2.0 ** 60, 1.1 * 2.0 ** -59, 0.9 * 2.0 ** 59], dtype=np.float32)
    kv = X.PagedKV(8, 4, 16, 4, 1, 32, 64, head_dim=hd, cache_dtype=torch.float8_e4m3fn)
    s = ends.astype(np.float64)[None, :, None]
    x = rng.normal(size=(32, 4, hd)) * 100 * s
    x[0, :, :6] = [0.0, -0.0, 3e38, -3e38, 1e-38, np.nan]
    d = torch.tensor(x).to(torch.bfloat16).cuda()
    x = d.double().cpu().numpy()
    c = [torch.zeros(kv.cache_shape, device="cuda").to(torch.float8_e4m3fn) for _ in range(2)]
    sc = torch.tensor(ends).cuda()
    kv.write(d, d, _i32(np.arange(32)), *c, k_scale=sc, v_scale=sc)
    want = R.to_e4m3(x / s)
    for a in c:
        got = a[:2].double().cpu().numpy().transpose(0, 2, 1, 3).reshape(32, 4, hd)
        np.testing.assert_array_equal(got, want)
    # scores by the small scales are next to nothing; V by the large ones far from it
    q = torch.tensor(rng.normal(size=(1, 8, hd))).to(torch.bfloat16).cuda()
    for ks, vs in ((ends[0], ends[1]), (ends[0], ends[0])):
        t = [torch.full((4,), float(e), device="cuda") for e in (ks, vs)]
        out = kv.attend(q, *c, _i32([[0, 1]]), _i32([31]), k_scale=t[0], v_scale=t[1],
                        window=20).double().cpu().numpy()
        v = want[11:31] * np.float64(vs)
        mean, spread = (np.repeat(y.mean(0), 2, axis=0) for y in (v, np.abs(v)))
        # one bf16 part of the numerators, the sums, half a bf16 step
        assert (np.abs(out[0] - mean) <= 2.0 ** -8 * np.abs(mean) + 1.01 * 2.0 ** -8 * spread).all()
    assert kv.device_errors() == 0
    kv.close()


def test_layer_over_pages_rejects_tensors_of_other_types_and_sizes():
    """Before any launch: the kernels read and write as many bytes as the layer's."""
    import torch
    layer, kv, d = _paged_layer(2, 2, 8, [20, 5], "bf16", seed=13)
    new = lambda *shape, t=torch.float32: torch.zeros(shape, dtype=t, device="cuda")  # noqa: E731
    for kw in (dict(x=d["x"].float()), dict(x=d["x"][:, :, :128].contiguous()),
               dict(x=d["x"].transpose(0, 1).contiguous().transpose(0, 1)), dict(x=d["x"].cpu()),
               dict(h_f32=new(2, 8, 256, t=torch.bfloat16)), dict(h_f32=new(1, 8, 256)),
               dict(h_f32=new(2, 8, 512)[:, :, :256]), dict(h_bf16=new(2, 8, 256)),
               dict(h_bf16=new(2, 4, 256, t=torch.bfloat16)), dict(ctx_len=d["cl"].long()),
               dict(ctx_len=d["cl"][:1])):
        a = dict(dict(x=d["x"], kv=kv, k_cache=d["pk"], v_cache=d["pv"], table=d["table"],
                      ctx_len=d["cl"]), **kw)
        with pytest.raises(ValueError):
            layer.forward_paged(**a)
    layer.close()
    kv.close()


def test_outputs_allocated_for_another_stream_are_that_streams():
    """Memory that was just freed on the current stream may still be in use there: a
    call on another stream does not get it for its results."""
    import torch
    c = Call(171, [900, 300], [16, 16], heads=8, n_kv=2)
    kv = c.device()
    layer, lkv, d = _paged_layer(2, 2, 8, [20, 5], "bf16", seed=14)
    want = c.run(kv)
    h32, h16 = layer.forward_paged(d["x"], lkv, d["pk"], d["pv"], d["table"], d["cl"])
    s = torch.cuda.Stream()
    torch.cuda.synchronize()
    for like, call in ((want, lambda: c.run(kv, stream=s)),
                       (h32, lambda: layer.forward_paged(d["x"], lkv, d["pk"], d["pv"], d["table"],
                                                         d["cl"], stream=s))):
        freed = [torch.empty_like(t) for t in (like, h16) for _ in range(20)]
        here = {t.data_ptr() for t in freed}
        del freed
        got = call()
        got = got if isinstance(got, tuple) else (got,)
        assert not here & {t.data_ptr() for t in got}
        s.synchronize()
        for a, b in zip(got, (like, h16)):
            assert a.equal(b)
    layer.close()
    for k in (kv, lkv):
        k.close()


@pytest.mark.parametrize("cache,prefix,window", [("bf16", 80, 0), ("e4m3", 16, 0), ("bf16", 144, 60)])
def test_requests_share_a_prefix_end_and_leave_its_pages_to_the_others(cache, prefix, window):
    """A prefix held by a request of its own; requests that share it take and return
    pages of their own, one ends and an unrelated one takes its pages, a new one joins,
    all end: no page is ever in the pool and in a table, or twice in the pool."""
    import torch
    from paper_2608_02438_amd.xpress import PagedKV
    rng = np.random.default_rng(180 + prefix)
    n, heads, n_kv, hd, P, n_pages, f = 6, 8, 2, 64, 16, 40, prefix // 16
    dt = torch.bfloat16 if cache == "bf16" else torch.float8_e4m3fn
    kv = PagedKV(heads, n_kv, P, n_pages, n, 256, 320, head_dim=hd, cache_dtype=dt, shared=True)
    kc, vc = (torch.full(kv.cache_shape, float("nan"), device="cuda").to(dt) for _ in range(2))
    sc = None if cache == "bf16" else np.array([0.011, 0.009], dtype=np.float32)
    dsc = None if sc is None else torch.tensor(sc).cuda()
    table = torch.full((n, 20), -1, dtype=torch.int32, device="cuda")
    held, pool, pool_n = _i32([0] * n), _i32(rng.permutation(n_pages)), _i32([n_pages])
    lens = torch.zeros(n, dtype=torch.int32, device="cuda")
    past = [[np.zeros((0, n_kv, hd))] * 2 for _ in range(n)]

    def pages_are_whole():
        t, h = table.cpu().numpy(), held.cpu().numpy()
        free = pool[:pool_n.item()].tolist()
        own = [p for b in range(n) for p in t[b, (f if b in sharers else 0):h[b]]]
        assert sorted(free + own) == list(range(n_pages))
        assert all((t[b, :f] == t[0, :f]).all() for b in sharers)

    def step(add, groups):
        T = sum(add)
        cu, kvl, slots = (torch.empty(m, dtype=torch.int32, device="cuda") for m in (n + 1, n, T))
        kv.map(lens, _i32(add), table, held, pool, pool_n, cu=cu, kv_len=kvl, slots=slots)
        q, k, v = (bf16(rng.normal(size=(T, h, hd)) * s) for h, s in
                   ((heads, 2), (n_kv, 1), (n_kv, 1)))
        dq, dk, dv = (torch.tensor(x).to(torch.bfloat16).cuda() for x in (q, k, v))
        kv.write(dk, dv, slots, kc, vc, k_scale=dsc, v_scale=dsc)
        starts, lengths = groups
        out = kv.attend_shared(dq, kc, vc, table, kvl, _i32(starts), _i32(lengths), cu_q=cu,
                               max_q=max(add), window=window, k_scale=dsc, v_scale=dsc)
        assert kv.device_errors() == 0
        pages_are_whole()
        got, at = out.double().cpu().numpy(), 0
        for b in range(n):
            new = slice(at, at + add[b])
            at += add[b]
            w = 1.0 if sc is None else sc.astype(np.float64)[None, :, None]
            past[b] = [np.concatenate([p, x[new] if sc is None else R.to_e4m3(x[new] / w) * w])
                       for p, x in zip(past[b], (k, v))]
            if add[b]:
                o, _, spread, score = R.attend(q[new], *past[b], window=window)
                m = past[b][0].shape[0]
                d = 2 * ((hd + 12) * 2.0 ** -23 * score + 2.0 ** -22) + m * 2.0 ** -23 + 2.0 ** -20
                c = d[..., None] + 2.0 ** -8                  # at most one part's rounding
                assert (np.abs(got[new] - o) <= 2.0 ** -8 * (np.abs(o) + c * spread) + c * spread).all()
        lens.add_(_i32(add))

    sharers = []

    def share(b):
        table[b, :f] = table[0, :f]
        held[b], lens[b] = f, prefix
        past[b] = past[0]
        sharers.append(b)

    def end(bs):
        """All of them at once: their own pages through the map, then held."""
        for b in bs:
            lens[b] = prefix if b in sharers else 0
        kv.map(lens, torch.zeros_like(lens), table, held, pool, pool_n)
        for b in bs:
            if b in sharers:
                held[b] = 0
                sharers.remove(b)
            lens[b] = 0
            past[b] = [x[:0] for x in past[b]]
        pages_are_whole()

    print(f"shared pages: {cache} prefix={prefix} window={window}", flush=True)
    none = ([0, n], [0])
    step([prefix, 0, 0, 0, 0, 33], none)
    for b in (1, 2, 3):
        share(b)
    group = ([0, 4, n], [prefix, 0])
    step([0, 20, 1, 7, 0, 1], group)
    step([0, 1, 16, 7, 0, 1], group)
    end([2])
    step([0, 3, 0, 1, 40, 1], group)                          # request 4 takes its pages
    share(2)
    step([0, 1, 50, 1, 1, 0], group)
    end([1, 2, 5])
    step([0, 0, 0, 5, 1, 0], group)
    end([3])
    end([0, 4])
    assert pool_n.item() == n_pages
    kv.close()


def test_lengths_up_to_whole_pages_are_allowed():
    """max_len stands for its whole pages: in the map, the write and the attention."""
    import torch
    from paper_2608_02438_amd import xpress as X
    c = Call(190, [112, 101], [12, 3], heads=4, n_kv=2, P=16)
    kv = c.device(max_len=100)
    out = c.run(kv)
    assert kv.device_errors() == 0
    c.check(out, causal=True, parts=2)
    wide = torch.cat([c.dtable, c.dtable], dim=1).contiguous()
    c.dkv[1] = 113                                            # the eighth page is past them
    got = kv.attend(c.dq, c.dk, c.dv, wide, c.dkv, cu_q=c.dcu, max_q=12)
    assert kv.device_errors() == X.XP_DEVERR_LENGTH
    assert got[:12].equal(out[:12])
    kv.close()


def test_write_quotients_that_fp32_moves_onto_a_middle():
    """Scales next to x / middle for all bf16 significands x and all middles between two
    neighbouring e4m3 values, subnormal ones among them: an fp32 quotient lies on the
    middle where the true one does not, and goes to the even neighbour."""
    import torch
    from paper_2608_02438_amd import xpress as X
    heads, hd, P = 1024, 64, 16
    grid = R.e4m3_values()[:127]
    mid = (grid[1:] + grid[:-1]) / 2
    x, m = (a.ravel() for a in np.meshgrid(np.arange(128, 256) * 2.0 ** -7, mid))
    near = (x / m).astype(np.float32)
    s = np.concatenate([near, np.nextafter(near, np.float32(0)), np.nextafter(near, np.float32(1e9))])
    x, s = np.concatenate([x] * 3), s
    pad = -len(s) % heads
    x, s = (np.concatenate([a, a[:pad]]).reshape(-1, heads) for a in (x, s))
    want = R.to_e4m3(x / s.astype(np.float64))
    once = R.to_e4m3((x.astype(np.float32) / s).astype(np.float64))
    assert (once != want).mean() > 0.1                        # what rounding twice would give
    kv = X.PagedKV(heads, heads, P, 1, 1, 1, P, head_dim=hd, cache_dtype=torch.float8_e4m3fn)
    c = [torch.zeros(kv.cache_shape, device="cuda").to(torch.float8_e4m3fn) for _ in range(2)]
    sign = torch.tensor([1.0, -1.0], device="cuda").repeat(hd // 2)
    for i in range(len(s)):
        d = (torch.tensor(x[i]).cuda()[None, :, None] * sign).to(torch.bfloat16)
        sc = torch.tensor(s[i]).cuda()
        kv.write(d, d, _i32([i % P]), *c, k_scale=sc, v_scale=sc)
        got = [a[0, :, i % P].double().cpu().numpy() for a in c]
        for g in got:
            np.testing.assert_array_equal(g[:, 0::2], np.repeat(want[i][:, None], hd // 2, 1))
            np.testing.assert_array_equal(g[:, 1::2], -g[:, 0::2])
    kv.close()


@pytest.mark.parametrize("cap,cache,shared", [(24, "bf16", False), (24, "e4m3", True), (5200, "bf16", False)])
def test_captured_step_of_all_calls(cap, cache, shared):
    """Map with lengths advanced in place, write, attention: one graph replayed step by
    step beside the same calls made eagerly on buffers of their own, with accepted
    lengths in between; a padded batch."""
    import torch
    from paper_2608_02438_amd.xpress import PagedKV
    n, heads, n_kv, hd, P, n_pages, width = 3, 8, 2, 128, 16, 80, 24
    dt = torch.bfloat16 if cache == "bf16" else torch.float8_e4m3fn
    g = torch.Generator(device="cuda").manual_seed(cap)
    sc = None if cache == "bf16" else torch.full((n_kv,), 0.02, device="cuda")
    q, k, v = (torch.empty(cap, h, hd, dtype=torch.bfloat16, device="cuda")
               for h in (heads, n_kv, n_kv))
    lens0, add, back = _i32([0, 0, 0]), _i32([0, 0, 0]), _i32([0, 0, 0])

    class Side:
        def __init__(self):
            self.kv = PagedKV(heads, n_kv, P, n_pages, n, cap, width * P, head_dim=hd,
                              cache_dtype=dt, shared=shared)
            self.c = [torch.zeros(self.kv.cache_shape, device="cuda").to(dt) for _ in range(2)]
            self.table = torch.full((n, width), -1, dtype=torch.int32, device="cuda")
            self.held, self.pool, self.pool_n = _i32([0] * n), _i32(range(n_pages)), _i32([n_pages])
            self.lens, self.cu = lens0.clone(), _i32([0] * (n + 1))
            self.slots = torch.zeros(cap, dtype=torch.int32, device="cuda")
            self.out = torch.zeros_like(q)
            self.starts, self.common = _i32([0, n]), _i32([0])

        def step(self):
            self.lens.sub_(back)                              # what verification rejected
            self.kv.map(self.lens, add, self.table, self.held, self.pool, self.pool_n, cu=self.cu,
                        kv_len=self.lens, slots=self.slots)
            self.kv.write(k, v, self.slots, *self.c, k_scale=sc, v_scale=sc)
            a = (q, *self.c, self.table, self.lens)
            kw = dict(cu_q=self.cu, max_q=8, k_scale=sc, v_scale=sc, out=self.out)
            if shared:
                self.kv.attend_shared(*a, self.starts, self.common, **kw)
            else:
                self.kv.attend(*a, **kw)

    a, b = Side(), Side()
    warm = Side()
    warm.step()
    graph = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        b.step()
    for new, less in (([8, 1, 5], [0, 0, 0]), ([8, 8, 8], [0, 0, 5]), ([1, 8, 0], [7, 1, 3]),
                      ([8, 0, 8], [0, 4, 0]), ([8, 8, 8], [8, 0, 2])):
        print(f"captured step: cap={cap} {cache} add={new}", flush=True)
        for t in (q, k, v):
            t.normal_(generator=g)
        add.copy_(_i32(new))
        back.copy_(_i32(less))
        a.step()
        graph.replay()
        torch.cuda.synchronize()
        used = sum(new)
        for x, y in ((a.lens, b.lens), (a.cu, b.cu), (a.slots, b.slots), (a.table, b.table),
                     (a.held, b.held), (a.pool_n, b.pool_n), (a.out[:used], b.out[:used])):
            assert x.equal(y)
        assert all(x.view(torch.uint8).equal(y.view(torch.uint8)) for x, y in zip(a.c, b.c))
        assert (a.slots[used:] == -1).all() and a.out[:used].abs().max() > 0
        assert a.kv.device_errors() == 0 and b.kv.device_errors() == 0
    for s in (a, b, warm):
        s.kv.close()


def _check_fp16_parts(c, out, **m):
    """The bound of tests/_kv.py with numerators of one fp16 part: 2^-11 of each (half
    a step) and, below 2^-21 of the row's greatest, 2^-25 beside a sum of 2^7 at least."""
    got = out.double().cpu().numpy()
    for b, (o, _, eb, _) in c.oracle(parts=2, **m).items():
        k, v = (R.gather(x, c.table[b], c.kv[b]) for x in (c.k, c.v))
        k, v = (x * s.astype(np.float64)[None, :, None] for x, s in ((k, c.ks), (v, c.vs)))
        q = c.q[c.cu[b]:c.cu[b + 1]]
        spread = R.attend(q, k, v, **m)[2]
        small = 2.0 ** -32 * np.repeat(np.abs(v).sum(0), c.heads // c.n_kv, axis=0)
        more = (2.0 ** -11 * spread + small) * (1 + 2.0 ** -8)
        r = (np.abs(got[c.cu[b]:c.cu[b + 1]] - o) / (eb + more)).max()
        print(f"    request {b}: {r:.3f} of the bound", flush=True)
        assert r <= 1


@pytest.mark.parametrize("hd", [64, 128])
@pytest.mark.parametrize("ql", [[1, 1, 1], [16, 9, 16], [40, 32, 1], [90, 16, 100]])
def test_numerators_over_8_bit_caches_keep_eleven_bits(hd, ql):
    c = Call(200 + hd + sum(ql), [300, 700, 130], ql, heads=4, n_kv=1, hd=hd, cache="e4m3", P=32)
    kv = c.device()
    for m in (dict(causal=True), dict(causal=False, window=200, sinks=5)):
        print(f"fp16 numerators: hd={hd} ql={ql} {m}", flush=True)
        _check_fp16_parts(c, c.run(kv, **m), **m)
    kv.close()


@pytest.mark.parametrize("hd", [64, 128])
@pytest.mark.parametrize("gap", [4, 11, 14, 17])
@pytest.mark.parametrize("late", [False, True])
def test_many_small_numerators_beside_a_great_one(hd, gap, late):
    """One key's score stands gap (in base 2) above 20000 equal ones, which together
    weigh as much or more: in the first tile, or in the last."""
    n = 20000
    c = Call(210 + gap, [n, n], [1, 16], heads=4, n_kv=1, hd=hd, cache="e4m3", P=256)
    c.q[:] = 0.0
    c.q[..., 0] = bf16(gap / 1.4426950408889634 * hd ** 0.5)
    c.ks[:] = 1.0
    c.k[:, :, :, 0] = 0.0
    for b in range(2):
        j = n - 20 if late else 3
        c.k[c.table[b, j // 256], :, j % 256, 0] = 1.0
    # what the small ones bring does not cancel
    c.v = np.abs(c.v)
    kv = c.device()
    print(f"small numerators: hd={hd} gap={gap} late={late}", flush=True)
    _check_fp16_parts(c, c.run(kv, causal=True), causal=True)
    kv.close()


def test_nan_with_a_weight_too_small_for_fp16():
    """A later token's key with NaN in V and a weight of 2^-40: NaN by the formula, for
    whoever sees it."""
    c = Call(220, [90, 64], [4, 64], heads=4, n_kv=1, hd=64, cache="e4m3", P=64)
    c.q[:] = 0.0
    c.q[..., 0] = 8.0
    c.ks[:] = 1.0
    c.k[:, :, :, 0] = 0.0
    for b, n in enumerate((90, 64)):
        c.k[c.table[b, (n - 2) // 64], :, (n - 2) % 64, 0] = -28.0   # 8 * -28 / 8 = -40 in base 2
        c.v[c.table[b, (n - 2) // 64], :, (n - 2) % 64, 5] = np.nan
    kv = c.device()
    out = c.run(kv).double().cpu().numpy()
    for b in range(2):
        got = out[c.cu[b]:c.cu[b + 1]]
        assert np.isfinite(got[:-2]).all() and np.isnan(got[-2:, :, 5]).all()
        assert np.isfinite(np.delete(got[-2:], 5, axis=2)).all()
    kv.close()
