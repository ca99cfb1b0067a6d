"""The token sampler on the device against the fp64 oracle: the same tokens, and their
log probabilities."""
import numpy as np
import pytest

from oracle import sample_ref

pytestmark = pytest.mark.gpu

# A token can differ only where u lies within both sides' rounding (about 2^-46 of the
# greatest weight a token, 2^-50 a sum) of a border between two: with the seeds below
# none does.  Log probabilities: the fp32 result's half step, and 2^-40 before it.


def _sampler(V, rows):
    from paper_2608_02438_amd.xpress import Sampler
    return Sampler(V, rows)


def _t(x, dt):
    import torch
    return torch.tensor(np.ascontiguousarray(x)).to(dt).cuda()


class Rows:
    """Random rows and settings of every kind."""

    def __init__(self, seed, rows, V, dtype="f32", sigma=2.0, ld=None, offset=0, greedy=5):
        import torch
        rng = np.random.default_rng(seed)
        self.dt = torch.float32 if dtype == "f32" else torch.bfloat16
        self.V, self.n = V, rows
        self.wide = _t(rng.normal(size=(rows, (ld or V) + offset)) * sigma, self.dt)
        self.logits = self.wide[:, offset:offset + V]
        self.temp = np.array([0 if greedy and r % greedy == 2 else 1 for r in range(rows)])
        self.T = rng.uniform(0.4, 1.6, size=rows).astype(np.float32)
        self.k = rng.choice([0, 0, 1, 2, 40, V // 2, V, V + 9], size=rows)
        self.p = rng.choice([1.0, 1.0, 0.95, 0.5, 1e-6, 0.9999, 2.0], size=rows).astype(np.float32)
        self.m = rng.choice([0.0, 0.0, 0.02, 0.3, 1.0], size=rows).astype(np.float32)
        self.u = rng.random(rows).astype(np.float32)
        self.u[::7] = np.float32(1 - 2.0 ** -24)

    def args(self):
        import torch
        f = torch.float32
        return dict(temp=_t(self.temp, torch.uint8), temperature=_t(self.T, f),
                    top_k=_t(self.k, torch.int32), top_p=_t(self.p, f), min_p=_t(self.m, f),
                    u=_t(self.u, f))

    def run(self, s, **kw):
        import torch
        lp = torch.full((self.n,), 9.0, device="cuda")
        a = dict(self.args(), **kw)
        ids = s.sample(self.logits, logprob=lp, **a)
        return ids.cpu().numpy(), lp.cpu().numpy()

    def check(self, ids, lp, **drop):
        l = self.logits.double().cpu().numpy()
        for r in range(self.n):
            kw = dict(T=float(self.T[r]), k=int(self.k[r]), p=float(self.p[r]),
                      min_p=float(self.m[r]), u=float(self.u[r]))
            kw.update(drop)
            y, want, _ = sample_ref.sample_row(l[r], bool(self.temp[r]), **kw)
            assert ids[r] == y, f"row {r}: {ids[r]} in place of {y}, {kw}"
            if np.isinf(want):
                assert lp[r] == want
            else:
                assert abs(lp[r] - want) <= 2.0 ** -24 * abs(want) + 2.0 ** -40


@pytest.mark.parametrize("V", [1, 2, 3, 63, 255, 1000, 4096, 4097, 8191, 33001, 151936, 262144])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_sample(V, dtype):
    rows = 40 if V < 30000 else 12
    c = Rows(V, rows, V, dtype)
    s = _sampler(V, rows)
    print(f"sample: V={V} {dtype}", flush=True)
    ids, lp = c.run(s)
    assert s.device_errors() == 0
    c.check(ids, lp)
    again, lp2 = c.run(s)
    assert np.array_equal(ids, again) and np.array_equal(lp, lp2)
    s.close()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("ld,offset", [(5000, 0), (5001, 1), (5003, 2), (5002, 3)])
def test_rows_of_any_distance_and_alignment(dtype, ld, offset):
    c = Rows(ld, 9, 4999, dtype, ld=ld, offset=offset)
    s = _sampler(4999, 16)
    ids, lp = c.run(s)
    c.check(ids, lp)
    s.close()


@pytest.mark.parametrize("levels", [1, 2, 5, 300])
@pytest.mark.parametrize("V", [4, 700, 40000])
def test_equal_logits(V, levels):
    """Ties at every threshold: they stay with top-k, and top-p cuts through them, lowest
    index first."""
    import torch
    c = Rows(V + levels, 30, V, greedy=6)
    rng = np.random.default_rng(levels)
    c.logits = _t(rng.integers(0, levels, size=(30, V)) / 4.0, torch.float32)
    s = _sampler(V, 30)
    print(f"equal logits: V={V} levels={levels}", flush=True)
    ids, lp = c.run(s)
    c.check(ids, lp)
    c.m[:] = 0
    c.k[:] = 0
    for p in (0.25, 0.5, 0.75, 0.1):
        c.p[:] = p
        ids, lp = c.run(s)
        c.check(ids, lp)
    s.close()


@pytest.mark.parametrize("k", [63, 64, 65, 255, 256, 257, 1023, 1024, 1025, 3000, 16384, 16385])
@pytest.mark.parametrize("p", [1.0, 0.9])
def test_top_k_of_any_size(k, p):
    """As many candidates as a wave, a sort or a list holds, and one more or less: of rows in
    which the k-th stands alone, and of rows of few levels, where many tie with it."""
    V = 40000
    c = Rows(k, 6, V, greedy=0)
    c.logits[3:] = (c.logits[3:] * 64).round() / 64
    c.k[:], c.p[:] = k, p
    c.m[::2] = 0.0
    s = _sampler(V, 6)
    ids, lp = c.run(s)
    assert s.device_errors() == 0
    c.check(ids, lp)
    s.close()


def test_two_graphs_of_one_sampler():
    """Two captured calls of different rows share the workspace; replayed in turn, with eager
    calls between."""
    import torch
    V = 30000
    s = _sampler(V, 20)
    cs = [Rows(31, 20, V), Rows(32, 7, V, "bf16", greedy=0)]
    args, outs, graphs = [c.args() for c in cs], [], []
    for c, a in zip(cs, args):
        out = torch.zeros(c.n, dtype=torch.int32, device="cuda")
        lp = torch.zeros(c.n, device="cuda")
        s.sample(c.logits, out=out, logprob=lp, **a)
        torch.cuda.synchronize()
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            s.sample(c.logits, out=out, logprob=lp, **a)
        outs.append((out, lp))
        graphs.append(g)
    for i in (0, 1, 1, 0, 1, 0):
        for c, a in zip(cs, args):                     # other uniforms for both, on the device
            c.u[:] = np.random.default_rng(100 + i).random(c.n).astype(np.float32)
            a["u"].copy_(torch.tensor(c.u))
        out, lp = outs[i]
        out.zero_()
        graphs[i].replay()
        cs[1 - i].run(s)
        cs[i].check(out.cpu().numpy(), lp.cpu().numpy())
    assert s.device_errors() == 0
    s.close()


def test_masked_nan_and_infinite_logits():
    import torch
    from paper_2608_02438_amd import xpress as X
    V = 5000
    c = Rows(3, 14, V)
    l = c.logits.double().cpu().numpy()
    rng = np.random.default_rng(1)
    l[0] = -np.inf
    l[1, :] = np.nan
    l[2, :] = -np.inf                                     # a greedy one
    l[3, rng.random(V) < 0.99] = -np.inf                  # few tokens left
    l[4, :] = -np.inf
    l[4, 4321] = -3e38                                    # one
    l[5, ::3] = np.nan
    l[6, [17, 400, 4999]] = np.inf
    l[7, 100] = np.inf                                    # greedy
    l[8] = -1e38 * rng.random(V)
    l[9, :] = np.where(np.arange(V) % 2, -0.0, 0.0)
    c.logits = _t(l, torch.float32)
    s = _sampler(V, 14)
    ids, lp = c.run(s)
    assert s.device_errors() == X.XP_DEVERR_EMPTY and s.device_errors() == 0
    assert (ids[:3] == -1).all() and np.isneginf(lp[:3]).all()
    c.check(ids, lp)
    s.close()


def test_uniforms_and_temperatures_at_their_ends():
    import torch
    V = 9000
    c = Rows(8, 24, V, greedy=0)
    c.u[:] = np.resize(np.float32([0.0, 2.0 ** -24, 1 - 2.0 ** -24, 0.5]), 24)
    c.T[:] = np.resize(np.float32([1e-30, 1e-3, 30.0, 1e30, 1.0, 3e38]), 24)
    c.logits = c.logits * 0.5
    s = _sampler(V, 24)
    ids, lp = c.run(s)
    assert s.device_errors() == 0
    c.check(ids, lp)
    # beyond: the last token with a weight; below 0 like 0
    one = np.ones(24, dtype=np.float32)
    for u, like in ((1.5, 1.0), (float("nan"), 1.0), (-2.0, 0.0)):
        ids, lp = c.run(s, u=_t(one * np.float32(u), torch.float32))
        c.u[:] = like
        c.check(ids, lp)
    s.close()


@pytest.mark.parametrize("T,scale", [(2.0 ** -126, 2.0 ** -126), (2.0 ** -130, 2.0 ** -128),
                                     (2.0 ** -121, 2.0 ** -120), (2.0 ** 121, 2.0 ** 122),
                                     (3e38, 2.0 ** 126)])
def test_temperatures_near_the_ends_of_fp32(T, scale):
    """Where 1 / T, or a difference of logits that has a weight, passes fp32's range."""
    V = 5000
    c = Rows(21, 24, V, greedy=0)
    c.T[:] = T
    c.logits = (c.logits.double() / 8 * scale).float()
    assert bool(c.logits.isfinite().all())
    s = _sampler(V, 24)
    ids, lp = c.run(s)
    assert s.device_errors() == 0
    c.check(ids, lp)
    s.close()


def test_settings_out_of_range_are_replaced_and_reported():
    import torch
    from paper_2608_02438_amd import xpress as X
    V = 300
    s = _sampler(V, 8)
    for field, values, like, bit in (("T", [0.0, -1.0, np.inf, np.nan], 1.0, X.XP_DEVERR_TEMPERATURE),
                                     ("k", [-1, -2 ** 31, -5, -1], 0, X.XP_DEVERR_FILTER),
                                     ("p", [0.0, -0.5, np.nan, -np.inf], 1.0, X.XP_DEVERR_FILTER),
                                     ("m", [-0.1, 1.5, np.nan, np.inf], 0.0, X.XP_DEVERR_FILTER)):
        c = Rows(11, 8, V, greedy=0)
        getattr(c, field)[:4] = values
        ids, lp = c.run(s)
        assert s.device_errors() == bit
        getattr(c, field)[:4] = like
        c.check(ids, lp)
    s.close()


def test_all_greedy_and_optional_settings():
    import torch
    V = 20000
    c = Rows(12, 10, V, greedy=0)
    s = _sampler(V, 10)
    ids = s.sample(c.logits)
    assert np.array_equal(ids.cpu().numpy(), c.logits.cpu().numpy().argmax(-1))
    a = c.args()
    ids, lp = c.run(s, top_k=None, top_p=None, min_p=None, temperature=None)
    c.check(ids, lp, T=1.0, k=0, p=1.0, min_p=0.0)
    ids, lp = c.run(s, top_k=None)
    c.check(ids, lp, k=0)
    out = torch.full((12,), 7, dtype=torch.int32, device="cuda")
    s.sample(c.logits[:4], temp=a["temp"][:4], u=a["u"][:4], out=out[2:6])
    assert (out[:2] == 7).all() and (out[6:] == 7).all()
    assert s.sample(c.logits[:0]).shape == (0,)
    s.close()


def test_frequencies():
    """200000 uniforms spread evenly give every token its probability to a part in that
    many."""
    import torch
    n, V = 50000, 7
    s = _sampler(V, n)
    l = torch.tensor([0.5, -1.0, 2.0, 0.0, 1.9, -3.0, 1.0], device="cuda").repeat(n, 1)
    u = (torch.arange(n, device="cuda") + 0.5) / n
    one = torch.ones(n, device="cuda")
    kw = dict(temp=one.to(torch.uint8), u=u, temperature=0.8 * one)
    for f, keep in (({}, range(7)), (dict(top_k=(3 * one).int()), (2, 4, 6)),
                    (dict(top_p=0.6 * one), (2, 4)), (dict(min_p=0.2 * one), (2, 4, 6))):
        ids = s.sample(l, **kw, **f).long()
        w = torch.exp(l[0].double() / float(np.float32(0.8)))
        w = torch.tensor([float(w[i]) if i in keep else 0.0 for i in range(7)], dtype=torch.float64)
        got = torch.bincount(ids.cpu(), minlength=7).double()
        # a token's count is off by less than the two borders of its interval
        assert ((got - n * w / w.sum()).abs() <= 2).all()
    s.close()


def test_captured_replayed_and_two_streams():
    import torch
    V = 30000
    c = Rows(21, 6, V)
    s, s2 = _sampler(V, 6), _sampler(V, 6)
    a = c.args()
    eager = s.sample(c.logits, **a).clone()
    st = [torch.cuda.Stream() for _ in range(2)]
    torch.cuda.synchronize()
    outs = []
    for _ in range(5):
        for x, stream in zip((s, s2), st):
            outs.append(x.sample(c.logits, stream=stream, **a))
    torch.cuda.synchronize()
    assert all(o.equal(eager) for o in outs)
    out = torch.zeros(6, dtype=torch.int32, device="cuda")
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        s.sample(c.logits, out=out, **a)
    for i in range(4):
        c.u = np.random.default_rng(i).random(6).astype(np.float32)
        a["u"].copy_(_t(c.u, torch.float32))
        if i == 2:
            c.logits.copy_(c.logits.flip(1))
        out.zero_()
        g.replay()
        torch.cuda.synchronize()
        assert out.equal(s.sample(c.logits, **a))
    s.close()
    s2.close()


def test_targets_for_verification():
    """Greedy targets and a first token feed xp_verify_block and xp_refine_block."""
    import torch
    B, V = 16, 1024
    rng = np.random.default_rng(2)
    l = _t(rng.normal(size=(3, B + 1, V)), torch.float32)
    s = _sampler(V, 64)
    t = s.sample(l.view(-1, V)).view(3, B + 1)
    assert t.dtype == torch.int32 and t.equal(l.argmax(-1).int())
    s.close()


# (rows, V): with 256 CUs a workgroup has rows * chunks / 1024 chunks of 4096 tokens of a
# row, and the last of a row what is left; rows go through the launches 128 at a time
@pytest.mark.parametrize("rows,V,ld,offset", [
    (64, 151936, None, 0),               # two chunks a workgroup
    (64, 135001, 135003, 1),             # two, one in the last; unaligned rows
    (100, 151936, None, 0),              # three, two in the last
    (128, 250000, None, 0),              # seven, six in the last
    (129, 5000, None, 0), (300, 40000, 40001, 0),   # a batch of one row, of 44
    (131, 151936, None, 0)])             # four chunks and two in the last, then one
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_chunks_of_a_workgroup_and_batches_of_rows(rows, V, ld, offset, dtype):
    """Rows, settings and logits all different."""
    print(f"sample: rows={rows} V={V} {dtype}", flush=True)
    c = Rows(rows + V, rows, V, dtype, ld=ld, offset=offset)
    s = _sampler(V, rows)
    ids, lp = c.run(s)
    assert s.device_errors() == 0
    c.check(ids, lp)
    ids = s.sample(c.logits).cpu().numpy()
    assert np.array_equal(ids, c.logits.float().cpu().numpy().argmax(-1))
    for kw, drop in ((dict(top_k=None, top_p=None), dict(k=0, p=1.0)), (dict(top_k=None), dict(k=0)),
                     (dict(top_p=None, min_p=None), dict(p=1.0, min_p=0.0))):
        if rows * V < 10 ** 7:
            ids, lp = c.run(s, **kw)
            c.check(ids, lp, **drop)
    s.close()


@pytest.mark.parametrize("rows,V", [(9, 4999), (9, 151936), (70, 151936)])
@pytest.mark.parametrize("k,p", [(20, 0.8), (20, 1.0), (1000, 0.8), (1000, 0.999), (1000, 1.0), (0, 0.8)])
def test_rows_of_few_tokens_with_a_weight(rows, V, k, p):
    """One to a few tokens far ahead of the others at low temperatures: fewer than k of them
    have a weight."""
    import torch
    c = Rows(rows + V + k, rows, V, greedy=0)
    rng = np.random.default_rng(k)
    l = c.logits.cpu().numpy()
    for r in range(rows):
        at = rng.choice(V, size=(1, 2, 5, 15, 19, 20, 21, 30, 500)[r % 9], replace=False)
        l[r, at] = 40 + rng.random(at.size)
    c.logits = _t(l, torch.float32)
    c.T[:] = rng.uniform(0.2, 0.7, size=rows)
    c.k[:], c.p[:] = k, p
    print(f"peaked rows: rows={rows} V={V} k={k} p={p}", flush=True)
    s = _sampler(V, rows)
    ids, lp = c.run(s)
    assert s.device_errors() == 0
    c.check(ids, lp)
    s.close()


def test_anchors_and_greedy_targets_of_a_block():
    """A first token and greedy targets go from the sampler into refine and verify."""
    import oracle as O
    import synth
    import torch
    from paper_2608_02438_amd.xpress import device_tensor, refiner_from_arrays
    w = synth.configs.TINY_F32
    batch, B, V = 3, w.B, w.V
    w = synth.scaled(w, index=w.index + 900, batch=batch)
    weights, inp = synth.make_weights(w), synth.make_inputs(w)
    ref = refiner_from_arrays(weights, w.H, w.r, V, B, batch)
    s = _sampler(V, batch * (B + 1))
    rng = np.random.default_rng(9)
    first = rng.normal(size=(batch, V)).astype(np.float32)
    anchor = s.sample(_t(first, torch.float32))
    seeds = rng.integers(0, V, size=(batch, B)).astype(np.int32)
    out = ref.refine_block(device_tensor(inp.h), anchor, seed_ids=device_tensor(seeds), K=w.K)
    P = O.Params.from_arrays(weights)
    res = O.refine_batch(P, inp.h, first.argmax(-1).astype(np.int32), inp.temp, inp.u_draft, w.K,
                         seed_ids=seeds)
    want = np.stack([r.ids for r in res.refined])
    assert np.array_equal(out.ids.cpu().numpy(), want)
    target = rng.normal(size=(batch, B + 1, V)).astype(np.float32)
    for b, n in enumerate((0, B // 2, B)):                # tokens that the target agrees with
        target[b, np.arange(n), want[b, :n]] = 9.0
        if n < B:
            target[b, n, want[b, n]] = -9.0
    t = s.sample(_t(target.reshape(-1, V), torch.float32)).view(batch, B + 1)
    n, nxt = ref.verify_block(out.ids, t)
    best = target.argmax(-1)
    for b, accepted in enumerate((0, B // 2, B)):
        assert (int(n[b]), int(nxt[b])) == O.verify_greedy(want[b], best[b])
        assert int(n[b]) == accepted
    ref.close()
    s.close()


def test_calls_reject_bad_arguments():
    import torch
    from paper_2608_02438_amd import xpress as X
    s = _sampler(100, 4)
    L = X.load_library()
    l = torch.zeros((4, 104), device="cuda")
    b = torch.zeros(64, device="cuda")
    p, q = l.data_ptr(), b.data_ptr()
    base = dict(rows=4, dt=X.XP_F32, l=p, ld=104, temp=q, T=q, k=q, tp=q, mp=q, u=q, ids=q, lp=None)
    call = lambda **kw: L.xp_sample(s._h, *dict(base, **kw).values(), None)  # noqa: E731
    for kw in (dict(rows=-1), dict(rows=5), dict(dt=X.XP_E4M3), dict(l=None), dict(l=p + 2),
               dict(ld=99), dict(ids=None), dict(temp=None, u=None), dict(u=None),
               dict(temp=None, T=None, k=None, tp=None, mp=None)):
        assert call(**kw) == X.XP_EINVAL, kw
        assert L.xp_sampler_last_error(s._h)
    assert call(rows=0) == X.XP_OK
    x = torch.zeros((4, 100), device="cuda")
    one = torch.ones(4, device="cuda")
    for f in (lambda: s.sample(x.double()), lambda: s.sample(x[:, :99]), lambda: s.sample(x.cpu()),
              lambda: s.sample(x.t().contiguous().t()), lambda: s.sample(x, temp=one, u=one),
              lambda: s.sample(x, temp=one.byte(), u=one[:3]),
              lambda: s.sample(x, out=one), lambda: s.sample(x, temp=one.byte(), u=one, top_k=one)):
        with pytest.raises(ValueError):
            f()
    for f in (lambda: s.sample(x, u=one), lambda: s.sample(x, top_p=one),
              lambda: s.sample(torch.zeros((5, 100), device="cuda"))):
        with pytest.raises(X.XpError):
            f()
    s.close()
