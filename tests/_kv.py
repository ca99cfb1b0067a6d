"""Shared helpers of the paged-cache tests: random calls, the oracle's results for
them, and what rounding may do to the device's."""
import numpy as np

import oracle as O

R = O.kv_ref


def bf16(x):
    return O.xpress_ref.round_bf16(np.asarray(x, dtype=np.float64))


class Call:
    """A random attention call.  kv: keys of each request; ql: its new tokens;
    groups: [(first, end, shared)] with whole pages shared."""

    def __init__(self, seed, kv, ql, heads=4, n_kv=2, hd=128, P=16, cache="bf16", groups=(),
                 spare=3, sigma_q=2.0):
        rng = np.random.default_rng(seed)
        self.kv, self.ql, self.heads, self.n_kv, self.hd, self.P = kv, ql, heads, n_kv, hd, P
        self.cache, self.groups = cache, groups
        n = len(kv)
        need = [R.pages_of(x, P) for x in kv]
        self.n_pages = sum(need) + spare
        pages = list(rng.permutation(self.n_pages))
        self.width = max(max(need, default=1), 1)
        self.table = np.full((max(n, 1), self.width), -1, dtype=np.int32)[:n]
        for b in range(n):
            self.table[b, :need[b]] = [pages.pop() for _ in range(need[b])]
        for s0, s1, shared in groups:
            for b in range(s0 + 1, s1):
                f = min(R.pages_of(shared, P), need[b])
                self.table[b, :f] = self.table[s0, :f]
        shape = (self.n_pages, n_kv, P, hd)
        if cache == "bf16":
            self.k, self.v = (bf16(rng.normal(size=shape)) for _ in range(2))
            self.ks = self.vs = None
        else:
            self.k, self.v = (R.to_e4m3(rng.normal(size=shape) * 100) for _ in range(2))
            self.ks, self.vs = (rng.uniform(0.008, 0.013, size=n_kv).astype(np.float32)
                                for _ in range(2))
        self.total = sum(ql)
        self.q = bf16(rng.normal(size=(self.total, heads, hd)) * sigma_q)
        self.cu = np.concatenate([[0], np.cumsum(ql)]).astype(np.int32)

    # -- the device's side ---------------------------------------------------
    def device(self, shared=False, max_batch=None, max_tokens=None, max_len=None):
        import torch
        from paper_2608_02438_amd.xpress import PagedKV
        self.dt = torch.bfloat16 if self.cache == "bf16" else torch.float8_e4m3fn
        kv = PagedKV(self.heads, self.n_kv, self.P, self.n_pages,
                     max_batch=max_batch or max(len(self.kv), 1),
                     max_tokens=max_tokens or max(self.total, 1),
                     max_len=max_len or self.width * self.P, head_dim=self.hd, cache_dtype=self.dt,
                     shared=shared)
        t = lambda x, d: torch.tensor(np.ascontiguousarray(x)).to(d).cuda()  # noqa: E731
        self.dk, self.dv = t(self.k, self.dt), t(self.v, self.dt)
        self.dq = t(self.q, torch.bfloat16)
        self.dtable, self.dkv = t(self.table, torch.int32), t(np.array(self.kv), torch.int32)
        self.dcu = t(self.cu, torch.int32)
        self.dks = None if self.ks is None else t(self.ks, torch.float32)
        self.dvs = None if self.vs is None else t(self.vs, torch.float32)
        if self.groups:
            starts = [g[0] for g in self.groups] + [self.groups[-1][1]]
            assert starts[1:-1] == [g[1] for g in self.groups[:-1]]
            self.dgs = t(np.array(starts), torch.int32)
            self.dgl = t(np.array([g[2] for g in self.groups]), torch.int32)
        return kv

    def run(self, kv, shared=False, q=None, **kw):
        args = [self.dq if q is None else q, self.dk, self.dv, self.dtable, self.dkv]
        kw = dict(dict(cu_q=self.dcu, max_q=max(self.ql, default=0), k_scale=self.dks,
                       v_scale=self.dvs), **kw)
        if shared:
            return kv.attend_shared(*args, self.dgs, self.dgl, **kw)
        return kv.attend(*args, **kw)

    # -- the oracle's side ---------------------------------------------------
    def rows(self, max_q=None):
        """Rows of a sequence's (or group's) tile: decides the numerators' parts."""
        return (max_q or max(self.ql, default=0)) * (self.heads // self.n_kv)

    def oracle(self, requests=None, **kw):
        """{request: (out, lse, bound of out, bound of lse)}; parts = 1 or 2 bf16
        parts of the numerators."""
        parts = kw.pop("parts")
        res = {}
        for b in range(len(self.kv)) if requests is None else requests:
            m, n = self.ql[b], self.kv[b]
            if m == 0:
                continue
            k, v = (R.gather(x, self.table[b], n) for x in (self.k, self.v))
            if self.ks is not None:
                k = k * self.ks.astype(np.float64)[None, :, None]
                v = v * self.vs.astype(np.float64)[None, :, None]
            q = self.q[self.cu[b]:self.cu[b + 1]]
            out, lse, spread, score = R.attend(q, k, v, **kw)
            # A weight's relative error d: the scores' fp32 sums (hd terms, bounded by
            # their absolute values), their scaling and the exponent's rounding (each
            # half a step, 2^-24, of at most three times the scores), the exponential
            # (2^-22); it enters the numerator and the sum, beside the sums' own fp32
            # roundings (a term for every key) and the merges of parts (2^-20).  The
            # numerators' bf16 parts: 2^-8 for one, 2^-16 for two.  Last, half a step
            # of the bf16 output (2^-8).
            d = (self.hd + 12) * 2.0 ** -24 * 2 * score + 2.0 ** -22
            d = 2 * d + 2 * n * 2.0 ** -24 + 2.0 ** -20
            c = d[..., None] + (2.0 ** -8 if parts == 1 else 2.0 ** -16)
            bound = 2.0 ** -8 * (np.abs(out) + c * spread) + c * spread + 1e-30
            res[b] = (out, lse, bound, d + 2.0 ** -21 * (1 + np.abs(np.where(np.isinf(lse), 0, lse))))
        return res

    def check(self, out, lse=None, requests=None, **kw):
        out = out.float().cpu().numpy().astype(np.float64)
        worst = 0.0
        for b, (o, l, eb, el) in self.oracle(requests, **kw).items():
            got = out[self.cu[b]:self.cu[b + 1]]
            assert np.isfinite(got).all(), f"request {b}: not finite"
            r = (np.abs(got - o) / eb).max()
            assert r <= 1, f"request {b}: {r:.3g} times the bound"
            worst = max(worst, r)
            if lse is not None:
                g = lse[self.cu[b]:self.cu[b + 1]].cpu().numpy().astype(np.float64)
                none = np.isinf(l)
                assert (g[none] == -np.inf).all()
                assert (np.abs(g - l)[~none] <= el[~none]).all(), f"request {b}: lse"
        print(f"    worst error {worst:.3f} of the bound", flush=True)


def parts_of(rows, cache="bf16"):
    # the bf16 parts of the numerators: two over a bf16 cache in calls of up to 64
    # rows, else one (its rounding is c's part of the bound above)
    return 2 if rows <= 64 and cache == "bf16" else 1
