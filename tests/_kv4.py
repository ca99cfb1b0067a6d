"""A random attention call over a 4-bit cache, beside tests/_kv.py's of 16 and 8 bits."""
import numpy as np

import oracle as O
from _kv import Call

R = O.kv_ref


class Call4(Call):
    """k and v hold the values that the pages stand for (their bounds are a bf16
    cache's: the values are exact in bf16); codes and exponents as the oracle packs them.
    spread: the rows' magnitudes are 2^-spread .. 2^spread."""

    def __init__(self, seed, kv, ql, spread=0, **kw):
        super().__init__(seed, kv, ql, **kw)
        rng = np.random.default_rng(seed + 1000)
        self.bits = []
        for name in ("k", "v"):
            x = getattr(self, name)
            if spread:
                x = x * 2.0 ** rng.integers(-spread, spread + 1, size=x.shape[:-1] + (1,))
            codes, exps = R.to_mxfp4(x)
            self.bits.append([codes, exps])
            setattr(self, name, R.mxfp4_values(codes, exps))

    def exponent(self, which, page, row, value, head=slice(None)):
        """A row's exponent bytes (255: NaN throughout)."""
        self.bits[which][1][page, head, row] = value
        x = (self.k, self.v)[which]
        codes, exps = self.bits[which]
        x[page, head, row] = R.mxfp4_values(codes[page, head, row], exps[page, head, row])

    def device(self, shared=False, max_batch=None, max_tokens=None, max_len=None):
        import torch
        from paper_2608_02438_amd.xpress import PagedKV
        kv = PagedKV(self.heads, self.n_kv, self.P, self.n_pages,
                     max_batch=max_batch or max(len(self.kv), 1),
                     max_tokens=max_tokens or max(self.total, 1),
                     max_len=max_len or self.width * self.P, head_dim=self.hd,
                     cache_dtype="mxfp4", shared=shared)
        t = lambda x, d: torch.tensor(np.ascontiguousarray(x)).to(d).cuda()  # noqa: E731
        self.dk, self.dv = (t(R.pack_mxfp4(*b), torch.uint8) for b in self.bits)
        assert self.dk.shape == kv.cache_shape
        self.dq = t(self.q, torch.bfloat16)
        self.dtable, self.dkv = t(self.table, torch.int32), t(np.array(self.kv), torch.int32)
        self.dcu = t(self.cu, torch.int32)
        self.dks = self.dvs = None
        if self.groups:
            starts = [g[0] for g in self.groups] + [self.groups[-1][1]]
            self.dgs = t(np.array(starts), torch.int32)
            self.dgl = t(np.array([g[2] for g in self.groups]), torch.int32)
        return kv


def parts_of4(rows):
    # the bf16 parts of the numerators: two in calls of up to 32 rows, else one
    return 2 if rows <= 32 else 1
