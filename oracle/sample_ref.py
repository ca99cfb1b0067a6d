"""fp64 CPU oracle of the token sampler.

TEST INFRASTRUCTURE.  Only the test suite imports this module; it shares no code with
the device path.  The rules are section 3.1's sampling at a temperature with the
truncations that serving adds to it, each stated here:

* order: logits descending, equal ones by index; NaN and -inf are no tokens;
* top-k keeps the k first and what ties with the last of them;
* top-p then keeps, in that order, every token before which less than p of the mass
  that top-k left lies;
* min-p then keeps e^{(l - max) / T} >= min_p;
* weights below 2^-46 of the greatest are 0;
* the token is the first in index order at which the kept mass exceeds u times its
  sum, the last one with mass where u is no number below 1.
"""
from __future__ import annotations

import numpy as np


def sample_row(l, sampled, T=1.0, k=0, p=1.0, min_p=0.0, u=0.0):
    """(id, log probability, kept ids)."""
    l = np.asarray(l, dtype=np.float64)
    ok = l > -np.inf                                   # False for NaN
    if not ok.any():
        return -1, -np.inf, []
    top = l[ok].max()
    if not sampled:
        return int(np.flatnonzero(l == top)[0]), 0.0, []
    ids = np.flatnonzero(ok)
    order = ids[np.argsort(-l[ids], kind="stable")]
    with np.errstate(over="ignore", invalid="ignore"):
        x = np.where(l[order] == top, 0.0, (l[order] - top) / T)
    w = np.exp(x)
    w[w < 2.0 ** -46] = 0.0
    keep = np.ones(order.size, dtype=bool)
    if 0 < k < order.size:
        keep = l[order] >= l[order][k - 1]
    if p < 1:
        m = np.where(keep, w, 0.0)
        before = np.concatenate([[0.0], np.cumsum(m)[:-1]])
        keep &= before < p * m.sum()
    if min_p > 0:
        keep &= x >= np.log(min_p)
    full = np.zeros(l.size)
    full[order[keep]] = w[keep]
    upto = np.cumsum(full)
    Z = upto[-1]
    over = np.flatnonzero((upto > u * Z) & (full > 0))
    y = int(over[0]) if over.size else int(np.flatnonzero(full > 0)[-1])
    return y, float(np.log(full[y] / Z)), np.sort(order[keep]).tolist()
