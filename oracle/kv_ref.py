"""fp64 CPU oracle of the paged context cache: pages and slots from lengths, the
write into the pages, and attention over them.

TEST INFRASTRUCTURE.  Only the test suite imports this module; it shares no code
with the device path.  The paper serves its refiner inside a paged engine and
gives no formula for the cache, so each definition is stated here:

* request b holds ceil((len + add) / P) pages; surplus pages go back to a stack,
  then requests take pages from its top, first come first served;
* a slot is page * P + row, key j of a request is row j % P of its page j // P;
* an 8-bit cache holds the nearest e4m3 value of x / scale, ties to even;
* token i of a request with m tokens and n keys has position p = n - m + i and sees
  key j iff j < n, j <= p (causal) and j > p - window or j < sinks (window > 0);
  o = sum_j softmax_j(scale q.k_j) v_j, 0 where it sees none.
"""
from __future__ import annotations

import numpy as np

F64 = np.float64


def pages_of(tokens, P):
    return -(-tokens // P)


class Pool:
    """Tables and free pages as Python lists; the last free page is the top."""

    def __init__(self, P, free, tables):
        self.P, self.free, self.tables = P, list(free), [list(t) for t in tables]

    def step(self, lens, add, max_pages):
        """One call: (cu, kv_len, slots, requests not served, requests out of range)."""
        P = self.P
        bad = [x < 0 or a < 0 or pages_of(x + a, P) > max_pages for x, a in zip(lens, add)]
        need = [len(t) if w else pages_of(x + a, P)
                for x, a, t, w in zip(lens, add, self.tables, bad)]
        back = []
        for t, m in zip(self.tables, need):
            back += t[m:]
            del t[m:]
        self.free += back[::-1]
        cu, kv_len, slots, unserved, full = [0], [], [], [], False
        for b, (x, a) in enumerate(zip(lens, add)):
            if bad[b]:
                kv_len.append(0)
                cu.append(cu[-1])
                continue
            more = need[b] - len(self.tables[b])
            full = full or more > len(self.free)
            served = more == 0 or not full
            if served:
                self.tables[b] += [self.free.pop() for _ in range(more)]
            else:
                unserved.append(b)
            kv_len.append(x + a if served else x)
            cu.append(cu[-1] + a)
            slots += [self.tables[b][p // P] * P + p % P if served else -1 for p in range(x, x + a)]
        return cu, kv_len, slots, unserved, [b for b, w in enumerate(bad) if w]


def e4m3_values():
    """The 256 values of the type (NaN at 0x7f and 0xff)."""
    out = np.empty(256, dtype=F64)
    for b in range(256):
        e, m = (b >> 3) & 15, b & 7
        v = np.nan if b & 127 == 127 else (m * 2.0 ** -9 if e == 0 else (8 + m) * 2.0 ** (e - 10))
        out[b] = -v if b & 128 else v
    return out


def to_e4m3(x):
    """The nearest e4m3 value of each x (ties to the even code), at most 448; NaN stays."""
    x = np.asarray(x, dtype=F64)
    grid = e4m3_values()[:127]
    mag = np.minimum(np.abs(x), 448.0)
    up = np.clip(np.searchsorted(grid, np.where(np.isnan(mag), 0, mag)), 0, 126)
    down = np.maximum(up - 1, 0)
    far, near = grid[up] - mag, mag - grid[down]
    pick = (far < near) | ((far == near) & (up % 2 == 0))
    return np.where(np.isnan(x), np.nan, np.copysign(np.where(pick, grid[up], grid[down]), x))


def visible(n_keys, m, causal, window, sinks):
    """[m][n_keys] truth values: which keys the m tokens of a request see."""
    p = (n_keys - m + np.arange(m))[:, None]
    j = np.arange(n_keys)[None]
    see = np.ones((m, n_keys), dtype=bool)
    if causal:
        see &= j <= p
    if window:
        see &= (j > p - window) | (j < sinks)
    return see


def attend(q, k, v, causal=True, window=0, sinks=0, scale=None):
    """One request: q [m][heads][hd], k and v [n][n_kv][hd] (its keys in order).
    Returns (out, lse, spread, score): spread = sum_j w_j |v_j| per output element
    and score = the greatest scale sum_d |q_d||k_d| of any visible key per row,
    what the rounding bounds need.  Keys that a row does not see do not enter it."""
    m, heads, hd = q.shape
    n, n_kv, _ = k.shape
    grp = heads // n_kv
    scale = hd ** -0.5 if scale is None else scale
    see = visible(n, m, causal, window, sinks)
    out = np.zeros((m, heads, hd), dtype=F64)
    spread = np.zeros_like(out)
    lse = np.full((m, heads), -np.inf)
    score = np.zeros((m, heads))
    for i in range(m):
        at = np.flatnonzero(see[i])
        if at.size == 0:
            continue
        for h in range(heads):
            kk, vv = k[at, h // grp].astype(F64), v[at, h // grp].astype(F64)
            s = kk @ q[i, h].astype(F64) * scale
            top = s.max()
            e = np.exp(s - top)
            w = e / e.sum()
            out[i, h] = w @ vv
            spread[i, h] = w @ np.abs(vv)
            lse[i, h] = top + np.log(e.sum())
            score[i, h] = (np.abs(kk) @ np.abs(q[i, h].astype(F64))).max() * scale
    return out, lse, spread, score


def gather(cache, table_row, n):
    """The n keys of a request from pages [n_pages][n_kv][P][hd], in order."""
    P = cache.shape[2]
    j = np.arange(n)
    return cache[np.asarray(table_row)[j // P], :, j % P]
