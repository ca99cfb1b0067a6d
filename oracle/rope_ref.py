"""fp64 CPU oracle of rotary positions of several axes (test infrastructure only): pair j
of a head as the complex number y[j] + i y[j + rot / 2], times e^{i p theta^(-2 j / rot)}
with p the position on the pair's axis, after the RMSNorm over the head."""
from __future__ import annotations

import numpy as np


def axis_of(sections, interleaved):
    """The axis of every pair."""
    axes, half = len(sections), sum(sections)
    if not interleaved:
        return [a for a, n in enumerate(sections) for _ in range(n)]
    return [j % axes if j // axes < sections[j % axes] else 0 for j in range(half)]


def rope(x, pos, sections, theta, g=None, eps=1e-6, interleaved=False):
    """x [tokens][heads][hd], pos [axes][tokens].  Returns (result, |a| + |b| of every
    element's pair after the norm)."""
    y = np.asarray(x, dtype=np.float64)
    if g is not None:
        y = y / np.sqrt((y * y).mean(-1, keepdims=True) + eps) * np.asarray(g, dtype=np.float64)
    half = sum(sections)
    axis = axis_of(sections, interleaved)
    j = np.arange(half)
    angle = np.asarray(pos, dtype=np.float64)[axis].T * float(np.float32(theta)) ** (-j / half)
    z = (y[..., :half] + 1j * y[..., half:2 * half]) * np.exp(1j * angle)[:, None]
    size = np.abs(y[..., :half]) + np.abs(y[..., half:2 * half])
    rest = y[..., 2 * half:]
    return (np.concatenate([z.real, z.imag, rest], -1),
            np.concatenate([size, size, np.abs(rest)], -1))
