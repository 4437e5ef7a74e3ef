"""The 4-bit cache in float64 on the CPU: quantised rows, attention over them
and eviction by accumulated weight.  Shares no code with the kernels.

A row of 128 channels is 4 groups of 32.  Of a group: minimum rounded down to
bf16, the smallest bf16 scale s with 15 s >= fl32(max - minimum), codes by the
exact quotient fl32(x - minimum) / s, ties to even.
"""
from __future__ import annotations

import numpy as np

GROUPS, GROUP = 4, 32


def _bf16_down(x: np.ndarray) -> np.ndarray:
    """float32 values rounded down to bf16 numbers (as float32)."""
    bits = x.astype(np.float32).view(np.uint32)
    cut = bits & np.uint32(0xFFFF0000)
    down = (x < 0) & (cut != bits)
    return np.where(down, cut + np.uint32(0x10000), cut).astype(np.uint32).view(np.float32)


def _next_bf16(x: np.ndarray) -> np.ndarray:
    """The next larger bf16 of non-negative bf16 numbers."""
    return (x.view(np.uint32) + np.uint32(0x10000)).view(np.float32)


def quantise(x: np.ndarray):
    """Codes [.., 128] (0..15), scales and minima [.., 4] (float32 that hold
    bf16 numbers) of float32 rows x [.., 128]."""
    g = np.ascontiguousarray(x, np.float32).reshape(*x.shape[:-1], GROUPS, GROUP)
    with np.errstate(invalid="ignore", over="ignore", divide="ignore"):
        m = _bf16_down(g.min(-1))
        spread = (g.max(-1) - m).astype(np.float32)
        s = _bf16_down((spread / np.float32(15)) * np.float32(0.98))
        for _ in range(8):  # 2 % are at most six bf16 steps
            low = s.astype(np.float64) * 15 < spread.astype(np.float64)
            s = np.where(low, _next_bf16(s), s)
        # no smaller scale holds: the start was below the quotient
        bad = ~np.isfinite(g).all(-1) | ~np.isfinite(spread)
        d = (g - m[..., None]).astype(np.float32).astype(np.float64)
        n = np.rint(d / np.where(s > 0, s, 1)[..., None].astype(np.float64))
    m, s = np.where(bad, np.float32(np.nan), m), np.where(bad, np.float32(np.nan), s)
    n = np.where(bad[..., None] | (s == 0)[..., None], 0, n)
    return n.astype(np.int64).reshape(x.shape), s, m


def values(codes, s, m) -> np.ndarray:
    """What codes stand for, float64."""
    rep = lambda a: np.repeat(np.asarray(a, np.float64), GROUP, -1)  # noqa: E731
    return np.asarray(codes, np.float64) * rep(s) + rep(m)


def pack(codes) -> np.ndarray:
    c = np.asarray(codes).astype(np.uint8)
    return c[..., 0::2] | (c[..., 1::2] << 4)


def unpack(packed) -> np.ndarray:
    p = np.asarray(packed)
    return np.stack([p & 15, p >> 4], -1).reshape(*p.shape[:-1], 128).astype(np.int64)


def attend(q, k, v, visible, scale):
    """One unit: q [R, 128], k and v [n, 128] float64, visible [R, n] bool.
    Returns out [R, 128], lse [R], p [R, n]; slots that a row does not see add
    nothing, whatever they hold."""
    R, n = visible.shape
    out, lse, p = np.zeros((R, 128)), np.full(R, -np.inf), np.zeros((R, n))
    for r in range(R):
        see = np.flatnonzero(visible[r])
        if see.size == 0:
            continue
        with np.errstate(invalid="ignore", over="ignore"):
            z = scale * (k[see] @ q[r])
            top = z.max()
            e = np.exp(z - top)
            p[r, see] = e / e.sum()
            lse[r] = top + np.log(e.sum())
            out[r] = p[r, see] @ v[see]
    return out, lse, p


def evict(positions, weights, budget, sinks, recent):
    """One unit: (destination slots, source slots, new length)."""
    n = len(positions)
    if budget < 0 or budget >= n:
        return np.zeros(0, int), np.zeros(0, int), n
    pos = np.asarray(positions, np.int64)
    forced = (pos < sinks) | (pos > pos.max() - recent)
    w = np.asarray(weights, np.float64)
    rank = sorted(range(n), key=lambda j: (not forced[j], 0 if forced[j] else bool(np.isnan(w[j])),
                                           0.0 if forced[j] or np.isnan(w[j]) else -w[j], j))
    keep = np.zeros(n, bool)
    keep[rank[:budget]] = True
    slot = np.arange(n)
    return slot[~keep & (slot < budget)], slot[keep & (slot >= budget)], budget
