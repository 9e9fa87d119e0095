"""Float64 reference of the key/value cache in pages: rotary positions with several axes, attention over a cache, eviction.

Plain numpy, sample by sample and head by head, written from the formulas in include/d3tom.h.  A cache is given as the dense rows of
each sample (the pages are a matter of where the rows lie); `pages` lays them out.
"""
from __future__ import annotations

import numpy as np


def axis_angles(pos, pairs, dh: int, theta: float, own: bool) -> np.ndarray:
    """[rows, dh / 2] angles; pairs behind the last section have none."""
    pos = np.asarray(pos, dtype=np.float64)
    out = np.zeros((pos.shape[0], dh // 2))
    at = 0
    for a, m in enumerate(pairs):
        for u in range(m):
            out[:, at + u] = pos[:, a] * theta ** -(u / m if own else 2.0 * (at + u) / dh)
        at += m
    return out


def rope_axes(x, pos, pairs, theta: float, own: bool) -> np.ndarray:
    """x [rows, heads, dh] turned."""
    x = np.asarray(x, dtype=np.float64)
    half = x.shape[2] // 2
    ang = axis_angles(pos, pairs, x.shape[2], theta, own)[:, None]
    a, b = x[:, :, :half], x[:, :, half:]
    return np.concatenate([a * np.cos(ang) - b * np.sin(ang), b * np.cos(ang) + a * np.sin(ang)], axis=2)


def attend(q, k, v, scale: float, causal: bool):
    """q [m, H, dh] over k, v [n, Hkv, dh]: (o [m, H, dh], lse [m, H], the probabilities added over rows and averaged over heads [n])."""
    q, k, v = (np.asarray(t, dtype=np.float64) for t in (q, k, v))
    (m, H, dh), (n, Hkv) = q.shape, k.shape[:2]
    o, lse, got = np.zeros((m, H, dh)), np.full((m, H), -np.inf), np.zeros(n)
    for i in range(m):
        seen = min(max(n - m + i + 1, 0), n) if causal else n
        if seen == 0:
            continue
        for h in range(H):
            g = h // (H // Hkv)
            x = scale * (k[:seen, g] @ q[i, h])
            top = x.max()
            p = np.exp(x - top)
            z = p.sum()
            lse[i, h] = top + np.log(z)
            o[i, h] = (p / z) @ v[:seen, g]
            got[:seen] += p / z / H
    return o, lse, got


def evict(weight, token, keep: int, first: int, recent: int) -> np.ndarray:
    """Which slot's row each of the remaining slots holds."""
    n = len(weight)
    k = min(max(keep, 0), n)
    newest = int(np.max(token)) if n else 0
    held = [t < first or t > newest - recent for t in np.asarray(token, dtype=np.int64)]
    order = sorted(range(n), key=lambda j: (not held[j], 0.0 if held[j] else -float(weight[j]), j))
    stays = set(order[:k])
    movers = iter([j for j in range(k, n) if j in stays])
    return np.array([j if j in stays else next(movers) for j in range(k)], dtype=np.int64)


def pages(lens, page_size: int, spare: int, rng, behind=-1):
    """(page table int32 [B, entries], number of pages): the samples' pages in no order; entries behind a sample's last page hold `behind`."""
    need = [-(-n // page_size) for n in lens]
    num = sum(need) + spare
    ids = rng.permutation(num)
    table = np.full((len(lens), max(max(need), 1) + 1), behind, dtype=np.int32)
    at = 0
    for b, m in enumerate(need):
        table[b, :m] = ids[at:at + m]
        at += m
    return table, num
