"""The paged cache's operators in plain float64 numpy, from their definitions in include/photon.h."""
import numpy as np
import torch


def rotated(x, position, theta):
    """Rows [n, heads, d_h] at positions [n]: pairs (i, i + d_h / 2) by position * theta^(-2 i / d_h); theta 0: as they are."""
    x = np.asarray(x, np.float64)
    if theta == 0:
        return x
    half = x.shape[-1] // 2
    angle = (np.asarray(position, np.float64)[:, None] * np.float64(theta) ** (-2.0 * np.arange(half) / x.shape[-1]))[:, None, :]
    a, b = x[..., :half], x[..., half:]
    return np.concatenate([a * np.cos(angle) - b * np.sin(angle), b * np.cos(angle) + a * np.sin(angle)], -1)


def values(pool):
    """A pool's values as float64 numpy."""
    if pool.dtype == torch.uint8:
        pool = pool.cpu().view(torch.float8_e4m3fn)
    return pool.to(torch.float32).cpu().numpy().astype(np.float64)


def entries(pool, table_row, n, d_h):
    """The first n entries [H_kv, n, d_h] of a sequence, from a pool's values."""
    P = pool.shape[2]
    pages = np.asarray(table_row)[: (n + P - 1) // P]
    return pool[pages].transpose(1, 0, 2, 3).reshape(pool.shape[1], -1, pool.shape[3])[:, :n, :d_h]


def seen(n, m, t, mask=None):
    """Which of a sequence's n entries its query t of m sees: bool [n]."""
    past = n - m
    see = np.arange(n) < past
    for j in range(m):
        if past + j >= 0 and (j <= t if mask is None else (int(mask) >> j) & 1):
            see[past + j] = True
    return see


def attended(q, k, v, see, scale):
    """q [H, d_h], k, v [H_kv, n, d_h], see [n] -> (out [H, d_h], sum of weight * |v| [H, d_h]); entries not seen are not touched."""
    H, d_h = q.shape
    group = H // k.shape[0]
    out, size = np.zeros((H, d_h)), np.zeros((H, d_h))
    if not see.any():
        return out, size
    for h in range(H):
        kk, vv = k[h // group][see], v[h // group][see]
        with np.errstate(invalid="ignore", over="ignore"):
            score = kk @ q[h].astype(np.float64) * scale
            p = np.exp(score - score.max())
            p /= p.sum()
            out[h], size[h] = (p[:, None] * vv).sum(0), (p[:, None] * np.abs(vv)).sum(0)
    return out, size


def tree_masks(parents):
    """Ancestors of every node as int64 words (bit t of node t set), and depths, from parents [T] (-1: a root)."""
    mask, depth = [], []
    for t, p in enumerate(parents):
        mask.append((mask[p] if p >= 0 else 0) | (1 << t))
        depth.append(depth[p] + 1 if p >= 0 else 0)
    return np.array(mask, np.uint64).astype(np.int64), np.array(depth)


def table_of(rng, lengths, P, spare=2, width=None):
    """A table that hands out pages in no order, -1 behind a sequence's last: (table int32 [Bt, width], number of pages)."""
    held = [(n + P - 1) // P for n in lengths]
    n_pages = sum(held) + spare
    order = rng.permutation(n_pages)
    table = np.full((len(lengths), max(1, max(held)) if width is None else width), -1, np.int32)
    at = 0
    for b, h in enumerate(held):
        table[b, :h] = order[at : at + h]
        at += h
    return table, n_pages
