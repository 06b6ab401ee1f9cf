"""The paged cache's operators in plain 64-bit arithmetic (numpy): the oracle of their tests.

Pools: keys [page][kv head][position][feature], values [page][kv head][position / 8][feature][position % 8].
"""
from __future__ import annotations

from typing import List, Optional

import numpy as np


def plan(cached, new, free, table, page: int, max_tokens: int):
    """(q_start, kv_len, positions, slots, n_used, status, table) of a step, request by request."""
    table = np.array(table, dtype=np.int64)
    b, width = table.shape
    q_start, kv_len, status = [0], [], []
    positions, slots = np.zeros(max_tokens, np.int64), np.full(max_tokens, -1, np.int64)
    taken, used, row = 0, 0, 0
    for i in range(b):
        c, n = max(int(cached[i]), 0), max(int(new[i]), 0)
        s = (2 if c + n > width * page else 0) | (4 if row + n > max_tokens else 0)
        have = -(-c // page)
        need = 0 if s else -(-(c + n) // page) - have
        if need and taken + need > len(free):
            s |= 1
        if need and not s:
            table[i, have:have + need] = free[taken:taken + need]
            used = taken + need
        taken += need
        for t in range(row, min(row + n, max_tokens)):
            p = c + t - row
            positions[t] = min(p, 2 ** 31 - 1)
            if not s and table[i, p // page] >= 0:
                slots[t] = table[i, p // page] * page + p % page
        row += n
        q_start.append(min(row, max_tokens))
        kv_len.append(c if s else c + n)
        status.append(s)
    return np.array(q_start), np.array(kv_len), positions, slots, np.array([used]), np.array(status), table


def rotate(x: np.ndarray, cos: np.ndarray, sin: np.ndarray) -> np.ndarray:
    """x [rows, heads, dim], cos, sin [rows, dim / 2]: the pair (i, i + dim / 2) turned."""
    half = x.shape[-1] // 2
    a, b, c, s = x[..., :half], x[..., half:], cos[:, None, :], sin[:, None, :]
    return np.concatenate([a * c - b * s, b * c + a * s], axis=-1)


def store(k_pages: np.ndarray, v_pages: np.ndarray, slots, k: np.ndarray, v: np.ndarray):
    """Keys and values of the rows into their slots, in place."""
    n_pages, _, page, _ = k_pages.shape
    for t, s in enumerate(int(s) for s in slots):
        if 0 <= s < n_pages * page:
            p, o = s // page, s % page
            k_pages[p, :, o] = k[t]
            v_pages[p, :, o // 8, :, o % 8] = v[t]


def gather(k_pages: np.ndarray, v_pages: np.ndarray, row, length: int):
    """(k, v [kv heads, length, dim], there [length]) of one request; positions in holes of its table row are not there."""
    n_pages, g, page, d = k_pages.shape
    k, v, there = np.zeros((g, length, d)), np.zeros((g, length, d)), np.zeros(length, bool)
    for i in range(-(-length // page)):
        p, m = int(row[i]), min(page, length - i * page)
        if 0 <= p < n_pages:
            there[i * page:i * page + m] = True
            k[:, i * page:i * page + m] = k_pages[p, :, :m]
            o = np.arange(m)
            v[:, i * page:i * page + m] = v_pages[p][:, o // 8, :, o % 8].transpose(1, 0, 2)
    return k, v, there


def attention(q, k_pages, v_pages, table, q_start, kv_len, scale: float = 0.0, softcap: float = 0.0, window: int = 0,
              slopes=None, prefix=None):
    """(out, mass, top): outputs of the rows below q_start[-1] (the others are zero), sum_j p_j |v_j| of every output, and the
    largest magnitude a row's scores reach on the way (what their rounding errors are relative to)."""
    t, h, d = q.shape
    g, page, width = k_pages.shape[1], k_pages.shape[2], np.asarray(table).shape[1]
    rep = h // g
    scale = scale or d ** -0.5
    out, mass, top = np.zeros((t, h, d)), np.zeros((t, h, d)), np.zeros((t, h))
    for b in range(len(kv_len)):
        lo, hi = min(int(q_start[b]), t), min(int(q_start[b + 1]), t)
        n, length = hi - lo, max(int(kv_len[b]), 0)
        if n <= 0:
            continue
        keys = min(length, width * page)
        k, v, there = gather(k_pages, v_pages, table[b], keys)
        p, j = (length - n + np.arange(n))[:, None], np.arange(keys)[None, :]
        sees = j <= p
        if window:
            sees &= j > p - window
        if prefix is not None:
            sees |= j < int(prefix[b])
        sees &= there[None, :]
        for head in range(h):
            kk, vv = k[head // rep], v[head // rep]
            x = scale * (q[lo:hi, head] @ kk.T)
            big = abs(scale) * (np.abs(q[lo:hi, head]) @ np.abs(kk).T)
            if softcap:
                x = softcap * np.tanh(x / softcap)
                big = big + softcap
            if slopes is not None:
                x = x + float(slopes[head]) * (j - p)
                big = big + np.abs(float(slopes[head]) * (j - p))
            x, big = np.where(sees, x, -np.inf), np.where(sees, big, 0.0)
            if keys == 0:
                continue
            m = x.max(axis=1, keepdims=True)
            e = np.exp(x - np.where(np.isfinite(m), m, 0.0))
            z = e.sum(axis=1, keepdims=True)
            w = np.divide(e, z, out=np.zeros_like(e), where=z > 0)
            # (a value that a row does not see plays no part, whatever it holds)
            safe = np.where(np.isfinite(vv), vv, 0.0)
            out[lo:hi, head], mass[lo:hi, head] = w @ safe, w @ np.abs(safe)
            for odd in np.nonzero(~np.isfinite(vv).all(axis=1))[0]:
                rows = np.nonzero(sees[:, odd])[0]
                bad = ~np.isfinite(vv[odd])
                with np.errstate(invalid="ignore"):
                    out[lo + rows[:, None], head, np.nonzero(bad)[0][None, :]] += w[rows, odd][:, None] * vv[odd][bad][None, :]
            top[lo:hi, head] = big.max(axis=1)
    return out, mass, top


def pages_of(lengths: List[int], page: int, rng: Optional[np.random.Generator] = None, spare: int = 3):
    """(table, n_pages): distinct pages for requests of these lengths, in random order when rng is given; unused entries -1."""
    counts = [-(-n // page) for n in lengths]
    total = sum(counts) + spare
    order = rng.permutation(total) if rng is not None else np.arange(total)
    table = np.full((len(lengths), max(1, max(counts, default=1))), -1, np.int32)
    at = 0
    for i, c in enumerate(counts):
        table[i, :c] = order[at:at + c]
        at += c
    return table, total
