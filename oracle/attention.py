"""Oracle of the cache append and of the attention over a paged cache: numpy in 64 bits, sequence by sequence, from the definitions.

A cache is two arrays [pages, kv_heads, page_tokens, head_dim].  A batch is a dict with ``lens`` (tokens of each sequence), ``starts``
(first row of each sequence and the end of the last), ``pages`` (table [sequences, entries], entries outside the pool are absent),
``prefix_len`` and ``prefix_pages``.
"""
from __future__ import annotations

import numpy as np


def place_of(batch, seq: int, pos: int, page_tokens: int, n_pages: int):
    """(page, place in the page) of a position, or None if it is not there."""
    p0 = batch["prefix_len"]
    if pos < 0:
        return None
    if pos < p0:
        page, place = int(batch["prefix_pages"][pos // page_tokens]), pos % page_tokens
    else:
        i = (pos - p0) // page_tokens
        if i >= batch["pages"].shape[1]:
            return None
        page, place = int(batch["pages"][seq, i]), (pos - p0) % page_tokens
    return (page, place) if 0 <= page < n_pages else None


def rotate(x: np.ndarray, cos: np.ndarray, sin: np.ndarray, neighbours: bool) -> np.ndarray:
    """One row's heads [heads, head_dim] with their first 2 * len(cos) values turned in pairs."""
    y = np.array(x, dtype=np.float64)
    half = len(cos)
    for i in range(half):
        a, b = (2 * i, 2 * i + 1) if neighbours else (i, i + half)
        y[:, a] = x[:, a] * cos[i] - x[:, b] * sin[i]
        y[:, b] = x[:, b] * cos[i] + x[:, a] * sin[i]
    return y


def append(k_pages, v_pages, batch, k, v, q, cos, sin, neighbours, positions=None):
    """(k_pages, v_pages, q_out) after the call, in fp64; rows of q_out that the call leaves alone are NaN."""
    k_pages, v_pages = np.array(k_pages, dtype=np.float64), np.array(v_pages, dtype=np.float64)
    n_pages, _, page_tokens, _ = k_pages.shape
    q_out = None if q is None else np.full(q.shape, np.nan)
    for b, length in enumerate(batch["lens"]):
        first, end = batch["starts"][b], batch["starts"][b + 1]
        for row in range(first, end):
            pos = int(length) - (end - row)
            kr, qr = k[row], None if q is None else q[row]
            if cos is not None and cos.shape[1]:
                at = pos if positions is None else int(positions[row])
                if not 0 <= at < len(cos):
                    continue
                kr = rotate(kr, cos[at], sin[at], neighbours)
                qr = None if q is None else rotate(qr, cos[at], sin[at], neighbours)
            if q is not None:
                q_out[row] = qr
            where = place_of(batch, b, pos, page_tokens, n_pages)
            if where is not None:
                k_pages[where[0], :, where[1]] = kr
                v_pages[where[0], :, where[1]] = v[row]
    return k_pages, v_pages, q_out


def attend(k_pages, v_pages, batch, q, scale: float, window: int = 0, sinks: int = 0):
    """(out, lse, size) for rows q [rows, heads, head_dim]: size has what a rounding error of a row is measured by: the same average
    over |v| ("v"), the largest |scale| * sum |q_i k_i| ("s"), the number of keys ("n") and the sum of |v| over them ("sum")."""
    rows, heads, d = q.shape
    n_pages, kv_heads, page_tokens, _ = k_pages.shape
    group = heads // kv_heads
    out, lse = np.full((rows, heads, d), np.nan), np.full((rows, heads), np.nan)
    size = {"v": np.zeros((rows, heads, d)), "s": np.zeros((rows, heads)), "n": np.zeros(rows), "sum": np.zeros((rows, heads, d))}
    for b, length in enumerate(batch["lens"]):
        first, end = int(batch["starts"][b]), int(batch["starts"][b + 1])
        if first == end:
            continue
        where = [place_of(batch, b, j, page_tokens, n_pages) for j in range(int(length))]
        there = np.array([w is not None for w in where], dtype=bool)
        for row in range(first, end):
            p = int(length) - (end - row)
            j = np.arange(int(length))
            sees = there & (j <= p)
            if window:
                sees &= (j > p - window) | (j < sinks)
            j = np.nonzero(sees)[0]
            out[row], lse[row], size["n"][row] = 0.0, -np.inf, len(j)
            if not len(j):
                continue
            at = np.array([where[i][0] for i in j]), np.array([where[i][1] for i in j])
            k, v = k_pages[at[0], :, at[1]].astype(np.float64), v_pages[at[0], :, at[1]].astype(np.float64)  # [keys, kv_heads, d]
            for h in range(heads):
                kh, vh, qh = k[:, h // group], v[:, h // group], q[row, h].astype(np.float64)
                s = scale * (kh @ qh)
                top = s.max()
                if top == -np.inf:
                    continue
                e = np.exp(s - top)
                out[row, h] = (e @ vh) / e.sum()
                lse[row, h] = top + np.log(e.sum())
                size["v"][row, h] = (e @ np.abs(vh)) / e.sum()
                size["sum"][row, h] = np.abs(vh).sum(0)
                size["s"][row, h] = abs(scale) * (np.abs(kh) @ np.abs(qh)).max()
    return out, lse, size
