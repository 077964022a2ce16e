"""Oracle of the cache held in 8 bits: numpy, token by token, from the definitions.  Batches are those of oracle.attention.

Keys turn in fp32 with every product and sum rounded (which is what the definition says), so whole numbers and scales have one right value."""
from __future__ import annotations

import numpy as np

from oracle.attention import place_of

LEAST = np.float32(2.0 ** -126)


def sound(s) -> np.float32:
    """A scale as it is read: a number above 0."""
    s = np.float32(s)
    return LEAST if not s > LEAST else min(s, np.float32(2.0 ** 127))


def scale_for(most) -> np.float32:
    """The smallest power of two, 2^-126 at least, of which 127 times is not below `most`."""
    e = -126
    while 127.0 * 2.0 ** e < float(most):
        e += 1
    return np.float32(2.0 ** e)


def rotate32(x: np.ndarray, cos: np.ndarray, sin: np.ndarray, neighbours: bool) -> np.ndarray:
    """One row's heads [heads, head_dim] in fp32 with their first 2 * len(cos) values turned in pairs."""
    x = np.asarray(x, dtype=np.float32)
    y, half = x.copy(), len(cos)
    with np.errstate(invalid="ignore", over="ignore"):
        for i in range(half):
            a, b = (2 * i, 2 * i + 1) if neighbours else (i, i + half)
            y[:, a] = x[:, a] * cos[i] - x[:, b] * sin[i]
            y[:, b] = x[:, b] * cos[i] + x[:, a] * sin[i]
    return y


def whole(x: np.ndarray, scale) -> np.ndarray:
    """The whole numbers nearest to x / scale.  A quotient of two fp32 numbers below 128 that is not the middle between two whole numbers is at least 2^-27 away from it,
    and its rounding in fp64 is off by 2^-47 at most."""
    with np.errstate(invalid="ignore", over="ignore"):
        n = np.clip(np.rint(np.asarray(x, np.float32).astype(np.float64) / np.float64(np.float32(scale))), -127, 127)
    return np.where(np.isnan(n), 0, n).astype(np.int8)


def append(k_pages, v_pages, k_scales, v_scales, batch, block: int, k, v, cos, sin, neighbours, positions=None, max_new=None):
    """(k_pages, v_pages, k_scales, v_scales) after the call; pools int8 [pages, kv_heads, page_tokens, head_dim], scales fp32
    [pages, kv_heads, page_tokens / block]; rows k, v in fp32."""
    pools, scales = (k_pages.copy(), v_pages.copy()), (k_scales.copy(), v_scales.copy())
    n_pages, kv_heads, page_tokens, _ = k_pages.shape
    for b, length in enumerate(batch["lens"]):
        first, end = int(batch["starts"][b]), int(batch["starts"][b + 1])
        rows = end - first if max_new is None else min(end - first, max_new)
        first_pos = int(length) - (end - first)
        groups = {}  # (page, block of the page) -> [(place in the page, row, keys, values)], and whether its first token is the call's
        reaches = {}
        for row in range(first, first + rows):
            pos = first_pos + row - first
            where = place_of(batch, b, pos, page_tokens, n_pages)
            if where is None:
                continue
            key = (where[0], where[1] // block)
            reaches[key] = reaches.get(key, False) or where[1] % block == 0
            groups.setdefault(key, [])
            x = np.asarray(k[row], np.float32)
            if cos is not None and cos.shape[1]:
                at = pos if positions is None else int(positions[row])
                if not 0 <= at < len(cos):
                    continue
                x = rotate32(x, cos[at], sin[at], neighbours)
            groups[key].append((where[1], x, np.asarray(v[row], np.float32)))
        for (page, n), new in groups.items():
            if not new:
                continue
            start = place_of(batch, b, max(first_pos, 0), page_tokens, n_pages)
            for which in (0, 1):
                for h in range(kv_heads):
                    values = np.concatenate([t[1 + which][h] for t in new])
                    finite = np.abs(values[np.isfinite(values)])
                    s = scale_for(finite.max() if len(finite) else 0.0)
                    if not reaches[page, n]:
                        old = sound(scales[which][page, h, n])
                        s = max(s, old)
                        if s != old:  # the tokens before the sequence's first new one
                            numbers = pools[which][page, h, n * block:start[1]].astype(np.float64)  # s is a power of two: exact
                            pools[which][page, h, n * block:start[1]] = np.rint(numbers * np.float64(old) / np.float64(s)).astype(np.int8)
                    for place, kr, vr in new:
                        pools[which][page, h, place] = whole((kr, vr)[which][h], s)
                    scales[which][page, h, n] = s
    return (*pools, *scales)


def values(pages: np.ndarray, scales: np.ndarray) -> np.ndarray:
    """What a pool stands for, in fp64."""
    block = pages.shape[2] // scales.shape[2]
    with np.errstate(invalid="ignore"):
        s = np.vectorize(sound, otypes=[np.float64])(scales)
    return pages.astype(np.float64) * np.repeat(s, block, axis=2)[..., None]
