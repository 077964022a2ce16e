"""Oracle of a step's tables: one sequence after the other, one entry after the other."""
from __future__ import annotations


def tables(held, new, pages, free, queue, n_rows: int, page_tokens: int, n_pages: int, prefix_len: int = 0, prefix_pages=(), window: int = 0,
           sinks: int = 0) -> dict:
    """pages: rows of entries; free: the ring; queue: (first place, number of free pages).  Everything as lists of whole numbers."""
    ring = [int(p) for p in free]
    first, count = int(queue[0]) % (1 << 32) % n_pages, min(max(int(queue[1]), 0), n_pages)
    taken, back, table, lens, starts = 0, [], [], [], [0]
    slots, positions, seqs = [], [], []
    for b, row in enumerate(pages):
        over = new[b] < 0
        h = 0 if over else max(int(held[b]), 0)
        n = max(int(new[b]), 0)
        out = []
        for i, page in enumerate(row):
            page = int(page)
            f = prefix_len + i * page_tokens
            there = 0 <= page < n_pages
            wanted = f < h + n and (not window or f + page_tokens - 1 > h - window or f < sinks)
            if there and wanted:
                out.append(page)
            elif there:
                out.append(-1)
                back.append(page)
            elif wanted and f >= h:
                out.append(ring[(first + taken) % n_pages] if taken < count else -1)
                taken += 1
            else:
                out.append(-1)
        table.append(out)
        n = min(n, n_rows - starts[-1])
        starts.append(starts[-1] + n)
        lens.append(h + n)
        for p in range(h, h + n):
            at = p if p < prefix_len else p - prefix_len
            i = at // page_tokens
            page = int(prefix_pages[i]) if p < prefix_len else out[i] if i < len(out) else -1
            slots.append(page * page_tokens + at % page_tokens if 0 <= page < n_pages else -1)
            positions.append(p)
            seqs.append(b)
    for j, page in enumerate(back):
        ring[(first + count + j) % n_pages] = page
    got = min(taken, count)
    rest = [-1] * (n_rows - len(slots))
    return {"pages": table, "free": ring, "queue": [(first + got) % n_pages, min(count - got + len(back), n_pages), taken - got], "lens": lens,
            "starts": starts, "slots": slots + rest, "positions": positions + rest, "seqs": seqs + rest}
