"""Recorded steps in place behind a common prefix, without the host: a sequence that is over leaves length 0, and the step itself makes that the prefix's length
for the one that takes its place, so that no row's place is on the prefix's pages."""
import numpy as np
import pytest

import oracle.tables as ot
import paper_2502_15443_amd as dc

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("prefix,page,seqs", [(21, 16, 5), (64, 32, 40), (1, 16, 3)])
def test_places_that_are_taken_again(prefix, page, seqs):
    print(f"case prefix again prefix={prefix} page={page} seqs={seqs}", flush=True)
    r = np.random.default_rng(2)
    entries, rows = 6, 8 * seqs
    n_prefix = -(-prefix // page)
    n_pages = n_prefix + seqs * entries
    prefix_pages = r.permutation(n_pages)[:n_prefix]
    free = [int(p) for p in r.permutation(n_pages) if p not in prefix_pages]
    state = {"held": [0] * seqs, "pages": [[-1] * entries for _ in range(seqs)], "free": free + [-1] * n_prefix, "queue": (0, len(free))}
    i32 = lambda a: torch.from_numpy(np.array(a, dtype=np.int32)).cuda()  # noqa: E731
    t = {n: i32(v) for n, v in (("lens", state["held"]), ("new", [0] * seqs), ("pages", state["pages"]), ("free", state["free"]), ("queue", [*state["queue"], 0]),
                                ("starts", [0] * (seqs + 1)), ("prefix", prefix_pages))}
    slots = torch.zeros(rows, dtype=torch.int64, device="cuda")
    q = dc.KVRequests(seqs, rows, page, entries, n_pages, held_dev=t["lens"], new_dev=t["new"], pages_in_dev=t["pages"], queue_in_dev=t["queue"], free_dev=t["free"],
                      len_dev=t["lens"], row_start_dev=t["starts"], pages_dev=t["pages"], queue_dev=t["queue"], slot_dev=slots, prefix_len=prefix,
                      prefix_pages_dev=t["prefix"])
    n = dc.kv_tables_workspace(q)
    ws = torch.empty(n, dtype=torch.uint8, device="cuda")
    graph, side = torch.cuda.CUDAGraph(), torch.cuda.Stream()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph, stream=side):
        t["lens"].clamp_(min=prefix)
        dc.kv_tables(q, ws, n, side.cuda_stream)
    over = 0
    for number in range(60):
        new = [-1 if h > prefix + 4 * page else int(r.integers(0, 9)) for h in state["held"]]
        over += sum(n < 0 for n in new)
        t["new"].copy_(i32(new))
        graph.replay()
        torch.cuda.synchronize()
        held = [max(h, prefix) for h in state["held"]]
        want = ot.tables(held, new, state["pages"], state["free"], state["queue"], rows, page, n_pages, prefix, prefix_pages)
        for name, key in (("lens", "lens"), ("pages", "pages"), ("free", "free"), ("queue", "queue"), ("starts", "starts")):
            assert t[name].flatten().tolist() == np.array(want[key]).flatten().tolist(), (number, name)
        assert slots.tolist() == want["slots"]
        mine = {s // page for s in want["slots"] if s >= 0}
        assert not mine & {int(p) for p in prefix_pages}
        state = {"held": want["lens"], "pages": want["pages"], "free": want["free"], "queue": tuple(want["queue"][:2])}
    assert over > 0
