"""dc_kv_tables against the oracle through the C ABI: every result is a whole number and has to be the same."""
import numpy as np
import pytest

import oracle.tables as ot
import paper_2502_15443_amd as dc

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

GUARD = 77


class Problem:
    """Requests with a table as a step before may have left it, and the arrays of a call."""

    def __init__(self, seed, seqs, page, entries, held, new, prefix=0, window=0, sinks=0, free=None, n_rows=None, absent=0.0, beyond=0.0, first=None):
        r = np.random.default_rng(seed)
        self.page, self.prefix, self.window, self.sinks = page, prefix, window, sinks
        self.held, self.new = np.array(held, dtype=np.int32), np.array(new, dtype=np.int32)
        f = prefix + np.arange(entries) * page
        there = (f < self.held[:, None]) & (r.random((seqs, entries)) >= absent)
        there |= r.random((seqs, entries)) < beyond  # pages of tokens that were taken back, or beyond the window
        prefix_pages, used = -(-prefix // page), int(there.sum())
        takes = int(np.clip(-(-(np.maximum(self.held, 0) + np.maximum(self.new, 0) - prefix) // page), 0, entries).sum())
        free = takes if free is None else free
        self.n_pages = max(1, prefix_pages + used + free)
        order = r.permutation(self.n_pages).astype(np.int32)
        self.pages = np.full((seqs, entries), -1, dtype=np.int32)
        self.pages[there] = order[prefix_pages:prefix_pages + used]
        self.prefix_pages = order[:prefix_pages]
        self.first = int(r.integers(self.n_pages)) if first is None else first
        self.free = np.full(self.n_pages, -1, dtype=np.int32)
        self.free[(self.first + np.arange(free)) % self.n_pages] = order[prefix_pages + used:][:free]
        self.count = free
        self.n_rows = n_rows or max(1, int(self.new.clip(min=0).sum()))

    def want(self):
        return ot.tables(self.held.tolist(), self.new.tolist(), self.pages.tolist(), self.free.tolist(), (self.first, self.count), self.n_rows, self.page,
                         self.n_pages, self.prefix, self.prefix_pages.tolist(), self.window, self.sinks)

    def device(self, in_place=False, rows=("slots", "positions", "seqs")):
        def guarded(n, dtype=torch.int32):
            w = torch.full((n + 2,), GUARD, dtype=dtype, device="cuda")
            return w, w[1:-1]

        t = lambda a: torch.from_numpy(np.ascontiguousarray(a)).cuda()  # noqa: E731
        seqs, entries = self.pages.shape
        d = {"new": t(self.new), "prefix_pages": t(self.prefix_pages)}
        self.wide = {}
        for name, n in (("pages", seqs * entries), ("free", self.n_pages), ("queue", 3), ("lens", seqs), ("starts", seqs + 1), ("slots", self.n_rows),
                        ("positions", self.n_rows), ("seqs", self.n_rows)):
            self.wide[name], d[name] = guarded(n, torch.int64 if name == "slots" else torch.int32)
        d["free"].copy_(t(self.free))
        queue = torch.tensor([self.first, self.count], dtype=torch.int32)
        if in_place:
            d["pages"].copy_(t(self.pages).flatten())
            d["queue"][:2] = queue.cuda()
            d["lens"].copy_(t(self.held))
            d["pages_in"], d["queue_in"], d["held"] = d["pages"], d["queue"], d["lens"]
        else:
            d["pages_in"], d["queue_in"], d["held"] = t(self.pages), queue.cuda(), t(self.held)
        self.d, self.rows = d, rows
        q = dc.KVRequests(seqs, self.n_rows, self.page, entries, self.n_pages, held_dev=d["held"], new_dev=d["new"], pages_in_dev=d["pages_in"],
                          queue_in_dev=d["queue_in"], free_dev=d["free"], len_dev=d["lens"], row_start_dev=d["starts"], pages_dev=d["pages"],
                          queue_dev=d["queue"], slot_dev=d["slots"] if "slots" in rows else None,
                          position_dev=d["positions"] if "positions" in rows else None, seq_dev=d["seqs"] if "seqs" in rows else None,
                          window=self.window, sinks=self.sinks, prefix_len=self.prefix, prefix_pages_dev=d["prefix_pages"] if self.prefix else None)
        n = dc.kv_tables_workspace(q)
        self.ws = torch.full((n + 64,), 0xA5, dtype=torch.uint8, device="cuda")
        self.n = n
        return q

    def check(self, want=None):
        torch.cuda.synchronize()
        want = want or self.want()
        for name, w in want.items():
            got = self.d[name].cpu().numpy()
            if name in ("slots", "positions", "seqs") and name not in self.rows:
                assert (got == GUARD).all()
                continue
            w = np.array(w).reshape(-1)
            assert np.array_equal(got, w), (name, np.argwhere(got != w)[:4].ravel().tolist(), got[got != w][:4], w[got != w][:4])
        assert all(int(w[0]) == GUARD and int(w[-1]) == GUARD for w in self.wide.values())
        assert (self.ws[self.n:] == 0xA5).all()


def run(*args, in_place=False, stream=None, rows=("slots", "positions", "seqs"), **kw):
    p = Problem(*args, **kw)
    print(f"case tables seqs={p.pages.shape[0]} entries={p.pages.shape[1]} page={p.page} prefix={p.prefix} window={p.window} sinks={p.sinks} free={p.count} "
          f"rows={p.n_rows} in_place={in_place}", flush=True)
    q = p.device(in_place, rows)
    torch.cuda.synchronize()
    dc.kv_tables(q, p.ws, p.n, torch.cuda.current_stream().cuda_stream if stream is None else stream.cuda_stream)
    p.check()
    return p


@pytest.mark.parametrize("page", [16, 32, 64, 128, 256])
@pytest.mark.parametrize("in_place", [False, True])
def test_pages_of_one_sequence(page, in_place):
    for held in (0, 1, page - 1, page, page + 1, 3 * page):
        for new in (0, 1, 2, page, 5 * page + 3, -1):
            run(1, 1, page, 9, [held], [new], in_place=in_place)


def batch(seed, seqs, most_held, most_new):
    r = np.random.default_rng(seed)
    held, new = r.integers(0, most_held + 1, seqs), r.integers(-1, most_new + 1, seqs)
    return held, new


@pytest.mark.parametrize("seqs", [2, 15, 16, 17, 64, 300, 1025, 2100])
@pytest.mark.parametrize("window,sinks", [(0, 0), (1, 0), (40, 5), (100, 64)])
def test_batches(seqs, window, sinks):
    held, new = batch(seqs, seqs, 200, 30)
    run(2, seqs, 16, 16, held, new, window=window, sinks=sinks, in_place=seqs % 2 == 0)


@pytest.mark.parametrize("entries", [1, 63, 64, 65, 1000, 1023, 1024, 1025, 2048, 5000])
@pytest.mark.parametrize("window,sinks", [(0, 0), (700, 40)])
def test_rows_of_the_table(entries, window, sinks):
    # from few runs of entries, one workgroup's, to many
    for seqs in (1, 3, 40):
        held, new = batch(entries + seqs, seqs, entries * 16, entries * 8)
        run(3, seqs, 16, entries, held, new, window=window, sinks=sinks, in_place=seqs == 3)


@pytest.mark.parametrize("seqs,entries", [(31, 7), (32, 256), (63, 7), (64, 256), (65, 9), (31, 300), (32, 512), (33, 257), (22, 700), (16, 1024), (13, 1200)])
@pytest.mark.parametrize("in_place", [False, True])
def test_runs_of_one_workgroup_and_beyond(seqs, entries, in_place):
    for most_new in (1, 63, 200):
        held, new = batch(seqs + most_new, seqs, entries * 16, most_new)
        run(14, seqs, 16, entries, held, new, window=500 * (most_new % 2), sinks=20, in_place=in_place, absent=0.1)
        run(15, seqs, 16, entries, held // 2, new * 8, prefix=33 if most_new > 1 else 0, in_place=in_place)


@pytest.mark.parametrize("prefix", [1, 15, 16, 100])
def test_a_common_prefix(prefix):
    held, new = batch(prefix, 30, 100, 50)
    run(4, 30, 16, 12, held, new, prefix=prefix)
    run(5, 30, 16, 12, held + prefix, new, prefix=prefix, window=30, sinks=prefix // 2)


@pytest.mark.parametrize("free", [0, 1, 7, 40])
@pytest.mark.parametrize("seqs", [4, 60])
def test_pages_that_are_missing(free, seqs):
    held, new = batch(free, seqs, 100, 60)
    p = run(6, seqs, 16, 12, held, new, free=free, in_place=True)
    assert p.want()["queue"][2] > 0 or (seqs, free) == (4, 40)  # four sequences need fewer


def test_entries_that_hold_no_page_or_one_too_many():
    # tokens that were taken back, and pages that were missing before: the first go back, the others stay away
    for seqs in (5, 80):
        held, new = batch(7, seqs, 150, 40)
        run(8, seqs, 16, 14, held, new, absent=0.3, beyond=0.2)
        run(9, seqs, 16, 14, held, new, absent=0.3, beyond=0.2, window=50, sinks=20, in_place=True)


def test_sequences_beyond_their_table():
    run(10, 3, 16, 4, [60, 64, 500], [10, 1, 3])
    run(11, 30, 16, 4, [60] * 30, [10] * 30, in_place=True)


def test_more_rows_than_there_is_room_for():
    for seqs in (4, 50):
        held, new = batch(12, seqs, 50, 20)
        total = int(np.maximum(new, 0).sum())
        for n_rows in (1, total // 2, total - 1, total, total + 1, total + 500):
            run(13, seqs, 16, 8, held, new, n_rows=n_rows)


def test_results_that_are_left_out():
    held, new = batch(14, 20, 50, 20)
    for rows in ((), ("slots",), ("positions",), ("seqs",)):
        run(15, 20, 16, 8, held, new, rows=rows)


def test_numbers_at_the_ends_of_their_range():
    big = 2 ** 31 - 1
    for seqs in (6, 40):
        held = [big, -5, 0, big - 3, -2 ** 31, 100] + [3] * (seqs - 6)
        new = [2, 3, big, 5, 7, -2 ** 31] + [1] * (seqs - 6)
        p = Problem(16, seqs, 16, 8, np.zeros(seqs), np.ones(seqs), n_rows=40)
        p.held, p.new = np.array(held, dtype=np.int32), np.array(new, dtype=np.int32)
        print(f"case tables ends of the range seqs={seqs}", flush=True)
        q = p.device()
        dc.kv_tables(q, p.ws, p.n, torch.cuda.current_stream().cuda_stream)
        torch.cuda.synchronize()
        # a length that no number holds is cut: what belongs to the table is the same
        want = p.want()
        for name in ("pages", "free", "queue", "starts", "seqs"):
            assert np.array_equal(p.d[name].cpu().numpy(), np.array(want[name]).reshape(-1)), name
        assert all(int(w[0]) == GUARD and int(w[-1]) == GUARD for w in p.wide.values())


def test_queues_that_cannot_be_are_survived():
    held, new = batch(17, 20, 50, 20)
    for first, count in ((-1, 5), (2 ** 31 - 1, 2 ** 31 - 1), (-2 ** 31, -7), (3, 10 ** 6)):
        p = Problem(18, 20, 16, 8, held, new)
        p.first, p.count = first, count
        print(f"case tables queue {first} {count}", flush=True)
        q = p.device()
        dc.kv_tables(q, p.ws, p.n, torch.cuda.current_stream().cuda_stream)
        torch.cuda.synchronize()
        assert all(int(w[0]) == GUARD and int(w[-1]) == GUARD for w in p.wide.values())
        assert np.array_equal(p.d["lens"].cpu().numpy(), np.array(p.want()["lens"]))
        assert 0 <= int(p.d["queue"][0]) < p.n_pages and 0 <= int(p.d["queue"][1]) <= p.n_pages


def test_another_stream_and_the_largest_batch():
    held, new = batch(19, 65535, 40, 3)
    run(20, 65535, 16, 3, held, new, stream=torch.cuda.Stream(), n_rows=250000)


def test_many_steps_lose_no_page():
    """A queue that goes round many times: sequences grow, end and begin anew, with a window; what is free and what is held are all pages at every step."""
    seqs, page, entries, window = 40, 16, 16, 60
    for runs_of_entries in (1, 2):  # few runs, and more than one workgroup takes
        p = Problem(21, seqs * runs_of_entries, page, entries, np.zeros(seqs * runs_of_entries), np.zeros(seqs * runs_of_entries), free=150, window=window,
                    sinks=3, n_rows=1200)
        n = seqs * runs_of_entries
        r = np.random.default_rng(22)
        q = p.device(in_place=True)
        for step in range(60):
            p.held = p.d["lens"].cpu().numpy().copy()
            p.new = np.where(p.held > 200, -1, r.integers(-1, 20, n) * (r.random(n) < 0.7)).astype(np.int32)
            p.d["new"].copy_(torch.from_numpy(p.new))
            p.pages = p.d["pages"].cpu().numpy().reshape(n, entries).copy()
            p.free = p.d["free"].cpu().numpy().copy()
            p.first, p.count = p.d["queue"][:2].tolist()
            dc.kv_tables(q, p.ws, p.n, torch.cuda.current_stream().cuda_stream)
            p.check()
            table, (first, count) = p.d["pages"].cpu().numpy(), p.d["queue"][:2].tolist()
            free = p.d["free"].cpu().numpy()[(first + np.arange(count)) % p.n_pages]
            assert sorted(np.concatenate([table[table >= 0], free]).tolist()) == list(range(p.n_pages))


def test_replays_of_a_recorded_call():
    for seqs in (5, 70):
        held, new = batch(23, seqs, 100, 30)
        p = Problem(24, seqs, 16, 12, held, new, window=40, n_rows=1500)
        q = p.device()
        want = p.want()
        side = torch.cuda.Stream()
        torch.cuda.synchronize()
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g, stream=side):
            dc.kv_tables(q, p.ws, p.n, side.cuda_stream)
        for _ in range(4):
            for name in ("pages", "lens", "starts", "slots", "positions", "seqs", "queue"):
                p.d[name].fill_(5)
            p.d["free"].copy_(torch.from_numpy(p.free))
            p.ws[:p.n] = 0x3C
            torch.cuda.synchronize()
            g.replay()
            p.check(want)
