"""Block tables made on the GPU against the definition, entry by entry: batches of one sequence to thousands, pools that
run dry, budgets that fill, holes, requests that cannot be, captured graphs, and the way back."""
import numpy as np
import pytest
import torch

from paper_2607_02963_amd import pdec

pytestmark = pytest.mark.gpu


def i32(x):
    return torch.from_numpy(np.ascontiguousarray(np.asarray(x, np.int32))).cuda()


class Pool:
    """A pool with sequences of `lens` keys, their pages in no order; absent: {(sequence, column)} without one."""

    def __init__(self, lens, page, cols, spare, seed=0, absent=()):
        rng = np.random.default_rng(seed)
        used = [-(-max(t, 0) // page) for t in lens]
        self.page, self.P = page, max(sum(used) + spare, 1)
        order, at = rng.permutation(self.P), 0
        self.table = np.full((len(lens), cols), -1, np.int64)
        for s, u in enumerate(used):
            u = min(u, cols)
            self.table[s, :u] = order[at:at + u]
            at += u
        self.free, self.count = np.full(self.P, -9, np.int64), self.P - at
        self.free[:self.count] = order[at:]
        for s, c in absent:
            self.table[s, c] = (-1, self.P, -2 ** 31, 2 ** 31 - 1)[c % 4]
        self.rows = 0

    def there(self, e):
        return 0 <= e < self.P

    def reserve(self, n, lens, room, max_len=0):
        """The definition; returns (cu, positions, slots)."""
        most = max_len or self.table.shape[1] * self.page
        cu, pos, slots, open_ = [0], [], [], True
        for s, (a, t) in enumerate(zip(n, lens)):
            if a < 0 or t < 0 or t + a > most:
                a = 0
            want = [c for c in range(t // self.page, -(-(t + a) // self.page)) if not self.there(self.table[s, c])] if a else []
            open_ = open_ and len(pos) + a <= room and len(want) <= self.count
            if open_ and a:
                for c in want:
                    self.count -= 1
                    self.table[s, c] = self.free[self.count]
                pos += range(t, t + a)
                slots += [self.table[s, x // self.page] * self.page + x % self.page for x in range(t, t + a)]
            cu.append(len(pos))
        return cu, pos, slots

    def release(self, keep, first=None, max_len=0):
        cols = min(self.table.shape[1], -(-(max_len or self.table.shape[1] * self.page) // self.page))
        for s in reversed(range(len(keep))):
            lo, hi = max(first[s], 0) if first is not None else 0, max(keep[s], 0)
            for c in reversed(range(cols)):
                held = max(c * self.page, lo) < min((c + 1) * self.page, hi)
                if not held and self.there(self.table[s, c]):
                    self.free[self.count] = self.table[s, c]
                    self.table[s, c] = -1
                    self.count += 1

    def put(self):
        self.d_table, self.d_free = i32(self.table), i32(self.free)
        self.d_count = [i32([self.count]), i32([-5])]
        return self

    def flip(self):
        self.d_count.reverse()

    def agrees(self):
        assert self.d_count[1].item() == self.count
        assert np.array_equal(self.d_table.cpu().numpy(), self.table)
        assert np.array_equal(self.d_free.cpu().numpy()[:self.count], self.free[:self.count])


def run(pool, n, lens, room, max_len=0, positions=True, slots=True):
    """One reservation on the device, checked."""
    cu = torch.full((len(n) + 1,), -3, dtype=torch.int32, device="cuda")
    pos = torch.full((room,), -4, dtype=torch.int32, device="cuda") if positions else None
    row = torch.full((room,), -4, dtype=torch.int64, device="cuda") if slots else None
    got = pdec.paged_reserve(i32(n), i32(lens), pool.d_table, pool.d_free, *pool.d_count, page_size=pool.page, cu_tokens=cu,
                             positions=pos, slots=row, num_tokens=room, max_len=max_len)
    assert got is cu
    want = pool.reserve(n, lens, room, max_len)
    assert cu.tolist() == want[0]
    for x, w in ((pos, want[1]), (row, want[2])):
        if x is not None:
            assert x[:len(w)].tolist() == w and (x[len(w):] == -4).all()
    pool.agrees()
    return want[0]


def batch(rng, S, page, cols, single=0.5):
    lens = [int(rng.integers(0, cols * page * 3 // 4)) for _ in range(S)]
    n = [1 if rng.random() < single else int(rng.integers(0, cols * page - t + 1)) for t in lens]
    return n, lens


@pytest.mark.parametrize("page", [16, 64, 128])
@pytest.mark.parametrize("S,cols", [(1, 1), (1, 700), (3, 40), (31, 17), (63, 5), (64, 130), (65, 9), (300, 20), (1025, 3), (4100, 2), (2, 1100), (40, 600), (70, 300)])
def test_reserve_and_release_against_the_definition(page, S, cols):
    rng = np.random.default_rng(S + page)
    n, lens = batch(rng, S, page, cols, 0.9 if S > 1000 or cols > 200 else 0.5)
    n[0] = max(n[0], min(cols * page - lens[0], 270 * page))  # a row of many entries
    pool = Pool(lens, page, cols, S * cols + 5, seed=S).put()
    before = pool.table.copy(), pool.free.copy(), pool.count
    run(pool, n, lens, sum(n) + 3)
    pool.flip()
    pdec.paged_release(i32(lens), pool.d_table, pool.d_free, *pool.d_count, page_size=page)
    pool.release(lens)
    pool.agrees()
    # one undoes the other
    assert np.array_equal(pool.table, before[0]) and pool.count == before[2]
    assert np.array_equal(pool.free[:pool.count], before[1][:pool.count])


@pytest.mark.parametrize("S", [7, 64, 200, 3000])
@pytest.mark.parametrize("pages,tokens", [(0.6, 2.0), (2.0, 0.6), (0.5, 0.45), (0.0, 2.0), (2.0, 0.0)])
def test_what_does_not_fit_is_not_served_nor_is_what_follows(S, pages, tokens):
    rng = np.random.default_rng(S)
    page, cols = 16, 12
    n, lens = batch(rng, S, page, cols, 0.7)
    lack = sum(-(-(t + a) // page) - (-(-t // page)) for a, t in zip(n, lens))
    pool = Pool(lens, page, cols, int(lack * pages), seed=S).put()
    cu = run(pool, n, lens, max(int(sum(n) * tokens), 1))
    assert (cu[-1] < sum(n)) == (min(pages, tokens) < 1)


@pytest.mark.parametrize("S", [40, 130])
def test_requests_that_cannot_be_are_passed_over(S):
    page, cols = 32, 6
    rng = np.random.default_rng(S)
    n, lens = batch(rng, S, page, cols)
    for s, (a, t) in {1: (-1, 5), 4: (3, -2), 7: (1, cols * page), 9: (2 ** 31 - 1, 7), 12: (2 ** 31 - 1, 2 ** 31 - 1),
                      15: (5, 160), 20: (-2 ** 31, -2 ** 31), 33: (0, -1)}.items():
        n[s], lens[s] = a, t
    clean = [t if 0 <= t <= cols * page else 0 for t in lens]
    pool = Pool(clean, page, cols, S * cols, seed=3).put()
    run(pool, n, lens, 100000, max_len=150)


def test_entries_that_are_there_stay_and_holes_are_filled():
    """Pages reserved for drafted tokens before, and a page lost from the last one's place."""
    page, lens, n = 16, [40, 33, 0, 100], [30, 2, 50, 1]
    pool = Pool([t + a for t, a in zip(lens, n)], page, 8, 9, absent=[(0, 3), (2, 0), (2, 3), (3, 0)]).put()
    run(pool, n, lens, 200)
    assert pool.table[3, 0] not in range(pool.P)  # not an entry that the new tokens need


@pytest.mark.parametrize("S,cols", [(9, 33), (64, 4), (70, 90), (1500, 7)])
def test_release_of_windows_prefixes_and_ended_sequences(S, cols):
    page = 16
    rng = np.random.default_rng(cols)
    lens = [int(rng.integers(0, cols * page + 1)) for _ in range(S)]
    pool = Pool(lens, page, cols, 3, seed=S, absent=[(s, 1) for s in range(0, S, 5)]).put()
    keep = [int(rng.choice([0, t, t // 2, max(t - 3, 0), -7, 2 ** 31 - 1])) for t in lens]
    first = [int(rng.choice([0, 0, max(t - 40, 0), t, t + 1, -3, 2 ** 31 - 1])) for t in lens]
    pdec.paged_release(i32(keep), pool.d_table, pool.d_free, *pool.d_count, page_size=page, keep_from=i32(first))
    pool.release([min(k, cols * page) for k in keep], first)
    pool.agrees()


def test_release_looks_at_the_entries_of_max_len_keys():
    pool = Pool([100, 64, 33], 16, 8, 2).put()
    pdec.paged_release(i32([0, 0, 0]), pool.d_table, pool.d_free, *pool.d_count, page_size=16, max_len=33)
    pool.release([0, 0, 0], max_len=33)
    pool.agrees()
    assert (pool.table[0, 3:7] >= 0).all()


@pytest.mark.parametrize("S", [5, 100])
def test_counts_and_lists_outside_the_contract_stay_inside_the_arrays(S):
    """A free count beyond the pool or below 0, a page in two tables: wrong pages, no stray access."""
    page, cols, P = 16, 4, 50
    guard = torch.full((3 * P,), 7, dtype=torch.int32, device="cuda")
    free = guard[P:2 * P]
    for count, left in ((-3, 0), (10 ** 6, P - min(S, P))):
        free.copy_(i32(np.arange(P)))
        table, out = i32(np.full((S, cols), -1)), i32([0])
        pdec.paged_reserve(i32([1] * S), i32([0] * S), table, free, i32([count]), out, page_size=page, num_tokens=1000)
        assert out.item() == left and (table.cpu().numpy()[:, 1:] == -1).all()
    table = i32(np.zeros((S, cols)))  # page 0 in every entry
    pdec.paged_release(i32([0] * S), table, free, i32([P - 3]), out, page_size=page)
    assert out.item() == P and (table == -1).all()
    assert (guard[:P] == 7).all() and (guard[2 * P:] == 7).all()


@pytest.mark.parametrize("S", [20, 400])
def test_without_positions_or_slots(S):
    rng = np.random.default_rng(1)
    n, lens = batch(rng, S, 16, 9)
    for kw in ({"positions": False}, {"slots": False}, {"positions": False, "slots": False}):
        run(Pool(lens, 16, 9, 9 * S).put(), n, lens, sum(n), **kw)


def test_many_sequences():
    """More than the lanes of many work-groups; sums past one chunk after another."""
    S = 30000
    n = (np.arange(S) % 3).tolist()
    lens = (np.arange(S) % 31).tolist()
    pool = Pool(lens, 16, 3, 12000, seed=2).put()
    run(pool, n, lens, 26001)


@pytest.mark.parametrize("S", [30, 300])
def test_captured_steps_replay_with_new_requests(S):
    """Release, reserve and the next step's in one graph, the requests changed between replays, two graphs in turn."""
    page, cols = 16, 30
    rng = np.random.default_rng(S)
    lens = [int(rng.integers(0, 200)) for _ in range(S)]
    pool = Pool(lens, page, cols, S * 8, seed=4).put()
    d_n, d_lens = i32([0] * S), i32(lens)
    room = S * 20
    out = [torch.zeros(room, dtype=torch.int32, device="cuda"), torch.zeros(room, dtype=torch.int64, device="cuda")]
    cu, mid = torch.zeros(S + 1, dtype=torch.int32, device="cuda"), i32([0])

    def step():
        pdec.paged_release(d_lens, pool.d_table, pool.d_free, pool.d_count[0], mid, page_size=page)
        pdec.paged_reserve(d_n, d_lens, pool.d_table, pool.d_free, mid, pool.d_count[1], page_size=page, cu_tokens=cu,
                           positions=out[0], slots=out[1])
        pool.d_count[0].copy_(pool.d_count[1])

    graphs = []
    for _ in range(2):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            step()
        graphs.append(g)
    for i in range(6):
        n = [int(rng.integers(0, 20)) for _ in range(S)]
        d_n.copy_(i32(n))
        graphs[i % 2].replay() if i < 5 else step()
        torch.cuda.synchronize()
        pool.release(lens)
        want = pool.reserve(n, lens, room)
        assert cu.tolist() == want[0] and out[0][:len(want[1])].tolist() == want[1] and out[1][:len(want[2])].tolist() == want[2]
        pool.agrees()
        lens = [t + int(rng.integers(0, b - a + 1)) for t, a, b in zip(lens, want[0], want[0][1:])]  # some are refused
        lens = [0 if rng.random() < 0.1 else t for t in lens]  # some end
        d_lens.copy_(i32(lens))


def test_on_another_stream():
    rng = np.random.default_rng(0)
    n, lens = batch(rng, 100, 16, 8)
    pool = Pool(lens, 16, 8, 900).put()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    a, b = i32(n), i32(lens)
    side.wait_stream(torch.cuda.current_stream())
    cu = pdec.paged_reserve(a, b, pool.d_table, pool.d_free, *pool.d_count, page_size=16, num_tokens=10 ** 5, stream=side)
    side.synchronize()
    assert cu.tolist() == pool.reserve(n, lens, 10 ** 5)[0]
    pool.agrees()
