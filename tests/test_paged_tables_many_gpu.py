"""Block tables of many sequences, whose counts are summed by a pass of their own: against the definition, with pools and
budgets that end in the first, a middle and the last of the sums' chunks and at their borders."""
import numpy as np
import pytest
import torch

from paper_2607_02963_amd import pdec

pytestmark = pytest.mark.gpu

PAGE, COLS, CHUNK = 16, 4, 2048


def i32(x):
    return torch.from_numpy(np.ascontiguousarray(np.asarray(x, np.int32))).cuda()


class Batch:
    """S sequences of up to 40 keys that ask for up to 20 more, a twentieth of them for what cannot be."""

    def __init__(self, S, seed=0):
        rng = np.random.default_rng(seed)
        self.lens, self.n = rng.integers(0, 41, S), rng.integers(0, 21, S)
        bad = rng.random(S) < 0.05
        self.asked = np.where(bad, rng.choice([-1, COLS * PAGE + 1], S), self.n)
        self.n = np.where(bad, 0, self.n)
        self.used, self.need = -(-self.lens // PAGE), -(-(self.lens + self.n) // PAGE) - -(-self.lens // PAGE)
        self.P = int(self.used.sum() + self.need.sum()) + 3
        order = rng.permutation(self.P)
        col = np.arange(COLS)
        first = np.concatenate([[0], np.cumsum(self.used)])
        at = np.minimum(first[:-1, None] + col, self.P - 1)
        self.table = np.where(col < self.used[:, None], order[at], -1)
        self.free, self.count = np.full(self.P, -9), self.P - int(first[-1])
        self.free[:self.count] = order[first[-1]:]

    def reserved(self, count, room):
        """(cu, positions, slots, table, pages left) by the definition."""
        served = (np.cumsum(self.need) <= count) & (np.cumsum(self.n) <= room)
        n, need = np.where(served, self.n, 0), np.where(served, self.need, 0)
        cu = np.concatenate([[0], np.cumsum(n)])
        col = np.arange(COLS)
        lack = served[:, None] & (col >= self.used[:, None]) & (col < (self.used + self.need)[:, None])
        table = self.table.copy()
        table[lack] = self.free[count - 1 - np.arange(lack.sum())]
        seq = np.repeat(np.arange(len(n)), n)
        pos = self.lens[seq] + np.arange(len(seq)) - cu[seq]
        return cu, pos, table[seq, pos // PAGE] * PAGE + pos % PAGE, table, count - int(need.sum())


def check(b, count, room):
    cu, pos, slots, table, left = b.reserved(count, room)
    d_table, d_free, d_in, d_mid, d_out = i32(b.table), i32(b.free), i32([count]), i32([-5]), i32([-5])
    d_lens, T = i32(b.lens), max(room, 1)
    got_pos, got_slots = torch.full((T,), -4, dtype=torch.int32, device="cuda"), torch.full((T,), -4, dtype=torch.int64, device="cuda")
    got = pdec.paged_reserve(i32(b.asked), d_lens, d_table, d_free, d_in, d_mid, page_size=PAGE, positions=got_pos, slots=got_slots)
    assert np.array_equal(got.cpu().numpy(), cu) and d_mid.item() == left
    for x, want in ((got_pos, pos), (got_slots, slots)):
        assert np.array_equal(x[:len(want)].cpu().numpy(), want) and (x[len(want):] == -4).all()
    assert np.array_equal(d_table.cpu().numpy(), table)
    # and back
    pdec.paged_release(d_lens, d_table, d_free, d_mid, d_out, page_size=PAGE)
    assert d_out.item() == count and np.array_equal(d_table.cpu().numpy(), b.table)
    assert np.array_equal(d_free.cpu().numpy()[:count], b.free[:count])


@pytest.mark.parametrize("S", [CHUNK - 1, CHUNK, CHUNK + 1, 4 * CHUNK, 8 * CHUNK, 8 * CHUNK + 1, 16 * CHUNK + 5, 100003])
def test_all_are_served(S):
    b = Batch(S, seed=S)
    check(b, b.count, int(b.n.sum()) + 7)


@pytest.mark.parametrize("S", [10 * CHUNK + 77, 40 * CHUNK - 1])
def test_what_does_not_fit_is_not_served_nor_is_what_follows(S):
    b = Batch(S, seed=S)
    pages, tokens = np.cumsum(b.need), np.cumsum(b.n)
    last = S - 1
    for s in (0, 3, CHUNK - 2, CHUNK - 1, CHUNK, 5 * CHUNK - 1, 5 * CHUNK, 5 * CHUNK + 5, 9 * CHUNK - 1, 9 * CHUNK + 900, last - 1, last):
        check(b, b.count, max(int(tokens[s]), 1))           # room for those up to s
        check(b, b.count, max(int(tokens[s]) - 1, 1))       # and for a token less
        check(b, min(int(pages[s]), b.count), int(tokens[-1]) + 1)
        check(b, max(int(pages[s]) - 1, 0), int(tokens[-1]) + 1)


def test_a_million_sequences():
    """The most that a call takes; its time grows with them, not with their square: 6.5 ms for the pair, a second by the
    square."""
    b = Batch(1 << 20, seed=1)
    check(b, b.count, int(b.n.sum()) + 1)
    n, lens, cu = i32(b.asked), i32(b.lens), i32(np.zeros((1 << 20) + 1))
    table, free, c = i32(b.table), i32(b.free), [i32([b.count]), i32([0]), i32([0])]
    ws = torch.empty(pdec.table_workspace_size(1 << 20), dtype=torch.uint8, device="cuda")
    times = []
    for _ in range(3):
        a, e = (torch.cuda.Event(enable_timing=True) for _ in "ae")
        a.record()
        pdec.paged_reserve(n, lens, table, free, c[0], c[1], page_size=PAGE, cu_tokens=cu, num_tokens=1 << 27, workspace=ws)
        pdec.paged_release(lens, table, free, c[1], c[2], page_size=PAGE, workspace=ws)
        e.record()
        torch.cuda.synchronize()
        times.append(a.elapsed_time(e))
    assert c[2].item() == b.count and min(times) < 50, times
