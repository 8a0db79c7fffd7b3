"""Sequences that share the pages of a prefix: their rows name the same pages, reservations add to them, and releases keep
them until the last sequence gives them back."""
import numpy as np
import pytest
import torch

from paper_2607_02963_amd import pdec

pytestmark = pytest.mark.gpu


def i32(x):
    return torch.from_numpy(np.ascontiguousarray(np.asarray(x, np.int32))).cuda()


@pytest.mark.parametrize("S", [5, 100])
def test_a_shared_prefix_is_given_back_once(S):
    page, cols, P, prefix = 16, 8, 10 * S, 3  # pages of the prefix
    table = np.full((S, cols), -1)
    table[:, :prefix] = [7, 2, 9]
    free = [x for x in range(P) if x not in (7, 2, 9)]
    d_table, d_free, count, mid = i32(table), i32(free + [-1] * prefix), i32([P - prefix]), i32([0])
    L, n = prefix * page, [1 + s % 40 for s in range(S)]
    cu = pdec.paged_reserve(i32(n), i32([L] * S), d_table, d_free, count, mid, page_size=page, num_tokens=sum(n))
    assert cu[-1].item() == sum(n) and mid.item() == P - prefix - sum(-(-x // page) for x in n)
    rows = d_table.cpu().numpy()
    own = rows[:, prefix:][rows[:, prefix:] >= 0]
    assert (rows[:, :prefix] == [7, 2, 9]).all() and len(set(own)) == len(own) and not {7, 2, 9} & set(own.tolist())
    # all but the first end; they keep the prefix
    keep = [L + n[0]] + [L] * (S - 1)
    pdec.paged_release(i32(keep), d_table, d_free, mid, count, page_size=page)
    rows = d_table.cpu().numpy()
    assert (rows[:, :prefix] == [7, 2, 9]).all() and (rows[1:, prefix:] == -1).all()
    assert count.item() == P - prefix - -(-n[0] // page)
    # the first ends too and gives all back; the others' rows are the caller's to clear
    pdec.paged_release(i32([0] + [L] * (S - 1)), d_table, d_free, count, mid, page_size=page)
    d_table[1:] = -1
    assert mid.item() == P and sorted(d_free.tolist()) == list(range(P)) and (d_table == -1).all()
