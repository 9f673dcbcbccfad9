"""The pool of pages of the paged cache where its lists are short, empty or wrong."""
import pytest
import torch

import kv_reference as R
from paper_2312_17238_amd import paged

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def i32(v):
    return torch.tensor(v, dtype=torch.int32, device=DEV)


@pytest.mark.parametrize("count", [3, 4, 5, 9, 12, 2 ** 31 - 1])
def test_nothing_behind_the_free_list_is_handed_out(count):
    """A count above the list's length counts as its length: entries behind it belong to somebody else."""
    store = i32([8, 9, 10, 11, 0, 1, 2, 3, 4, 5, 6, 7])
    free, table = store[:4], i32([[-1] * 3] * 5)
    step = paged.Step(5, 5 * 16, 16, 3, 12, 16, 4, 2, 64)
    step.plan(i32([0, 5, 0, 0, 0]), i32([16, 1, 16, 16, 16]), table, free, i32([count]))
    want = torch.full((5, 3), -1).int().numpy()
    lists = R.plan([0, 5, 0, 0, 0], [16, 1, 16, 16, 16], want, free.tolist(), min(count, 4), n_tokens=80, max_new=16, n_pages=12, page=16)
    start, positions, slots, kv, status, left = lists
    assert step.status.tolist() == status and step.free_left.tolist() == [left] and step.slots.tolist() == slots and step.kv_len.tolist() == kv
    assert table.tolist() == want.tolist() and not (set(table.flatten().tolist()) & set(range(8)))


def test_giving_back_nothing():
    table, ctx, free, count = i32([[3, 4]]), i32([20]), i32([0, 1, -7, -7]), i32([2])
    paged.release(i32([]), 8, 16, ctx, table, free, count)
    assert ctx.tolist() == [20] and count.tolist() == [2] and free.tolist() == [0, 1, -7, -7]
