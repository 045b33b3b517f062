"""Pages of the paged cache over many steps: whoever is refused, every page has one owner, a request or the free list, and none is lost."""
import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu

from paper_2601_07048_amd import jx  # noqa: E402


def i32(x):
    return torch.tensor(np.asarray(x), dtype=torch.int32, device="cuda")


def held(table, free, n_free):
    """Every page that a row or the free list names."""
    rows = table.cpu().numpy().ravel()
    return sorted(rows[rows >= 0].tolist() + free.cpu().numpy()[:int(n_free)].tolist())


def test_a_request_too_long_for_its_table_keeps_nobody_from_a_page():
    page, width = 16, 8
    table = np.full((3, width), -1, np.int32)
    table[0] = range(width)  # 128 tokens: its table is full
    table, free = i32(table), i32([10, 11, 12, 13] + [-1] * 10)
    plan = jx.kv_plan(i32([128, 0, 0]), i32([1, 1, 0]), table, free, i32([4]), page, 2)
    assert plan.kv_len.tolist() == [0, 1, 0] and plan.slot.tolist() == [-1, 13 * page] and int(plan.n_free) == 3
    plan = jx.kv_plan(i32([128, 1, 0]), i32([0, 0, 1]), table, free, plan.n_free, page, 1)
    assert plan.kv_len.tolist() == [128, 1, 1] and plan.slot.tolist() == [12 * page] and int(plan.n_free) == 2
    assert table[1:, 0].tolist() == [13, 12]
    assert held(table, free, plan.n_free) == list(range(8)) + [10, 11, 12, 13]


@pytest.mark.parametrize("n_req,page,width,n_pages", [(6, 16, 5, 24), (40, 8, 4, 120), (1500, 4, 3, 3000), (3, 1, 9, 20)])
def test_pages_have_one_owner(n_req, page, width, n_pages):
    """Requests grow by chunks until they are too long for their table, are refused there, finish and begin again; the pool is too
    small for all, and now and then the step has too few rows.  By the definition: requests in turn, where one whose tokens exceed
    its table or whose rows exceed the step's asks for nothing."""
    rng = np.random.default_rng(n_req)
    total = n_pages + 3
    free = i32(rng.permutation(total))
    n_free = i32([total])
    table = torch.full((n_req, width), -1, dtype=torch.int32, device="cuda")
    lens = np.zeros(n_req, np.int64)
    refused = 0
    for step in range(25):
        new = rng.integers(0, page + 3, n_req)
        rows = max(int(new.sum()) - (int(rng.integers(1, page + 3)) if step % 5 == 4 else -2), 0)
        before, stack, left = table.cpu().numpy(), free.cpu().numpy(), int(n_free)
        want_table, want_len, begin, slots = before.copy(), [], 0, []
        asked = 0
        for r in range(n_req):
            a, n = int(lens[r]), int(new[r])
            first, end = -(-a // page), -(-(a + n) // page)
            begin += n
            fits = end <= width and begin <= rows
            if fits:
                asked += end - first
            if not fits or (end > first and asked > left):
                want_len.append(0)
                slots += [-1] * n
                refused += end > width
                continue
            for i in range(first, end):
                want_table[r, i] = stack[left - asked + end - 1 - i]
            want_len.append(a + n)
            slots += [int(want_table[r, p // page]) * page + p % page for p in range(a, a + n)]
        got = jx.kv_plan(i32(lens), i32(new), table, free, n_free, page, rows)
        assert np.array_equal(table.cpu().numpy(), want_table) and got.kv_len.tolist() == want_len, step
        assert got.slot.tolist() == (slots + [-1] * max(0, rows - len(slots)))[:rows], step
        lens = np.where(np.asarray(want_len) > 0, want_len, lens)
        n_free = got.n_free.clone()
        assert held(table, free, n_free) == list(range(total)), step
        over = rng.random(n_req) < np.where(lens > (width - 1) * page, 0.4, 0.05)  # finished
        jx.kv_release(i32(np.zeros(n_req)), i32(np.where(over, width, 0)), table, free, n_free)
        lens[over] = 0
        assert held(table, free, n_free) == list(range(total)), step
    assert refused > 0
