"""The plan from lengths, heads and pages that no cache has: nothing outside its arrays is read or written, and the fault bits say so."""
import pytest

import window_reference as W
from test_gpu_operators import R, i32

pytestmark = pytest.mark.gpu


def bounded_plan(ctx, new, P, free, head, table, max_rows):
    """The plan sequence by sequence, its sums held at 2^31 - 1; only rows and table places that exist are gone through."""
    most = 2 ** 31 - 1
    total, starts, slots, pos = [], [0], [-1] * max_rows, [0] * max_rows
    at, faults, width = head, 2 if head > len(free) else 0, len(table[0])
    for s, (c, n) in enumerate(zip(ctx, new)):
        if c < 0 or n < 0 or max(c, 0) + max(n, 0) > most:
            faults |= 8
        c = max(c, 0)
        n = min(max(n, 0), most - c)
        had, need = -(-c // P), -(-(c + n) // P)
        faults |= 4 if need > width else 0

        def page(e):
            return table[s][e] if e < had else free[at + e - had] if at + e - had < len(free) else -1

        for e in range(had, min(need, width)):
            table[s][e] = page(e)
        for r in range(starts[-1], min(starts[-1] + n, max_rows)):
            p = c + r - starts[-1]
            e, x = p // P, -1
            if e < width:
                x = table[s][e]
            slots[r], pos[r] = (x * P + p % P if x >= 0 else -1), p
        at += need - had
        total.append(c + n)
        starts.append(min(starts[-1] + n, most))
    faults |= (2 if at > len(free) else 0) | (1 if starts[-1] > max_rows or starts[-1] == most else 0)
    return total, starts, slots, pos, [starts[-1], min(at, len(free)), max(total), faults]


MOST = 2 ** 31 - 1


def check(ctx, new, P, free, head, width, max_rows, seed=0):
    table = [[s * width + e + 100 if e < -(-max(c, 0) // P) else -7 for e in range(width)] for s, c in enumerate(ctx)]
    t = i32(table)
    got = R.rlgen_plan_pages(i32(ctx), i32(new), P, i32(free), t, max_rows, i32([head]))
    want = bounded_plan(ctx, new, P, free, head, table, max_rows)
    for name, g, w in zip(got._fields, got, want):
        assert g.tolist() == list(w), name
    assert t.tolist() == table


def test_the_bounded_form_is_the_plain_one():
    for ctx, new, free, head, rows in (([3, 0, 8], [6, 2, 1], [9, 4, 1, 6], 0, 10), ([-4, 30], [40, 9], [1, 2], 1, 20), ([0, 3], [20, 9], [1, 2, 3], 0, 29)):
        a, b = [[5, -7, 1] for _ in ctx], [[5, -7, 1] for _ in ctx]
        assert bounded_plan(ctx, new, 8, free, head, a, rows) == W.plan(ctx, new, 8, free, head, b, rows) and a == b


@pytest.mark.parametrize("P", [8, 16, 1024])
@pytest.mark.parametrize("new", [[MOST, MOST, 1], [1, MOST, 7, MOST, 3], [MOST - 2, 1, 1, 1, 5], [5, MOST - 5, 0], [2, MOST - 4, 1]])
def test_rows_that_pass_2_to_the_31(P, new):
    check([0] * len(new), new, P, [7, 8, 9, 2], 0, 3, 40)
    check([9] + [0] * (len(new) - 1), new, P, [7, 8, 9, 2], 1, 2, 0)


@pytest.mark.parametrize("S", [700, 1100, 3000])
def test_many_requests_whose_sums_pass_2_to_the_31(S):
    """Several requests to a block, the sums passing the limit within it and in front of it, in rows alone and in pages too."""
    check([i % 5 for i in range(S)], [3 if i % 7 else 2 ** 27 for i in range(S)], 16, list(range(50)), 0, 2, 300)
    check([i % 20 for i in range(S)], [1 if i < S - 40 else MOST for i in range(S)], 8, list(range(S)), 3, 2, S)


@pytest.mark.parametrize("ctx, new", [([MOST, 3], [5, 2]), ([MOST - 3, 0], [4, 1]), ([2 ** 30, 2 ** 30], [2 ** 30, 2 ** 30 - 1]), ([MOST, MOST], [MOST, MOST])])
def test_lengths_that_pass_2_to_the_31(ctx, new):
    check(ctx, new, 16, [4, 5, 6], 0, 2, 20)


@pytest.mark.parametrize("head", [3, 4, 5, 1000, MOST - 1, MOST])
def test_a_head_past_the_free_list(head):
    check([0, 3, 8], [6, 9, 20], 8, [4, 5, 6, 9], head, 3, 40)
    check([0, 3, 8], [0, 0, 0], 8, [4, 5, 6, 9], head, 3, 2)
    check([0] * 600, [30] * 600, 8, list(range(9)), head, 3, 600)


@pytest.mark.parametrize("page_size, page", [(16, 2 ** 28 + 5), (16, 2 ** 27 + 3), (16, 2 ** 31 - 1), (8, 2 ** 29 + 2), (1024, 2 ** 22), (1024, 2 ** 21)])
def test_a_page_whose_slots_pass_32_bits_has_none(page_size, page):
    """Both from the table (a page already begun) and from the free list; pages next to them keep their slots."""
    table = i32([[page, -7], [4, -7]])
    plan = R.rlgen_plan_pages(i32([3, page_size]), i32([2, 2]), page_size, i32([page]), table, 4)
    assert plan.slots.tolist() == [-1] * 4 and plan.positions.tolist() == [3, 4, page_size, page_size + 1]
    assert table.tolist() == [[page, -7], [4, page]]
    last = (2 ** 31 - 1) // page_size - 1                  # (the last page that has slots in 32 bits, all of it)
    table = i32([[last, -7]])
    assert R.rlgen_plan_pages(i32([3]), i32([1]), page_size, i32([0]), table, 1).slots.tolist() == [last * page_size + 3]
