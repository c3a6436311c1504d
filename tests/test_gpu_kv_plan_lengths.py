"""dcl_kv_plan: what it tells of sequences that get no rows because their numbers do not fit, apart from the starts and in
their place.  Whole numbers, equal to those of lists on the host."""
import numpy as np
import pytest
import torch

import paper_2607_20467_gb300 as dcl
import test_gpu_kv_plan as plan
from test_gpu_kv_plan import ops  # noqa: F401 (a fixture)

pytestmark = pytest.mark.gpu

P, WIDTH = 16, 3  # a table of 48 positions


@pytest.mark.parametrize("in_place", [False, True])
@pytest.mark.parametrize("new", [9, -2, 2 ** 31 - 1])
@pytest.mark.parametrize("batch,rows", [(3, 100), (300, 2000), (1500, 9000), (2049, 9000)])  # (one kernel, and two)
def test_a_sequence_that_does_not_fit_keeps_its_length_and_pages(ops, batch, rows, new, in_place):  # noqa: F811
    """Sequences of 40 positions, the whole of their pages, ask for rows past the table (or fewer than none) and are left
    out: told as 40 positions, after which they go on as if they had not asked."""
    pages, lists, call = dcl.KvPages.new(3 * batch, P, batch, WIDTH), plan.Lists(3 * batch, P, batch), plan.Call(batch, rows)
    full = sorted({1, batch // 2, batch - 1})
    at = [0] * batch

    def step(news, reported=False):
        nonlocal at
        starts = plan._i32(at)
        ops.kv_plan(pages, starts, plan._i32(news), call.q_start, starts if in_place else call.seq_len, call.slots, call.pos)
        if reported:
            plan._reported(ops)
        else:
            ops.synchronise()
        if in_place:
            call.seq_len = starts
        want = lists.plan(at, [0 if b in full and reported else n for b, n in enumerate(news)])
        plan._same(pages, lists, call, want)
        at = call.seq_len.tolist()  # (a loop on the device goes on from what it was told)

    some = lambda b: b % 5
    step([40 if b in full else some(b) for b in range(batch)])
    held = [list(lists.of[b]) for b in full]
    step([new if b in full else some(b) for b in range(batch)], reported=True)
    assert [at[b] for b in full] == [40] * len(full)
    step([0 if b in full else some(b) for b in range(batch)])
    step([8 if b in full else 0 for b in range(batch)])
    assert [at[b] for b in full] == [48] * len(full) and [lists.of[b] for b in full] == held


@pytest.mark.parametrize("batch", [2, 600])
@pytest.mark.parametrize("held", [-1, 4])
def test_pages_that_no_table_has_leave_the_length(ops, batch, held):  # noqa: F811
    """More pages held than a table has, or fewer than none: the sequence is left out, its length as it was."""
    pages, call = dcl.KvPages.new(3 * batch, P, batch, WIDTH), plan.Call(batch, 5000 if batch > 2 else 50)
    call(ops, pages, [0] * batch, [20] + [3] * (batch - 1))
    ops.synchronise()
    pages.held[0] = held
    table = pages.table.clone()
    call(ops, pages, [20] + [3] * (batch - 1), [1] * batch)
    plan._reported(ops)
    assert call.seq_len.tolist() == [20] + [4] * (batch - 1) and torch.equal(pages.table, table)
    assert pages.held.tolist() == [held] + [1] * (batch - 1)
    assert call.q_start.tolist() == np.concatenate([[0], np.arange(batch)]).tolist()


@pytest.mark.parametrize("start", [-1, 49, 2 ** 31 - 1])
def test_a_start_that_is_no_position_is_told_as_none(ops, start):  # noqa: F811
    pages, call = dcl.KvPages.new(9, P, 2, WIDTH), plan.Call(2, 60)
    call(ops, pages, [0, 0], [40, 5])
    ops.synchronise()
    table = pages.table.clone()
    call(ops, pages, [start, 5], [1, 1])
    plan._reported(ops)
    assert call.seq_len.tolist() == [0, 6] and call.q_start.tolist() == [0, 0, 1] and pages.held.tolist() == [3, 1]
    assert torch.equal(pages.table, table)
