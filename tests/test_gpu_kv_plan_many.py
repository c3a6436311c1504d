"""dcl_kv_plan of more sequences than one block keeps in shared memory (2048), and of the largest pages: the steps of
test_gpu_kv_plan."""
import pytest
import torch

import paper_2607_20467_gb300 as dcl
import test_gpu_kv_plan as plan
from test_gpu_kv_plan import ops  # noqa: F401 (a fixture)

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("batch,page_len,width,n_pages", [
    (2047, 16, 3, 4000), (2048, 32, 4, 5000), (2049, 16, 4, 5000), (5000, 64, 3, 9000), (40, 256, 5, 110), (256, 16, 4, 600), (257, 16, 4, 600)])
def test_steps_of_growing_shrinking_and_ending_sequences(ops, batch, page_len, width, n_pages):  # noqa: F811
    plan.test_steps_of_growing_shrinking_and_ending_sequences(ops, batch, page_len, width, n_pages)


@pytest.mark.parametrize("batch,rows", [(256, 4096), (256, 4097), (257, 4000), (2048, 9000), (2049, 9000), (5000, 12000)])
def test_lengths_that_take_the_place_of_the_starts(ops, batch, rows):  # noqa: F811
    plan.test_lengths_that_take_the_place_of_the_starts(ops, batch, rows)


def test_rows_up_to_two_to_the_31st(ops):  # noqa: F811
    """As many rows as an int counts: the last ones of a thread's four would pass 2^31."""
    n, P, width = 2 ** 31 - 1, 256, 2 ** 31 // 256 // 2
    pages = dcl.KvPages.new(7, P, 2, width)
    pages.table.fill_(3)  # (every place of both sequences in one page)
    pages.held.fill_(width)
    pages.n_free.fill_(0)
    call = plan.Call(2, 0)
    call.slots, call.pos = (torch.full((n,), 99, dtype=torch.int32, device="cuda") for _ in range(2))
    call(ops, pages, [0, 1], [width * P, width * P - 1])
    ops.synchronise()
    half = width * P
    assert call.q_start.tolist() == [0, half, n] and call.seq_len.tolist() == [half, half]
    for first, count, pos in ((0, 1000, 0), (half - 1000, 1000, half - 1000), (half, 1000, 1), (n - 1003, 1003, half - 1003)):
        want = torch.arange(pos, pos + count, dtype=torch.int32, device="cuda")
        assert torch.equal(call.pos[first:first + count], want)
        assert torch.equal(call.slots[first:first + count], 3 * P + want % P)
    step = 1 << 27
    for at in range(0, n, step):  # (whole rows, a part at a time)
        row = torch.arange(at, min(at + step, n), dtype=torch.int64, device="cuda")
        want = torch.where(row < half, row, row - half + 1).to(torch.int32)
        assert torch.equal(call.pos[at:at + step], want) and torch.equal(call.slots[at:at + step], 3 * P + want % P)
