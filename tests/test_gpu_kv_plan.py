"""dcl_kv_plan against lists of pages on the host: everything it writes is a whole number and has to be equal."""
import numpy as np
import pytest
import torch

import paper_2607_20467_gb300 as dcl

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def ops():
    import __graft_entry__
    __graft_entry__.build()
    ctx = dcl.Context(None, 1, 1)
    yield ctx
    ctx.close()


class Lists:
    """Pages of sequences, and the free ones, as lists."""

    def __init__(self, n_pages, page_len, batch):
        self.free, self.of, self.page_len = list(range(n_pages)), [[] for _ in range(batch)], page_len

    def plan(self, start, new):
        """Rows of every sequence (slots, positions), q_start and seq_len."""
        P = self.page_len
        need = [-(-(a + n) // P) for a, n in zip(start, new)]
        for pages, k in zip(self.of, need):
            self.free += pages[k:]
            del pages[k:]
        there, total, slots, pos, q_start, lens = len(self.free), 0, [], [], [0], []
        for b, (pages, k) in enumerate(zip(self.of, need)):
            lack = k - len(pages)
            total += lack
            ok = lack == 0 or total <= there
            if ok:
                pages += [self.free.pop() for _ in range(lack)]
                at = np.arange(start[b], start[b] + new[b])
                slots += (np.asarray(pages + [0])[at // P] * P + at % P).tolist()
                pos += at.tolist()
            q_start.append(len(pos))
            lens.append(start[b] + new[b] if ok else start[b])
        return slots, pos, q_start, lens


def _i32(a):
    return torch.tensor(np.asarray(a, np.int64), dtype=torch.int32, device="cuda")


class Call:
    def __init__(self, batch, rows):
        full = lambda n: torch.full((n,), 99, dtype=torch.int32, device="cuda")
        self.q_start, self.seq_len, self.slots, self.pos = full(batch + 1), full(batch), full(rows), full(rows)

    def __call__(self, ops, pages, start, new):
        ops.kv_plan(pages, _i32(start), _i32(new), self.q_start, self.seq_len, self.slots, self.pos)


def _same(pages, lists, call, want):
    slots, pos, q_start, lens = want
    assert call.q_start.tolist() == q_start and call.seq_len.tolist() == lens
    pad = [-1] * (len(call.slots) - len(slots))
    assert call.slots.tolist() == slots + pad and call.pos.tolist() == pos + pad
    held, table = pages.held.tolist(), pages.table.cpu().numpy()
    assert held == [len(p) for p in lists.of]
    for b, p in enumerate(lists.of):
        assert table[b, :len(p)].tolist() == p and (table[b, len(p):] == -1).all()
    n = int(pages.n_free)
    assert n == len(lists.free) and pages.free[:n].tolist() == lists.free


@pytest.mark.parametrize("batch,page_len,width,n_pages", [
    (1, 16, 4, 3), (3, 32, 7, 21), (8, 64, 30, 200), (33, 16, 12, 120), (512, 16, 5, 900), (513, 128, 3, 1600), (1500, 16, 6, 3000)])
def test_steps_of_growing_shrinking_and_ending_sequences(ops, batch, page_len, width, n_pages):
    """Several plans in a row over one pool, which is too small at times where it has less than half of them all."""
    rng = np.random.default_rng(batch)
    pages, lists = dcl.KvPages.new(n_pages, page_len, batch, width), Lists(n_pages, page_len, batch)
    room, start = width * page_len, np.zeros(batch, np.int64)
    refused = 0
    for step in range(8):
        new = np.minimum(rng.integers(0, rng.choice([2, 40, room]) + 1, batch), room - start)
        new[rng.random(batch) < 0.2] = 0
        rows = int(new.sum()) + int(rng.integers(0, 4))
        call = Call(batch, rows)
        call(ops, pages, start, new)
        ops.synchronise()
        want = lists.plan(start.tolist(), new.tolist())
        _same(pages, lists, call, want)
        got = np.diff(want[2])
        refused += int((got < new).sum())
        start = np.where(got == new, start + new, start)
        gone = rng.random(batch) < 0.3
        start[gone] = 0  # (ended)
        back = rng.random(batch) < 0.3
        start[back] = (start[back] * rng.random(back.sum())).astype(np.int64)  # (positions given up)
    assert refused > 0 or 2 * n_pages > batch * width
    every = sorted(lists.free + sum(lists.of, []))
    assert every == list(range(n_pages))


def test_a_large_admission(ops):
    """Prompts of unlike lengths, one of them most of the rows, at once."""
    lens = [1, 70000, 3, 1536, 0, 16, 17, 30001]
    P, width = 16, 4400
    pages, lists = dcl.KvPages.new(7000, P, 8, width), Lists(7000, P, 8)
    call = Call(8, sum(lens) + 5)
    call(ops, pages, [0] * 8, lens)
    ops.synchronise()
    _same(pages, lists, call, lists.plan([0] * 8, lens))
    call(ops, pages, lens, [1] * 8)  # one more each; rows of the rest are cleared
    ops.synchronise()
    _same(pages, lists, call, lists.plan(lens, [1] * 8))


def test_the_same_step_again_changes_nothing(ops):
    pages, call = dcl.KvPages.new(50, 16, 4, 20), Call(4, 130)
    for _ in range(2):
        call(ops, pages, [3, 0, 40, 16], [32, 32, 32, 32])
        ops.synchronise()
        state = [t.clone() for t in (pages.table, pages.held, pages.free, pages.n_free, call.slots, call.pos, call.q_start)]
        if _:
            assert all(torch.equal(a, b) for a, b in zip(state, before))
        before = state


def test_no_sequences_and_no_rows(ops):
    pages, call = dcl.KvPages.new(5, 16, 0, 3), Call(0, 7)
    call(ops, pages, [], [])
    ops.synchronise()
    assert call.q_start.tolist() == [0] and call.slots.tolist() == [-1] * 7 and call.pos.tolist() == [-1] * 7
    pages, call = dcl.KvPages.new(5, 16, 2, 3), Call(2, 0)
    call(ops, pages, [5, 0], [0, 0])
    ops.synchronise()
    assert call.q_start.tolist() == [0, 0, 0] and call.seq_len.tolist() == [5, 0] and pages.held.tolist() == [1, 0]


def _reported(ops):
    with pytest.raises(dcl.DcleapError, match="outside the paged cache") as e:
        ops.synchronise()
    assert e.value.status == dcl.DCL_ERR_INVALID_ARG


@pytest.mark.parametrize("start,new", [(-1, 5), (3, -2), (40, 9), (2 ** 31 - 1, 2 ** 31 - 1)])
def test_a_sequence_past_its_table_is_reported_and_left_out(ops, start, new):
    pages, lists, call = dcl.KvPages.new(20, 16, 3, 3), Lists(20, 16, 3), Call(3, 40)
    call(ops, pages, [0, 0, 0], [17, 20, 3])
    ops.synchronise()
    _same(pages, lists, call, lists.plan([0, 0, 0], [17, 20, 3]))
    call(ops, pages, [17, start, 3], [1, new, 30])
    _reported(ops)
    want = lists.plan([17, 20, 3], [1, 0, 30])
    want[3][1] = 0
    _same(pages, lists, call, want)


def test_more_rows_than_there_is_room_for(ops):
    pages, lists, call = dcl.KvPages.new(20, 16, 3, 5), Lists(20, 16, 3), Call(3, 25)
    call(ops, pages, [0, 0, 0], [10, 20, 30])
    _reported(ops)
    slots, pos, _, lens = lists.plan([0, 0, 0], [10, 20, 30])
    _same(pages, lists, call, (slots[:25], pos[:25], [0, 10, 25, 25], lens))


def test_a_broken_stack_moves_nothing(ops):
    for count, held in ((-1, 2), (21, 2), (19, 2), (5, 7)):
        pages, call = dcl.KvPages.new(20, 16, 2, 3), Call(2, 60)
        call(ops, pages, [0, 0], [20, 32])
        ops.synchronise()
        pages.n_free.fill_(count)
        pages.held.copy_(_i32([held, 2]))
        state = [t.clone() for t in (pages.table, pages.held, pages.free, pages.n_free)]
        call(ops, pages, [0, 0], [0, 0])
        _reported(ops)
        if held == 2:
            assert all(torch.equal(a, b) for a, b in zip(state, (pages.table, pages.held, pages.free, pages.n_free)))
            assert call.q_start.tolist() == [0, 0, 0] and call.slots.tolist() == [-1] * 60
        else:  # (more pages held than a table has: that sequence is left as it is, the other ends)
            assert pages.held.tolist() == [7, 0] and int(pages.n_free) == 7


def test_a_page_outside_the_pool_gives_no_slot(ops):
    pages, call = dcl.KvPages.new(20, 16, 2, 3), Call(2, 40)
    call(ops, pages, [0, 0], [20, 20])
    ops.synchronise()
    pages.table[0, 1] = 20
    pages.table[1, 0] = -7
    call(ops, pages, [0, 0], [20, 20])
    _reported(ops)
    slots = call.slots.tolist()
    assert slots[16:20] == [-1] * 4 and slots[20:36] == [-1] * 16 and min(slots[:16] + slots[36:40]) >= 0
    assert call.pos.tolist() == list(range(20)) * 2


def test_rows_at_any_address(ops):
    """Slots and positions that begin between 16-byte borders."""
    for shift in (1, 2, 3):
        pages, lists, call = dcl.KvPages.new(500, 16, 3, 400), Lists(500, 16, 3), Call(3, 0)
        bufs = [torch.full((5010,), 99, dtype=torch.int32, device="cuda") for _ in range(2)]
        call.slots, call.pos = (b[shift:5003] for b in bufs)
        call(ops, pages, [0, 0, 0], [1, 4990, 3])
        ops.synchronise()
        _same(pages, lists, call, lists.plan([0, 0, 0], [1, 4990, 3]))
        assert all((b[:shift] == 99).all() and (b[5003:] == 99).all() for b in bufs)


@pytest.mark.parametrize("rows", [200, 5000])  # (one kernel, and two)
def test_a_captured_plan_follows_its_inputs(rows):
    stream = torch.cuda.Stream()
    B, P, width, n_pages = 5, 16, 20, 60
    start, new = _i32([0] * B), _i32([0] * B)
    pages, lists, call = dcl.KvPages.new(n_pages, P, B, width), Lists(n_pages, P, B), Call(B, rows)
    with dcl.Context(None, 1, 1, stream=stream.cuda_stream) as ctx:
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=stream):
            ctx.kv_plan(pages, start, new, call.q_start, call.seq_len, call.slots, call.pos)
        rng, at = np.random.default_rng(1), np.zeros(B, np.int64)
        for _ in range(6):
            n = rng.integers(0, 40, B)
            n = np.minimum(n, width * P - at)
            start.copy_(_i32(at))
            new.copy_(_i32(n))
            torch.cuda.synchronize()
            graph.replay()
            torch.cuda.synchronize()
            want = lists.plan(at.tolist(), n.tolist())
            _same(pages, lists, call, want)
            at = np.where(rng.random(B) < 0.4, 0, want[3])
        ctx.synchronise()


@pytest.mark.parametrize("batch,rows", [(5, 60), (300, 2000), (1500, 9000), (3, 9000)])
def test_lengths_that_take_the_place_of_the_starts(ops, batch, rows):
    """seq_len is start: steps in a row, each from where the last one ended, with one kernel and with two (from 256
    sequences or 4096 rows on), and more sequences than a block has threads; one that gets no pages stays where it is."""
    rng = np.random.default_rng(batch)
    P, width = 16, 1200
    n_pages = batch + rows // 8
    pages, lists = dcl.KvPages.new(n_pages, P, batch, width), Lists(n_pages, P, batch)
    call = Call(batch, rows)
    call.seq_len.zero_()
    at = [0] * batch
    for step in range(6):
        new = rng.multinomial(int(rng.integers(rows // 2, rows + 1)), [1 / batch] * batch).tolist()
        ops.kv_plan(pages, call.seq_len, _i32(new), call.q_start, call.seq_len, call.slots, call.pos)
        ops.synchronise()
        want = lists.plan(at, new)
        _same(pages, lists, call, want)
        at = want[3]
