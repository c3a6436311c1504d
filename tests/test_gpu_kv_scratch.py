"""What dcl_kv_attention keeps between calls: the scratch in which CTAs that share a sequence's keys leave
their parts."""
import numpy as np
import pytest
import torch

import paper_2607_20467_gb300 as dcl

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def built():
    import __graft_entry__
    __graft_entry__.build()


class Call:
    """One sequence of n positions (random FP8 codes) and its rows; a table of `wide` positions chooses the
    kernel."""

    def __init__(self, n, new, wide, heads=4, hd=64, page_len=64):
        gen = torch.Generator(device="cuda").manual_seed(n + new)
        pages = -(-n // page_len)
        self.cache = dcl.KvCache.empty(pages, page_len, 1, hd)
        for t in (self.cache.k, self.cache.v):  # codes of finite values
            t.copy_(torch.randint(0, 0x70, t.shape, generator=gen, device="cuda", dtype=torch.uint8))
        self.cache.k_exp.fill_(-8)
        self.cache.v_exp.fill_(0)
        self.q = torch.randn(new, heads, hd, generator=gen, device="cuda").to(torch.bfloat16)
        i32 = lambda a: torch.tensor(a, dtype=torch.int32, device="cuda")
        self.starts, self.lens, self.new = i32([0, new]), i32([n]), new
        self.table = torch.full((1, max(pages, -(-wide // page_len))), -1, dtype=torch.int32, device="cuda")
        self.table[0, :pages] = torch.arange(pages, device="cuda")
        self.bad = self.table.clone()
        self.bad[0, 1] = pages
        torch.cuda.synchronize()

    def out(self):
        return torch.full(self.q.shape, 7.0, dtype=torch.bfloat16, device="cuda")

    def run(self, ctx, out, table=None):
        ctx.kv_attention(self.cache, self.q, self.starts, self.table if table is None else table, self.lens, out,
                         max_new=self.new)


KINDS = {"few rows": (40_000, 2, 0), "many rows": (20_000, 40, 3_400_000)}


@pytest.mark.parametrize("kind", list(KINDS))
def test_a_call_right_after_a_reported_error(kind):
    """On a stream that is not ordered with the default one: what the report clears is clear before the next
    call's CTAs count their parts."""
    call = Call(*KINDS[kind])
    s = torch.cuda.Stream()
    with dcl.Context(None, 1, 1, stream=s.cuda_stream) as ctx, torch.cuda.stream(s):
        want = call.out()
        call.run(ctx, want)
        ctx.synchronise()
        assert torch.isfinite(want).all()
        outs = [call.out() for _ in range(30)]
        for out in outs:
            call.run(ctx, call.out(), call.bad)
            with pytest.raises(dcl.DcleapError, match="outside the paged cache"):
                ctx.synchronise()
            call.run(ctx, out)
            call.run(ctx, out)
        ctx.synchronise()
        assert all(torch.equal(out, want) for out in outs)


def _captured(ctx, s, call, out):
    """A graph of one call, made on the stream s (the context's)."""
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g, stream=s):
        call.run(ctx, out)
    return g


@pytest.mark.parametrize("first", list(KINDS))
def test_one_call_of_any_size_prepares_every_capture(first):
    """After a small call of either kernel a call of both can be captured, and replays give what they gave."""
    calls = {kind: Call(*KINDS[kind]) for kind in KINDS}
    s = torch.cuda.Stream()
    with dcl.Context(None, 1, 1, stream=s.cuda_stream) as ctx:
        with torch.cuda.stream(s):
            n, new, wide = KINDS[first]
            small = Call(100, new, wide)
            small.run(ctx, small.out())
            outs = {kind: call.out() for kind, call in calls.items()}
            ctx.synchronise()
        graphs = {kind: _captured(ctx, s, call, outs[kind]) for kind, call in calls.items()}
        with torch.cuda.stream(s):
            want = {kind: call.out() for kind, call in calls.items()}
            for kind, call in calls.items():
                call.run(ctx, want[kind])
            for _ in range(3):
                for out in outs.values():
                    out.fill_(7.0)
                for g in graphs.values():
                    g.replay()
                ctx.synchronise()
                for kind in KINDS:
                    assert torch.equal(outs[kind], want[kind])


@pytest.mark.parametrize("kind", list(KINDS))
def test_the_first_call_is_not_captured(kind):
    """It is refused, and the capture and the context stay usable."""
    call = Call(*KINDS[kind])
    s = torch.cuda.Stream()
    with dcl.Context(None, 1, 1, stream=s.cuda_stream) as ctx:
        out, other = call.out(), torch.zeros(4, device="cuda")
        torch.cuda.synchronize()
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g, stream=s):
            other.add_(1.0)
            with pytest.raises(dcl.DcleapError, match="cannot be captured") as e:
                call.run(ctx, out)
        assert e.value.status == dcl.DCL_ERR_STATE
        with torch.cuda.stream(s):
            g.replay()
            call.run(ctx, out)
            ctx.synchronise()
        assert (other == 1).all() and (out != 7).any()
