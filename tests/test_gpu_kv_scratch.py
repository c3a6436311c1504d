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
