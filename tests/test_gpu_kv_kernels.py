"""dcl_kv_attention's kernels on the same inputs, and blocks longer than a row tile.

The kernel is chosen by max_new and the page table's width: up to 8, 16 and 32 rows of a kv head (max_new x
the query heads that share it), and, where the table has room for millions of positions, the one for many
rows.  Every one serves whatever rows there are.  Tolerance against the definition in 64 bits: 2^-8 of
the output (its bf16 rounding) and 2^-12 A, A = sum p |v|; two kernels may differ by twice that."""
import numpy as np
import pytest
import torch

import paper_2607_20467_gb300 as dcl
from test_gpu_kv_range import Case

pytestmark = pytest.mark.gpu

WIDE = 3_400_000


@pytest.fixture(scope="module")
def ops():
    import __graft_entry__
    __graft_entry__.build()
    ctx = dcl.Context(None, 1, 1)
    yield ctx
    ctx.close()


def _attend(ops, c, q, max_new, wide, causal=False):
    new, heads, hd = q.shape
    width = max(len(c.order), -(-wide // c.page_len))
    table = torch.full((1, width), -1, dtype=torch.int32, device="cuda")
    table[0, :len(c.order)] = torch.from_numpy(c.order.astype(np.int32))
    out = torch.full((new, heads, hd), 77.0, dtype=torch.bfloat16, device="cuda")
    lse = torch.full((new, heads), 77.0, device="cuda")
    i32 = lambda a: torch.tensor(a, dtype=torch.int32, device="cuda")
    ops.kv_attention(c.cache, q, i32([0, new]), table, i32([c.n]), out, max_new=max_new, causal=causal, lse=lse)
    ops.synchronise()
    return out.double(), lse.double()


@pytest.mark.parametrize("fp8", [True, False])
@pytest.mark.parametrize("hd", [64, 128])
@pytest.mark.parametrize("n,new", [(1, 1), (37, 2), (700, 2), (5001, 2), (900, 30)])
def test_each_kernel_on_the_same_rows(ops, n, new, hd, fp8):
    rng = np.random.default_rng(n + new)
    k, v = rng.normal(0, 1, (2, n, 2, hd))
    c = Case(ops, k, v, fp8)
    q = torch.from_numpy(rng.normal(0, 2, (new, 8, hd))).to(torch.bfloat16).cuda()  # 4 heads a kv head
    o, A, l = c.reference(q)
    room = 2.0 ** -8 * o.abs() + 2.0 ** -12 * A
    outs = []
    for max_new, wide in ((2, 0), (4, 0), (8, 0), (64, WIDE)):
        out, lse = _attend(ops, c, q, max_new, wide)
        assert ((out - o).abs() <= room).all(), (max_new, wide)
        assert ((lse - l).abs() <= 1e-4 * (1 + l.abs())).all(), (max_new, wide)
        assert all(((out - x).abs() <= 2 * room).all() for x in outs), (max_new, wide)
        outs.append(out)


@pytest.mark.parametrize("fp8", [True, False])
@pytest.mark.parametrize("causal", [False, True])
@pytest.mark.parametrize("n,new,heads,kv,hd", [(300, 300, 4, 2, 64), (1025, 257, 7, 1, 128), (700, 511, 2, 2, 128)])
def test_a_whole_prompt(ops, n, new, heads, kv, hd, causal, fp8):
    """Hundreds of new positions: tens of row tiles of the kernel for 32 rows (causal), several of the one
    for many (a wide table)."""
    rng = np.random.default_rng(n + new)
    k, v = rng.normal(0, 1, (2, n, kv, hd))
    c = Case(ops, k, v, fp8)
    q = torch.from_numpy(rng.normal(0, 1, (new, heads, hd))).to(torch.bfloat16).cuda()
    o, A, l = c.reference(q, causal)
    for wide in (0, WIDE):
        out, lse = _attend(ops, c, q, new, wide, causal)
        assert ((out - o).abs() <= 2.0 ** -8 * o.abs() + 2.0 ** -12 * A).all()
        assert ((lse - l).abs() <= 1e-4 * (1 + l.abs())).all()
