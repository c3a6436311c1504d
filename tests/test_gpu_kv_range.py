"""dcl_kv_attention over the range of what a cache can hold, by each of its kernels, against a plain
attention in 64 bits over the stored values (dcl_kv_read gives them exactly).

Tolerance.  A component's error is at most 2^-8 of itself for the output's bf16 (half a unit in the last place
of a number just above a power of two), and 2^-12 of A = sum p |v| for the weights' two parts (2^-16
of each and less), the scores and the sums."""
import numpy as np
import pytest
import torch

import paper_2607_20467_gb300 as dcl

pytestmark = pytest.mark.gpu

# (query heads of a kv head, new positions, positions that the page table has room for): how many rows share
# a kv head's keys, and a table wide enough for the kernel of many rows
KERNELS = {"8 rows": (4, 2, 0), "16 rows": (4, 4, 0), "32 rows": (4, 8, 0), "many rows": (4, 40, 3_400_000)}
FEW = ["8 rows", "16 rows", "32 rows"]


@pytest.fixture(scope="module")
def ops():
    import __graft_entry__
    __graft_entry__.build()
    ctx = dcl.Context(None, 1, 1)
    yield ctx
    ctx.close()


class Case:
    """One sequence of the keys and values k, v [n][kv][hd] (rounded to bf16, then stored), and what a
    cache returns of them in 64 bits."""

    def __init__(self, ops, k, v, fp8, page_len=32, seed=0):
        n, kv, hd = k.shape
        self.n, self.page_len = n, page_len
        pages = -(-n // page_len)
        self.cache = dcl.KvCache.empty(pages, page_len, kv, hd, fp8=fp8)
        for t in (self.cache.k, self.cache.v):
            t.view(torch.uint8).fill_(0x7F)  # (what no key was written to is no number)
        order = np.random.default_rng(seed).permutation(pages)
        at = np.arange(n)
        slots = torch.from_numpy((order[at // page_len] * page_len + at % page_len).astype(np.int32)).cuda()
        bf = [torch.as_tensor(x).to(torch.bfloat16).cuda().contiguous() for x in (k, v)]
        ops.kv_write(self.cache, bf[0], bf[1], slots)
        back = [torch.empty_like(x) for x in bf]
        ops.kv_read(self.cache, slots, *back)
        ops.synchronise()
        self.k, self.v = (x.double() for x in back)
        self.order = order

    def attend(self, ops, q, causal=False, scale=None, wide=0):
        """out, lse of the rows q [new][heads][hd]."""
        new, heads, hd = q.shape
        width = max(len(self.order), -(-wide // self.page_len))
        table = torch.full((1, width), -1, dtype=torch.int32, device="cuda")
        table[0, :len(self.order)] = torch.from_numpy(self.order.astype(np.int32))
        out = torch.full((new, heads, hd), 77.0, dtype=torch.bfloat16, device="cuda")
        lse = torch.full((new, heads), 77.0, device="cuda")
        i32 = lambda a: torch.tensor(a, dtype=torch.int32, device="cuda")
        ops.kv_attention(self.cache, q, i32([0, new]), table, i32([self.n]), out, max_new=new, causal=causal,
                         scale=scale or 0.0, lse=lse)
        ops.synchronise()
        return out.double(), lse.double()

    def reference(self, q, causal=False, scale=None):
        """o, A, lse in 64 bits."""
        new, heads, hd = q.shape
        kv = self.k.shape[1]
        rep = heads // kv
        k, v = (x.repeat_interleave(rep, 1) for x in (self.k, self.v))
        s = torch.einsum("ihd,jhd->hij", q.double(), k) * (scale or hd ** -0.5)
        if causal:
            j, i = torch.arange(self.n, device="cuda"), torch.arange(new, device="cuda")
            s = s.masked_fill(j[None, :] > (self.n - new + i)[:, None], -np.inf)
        p = torch.softmax(s, -1)
        return (torch.einsum("hij,jhd->ihd", p, v), torch.einsum("hij,jhd->ihd", p, v.abs()), torch.logsumexp(s, -1).T)

    def check(self, ops, q, causal=False, scale=None, wide=0):
        out, lse = self.attend(ops, q, causal, scale, wide)
        o, A, l = self.reference(q, causal, scale)
        bad = (out - o).abs() - (2.0 ** -8 * o.abs() + 2.0 ** -12 * A)
        assert (bad <= 0).all(), float(((out - o).abs() / A).max())
        S = torch.einsum("ihd,jhd->ihj", q.double().abs(), self.k.abs().repeat_interleave(q.shape[1] // self.k.shape[1], 1))
        S = S.amax(-1) * (scale or q.shape[2] ** -0.5)
        assert ((lse - l).abs() <= 1e-5 * (1 + S)).all()


def _q(rng, kernel, kv, hd, scale=1.0):
    rep, new, _ = KERNELS[kernel]
    return torch.from_numpy(rng.normal(0, scale, (new, rep * kv, hd))).to(torch.bfloat16).cuda()


def _sharp(rng, kernel, k):
    """Rows that each see one key of its own (77 binades above the rest, and more), and which."""
    rep, new, _ = KERNELS[kernel]
    n, kv, hd = k.shape
    which = rng.integers(0, n, (new, rep * kv))
    unit = k / np.sqrt((k ** 2).mean(-1, keepdims=True))
    q = np.stack([unit[which[:, h], h // rep] for h in range(rep * kv)], 1) / np.sqrt((k ** 2).mean())
    return torch.from_numpy(8.0 * q).to(torch.bfloat16).cuda()


@pytest.mark.parametrize("kernel", FEW)
@pytest.mark.parametrize("fp8", [True, False])
def test_weights_keep_more_bits_than_the_output(ops, kernel, fp8):
    """Fifteen of sixteen keys have a weight just under half-way between two numbers of 11 bits, all to the same
    side, and every component another mixture of 1 and 1.125: weights of 11 bits would be off by 2^-11 in all of
    them, on top of the output's rounding wherever that comes out at its worst."""
    hd, n = 64, 4096
    rep, new, wide = KERNELS[kernel]
    first = np.arange(n) % 16 == 5  # (one in every step of 16 keys: the reference is theirs)
    k = np.zeros((n, 1, hd))
    k[~first, 0, 0], k[~first, 0, 1] = -1.0, 1.0
    order = np.random.default_rng(3).permutation(np.flatnonzero(~first))
    v = np.ones((n, 1, hd))
    for d in range(hd):
        v[order[:100 + 2 * d], 0, d] = 1.125
    q = torch.zeros(new, rep, hd, dtype=torch.bfloat16, device="cuda")
    q[:, :, 0] = 1.0
    q[:, :, 1] = 0.97 * 2.0 ** -11 * np.log2(np.e)
    Case(ops, k, v, fp8).check(ops, q, scale=float(np.log(2.0)), wide=wide)


@pytest.mark.parametrize("kernel", FEW)
@pytest.mark.parametrize("hd", [64, 128])
@pytest.mark.parametrize("down", [16, 24, 32, 50])
def test_zero_vectors_do_not_cost_small_values_their_bits(ops, kernel, hd, down):
    """Zero vectors are stored with exponent 0, whatever the others' sizes."""
    rng = np.random.default_rng(down)
    n = 300
    for zero in (rng.random(n) < 0.3, np.arange(n) < 150, np.arange(n) >= 150, np.arange(n) % 32 != 7):
        k, v = rng.normal(0, 1, (2, n, 2, hd))
        v = np.where(zero[:, None, None], 0.0, v * 2.0 ** -down)
        c = Case(ops, k, v, True)
        c.check(ops, _q(rng, kernel, 2, hd), wide=KERNELS[kernel][2])
        c.check(ops, _q(rng, kernel, 2, hd, 5.0), causal=True, wide=KERNELS[kernel][2])


@pytest.mark.parametrize("kernel", FEW)
def test_zero_vectors_alone(ops, kernel):
    rng = np.random.default_rng(1)
    k = rng.normal(0, 1, (200, 1, 64))
    Case(ops, k, np.zeros_like(k), True).check(ops, _q(rng, kernel, 1, 64), wide=KERNELS[kernel][2])


@pytest.mark.parametrize("kernel", FEW)
@pytest.mark.parametrize("hd", [64, 128])
def test_sizes_at_both_ends_of_the_exponents(ops, kernel, hd):
    """Values of 2^-55 that have nearly all of the weight beside some of 2^118 that have 2^-30 of it, and so
    decide the result: the sum of the weights counts the first."""
    rng = np.random.default_rng(2)
    n, rep, new = 260, *KERNELS[kernel][:2]
    large = rng.permutation(n) < 40
    k = np.zeros((n, 1, hd))
    k[:, 0, 0] = np.where(large, -30.0, 0.0)
    k[:, 0, 1:] = 0.05 * rng.normal(0, 1, (n, hd - 1))
    v = rng.normal(0, 1, (n, 1, hd)) * np.where(large, 2.0 ** 118, 2.0 ** -55)[:, None, None]
    c = Case(ops, k, v, True)
    q = rng.normal(0, 1, (new, rep, hd))
    q[:, :, 0] = 1.0
    q = torch.from_numpy(q).to(torch.bfloat16).cuda()
    c.check(ops, q, scale=float(np.log(2.0)), wide=KERNELS[kernel][2])


@pytest.mark.parametrize("kernel", list(KERNELS))
@pytest.mark.parametrize("hd", [64, 128])
@pytest.mark.parametrize("spread", [12, 20, 30])
def test_a_row_that_sees_one_small_value_among_large_ones(ops, kernel, hd, spread):
    """Values of sizes 2^-spread to 2^spread side by side."""
    rng = np.random.default_rng(spread)
    n = 200
    k, v = rng.normal(0, 1, (2, n, 2, hd))
    v *= np.exp2(rng.integers(-spread, spread + 1, (n, 2, 1)))
    for fp8 in (True, False):
        Case(ops, k, v, fp8).check(ops, _sharp(rng, kernel, k), wide=KERNELS[kernel][2])


@pytest.mark.parametrize("kernel", list(KERNELS))
def test_small_keys_beside_large_ones_that_have_no_weight(ops, kernel):
    """Keys of 2^25 against the rows' direction, between keys of 2^-8 whose scores are small numbers."""
    rng = np.random.default_rng(4)
    n, hd = 150, 64
    rep, new, wide = KERNELS[kernel]
    k = 2.0 ** -8 * rng.normal(0, 1, (n, 1, hd))
    k[:, :, 0] = 0.0
    k[::5] = 0.0
    k[::5, :, 0] = -2.0 ** 25
    v = rng.normal(0, 1, (n, 1, hd))
    q = 2.0 ** 8 * rng.normal(0, 1, (new, rep, hd))
    q[:, :, 0] = 2.0 ** 8
    q = torch.from_numpy(q).to(torch.bfloat16).cuda()
    for fp8 in (True, False):
        Case(ops, k, v, fp8).check(ops, q, wide=wide)


@pytest.mark.parametrize("kernel", list(KERNELS))
@pytest.mark.parametrize("down", [16, 24, 32, 50])
def test_pages_of_zeros_between_small_values(ops, kernel, down):
    rng = np.random.default_rng(down)
    n, hd = 320, 64
    k, v = rng.normal(0, 1, (2, n, 2, hd))
    v *= 2.0 ** -down
    for zero in (np.arange(n) // 32 % 2 == 0, rng.random(n) < 0.3):
        for fp8 in (True, False):
            c = Case(ops, k, np.where(zero[:, None, None], 0.0, v), fp8)
            c.check(ops, _q(rng, kernel, 2, hd), wide=KERNELS[kernel][2])


@pytest.mark.parametrize("kernel", list(KERNELS))
@pytest.mark.parametrize("fp8", [True, False])
def test_the_largest_values(ops, kernel, fp8):
    """Values up to 2^126: their weighted sum is no larger, and no step on the way may overflow."""
    rng = np.random.default_rng(5)
    k, v = rng.normal(0, 1, (2, 40, 1, 64))
    v = np.clip(v, -3.9, 3.9) * 2.0 ** 124
    Case(ops, k, v, fp8).check(ops, _q(rng, kernel, 1, 64), wide=KERNELS[kernel][2])


@pytest.mark.parametrize("kernel", list(KERNELS))
@pytest.mark.parametrize("hd", [64, 128])
def test_infinite_values_of_bf16_pages(ops, kernel, hd):
    """An infinity that a row sees is its component's result, two of unlike sign or a NaN are no number, and
    the other components are what they were."""
    rng = np.random.default_rng(6)
    n = 700
    k, v = rng.normal(0, 1, (2, n, 2, hd))
    c = Case(ops, k, v, False)
    at = rng.permutation(n)[:6]
    w = c.v.clone()
    for j, d, x in ((at[0], 3, np.inf), (at[1], 9, -np.inf), (at[2], 20, np.inf), (at[3], 20, -np.inf),
                    (at[4], 33, np.nan), (at[5], 40, np.inf), (at[0], 40, np.inf)):
        c.cache.v[int(c.order[j // 32]), 1, int(j % 32), d] = x
        w[int(j), 1, d] = x
    q = _q(rng, kernel, 2, hd)
    rep = KERNELS[kernel][0]
    for causal in (False, True):
        o, A, _ = c.reference(q, causal)
        out, _ = c.attend(ops, q, causal, wide=KERNELS[kernel][2])
        seen = torch.ones(q.shape[0], n, dtype=torch.bool, device="cuda")
        if causal:
            j, i = torch.arange(n, device="cuda"), torch.arange(q.shape[0], device="cuda")
            seen = j[None, :] <= (n - q.shape[0] + i)[:, None]
        # the sum over the seen keys of what is no finite number of w, rows x hd
        odd = torch.where(torch.isfinite(w[:, 1]), torch.zeros_like(w[:, 1]), w[:, 1])
        odd = torch.where(seen[:, :, None], odd[None], torch.zeros_like(odd[None])).sum(1)
        odd = odd[:, None].expand(-1, rep, -1)
        got, fine = out[:, rep:], odd == 0
        assert torch.equal(got.isnan(), odd.isnan())
        assert (got[odd.isinf()] == odd[odd.isinf()]).all()
        bad = (got - o[:, rep:]).abs() - (2.0 ** -8 * o[:, rep:].abs() + 2.0 ** -12 * A[:, rep:])
        assert (bad[fine] <= 0).all()
        assert ((out - o).abs()[:, :rep] <= 2.0 ** -8 * o.abs()[:, :rep] + 2.0 ** -12 * A[:, :rep]).all()
