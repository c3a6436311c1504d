"""dcl_kv_attention over a 4-bit cache against a plain attention in 64 bits over the values it stores.

Tolerance.  The operands are exact (q and every stored value are bf16).  A score is a sum of hd products
in fp32, off by at most d = hd 2^-24 S, S the largest sum |q_i k_i| scale of the row; weights are off by
that much of themselves, by 2^-16 (two bf16 parts) and 2^-20 (exp2, factors); sums over n keys by n 2^-23.  The
weights' errors stand in the numerator and in the denominator, so with A = sum p |v| a component is off by
at most (2 d + 2^-14 + n 2^-22) A, and by half a step of bf16, 2^-8 |o|.  Weights are held in fp32 and bf16 down to
2^-126, against a reference of which the row's largest is 2^-32 at least (the reference stands 32 above it when it
is taken, and it only grows until it is taken again): those below 2^-94 of the row's largest are none, and those
below 2^-86 may lose their second part, 2^-8 of them; both are at most 2^-94 of the largest each, so n 2^-93
max |v| in all.  The log-sum-exp is off by d + 2^-20 (1 + |lse|) + n 2^-23."""
import numpy as np
import pytest
import torch

import paper_2607_20467_gb300 as dcl
import synthetic as syn
from oracle import q4

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def ops():
    import __graft_entry__
    __graft_entry__.build()
    ctx = dcl.Context(None, 1, 1)
    yield ctx
    ctx.close()


def _pool(rng, lens, kv, hd, page_len, spread=3, k_scale=1.0):
    """A 4-bit cache holding sequences of these lengths in shuffled pages, every place past a length with a
    scale that reads as NaN, its page table, and what it stores in 64 bits (per sequence [n][kv][hd])."""
    need = [-(-n // page_len) for n in lens]
    pages = sum(need) + 2
    order = rng.permutation(pages)
    table = np.full((len(lens), max(max(need), 1) + 1), -1, np.int32)
    host, at = {}, 0
    for name in ("k", "v"):
        size = np.exp2(rng.integers(-spread, spread + 1, (pages, kv, page_len, hd // 32, 1)).astype(np.float64))
        a = rng.normal(0, 1, (pages, kv, page_len, hd // 32, 32)) * size * (k_scale if name == "k" else 1.0)
        host[name] = q4.encode(a.reshape(pages, kv, page_len, hd))
    used = np.zeros((pages, page_len), bool)
    values = {"k": [], "v": []}
    for b, n in enumerate(lens):
        table[b, :need[b]] = order[at:at + need[b]]
        at += need[b]
        for j in range(n):
            used[table[b, j // page_len], j % page_len] = True
        for name in ("k", "v"):
            full = q4.decode(*(x[table[b, :need[b]]] for x in host[name]))
            values[name].append(full.transpose(0, 2, 1, 3).reshape(-1, kv, hd)[:n])
    cache = dcl.KvCache.empty(pages, page_len, kv, hd, q4=True)
    for name in ("k", "v"):
        codes, b = host[name]
        b = np.where(used[:, None, :, None], b, rng.integers(252, 256, b.shape)).astype(np.uint8)
        getattr(cache, name).copy_(torch.from_numpy(q4.pack(codes)))
        getattr(cache, name + "_exp").copy_(torch.from_numpy(b))
    return cache, torch.from_numpy(table).cuda(), values


def _reference(q, k, v, causal, scale):
    """o, lse, A, S of one sequence: q [new][H][hd], k, v [n][kv][hd] in 64 bits."""
    new, H, hd = q.shape
    n, kv, _ = k.shape
    o, A = np.zeros((new, H, hd)), np.zeros((new, H, hd))
    lse, S = np.full((new, H), -np.inf), np.zeros((new, H))
    for h in range(H):
        s = q[:, h] @ k[:, h // (H // kv)].T * scale
        big = np.abs(q[:, h]) @ np.abs(k[:, h // (H // kv)]).T * scale
        seen = np.ones((new, n), bool)
        if causal:
            seen = np.arange(n) <= (n - new + np.arange(new))[:, None]
        rows = seen.any(1)
        if not rows.any():
            continue
        s = np.where(seen, s, -np.inf)[rows]
        w = np.exp(s - s.max(1, keepdims=True))
        t = w.sum(1, keepdims=True)
        with np.errstate(invalid="ignore"):
            o[rows, h], A[rows, h] = w / t @ v[:, h // (H // kv)], w / t @ np.abs(v[:, h // (H // kv)])
        lse[rows, h] = (s.max(1, keepdims=True) + np.log(t))[:, 0]
        S[rows, h] = np.where(seen, big, 0)[rows].max(1)
    return o, lse, A, S


def _check(ops, rng, lens, news, heads, kv, hd, page_len, causal=False, scale=None, max_new=None, q_scale=1.0, wide=0, **pool):
    cache, table, values = _pool(rng, lens, kv, hd, page_len, **pool)
    if wide:  # a page table for sequences of up to `wide` positions
        pad = torch.full((len(lens), -(-wide // page_len)), -1, dtype=torch.int32, device="cuda")
        table = torch.cat([table, pad], 1).contiguous()
    rows, gap = sum(news), 2  # gap: rows of no sequence, before the first and after the last
    q = torch.from_numpy(rng.normal(0, q_scale, (rows + 2 * gap, heads + 2, hd))).to(torch.bfloat16).cuda()
    q = q[:, 1:heads + 1]  # rows of a wider matrix
    starts = np.concatenate([[0], np.cumsum(news)]).astype(np.int32) + gap
    out = torch.full((rows + 2 * gap, heads, hd), 77.0, dtype=torch.bfloat16, device="cuda")
    lse = torch.full((rows + 2 * gap, heads), 77.0, device="cuda")
    args = (cache, q, torch.from_numpy(starts).cuda(), table, torch.tensor(lens, dtype=torch.int32, device="cuda"))
    kw = dict(max_new=max_new or max(max(news), 1), causal=causal, scale=scale or 0.0)
    ops.kv_attention(*args, out, lse=lse, **kw)
    ops.synchronise()
    for t in (out, lse):
        assert (t[:gap] == 77).all() and (t[gap + rows:] == 77).all()
    got, got_lse = out.float().cpu().numpy().astype(np.float64), lse.cpu().numpy().astype(np.float64)
    for b, n in enumerate(lens):
        sl = slice(starts[b], starts[b + 1])
        o, l, A, S = _reference(q[sl].float().cpu().numpy().astype(np.float64), values["k"][b], values["v"][b], causal,
                                scale or hd ** -0.5)
        empty = np.isneginf(l)
        assert (np.isneginf(got_lse[sl]) == empty).all() and (got[sl][empty] == 0).all()
        d = hd * 2.0 ** -24 * S
        err, most = np.abs(got[sl] - o), 2.0 ** -8 * np.abs(o) + (2 * d + 2.0 ** -14 + n * 2.0 ** -22)[..., None] * A
        most = most + n * 2.0 ** -93 * np.abs(values["v"][b]).max(initial=0.0)
        assert (err <= most + 1e-30).all(), (b, (err / (most + 1e-30)).max())
        off = np.abs(got_lse[sl][~empty] - l[~empty]) - (d + 2.0 ** -20 * (1 + np.abs(np.where(empty, 0, l))) + n * 2.0 ** -23)[~empty]
        assert (off <= 0).all(), (b, off.max())
    again, lse2 = torch.zeros_like(out), torch.zeros_like(lse)
    ops.kv_attention(*args, again, lse=lse2, **kw)
    ops.synchronise()
    assert torch.equal(again[gap:gap + rows], out[gap:gap + rows]) and torch.equal(lse2[gap:gap + rows], lse[gap:gap + rows])
    return out


HEADS = [(4, 4, 64), (2, 2, 128), (7, 1, 128), (12, 4, 64), (16, 1, 128), (20, 1, 64)]


@pytest.mark.parametrize("heads,kv,hd", HEADS)
@pytest.mark.parametrize("page_len", [16, 64])
def test_one_new_position(ops, heads, kv, hd, page_len):
    lens = [1, 0, 15, 16, 17, 127, 128, 129, 300]
    _check(ops, np.random.default_rng(heads + hd), lens, [1] * 9, heads, kv, hd, page_len)


@pytest.mark.parametrize("heads,kv,hd", HEADS)
@pytest.mark.parametrize("causal", [False, True])
def test_ragged_blocks(ops, heads, kv, hd, causal):
    lens, news = [40, 5, 0, 129, 33, 257, 3], [32, 5, 2, 0, 33, 7, 9]  # (the last has more rows than positions)
    _check(ops, np.random.default_rng(7 * heads + hd), lens, news, heads, kv, hd, 32, causal=causal)


@pytest.mark.parametrize("lens,news,heads,kv,hd,wide", [
    ([20000], [1], 7, 1, 128, 0), ([9000, 1, 3000], [1, 1, 1], 4, 2, 64, 0), ([6001], [3], 28, 4, 128, 0),
    ([4097, 2000], [32, 32], 14, 2, 128, 0), ([1500], [64], 4, 1, 64, 0), ([700, 90], [40, 9], 28, 4, 128, 30000)])
def test_sequences_that_many_ctas_share(ops, lens, news, heads, kv, hd, wide):
    _check(ops, np.random.default_rng(lens[0]), lens, news, heads, kv, hd, 64, wide=wide)


@pytest.mark.parametrize("lens,new", [([768] * 29, 1), ([768] * 28 + [897], 1), ([760, 768] * 14, 3), ([768] * 28 + [100], 2)])
def test_as_many_items_as_there_are_ctas(ops, lens, new):
    """Sequences of one length, about a CTA's share (none is cut), of almost one, and one that is none of it."""
    _check(ops, np.random.default_rng(len(lens) + new), lens, [new] * len(lens), 4, 4, 64, 64)


@pytest.mark.parametrize("lens,news,heads,kv,hd", [
    ([9000], [3], 5, 1, 64), ([7000], [29], 1, 1, 128), ([6100, 9300, 50], [8, 4, 1], 3, 1, 128), ([6000, 15000], [14, 2], 1, 1, 64),
    ([40000], [1], 1, 1, 64), ([33000], [7], 1, 1, 128), ([18000, 29000, 5], [1, 2, 1], 4, 1, 64), ([16500, 0, 29000], [1, 1, 1], 2, 2, 128)])
def test_joins_in_two_steps(ops, lens, news, heads, kv, hd):
    """Items that more than 10 CTAs share (48 of up to 8 rows), beside ones that fewer do."""
    _check(ops, np.random.default_rng(lens[0]), lens, news, heads, kv, hd, 128)


@pytest.mark.parametrize("page_len", [16, 256])
@pytest.mark.parametrize("hd", [64, 128])
def test_many_rows_of_a_kv_head(ops, hd, page_len):
    _check(ops, np.random.default_rng(hd + page_len), [3000, 1000, 64, 1], [33, 40, 20, 1], 28, 4, hd, page_len)


@pytest.mark.parametrize("page_len,heads,kv", [(16, 28, 4), (64, 16, 1), (128, 33, 3)])
@pytest.mark.parametrize("hd", [64, 128])
def test_many_rows_under_a_wide_table(ops, hd, page_len, heads, kv):
    """Page tables as wide as those of long sequences: the kernel for many rows."""
    _check(ops, np.random.default_rng(hd + page_len), [700, 0, 90, 129], [40, 3, 9, 32], heads, kv, hd, page_len, wide=40000)


def test_pages_past_four_gigabytes(ops):
    heads, hd, page_len, pages = 32, 128, 256, 8300  # 4.35 GB of codes each
    cache = dcl.KvCache.empty(pages, page_len, heads, hd, q4=True)
    rng = np.random.default_rng(4)
    k, v = (syn.round_bf16(rng.normal(0, 1, (300, heads, hd)).astype(np.float32)) for _ in range(2))
    table = torch.tensor([[8299, 8250]], dtype=torch.int32, device="cuda")
    at = np.arange(300)
    slots = torch.from_numpy((np.array([8299, 8250])[at // 256] * 256 + at % 256).astype(np.int32)).cuda()
    bf = lambda a: torch.from_numpy(a).to(torch.bfloat16).cuda()
    ops.kv_write(cache, bf(k), bf(v), slots)
    i32 = lambda *a: torch.tensor(a, dtype=torch.int32, device="cuda")
    for new in (1, 12, 40):
        q = bf(rng.normal(0, 1, (new, heads, hd)).astype(np.float32))
        out = torch.empty_like(q)
        ops.kv_attention(cache, q, i32(0, new), table, i32(300), out, max_new=new)
        ops.synchronise()
        o, _, A, _ = _reference(q.double().cpu().numpy(), q4.decode(*q4.encode(k)), q4.decode(*q4.encode(v)), False, hd ** -0.5)
        assert (np.abs(out.double().cpu().numpy() - o) <= 2.0 ** -8 * np.abs(o) + 2.0 ** -12 * A).all()


def test_sizes_far_apart_and_sharp_scores(ops):
    rng = np.random.default_rng(11)
    _check(ops, rng, [500, 130], [3, 20], 8, 2, 128, 16, spread=14, k_scale=2.0 ** -10)  # groups 2^28 apart
    _check(ops, rng, [500, 130], [1, 5], 8, 2, 64, 16, q_scale=8.0, scale=0.7)


def test_max_new_above_the_rows_there_are(ops):
    _check(ops, np.random.default_rng(5), [300, 200], [1, 3], 8, 8, 128, 32, max_new=17)


@pytest.mark.parametrize("new,H", [(20, 4), (4, 2), (7, 1)])  # (a pass for many rows, and one for up to 8)
@pytest.mark.parametrize("hd", [64, 128])
def test_a_group_without_numbers_is_seen_by_its_rows_only(ops, hd, new, H):
    """A key's group makes every row that sees it NaN, a value's group its components; rows before it (causal) and
    other groups are as without it."""
    rng = np.random.default_rng(hd)
    n = 70
    cache, table, _ = _pool(rng, [n], 1, hd, 16)
    q = torch.from_numpy(rng.normal(0, 1, (new, H, hd))).to(torch.bfloat16).cuda()
    i32 = lambda *a: torch.tensor(a, dtype=torch.int32, device="cuda")
    args = (q, i32(0, new), table, i32(n))
    def run(causal):
        out = torch.empty_like(q)
        ops.kv_attention(cache, *args, out, max_new=new, causal=causal)
        ops.synchronise()
        return out
    plain = run(True)
    for pos in (5, 55, 67, 69):  # 5 is seen by all rows, 69 by the last alone
        page, place = int(table[0, pos // 16]), pos % 16
        sees = np.arange(new) + n - new >= pos
        g = 1
        was = int(cache.v_exp[page, 0, place, g])
        cache.v_exp[page, 0, place, g] = 254
        out, full = run(True), run(False)
        cache.v_exp[page, 0, place, g] = was
        nan = torch.isnan(out)
        assert nan[sees][:, :, 32 * g:32 * g + 32].all() and not nan[~sees].any()
        other = torch.ones(hd, dtype=torch.bool, device="cuda")
        other[32 * g:32 * g + 32] = False
        assert torch.equal(out[:, :, other], plain[:, :, other]) and torch.equal(out[~sees], plain[~sees])
        assert torch.isnan(full[:, :, 32 * g:32 * g + 32]).all() and not torch.isnan(full[:, :, other]).any()
        was = int(cache.k_exp[page, 0, place, 0])
        cache.k_exp[page, 0, place, 0] = 255
        out = run(True)
        cache.k_exp[page, 0, place, 0] = was
        assert torch.isnan(out[sees]).all() and torch.equal(out[~sees], plain[~sees])


@pytest.mark.parametrize("P", [16, 32])
@pytest.mark.parametrize("heads", [4, 24])
def test_a_page_outside_the_cache_is_reported_and_left_out(ops, P, heads):
    rng = np.random.default_rng(2)
    cache, table, values = _pool(rng, [3 * P, 20], 2, 64, P)
    table[0, 1] = 1 << 20
    q = torch.from_numpy(rng.normal(0, 1, (2, heads, 64))).to(torch.bfloat16).cuda()
    i32 = lambda *a: torch.tensor(a, dtype=torch.int32, device="cuda")
    out = torch.empty_like(q)
    ops.kv_attention(cache, q, i32(0, 1, 2), table, i32(3 * P, 20), out, max_new=1)
    with pytest.raises(dcl.DcleapError, match="outside the paged cache"):
        ops.synchronise()
    assert torch.isfinite(out.float()).all()
    keep = np.r_[0:P, 2 * P:3 * P]
    for b, (k, v) in enumerate(((values["k"][0][keep], values["v"][0][keep]), (values["k"][1], values["v"][1]))):
        o, _, A, _ = _reference(q[b:b + 1].float().cpu().numpy().astype(np.float64), k, v, False, 0.125)
        assert (np.abs(out[b].float().cpu().numpy() - o[0]) <= 2.0 ** -8 * np.abs(o[0]) + 2.0 ** -12 * A[0]).all()
    ops.synchronise()


def test_a_captured_call_follows_the_lengths(ops):
    """One graph, replayed with other lengths and pages, gives what eager calls give."""
    rng = np.random.default_rng(9)
    cache, table, _ = _pool(rng, [400, 90], 2, 128, 16)
    q = torch.from_numpy(rng.normal(0, 1, (2, 8, 128))).to(torch.bfloat16).cuda()
    i32 = lambda *a: torch.tensor(a, dtype=torch.int32, device="cuda")
    starts, lens = i32(0, 1, 2), i32(400, 90)
    out, eager = torch.empty_like(q), torch.empty_like(q)
    stream = torch.cuda.Stream()
    with dcl.Context(None, 1, 1, stream=stream.cuda_stream) as ctx:
        torch.cuda.synchronize()
        ctx.kv_attention(cache, q, starts, table, lens, out, max_new=1)
        ctx.synchronise()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=stream):
            ctx.kv_attention(cache, q, starts, table, lens, out, max_new=1)
        for a, b in ((400, 90), (1, 0), (33, 89)):
            lens.copy_(i32(a, b))
            ops.kv_attention(cache, q, starts, table, lens, eager, max_new=1)
            ops.synchronise()
            torch.cuda.synchronize()
            graph.replay()
            torch.cuda.synchronize()
            assert torch.equal(out, eager)
        ctx.synchronise()


@pytest.mark.parametrize("page_len,heads,kv", [(16, 28, 4), (64, 16, 1), (128, 33, 3)])
@pytest.mark.parametrize("hd", [64, 128])
def test_many_causal_rows_under_a_wide_table(ops, hd, page_len, heads, kv):
    """The kernel for many rows, each of which sees the keys up to its own: as many new positions as there are (a
    prompt), more, which leaves rows that see none, and few; lengths that end inside units and pages."""
    lens, news = [700, 0, 90, 129, 300, 33, 257], [40, 3, 9, 32, 300, 50, 1]
    _check(ops, np.random.default_rng(hd + page_len), lens, news, heads, kv, hd, page_len, causal=True, wide=200000)


def test_a_long_causal_block_that_many_ctas_share(ops):
    _check(ops, np.random.default_rng(21), [4500, 900], [90, 600], 14, 2, 128, 64, causal=True, wide=200000)


@pytest.mark.parametrize("hd", [64, 128])
def test_a_group_without_numbers_under_many_causal_rows(ops, hd):
    """As for few rows: every row that sees a key without numbers gets NaN, those before it nothing of it; two values'
    groups at once, one of them in a unit that only some rows see."""
    rng = np.random.default_rng(hd)
    n, new, H = 300, 200, 7
    cache, table, _ = _pool(rng, [n, 140], 1, hd, 16)
    table = torch.cat([table, torch.full((2, 60000), -1, dtype=torch.int32, device="cuda")], 1).contiguous()
    news = [new, 20]
    q = torch.from_numpy(rng.normal(0, 1, (sum(news), H, hd))).to(torch.bfloat16).cuda()
    i32 = lambda *a: torch.tensor(a, dtype=torch.int32, device="cuda")

    def run():
        out = torch.empty_like(q)
        ops.kv_attention(cache, q, i32(0, new, sum(news)), table, i32(n, 140), out, max_new=new, causal=True)
        ops.synchronise()
        return out[:new], out[new:]

    plain, plain2 = run()
    last = hd // 32 - 1
    for first, second in ((5, 101), (99, 100), (100, 127), (128, 299), (299, 200), (255, 256)):
        sees = [torch.from_numpy(np.arange(new) + n - new >= pos).cuda() for pos in (first, second)]
        where = [(int(table[0, pos // 16]), 0, pos % 16, g) for pos, g in ((first, 0), (second, last))]
        was = [int(cache.v_exp[w]) for w in where]
        for w, byte in zip(where, (252, 255)):
            cache.v_exp[w] = byte
        out, out2 = run()
        for w, byte in zip(where, was):
            cache.v_exp[w] = byte
        want = torch.zeros(new, H, hd, dtype=torch.bool, device="cuda")
        want[:, :, :32] |= sees[0][:, None, None]
        want[:, :, 32 * last:] |= sees[1][:, None, None]
        assert torch.equal(torch.isnan(out), want) and torch.equal(out[~want], plain[~want]) and torch.equal(out2, plain2)
        was = int(cache.k_exp[where[1]])
        cache.k_exp[where[1]] = 253
        out, out2 = run()
        cache.k_exp[where[1]] = was
        assert torch.isnan(out[sees[1]]).all() and torch.equal(out[~sees[1]], plain[~sees[1]]) and torch.equal(out2, plain2)
