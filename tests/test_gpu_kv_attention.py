"""dcl_kv_attention against a plain attention in 64 bits over the values the cache stores.

Tolerance.  The output is rounded to bf16 (2^-9 of itself), the probabilities to 16 bits (bf16 at
worst: 2^-9 of each), scores and sums are fp32.  With A = sum_j p_j |v_j| >= |o| the error of a
component is at most (2^-9 + 2^-9) A, and 2^-12 A more for the rest.  The log-sum-exp is fp32
throughout: a score is a sum of hd products, off by at most hd 2^-24 of sum |q_d k_d| scale (8e-6
of it at hd = 128), so within 1e-5 (1 + the largest such sum)."""
import numpy as np
import pytest
import torch

import paper_2607_20467_gb300 as dcl
from oracle import fp8

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def ops():
    import __graft_entry__
    __graft_entry__.build()
    ctx = dcl.Context(None, 1, 1)
    yield ctx
    ctx.close()


def _pool(rng, lens, heads, kv, hd, page_len, fp8_format, spread=3, k_scale=1.0, jump=0):
    """A cache holding sequences of these lengths in shuffled pages, every place past a length filled
    with NaN, and the values it stores in 64 bits (per sequence [n][kv][hd])."""
    need = [-(-n // page_len) for n in lens]
    pages = sum(need) + 2
    order = rng.permutation(pages)
    width = max(max(need), 1) + 1
    table = np.full((len(lens), width), -1, np.int32)
    cache = dcl.KvCache.empty(pages, page_len, kv, hd, fp8=fp8_format)
    host = {}
    for name in ("k", "v"):
        size = np.exp2(rng.integers(-spread, spread + 1, (pages, kv, page_len, 1)).astype(np.float64))
        if name == "v" and jump:  # whole pages of large and of small values
            size = size * np.exp2(jump * (np.arange(pages) % 2 * 2.0 - 1.0))[:, None, None, None]
        a = rng.normal(0, 1, (pages, kv, page_len, hd)) * size * (k_scale if name == "k" else 1.0)
        if fp8_format:
            flat = a.reshape(-1, hd)
            e = fp8.row_exponents(flat)
            codes = fp8.e4m3_encode(fp8.e4m3_round(flat * np.exp2(-e.astype(np.float64))[:, None])).reshape(a.shape)
            host[name] = [codes, e.reshape(a.shape[:3]).astype(np.int8)]
        else:
            host[name] = [torch.from_numpy(a).to(torch.bfloat16)]
    at, values = 0, {"k": [], "v": []}
    used = np.zeros((pages, page_len), bool)
    for b, n in enumerate(lens):
        table[b, :need[b]] = order[at:at + need[b]]
        at += need[b]
        for j in range(n):
            used[table[b, j // page_len], j % page_len] = True
        for name in ("k", "v"):
            if fp8_format:
                full = fp8.e4m3_decode(host[name][0]) * np.exp2(host[name][1].astype(np.float64))[..., None]
            else:
                full = host[name][0].double().numpy()
            rows = full[table[b, :need[b]]].transpose(0, 2, 1, 3).reshape(-1, kv, hd)[:n]
            values[name].append(rows)
    for name in ("k", "v"):
        dst = getattr(cache, name)
        if fp8_format:
            codes, e = host[name]
            codes = np.where(used[:, None, :, None], codes, 0x7F).astype(np.uint8)
            e = np.where(used[:, None, :], e, -128).astype(np.int8)
            dst.copy_(torch.from_numpy(codes))
            getattr(cache, name + "_exp").copy_(torch.from_numpy(e))
        else:
            a = host[name][0].clone()
            a[~torch.from_numpy(used)[:, None, :].expand(pages, kv, page_len)] = float("nan")
            dst.copy_(a)
    return cache, torch.from_numpy(table).cuda(), values


def _reference(q, k, v, new, causal, scale):
    """o, lse, A, S of one sequence: q [new][H][hd], k, v [n][kv][hd] in 64 bits."""
    n, kv, hd = k.shape
    H = q.shape[1]
    rep = H // kv
    o, lse = np.zeros((new, H, hd)), np.full((new, H), -np.inf)
    A, S = np.zeros((new, H, hd)), np.zeros((new, H))
    for i in range(new):
        m = min(n, n - new + i + 1) if causal else n
        if m <= 0:
            continue
        for h in range(H):
            kk, vv = k[:m, h // rep], v[:m, h // rep]
            s = kk @ q[i, h] * scale
            top = s.max()
            w = np.exp(s - top)
            o[i, h] = w @ vv / w.sum()
            A[i, h] = w @ np.abs(vv) / w.sum()
            S[i, h] = (np.abs(kk) @ np.abs(q[i, h])).max() * scale
            lse[i, h] = top + np.log(w.sum())
    return o, lse, A, S


def _check(ops, rng, lens, news, heads, kv, hd, page_len, fp8_format, causal=False, scale=None, max_new=None,
           q_scale=1.0, wide=0, **pool):
    cache, table, values = _pool(rng, lens, heads, kv, hd, page_len, fp8_format, **pool)
    if wide:  # a page table for sequences of up to `wide` positions
        pad = torch.full((len(lens), -(-wide // page_len)), -1, dtype=torch.int32, device="cuda")
        table = torch.cat([table, pad], 1).contiguous()
    rows = sum(news)
    gap = 2  # rows of no sequence, before the first
    q = torch.from_numpy(rng.normal(0, q_scale, (rows + gap, heads + 2, hd))).to(torch.bfloat16).cuda()
    q = q[:, 1:heads + 1]  # rows of a wider matrix
    starts = np.concatenate([[0], np.cumsum(news)]).astype(np.int32) + gap
    out = torch.full((rows + gap, heads, hd), 77.0, dtype=torch.bfloat16, device="cuda")
    lse = torch.full((rows + gap, heads), 77.0, device="cuda")
    lens_d = torch.tensor(lens, dtype=torch.int32, device="cuda")
    args = (cache, q, torch.from_numpy(starts).cuda(), table, lens_d)
    ops.kv_attention(*args, out, max_new=max_new or max(max(news), 1), causal=causal, scale=scale or 0.0, lse=lse)
    ops.synchronise()
    assert (out[:gap] == 77).all() and (lse[:gap] == 77).all()
    got, got_lse = out.float().cpu().numpy().astype(np.float64), lse.cpu().numpy().astype(np.float64)
    for b, (n, new) in enumerate(zip(lens, news)):
        sl = slice(starts[b], starts[b + 1])
        o, l, A, S = _reference(q[sl].float().cpu().numpy().astype(np.float64), values["k"][b], values["v"][b], new,
                                causal, scale or hd ** -0.5)
        empty = np.isneginf(l)
        assert (np.isneginf(got_lse[sl]) == empty).all()
        assert (got[sl][empty] == 0).all()
        err = np.abs(got[sl] - o)
        assert (err <= (2.0 ** -8 + 2.0 ** -12) * A + 1e-30).all(), (b, (err / (A + 1e-30)).max())
        bad = np.abs(got_lse[sl][~empty] - l[~empty]) - 1e-5 * (1 + S[~empty])
        assert (bad <= 0).all(), (b, bad.max())
    again, lse2 = torch.zeros_like(out), torch.zeros_like(lse)
    ops.kv_attention(*args, again, max_new=max_new or max(max(news), 1), causal=causal, scale=scale or 0.0, lse=lse2)
    ops.synchronise()
    assert torch.equal(again[gap:], out[gap:]) and torch.equal(lse2[gap:], lse[gap:])  # bit for bit
    return out[gap:]


HEADS = [(4, 4, 64), (2, 2, 128), (7, 1, 128), (12, 4, 64), (16, 1, 128), (20, 1, 64)]


@pytest.mark.parametrize("fp8_format", [True, False])
@pytest.mark.parametrize("heads,kv,hd", HEADS)
def test_one_token(ops, heads, kv, hd, fp8_format):
    rng = np.random.default_rng(heads * hd)
    lens = [1, 0, 2, 15, 16, 17, 31, 33, 64, 127, 128, 129, 500, 1031]
    _check(ops, rng, lens, [1] * len(lens), heads, kv, hd, 16, fp8_format)


@pytest.mark.parametrize("fp8_format", [True, False])
@pytest.mark.parametrize("causal", [False, True])
@pytest.mark.parametrize("heads,kv,hd,page_len", [(4, 4, 64, 32), (2, 2, 128, 64), (14, 2, 128, 16), (8, 1, 64, 128),
                                                  (28, 4, 128, 256)])
def test_ragged_blocks(ops, heads, kv, hd, page_len, causal, fp8_format):
    """From no new position to 70 of each sequence; causal rows that see nothing (fewer cached than
    new positions) among them."""
    rng = np.random.default_rng(heads * hd + page_len)
    lens = [40, 0, 300, 129, 5, 64, 70, 257, 1]
    news = [32, 3, 1, 17, 9, 0, 70, 33, 1]
    _check(ops, rng, lens, news, heads, kv, hd, page_len, fp8_format, causal=causal)


# Many rows that share a kv head are given to another kernel where the table's width promises enough
# keys: at this width all that follow.
WIDE = 3_400_000


@pytest.mark.parametrize("fp8_format", [True, False])
@pytest.mark.parametrize("heads,kv,hd,page_len", [(4, 4, 64, 32), (2, 2, 128, 64), (14, 2, 128, 16), (8, 1, 64, 128),
                                                  (28, 4, 128, 256), (20, 1, 128, 16)])
def test_many_rows(ops, heads, kv, hd, page_len, fp8_format):
    """Up to 70 new positions (1400 rows of a kv head), ragged, one and two row tiles and several."""
    rng = np.random.default_rng(heads * hd + page_len + 1)
    lens = [40, 0, 300, 129, 5, 64, 70, 257, 1, 128, 511]
    news = [32, 3, 1, 17, 9, 0, 70, 33, 1, 40, 13]
    _check(ops, rng, lens, news, heads, kv, hd, page_len, fp8_format, wide=WIDE)


@pytest.mark.parametrize("fp8_format", [True, False])
@pytest.mark.parametrize("hd", [64, 128])
def test_many_rows_split_and_joined(ops, hd, fp8_format):
    rng = np.random.default_rng(20 + hd)
    _check(ops, rng, [9001, 700], [33, 40], 7, 1, hd, 64, fp8_format, wide=WIDE)
    _check(ops, rng, [5000], [70], 2, 2, hd, 16, fp8_format, wide=WIDE)


@pytest.mark.parametrize("fp8_format", [True, False])
@pytest.mark.parametrize("wide,news", [(0, [1, 3]), (0, [20, 30]), (WIDE, [40, 64])])
def test_values_of_unlike_size(ops, wide, news, fp8_format):
    """Values that differ by 2^24 from page to page, and by 2^40 within one: what is small is not lost where
    it is all that a row sees much of, and what it adds to the sum of the weights counts."""
    rng = np.random.default_rng(21)
    _check(ops, rng, [100, 999], news, 4, 1, 64, 64, fp8_format, wide=wide, jump=12, spread=0, k_scale=2.0 ** -6)
    _check(ops, rng, [150, 600], news, 4, 1, 128, 32, fp8_format, wide=wide, jump=12, spread=1, k_scale=6.0)
    _check(ops, rng, [100, 999], news, 4, 1, 128, 32, fp8_format, wide=wide, spread=20, k_scale=2.0 ** -20)


@pytest.mark.parametrize("fp8_format", [True, False])
def test_many_rows_of_peaked_scores(ops, fp8_format):
    rng = np.random.default_rng(22)
    _check(ops, rng, [100, 999], [40, 64], 4, 1, 64, 32, fp8_format, wide=WIDE, k_scale=30.0, q_scale=3.0)


@pytest.mark.parametrize("fp8_format", [True, False])
def test_many_rows_a_page_outside_the_cache_is_reported(ops, fp8_format):
    rng = np.random.default_rng(23)
    cache, table, values = _pool(rng, [40, 200], 4, 1, 64, 16, fp8_format)
    q = torch.from_numpy(rng.normal(0, 1, (64, 4, 64))).to(torch.bfloat16).cuda()
    starts = torch.tensor([0, 24, 64], dtype=torch.int32, device="cuda")
    out = torch.zeros(64, 4, 64, dtype=torch.bfloat16, device="cuda")
    lens = torch.tensor([40, 200], dtype=torch.int32, device="cuda")
    wide = torch.full((2, 212_500), -1, dtype=torch.int32, device="cuda")
    wide[:, :table.shape[1]] = table
    wide[0, 1] = cache.n_pages
    ops.kv_attention(cache, q, starts, wide, lens, out, max_new=40)
    with pytest.raises(dcl.DcleapError, match="outside the paged cache"):
        ops.synchronise()
    o, _, A, _ = _reference(q[24:].float().cpu().numpy().astype(np.float64), values["k"][1], values["v"][1], 40, False,
                            64 ** -0.5)
    assert (np.abs(out[24:].float().cpu().numpy() - o) <= (2.0 ** -8 + 2.0 ** -12) * A).all()


@pytest.mark.parametrize("fp8_format", [True, False])
def test_long_sequences_split_and_joined(ops, fp8_format):
    rng = np.random.default_rng(1)
    _check(ops, rng, [20011, 3], [1, 1], 7, 1, 128, 64, fp8_format)
    _check(ops, rng, [9973], [32], 4, 2, 64, 16, fp8_format, causal=True)


@pytest.mark.parametrize("fp8_format", [True, False])
def test_many_short_sequences(ops, fp8_format):
    rng = np.random.default_rng(2)
    lens = [int(x) for x in rng.integers(0, 60, 300)]
    news = [int(x) for x in rng.integers(0, 4, 300)]
    _check(ops, rng, lens, news, 4, 2, 64, 16, fp8_format, causal=True)


@pytest.mark.parametrize("fp8_format", [True, False])
def test_peaked_scores_and_unlike_vectors(ops, fp8_format):
    """Scores of several hundred (one key takes all), and vectors whose sizes differ by 2^40, so
    that a small probability may carry a large value."""
    rng = np.random.default_rng(4)
    _check(ops, rng, [100, 999], [1, 20], 4, 1, 64, 32, fp8_format, k_scale=30.0, q_scale=3.0)
    _check(ops, rng, [100, 999], [3, 40], 4, 1, 128, 32, fp8_format, spread=20, k_scale=2.0 ** -20)


def test_the_choice_of_kernel_does_not_change_a_row_beyond_rounding(ops):
    """max_new chooses the kernel; both answers are within the tolerance of the definition."""
    for most in (1, 8, 64):
        _check(ops, np.random.default_rng(5), [300, 77], [5, 8], 8, 2, 128, 32, True, max_new=max(most, 8))


def test_nan_in_a_seen_vector_reaches_the_row_and_no_other(ops):
    rng = np.random.default_rng(6)
    cache, table, _ = _pool(rng, [50, 50], 2, 2, 64, 16, True)
    cache.v[int(table[0, 1]), 0, 3, 5] = 0x7F  # sequence 0, kv head 0, one component
    q = torch.from_numpy(rng.normal(0, 1, (2, 2, 64))).to(torch.bfloat16).cuda()
    out = torch.zeros(2, 2, 64, dtype=torch.bfloat16, device="cuda")
    ops.kv_attention(cache, q, torch.tensor([0, 1, 2], dtype=torch.int32, device="cuda"), table,
                     torch.tensor([50, 50], dtype=torch.int32, device="cuda"), out, max_new=1)
    ops.synchronise()
    nan = torch.isnan(out)
    assert nan[0, 0, 5] and nan.sum() == 1


@pytest.mark.parametrize("fp8_format", [True, False])
@pytest.mark.parametrize("heads,kv,hd,new", [(2, 2, 64, 5), (2, 2, 128, 12), (4, 1, 128, 40), (8, 2, 64, 20)])
def test_causal_rows_before_a_value_that_is_no_number_do_not_see_it(ops, heads, kv, hd, new, fp8_format):
    rng = np.random.default_rng(16)
    n = 50
    cache, table, values = _pool(rng, [n], heads, kv, hd, 16, fp8_format)
    at = n - 3  # seen by the last three rows only
    page, pos = int(table[0, at // 16]), at % 16
    cache.v[page, 0, pos, 7] = 0xFF if fp8_format else float("nan")
    if not fp8_format:
        cache.v[page, 0, pos, 9] = float("inf")
    q = torch.from_numpy(rng.normal(0, 1, (new, heads, hd))).to(torch.bfloat16).cuda()
    out = torch.zeros(new, heads, hd, dtype=torch.bfloat16, device="cuda")
    ops.kv_attention(cache, q, torch.tensor([0, new], dtype=torch.int32, device="cuda"), table,
                     torch.tensor([n], dtype=torch.int32, device="cuda"), out, max_new=new, causal=True)
    ops.synchronise()
    got = out.float().cpu().numpy().astype(np.float64)
    o, _, A, _ = _reference(q.float().cpu().numpy().astype(np.float64), values["k"][0], values["v"][0], new, True,
                            hd ** -0.5)
    strange = np.zeros_like(o, bool)
    strange[-3:, :heads // kv, 7] = True
    if not fp8_format:
        strange[-3:, :heads // kv, 9] = True
        assert np.isinf(got[-3:, :heads // kv, 9]).all()
    assert np.isnan(got[-3:, :heads // kv, 7]).all()
    assert (np.abs(got - o)[~strange] <= ((2.0 ** -8 + 2.0 ** -12) * A)[~strange]).all()


def test_a_page_or_length_outside_the_cache_is_reported(ops):
    rng = np.random.default_rng(7)
    cache, table, values = _pool(rng, [40, 40], 2, 2, 64, 16, True)
    q = torch.from_numpy(rng.normal(0, 1, (2, 2, 64))).to(torch.bfloat16).cuda()
    starts = torch.tensor([0, 1, 2], dtype=torch.int32, device="cuda")
    out = torch.zeros(2, 2, 64, dtype=torch.bfloat16, device="cuda")
    lens = torch.tensor([40, 40], dtype=torch.int32, device="cuda")
    bad = table.clone()
    bad[0, 1] = cache.n_pages
    for t, n in ((bad, lens), (table, torch.tensor([table.shape[1] * 16 + 1, 40], dtype=torch.int32, device="cuda")),
                 (table, torch.tensor([-1, 40], dtype=torch.int32, device="cuda"))):
        ops.kv_attention(cache, q, starts, t, n, out, max_new=1)
        with pytest.raises(dcl.DcleapError, match="outside the paged cache"):
            ops.synchronise()
        o, _, A, _ = _reference(q[1:].float().cpu().numpy().astype(np.float64), values["k"][1], values["v"][1], 1,
                                False, 64 ** -0.5)
        assert (np.abs(out[1:].float().cpu().numpy() - o) <= (2.0 ** -8 + 2.0 ** -12) * A).all()  # the other is right


def test_pages_past_four_gigabytes(ops):
    heads, hd, page_len, pages = 32, 128, 256, 4400
    cache = dcl.KvCache.empty(pages, page_len, heads, hd)
    rng = np.random.default_rng(8)
    n = 300
    table = np.array([[4399, 4200]], np.int32)
    a = [torch.from_numpy(rng.normal(0, 1, (n, heads, hd))).to(torch.bfloat16).cuda() for _ in range(2)]
    slots = torch.from_numpy((table[0][np.arange(n) // page_len] * page_len + np.arange(n) % page_len).astype(np.int32))
    ops.kv_write(cache, a[0], a[1], slots.cuda())
    back = [torch.empty_like(x) for x in a]
    ops.kv_read(cache, slots.cuda(), *back)
    q = torch.from_numpy(rng.normal(0, 1, (1, heads, hd))).to(torch.bfloat16).cuda()
    out = torch.zeros_like(q)
    ops.kv_attention(cache, q, torch.tensor([0, 1], dtype=torch.int32, device="cuda"), torch.from_numpy(table).cuda(),
                     torch.tensor([n], dtype=torch.int32, device="cuda"), out, max_new=1)
    ops.synchronise()
    k, v = (x.float().cpu().numpy().astype(np.float64) for x in back)
    o, _, A, _ = _reference(q.float().cpu().numpy().astype(np.float64), k, v, 1, False, hd ** -0.5)
    assert (np.abs(out.float().cpu().numpy() - o) <= (2.0 ** -8 + 2.0 ** -12) * A).all()


def test_on_a_stream_of_its_own():
    """Work goes to the stream the context was made with."""
    s = torch.cuda.Stream()
    with dcl.Context(None, 1, 1, stream=s.cuda_stream) as ctx, torch.cuda.stream(s):
        _check(ctx, np.random.default_rng(9), [100], [2], 4, 2, 64, 16, True)
