"""The paged key / value cache against the CPU oracle: what dcl_kv_write stores (codes and exponents
exactly those of the oracle's E4M3 quantiser), what dcl_kv_read returns (exactly what is
stored), and what neither touches."""
import numpy as np
import pytest
import torch

import paper_2607_20467_gb300 as dcl
import synthetic as syn
from oracle import fp8

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def ops():
    import __graft_entry__
    __graft_entry__.build()
    ctx = dcl.Context(None, 1, 1)
    yield ctx
    ctx.close()


def _values(rng, n, heads, hd):
    """Vectors of unlike sizes, some with channels far above the rest, zeros among them."""
    a = rng.normal(0, 1, (n, heads, hd)) * np.exp2(rng.integers(-12, 13, (n, heads, 1)))
    a *= np.where(rng.random((1, heads, hd)) < 0.05, 30.0, 1.0)
    a[rng.random((n, heads)) < 0.1] = 0.0
    return syn.round_bf16(a.astype(np.float32))


def _bf16(a):
    return torch.from_numpy(np.ascontiguousarray(a, np.float32)).to(torch.bfloat16).cuda()


def _oracle(a):
    """Codes and exponents of [n][heads][hd], the exponent at least DCL_KV_EXP_MIN."""
    flat = a.reshape(-1, a.shape[-1]).astype(np.float64)
    e = np.where(np.abs(flat).max(1) > 0, np.maximum(fp8.row_exponents(flat), dcl.DCL_KV_EXP_MIN), 0)
    codes = fp8.e4m3_encode(fp8.e4m3_round(flat * np.exp2(-e.astype(np.float64))[:, None]))
    # (the oracle's encode keeps the sign of a value; a rounded-away negative is -0)
    return codes.reshape(a.shape), e.reshape(a.shape[:-1])


def _filled(cache, byte=0x5A):
    for t in (cache.k, cache.v, cache.k_exp, cache.v_exp):
        if t is not None:
            t.view(torch.uint8).fill_(byte)


def _at(t, slots, page_len):
    """Rows [n][heads][...] of a pool tensor at the slots."""
    s = torch.from_numpy(slots.astype(np.int64)).cuda()
    return t[s // page_len, :, s % page_len].cpu()


@pytest.mark.parametrize("hd", [64, 128])
@pytest.mark.parametrize("page_len,heads,n", [(16, 1, 1), (16, 4, 33), (32, 5, 100), (64, 32, 257), (256, 3, 700)])
def test_write_matches_the_oracles_codes(ops, hd, page_len, heads, n):
    rng = np.random.default_rng(n * hd)
    pages = n // page_len + 2
    slots = rng.permutation(pages * page_len)[:n].astype(np.int32)
    slots[rng.random(n) < 0.1] = -1
    k, v = _values(rng, n, heads, hd), _values(rng, n, heads, hd)
    cache = dcl.KvCache.empty(pages, page_len, heads, hd)
    _filled(cache)
    # k and v as column blocks of wider rows
    wide = torch.zeros(n, (2 + 2 * heads) * hd, dtype=torch.bfloat16, device="cuda")
    wide[:, 2 * hd:(2 + heads) * hd] = _bf16(k).flatten(1)
    wide[:, (2 + heads) * hd:] = _bf16(v).flatten(1)
    ops.kv_write(cache, wide[:, 2 * hd:(2 + heads) * hd].unflatten(1, (heads, hd)),
                 wide[:, (2 + heads) * hd:].unflatten(1, (heads, hd)), torch.from_numpy(slots).cuda())
    ops.synchronise()
    live = slots >= 0
    for a, codes, exps in ((k, cache.k, cache.k_exp), (v, cache.v, cache.v_exp)):
        want, e = _oracle(a[live])
        got = _at(codes, slots[live], page_len).numpy()
        assert (got == want).all()
        assert (_at(exps, slots[live], page_len).numpy() == e).all()
        # every other slot is as it was
        rest = torch.ones(pages * page_len, dtype=torch.bool)
        rest[torch.from_numpy(slots[live].astype(np.int64))] = False
        assert (codes.transpose(1, 2).reshape(pages * page_len, -1).cpu()[rest] == 0x5A).all()
        assert (exps.transpose(1, 2).reshape(pages * page_len, -1).cpu()[rest] == 0x5A).all()


def test_write_corner_values(ops):
    """The largest bf16 value, subnormals, exponents at the floor, ties, signed zeros, NaN and
    infinities (stored as NaN, and left out of the exponent)."""
    hd = 64
    bits = np.zeros((8, hd), np.uint16)
    bits[0, :] = 0x7F7F  # the largest bf16
    bits[1, :4] = [0x0001, 0x8001, 0x007F, 0x0080]  # subnormals
    bits[2, :3] = [0x1F80, 0x9F80, 0x1F00]  # 2^-64 and 2^-65: below 448 * 2^KV_EXP_MIN
    bits[3, :] = (np.arange(hd) + 0x3F80).astype(np.uint16)  # 1 .. 1.49, every bf16 step: all ties
    bits[4, :2] = [0x8000, 0x0000]
    bits[5, :3] = [0x7FC0, 0x3F80, 0xBF80]  # NaN, 1, -1
    bits[6, :3] = [0x7F80, 0xFF80, 0x4000]  # infinities, 2
    bits[7, :2] = [0x43E0, 0x43E1]  # 448 and the next value: e = 1
    x = torch.from_numpy(bits.view(np.int16)).cuda().view(torch.bfloat16).view(8, 1, hd)
    cache = dcl.KvCache.empty(1, 16, 1, hd)
    slots = torch.arange(8, dtype=torch.int32, device="cuda")
    ops.kv_write(cache, x, x, slots)
    ops.synchronise()
    got, e = cache.k[0, 0, :8].cpu().numpy(), cache.k_exp[0, 0, :8].cpu().numpy()
    assert (got == cache.v[0, 0, :8].cpu().numpy()).all() and (e == cache.v_exp[0, 0, :8].cpu().numpy()).all()
    f = syn.bf16_to_f32(bits).astype(np.float64)
    nan = ~np.isfinite(f)
    want, we = _oracle(np.where(nan, 0.0, f))
    assert (e == we).all()
    assert ((got & 0x7F)[nan] == 0x7F).all()
    assert (got[~nan] == want[~nan]).all()
    assert e[2] == dcl.DCL_KV_EXP_MIN and e[7] == 1
    back = torch.empty(8, 1, hd, dtype=torch.bfloat16, device="cuda")
    ops.kv_read(cache, slots, back, torch.empty_like(back))
    ops.synchronise()
    vals = np.where(nan, np.nan, fp8.e4m3_decode(got) * np.exp2(e.astype(np.float64))[:, None])
    assert (vals[0] == 2.0 ** 128).all()  # the code nearest to the largest bf16: bf16 holds it as infinity
    vals[0] = np.inf
    assert np.array_equal(back.view(8, hd).float().cpu().numpy().astype(np.float64), vals, equal_nan=True)


@pytest.mark.parametrize("fp8_format", [True, False])
@pytest.mark.parametrize("hd,heads,n", [(64, 3, 1), (128, 4, 50), (128, 32, 300)])
def test_read_returns_what_is_stored(ops, fp8_format, hd, heads, n):
    rng = np.random.default_rng(n)
    page_len, pages = 32, n // 32 + 3
    cache = dcl.KvCache.empty(pages, page_len, heads, hd, fp8=fp8_format)
    _filled(cache)
    slots = rng.permutation(pages * page_len)[:n].astype(np.int32)
    k, v = _values(rng, n, heads, hd), _values(rng, n, heads, hd)
    ops.kv_write(cache, _bf16(k), _bf16(v), torch.from_numpy(slots).cuda())
    # read in another order, with padding, into the column blocks of wider rows
    order = rng.permutation(n)
    ask = slots[order].copy()
    ask[::7] = -1
    out = torch.full((n, 2, heads, hd), 9.0, dtype=torch.bfloat16, device="cuda")
    ops.kv_read(cache, torch.from_numpy(ask).cuda(), out[:, 0], out[:, 1])
    ops.synchronise()
    for i, a in enumerate((k, v)):
        want = a[order].astype(np.float64)
        if fp8_format:
            codes, e = _oracle(want)
            want = fp8.e4m3_decode(codes) * np.exp2(e.astype(np.float64))[..., None]
        want[::7] = 0.0
        assert (out[:, i].float().cpu().numpy().astype(np.float64) == want).all()


def test_rows_of_none_are_a_no_op(ops):
    cache = dcl.KvCache.empty(1, 16, 2, 64)
    none = torch.empty(0, 2, 64, dtype=torch.bfloat16, device="cuda")
    slots = torch.empty(0, dtype=torch.int32, device="cuda")
    ops.kv_write(cache, none, none, slots)
    ops.kv_read(cache, slots, none, none)
    ops.synchronise()


def test_a_slot_outside_the_cache_is_reported_and_not_followed(ops):
    whole = torch.full((3, 2, 16, 64), 7, dtype=torch.uint8, device="cuda")
    other = torch.full((3, 2, 16, 64), 7, dtype=torch.uint8, device="cuda")
    exps = torch.full((2, 3, 2, 16), 7, dtype=torch.int8, device="cuda")
    cache = dcl.KvCache(whole[:2], other[:2], exps[0, :2], exps[1, :2])  # the third page is not the cache's
    x = torch.ones(2, 2, 64, dtype=torch.bfloat16, device="cuda")
    slots = torch.tensor([3, 32], dtype=torch.int32, device="cuda")
    ops.kv_write(cache, x, x, slots)
    with pytest.raises(dcl.DcleapError, match="outside the paged cache") as e:
        ops.synchronise()
    assert e.value.status == dcl.DCL_ERR_INVALID_ARG
    assert (whole[2] == 7).all() and (other[2] == 7).all() and (exps[:, 2] == 7).all()
    out = torch.full((2, 2, 64), 5.0, dtype=torch.bfloat16, device="cuda")
    out2 = out.clone()
    ops.kv_read(cache, slots, out, out2)
    with pytest.raises(dcl.DcleapError, match="outside the paged cache"):
        ops.synchronise()
    assert (out[0] == 1).all() and (out[1] == 0).all()  # the other row is served, this one reads as zeros
    ops.synchronise()  # reported once


def test_pages_past_four_gigabytes(ops):
    """Codes at byte offsets above 2^32 (and vectors whose element index passes 2^31)."""
    heads, hd, page_len, pages = 32, 128, 256, 4400  # 4.6 GB of codes each
    cache = dcl.KvCache.empty(pages, page_len, heads, hd)
    n = 5
    rng = np.random.default_rng(3)
    slots = np.array([pages * page_len - 1, 0, 4200 * page_len + 17, 2048 * page_len, 4399 * page_len], np.int32)
    k, v = _values(rng, n, heads, hd), _values(rng, n, heads, hd)
    d = torch.from_numpy(slots).cuda()
    ops.kv_write(cache, _bf16(k), _bf16(v), d)
    outs = [torch.empty(n, heads, hd, dtype=torch.bfloat16, device="cuda") for _ in range(2)]
    ops.kv_read(cache, d, *outs)
    ops.synchronise()
    for a, codes, exps, out in ((k, cache.k, cache.k_exp, outs[0]), (v, cache.v, cache.v_exp, outs[1])):
        want, e = _oracle(a)
        assert (_at(codes, slots, page_len).numpy() == want).all()
        assert (_at(exps, slots, page_len).numpy() == e).all()
        assert (out.float().cpu().numpy() == fp8.e4m3_decode(want) * np.exp2(e.astype(np.float64))[..., None]).all()
