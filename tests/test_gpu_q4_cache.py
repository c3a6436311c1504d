"""The paged cache in 4 bits against the format's oracle: what dcl_kv_write stores (codes and scale bytes
exactly the oracle's), what dcl_kv_read returns (exactly what is stored), and what neither touches."""
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


def _values(rng, n, heads, hd):
    """Vectors of unlike sizes, some with channels far above the rest, whole vectors and groups of zeros among them."""
    a = rng.normal(0, 1, (n, heads, hd)) * np.exp2(rng.integers(-12, 13, (n, heads, 1)))
    a *= np.where(rng.random((1, heads, hd)) < 0.05, 30.0, 1.0)
    a[rng.random((n, heads)) < 0.1] = 0.0
    a[rng.random((n, heads)) < 0.1, :32] = 0.0
    return syn.round_bf16(a.astype(np.float32))


def _bf16(a):
    return torch.from_numpy(np.ascontiguousarray(a, np.float32)).to(torch.bfloat16).cuda()


def _filled(cache, byte=0x5A):
    for t in (cache.k, cache.v, cache.k_exp, cache.v_exp):
        t.fill_(byte)


def _at(t, slots, page_len):
    s = torch.from_numpy(slots.astype(np.int64)).cuda()
    return t[s // page_len, :, s % page_len].cpu().numpy()


@pytest.mark.parametrize("hd", [64, 128])
@pytest.mark.parametrize("page_len,heads,n", [(16, 1, 1), (16, 4, 33), (32, 5, 100), (64, 32, 257), (256, 3, 700)])
def test_write_and_read_match_the_oracle(ops, hd, page_len, heads, n):
    rng = np.random.default_rng(n * hd)
    pages = n // page_len + 2
    slots = rng.permutation(pages * page_len)[:n].astype(np.int32)
    slots[rng.random(n) < 0.1] = -1
    k, v = _values(rng, n, heads, hd), _values(rng, n, heads, hd)
    cache = dcl.KvCache.empty(pages, page_len, heads, hd, q4=True)
    assert cache.format == dcl.DCL_KV_Q4 and cache.head_dim == hd
    _filled(cache)
    wide = torch.zeros(n, (2 + 2 * heads) * hd, dtype=torch.bfloat16, device="cuda")  # k and v in wider rows
    wide[:, 2 * hd:(2 + heads) * hd] = _bf16(k).flatten(1)
    wide[:, (2 + heads) * hd:] = _bf16(v).flatten(1)
    d = torch.from_numpy(slots).cuda()
    ops.kv_write(cache, wide[:, 2 * hd:(2 + heads) * hd].unflatten(1, (heads, hd)),
                 wide[:, (2 + heads) * hd:].unflatten(1, (heads, hd)), d)
    out = torch.full((n, 2, heads, hd), 9.0, dtype=torch.bfloat16, device="cuda")
    ops.kv_read(cache, d, out[:, 0], out[:, 1])
    ops.synchronise()
    live = slots >= 0
    rest = np.ones(pages * page_len, bool)
    rest[slots[live]] = False
    for i, (a, codes, scales) in enumerate(((k, cache.k, cache.k_exp), (v, cache.v, cache.v_exp))):
        want, b = q4.encode(a[live])
        assert (_at(scales, slots[live], page_len) == b).all()
        assert (_at(codes, slots[live], page_len) == q4.pack(want)).all()
        for t in (codes, scales):  # every other slot is as it was
            assert (t.transpose(1, 2).reshape(pages * page_len, -1).cpu().numpy()[rest] == 0x5A).all()
        got = out[:, i].float().cpu().numpy().astype(np.float64)
        assert (got[live] == q4.decode(want, b)).all() and (got[~live] == 0).all()


def test_every_step_of_a_binade_and_every_tie(ops):
    """All 128 bf16 values of a binade as a group's largest, with halves, quarters, eighths and every multiple of
    a 14th of it below: the borders between scales and the ties between codes."""
    hd = 64
    top = (np.arange(128) + 0x4000).astype(np.uint16)
    f = syn.bf16_to_f32(top).astype(np.float64)
    a = np.zeros((128, 1, hd))
    a[:, 0, 0] = f
    for i in range(1, 32):
        a[:, 0, i] = f * (i - 16) / 16
        a[:, 0, 32 + i] = f * (i - 16) / 14
    a[:, 0, 32] = -f
    a = syn.round_bf16(a.astype(np.float32)).astype(np.float64)
    s = q4.scale_value(q4.encode(a)[1])  # (and exact ties: odd halves of the scale)
    a[:, 0, 1:8] = s[:, 0, :1] * (np.arange(7) - 3.5)
    assert (syn.round_bf16(a.astype(np.float32)) == a).all()
    cache = dcl.KvCache.empty(8, 16, 1, hd, q4=True)
    slots = torch.arange(128, dtype=torch.int32, device="cuda")
    ops.kv_write(cache, _bf16(a), _bf16(-a), slots)
    ops.synchronise()
    n = np.arange(128)
    for x, codes, scales in ((a, cache.k, cache.k_exp), (-a, cache.v, cache.v_exp)):
        want, b = q4.encode(x)
        assert (_at(scales, n, 16) == b).all() and (_at(codes, n, 16) == q4.pack(want)).all()


def test_corner_values(ops):
    """The largest bf16 value (cut off), subnormals, below the least scale, signed zeros, NaN and infinities."""
    hd = 64
    bits = np.zeros((7, hd), np.uint16)
    bits[0, :3] = [0x7F7F, 0xFF7F, 0x4D00]  # the largest; 1.34e8 beside it
    bits[1, :4] = [0x0001, 0x8001, 0x007F, 0x0080]  # subnormals
    bits[2, :4] = [0x2C80, 0x2C7F, 0x2C00, 0xAC81]  # about half the least scale
    bits[3, :2] = [0x8000, 0x0000]
    bits[4, :3] = [0x7FC0, 0x3F80, 0xBF80]  # NaN beside numbers
    bits[5, 40:43] = [0x7F80, 0xFF80, 0x4000]  # infinities in the second group
    bits[6, :2] = [0x4D43, 0x4D44]  # around the largest that a scale reaches
    x = torch.from_numpy(bits.view(np.int16)).cuda().view(torch.bfloat16).view(7, 1, hd)
    cache = dcl.KvCache.empty(1, 16, 1, hd, q4=True)
    slots = torch.arange(7, dtype=torch.int32, device="cuda")
    back = torch.empty(7, 1, hd, dtype=torch.bfloat16, device="cuda")
    ops.kv_write(cache, x, x, slots)
    ops.kv_read(cache, slots, back, torch.empty_like(back))
    ops.synchronise()
    want, b = q4.encode(syn.bf16_to_f32(bits).astype(np.float64))
    for codes, scales in ((cache.k, cache.k_exp), (cache.v, cache.v_exp)):
        got, gb = codes[0, 0, :7].cpu().numpy(), scales[0, 0, :7].cpu().numpy()
        assert (gb == b).all()
        assert (q4.unpack(got).reshape(7, 2, 32)[b < 252] == want.reshape(7, 2, 32)[b < 252]).all()
    vals = q4.decode(want, b)
    assert np.isnan(vals[4, :32]).all() and np.isnan(vals[5, 32:]).all() and (vals[5, :32] == 0).all()
    assert vals[0, 0] == 49.0 * 2.0 ** 22
    assert np.array_equal(back.view(7, hd).float().cpu().numpy().astype(np.float64), vals, equal_nan=True)


def test_every_scale_byte_and_code_reads_as_the_oracles_value(ops):
    hd, n = 128, 256
    cache = dcl.KvCache.empty(16, 16, 1, hd, q4=True)
    b = np.arange(n)[:, None] + np.array([0, 64, 128, 192])
    codes = (np.arange(hd) + np.arange(n)[:, None]) % 16
    cache.k.copy_(torch.from_numpy(q4.pack(codes.astype(np.uint8))).view(16, 1, 16, hd // 2))
    cache.v.copy_(cache.k.flip(0))
    cache.k_exp.copy_(torch.from_numpy((b % 256).astype(np.uint8)).view(16, 1, 16, hd // 32))
    cache.v_exp.copy_(cache.k_exp)
    k, v = (torch.empty(n, 1, hd, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    ops.kv_read(cache, torch.arange(n, dtype=torch.int32, device="cuda"), k, v)
    ops.synchronise()
    want = q4.decode(codes.astype(np.uint8), b % 256)
    assert np.array_equal(k.view(n, hd).float().cpu().numpy().astype(np.float64), want, equal_nan=True)


def test_slots_outside_the_cache_are_reported_and_not_followed(ops):
    codes = torch.full((2, 3, 2, 16, 32), 7, dtype=torch.uint8, device="cuda")
    scales = torch.full((2, 3, 2, 16, 2), 7, dtype=torch.uint8, device="cuda")
    cache = dcl.KvCache(codes[0, :2], codes[1, :2], scales[0, :2], scales[1, :2])  # the third page is not the cache's
    x = torch.ones(2, 2, 64, dtype=torch.bfloat16, device="cuda")
    slots = torch.tensor([3, 32], dtype=torch.int32, device="cuda")
    ops.kv_write(cache, x, x, slots)
    with pytest.raises(dcl.DcleapError, match="outside the paged cache"):
        ops.synchronise()
    assert (codes[:, 2] == 7).all() and (scales[:, 2] == 7).all()
    out = torch.full((2, 2, 2, 64), 5.0, dtype=torch.bfloat16, device="cuda")
    ops.kv_read(cache, slots, out[0], out[1])
    with pytest.raises(dcl.DcleapError, match="outside the paged cache"):
        ops.synchronise()
    want = float(q4.decode(*q4.encode(np.ones((1, 64))))[0, 0])
    assert (out[:, 0] == want).all() and (out[:, 1] == 0).all()
    none = torch.empty(0, 2, 64, dtype=torch.bfloat16, device="cuda")
    ops.kv_write(cache, none, none, slots[:0])
    ops.kv_read(cache, slots[:0], none, none)
    ops.synchronise()


def test_pages_past_four_gigabytes(ops):
    heads, hd, page_len, pages = 32, 128, 256, 8500  # 4.5 GB of codes each
    cache = dcl.KvCache.empty(pages, page_len, heads, hd, q4=True)
    rng = np.random.default_rng(3)
    slots = np.array([pages * page_len - 1, 0, 8300 * page_len + 17, 4096 * page_len, 8499 * page_len], np.int32)
    k, v = _values(rng, 5, heads, hd), _values(rng, 5, heads, hd)
    d = torch.from_numpy(slots).cuda()
    outs = [torch.empty(5, heads, hd, dtype=torch.bfloat16, device="cuda") for _ in range(2)]
    ops.kv_write(cache, _bf16(k), _bf16(v), d)
    ops.kv_read(cache, d, *outs)
    ops.synchronise()
    for a, codes, out in ((k, cache.k, outs[0]), (v, cache.v, outs[1])):
        want, b = q4.encode(a)
        assert (_at(codes, slots, page_len) == q4.pack(want)).all()
        assert (out.float().cpu().numpy() == q4.decode(want, b)).all()
