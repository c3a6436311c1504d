"""Refusals of the 4-bit cache, the plan and the norm and rotation of queries and keys: what the binding
refuses before a call (CPU only), and what the C ABI refuses before it touches a device."""
import ctypes

import pytest
import torch

import paper_2607_20467_gb300 as dcl
from test_serving_args import FakeCuda, _context


def _q4(pages=4, heads=2, page_len=16, hd=64):
    t = lambda d: FakeCuda((pages, heads, page_len, hd // d), 1)
    return dcl.KvCache(t(2), t(2), t(32), t(32))


def test_a_4_bit_cache_takes_only_matching_tensors():
    c = _q4()
    assert (c.format, c.head_dim, c.row) == (dcl.DCL_KV_Q4, 64, 128)
    codes, scales = FakeCuda((4, 2, 16, 32), 1), FakeCuda((4, 2, 16, 2), 1)
    for bad in (FakeCuda((4, 2, 16, 1), 1), FakeCuda((3, 2, 16, 2), 1), FakeCuda((4, 2, 16), 1)):
        with pytest.raises(ValueError):
            dcl.KvCache(codes, codes, scales, bad)
    with pytest.raises(ValueError, match="differ"):
        dcl.KvCache(codes, FakeCuda((4, 2, 16, 64), 1), scales, scales)
    with pytest.raises(ValueError, match="contiguous"):
        dcl.KvCache(codes, codes, scales, FakeCuda((4, 2, 16, 2), 1, (64, 32, 4, 1)))
    with pytest.raises(ValueError, match="scales"):
        dcl.KvCache(codes, codes)
    with pytest.raises(TypeError):  # E4M3 codes are no 4-bit codes
        t = torch.zeros(4, 2, 16, 32).to(torch.float8_e4m3fn)
        fake = FakeCuda((4, 2, 16, 32), 1)
        fake.dtype = t.dtype
        dcl.KvCache(fake, fake, scales, scales)


def _pages(batch=3, width=5, pages=20):
    i = lambda *s: FakeCuda(s, 4)
    return dcl.KvPages(i(batch, width), i(batch), i(pages), i(1), 16)


def test_the_plan_takes_only_matching_tensors():
    i = lambda *s: FakeCuda(s, 4)
    for bad in ((i(15), i(3), i(20), i(1)), (i(3, 5), i(2), i(20), i(1)), (i(3, 5), i(3), i(4, 5), i(1)), (i(3, 5), i(3), i(20), i(0)),
                (FakeCuda((3, 5), 4, (8, 1)), i(3), i(20), i(1)), (torch.zeros(3, 5, dtype=torch.int32), i(3), i(20), i(1))):
        with pytest.raises(ValueError):
            dcl.KvPages(*bad, 16)
    with pytest.raises(TypeError):
        dcl.KvPages(FakeCuda((3, 5), 8), i(3), i(20), i(1), 16)
    ctx, pages = _context(), _pages()
    good = dict(start=i(3), new=i(3), q_start=i(4), seq_len=i(3), slots=i(10), pos=i(10))
    for name, bad in (("start", i(2)), ("new", i(2)), ("q_start", i(3)), ("seq_len", i(2)), ("pos", i(9)), ("slots", FakeCuda((10,), 4, (2,)))):
        with pytest.raises(ValueError):
            ctx.kv_plan(pages, **{**good, name: bad})
    with pytest.raises(TypeError):
        ctx.kv_plan(pages, **{**good, "start": FakeCuda((3,), 8)})
    assert ctx._L.calls == []
    ctx.kv_plan(pages, **good)
    (name, args), = ctx._L.calls
    assert name == "dcl_kv_plan" and args[1] == pages.ptr and args[-1] == 10


def test_the_rotation_refuses_what_a_kernel_would_read_past():
    ctx = _context()
    b = lambda *s, **k: FakeCuda(s, 2, **k)
    good = dict(q=b(5, 4, 64), k=b(5, 2, 64), pos=FakeCuda((5,), 4), q_out=b(5, 4, 64), k_out=b(5, 2, 64), theta=1e4, q_gain=b(64))
    for name, bad in (("k", b(4, 2, 64)), ("k", b(5, 2, 128)), ("q_out", b(5, 3, 64)), ("k_out", b(4, 2, 64)), ("pos", FakeCuda((4,), 4)),
                      ("q_gain", b(63)), ("q", b(5, 4, 64, stride=(256, 1, 4))), ("q", torch.zeros(5, 4, 64, dtype=torch.bfloat16))):
        with pytest.raises(ValueError):
            ctx.qk_norm_rope(**{**good, name: bad})
    for name in ("q", "k", "q_out", "k_out"):
        with pytest.raises(TypeError):
            ctx.qk_norm_rope(**{**good, name: FakeCuda(good[name].shape, 4)})
    assert ctx._L.calls == []
    ctx.qk_norm_rope(**{**good, "k": b(5, 2, 64, stride=(512, 64, 1))})
    (name, args), = ctx._L.calls
    assert name == "dcl_qk_norm_rope" and args[2] == 256 and args[4] == 512 and args[6:11] == (5, 4, 2, 64, 64)


@pytest.fixture(scope="module")
def built():
    import __graft_entry__
    __graft_entry__.build()
    return dcl.lib()


def test_null_context_is_rejected(built):
    n = dcl.DCL_ERR_INVALID_ARG
    assert built.dcl_kv_plan(None, None, None, None, None, None, None, None, 0) == n
    assert built.dcl_qk_norm_rope(None, None, 0, None, 0, None, 0, 0, 0, 0, 0, 0.0, None, None, 0.0, None, 0, None, 0) == n


@pytest.mark.gpu
def test_the_abi_refuses_bad_arguments(built):
    """Every refusal is a status with a message, decided on the host (no pointer is followed)."""
    with dcl.Context(None, 1, 1) as ctx:
        P = 0x7000_0000  # never dereferenced: each call is refused

        def refused(st, words):
            assert st == dcl.DCL_ERR_INVALID_ARG
            assert words in built.dcl_last_error(ctx.ptr).decode()

        def plan(start=P, new=P, q_start=P, seq=P, slot=P, pos=P, rows=4, **kw):
            d = dict(n_pages=8, page_len=16, batch=2, max_pages=3, table_dev=P, held_dev=P, free_dev=P, n_free_dev=P)
            d.update(kw)
            return built.dcl_kv_plan(ctx.ptr, ctypes.byref(dcl.KvPagesDesc(**d)), start, new, q_start, seq, slot, pos, rows)

        refused(built.dcl_kv_plan(ctx.ptr, None, P, P, P, P, P, P, 1), "NULL")
        for kw, words in ((dict(page_len=8), "page_len"), (dict(page_len=48), "page_len"), (dict(page_len=512), "page_len"),
                          (dict(n_pages=0), "n_pages"), (dict(n_pages=1 << 27), "2^31"), (dict(batch=-1), "batch"),
                          (dict(rows=-1), "n_rows"), (dict(max_pages=0), "max_pages"), (dict(max_pages=1 << 27), "max_pages"),
                          (dict(batch=1 << 20, max_pages=1 << 11), "batch"), (dict(table_dev=None), "NULL"), (dict(held_dev=None), "NULL"),
                          (dict(free_dev=None), "NULL"), (dict(n_free_dev=None), "NULL"), (dict(start=None), "NULL"),
                          (dict(new=None), "NULL"), (dict(q_start=None), "NULL"), (dict(seq=None), "NULL"), (dict(slot=None), "NULL"),
                          (dict(pos=None), "NULL")):
            refused(plan(**kw), words)

        def rope(q=P, qs=256, k=P, ks=128, pos=P, n=1, H=4, G=2, hd=64, rot=64, theta=1e4, qg=P, kg=P, eps=1e-6, qo=P + 4096, qos=256,
                 ko=P + 8192, kos=128):
            return built.dcl_qk_norm_rope(ctx.ptr, q, qs, k, ks, pos, n, H, G, hd, rot, theta, qg, kg, eps, qo, qos, ko, kos)

        for kw, words in ((dict(hd=96), "head_dim"), (dict(rot=24), "rot_dim"), (dict(rot=80), "rot_dim"), (dict(rot=-16), "rot_dim"),
                          (dict(n=-1), "n must"), (dict(H=0), "n_heads"), (dict(G=0), "n_kv_heads"), (dict(theta=0.5), "theta"),
                          (dict(theta=float("nan")), "theta"), (dict(theta=float("inf")), "theta"), (dict(eps=0.0), "eps"),
                          (dict(eps=-1.0), "eps"), (dict(eps=float("nan")), "eps"), (dict(eps=3e38), "eps"), (dict(eps=1e-44), "eps"),
                          (dict(eps=3e38, qg=None), "eps"), (dict(q=None), "NULL"), (dict(k=None), "NULL"),
                          (dict(pos=None), "NULL"), (dict(qo=None), "NULL"), (dict(ko=None), "NULL"), (dict(qs=255), "strides"),
                          (dict(ks=132), "strides"), (dict(qos=128), "strides"), (dict(kos=129), "strides"), (dict(q=P + 8), "aligned"),
                          (dict(kg=P + 2), "aligned"), (dict(ko=P + 4), "aligned"), (dict(qo=P, qos=512), "in place")):
            refused(rope(**kw), words)
        assert rope(n=0) == dcl.DCL_OK and rope(n=0, eps=0.0, qg=None, kg=None) == dcl.DCL_OK

        def write(**kw):
            d = dict(n_pages=4, page_len=16, n_kv_heads=2, head_dim=64, format=dcl.DCL_KV_Q4, k_dev=P, v_dev=P, k_exp_dev=P, v_exp_dev=P)
            d.update(kw)
            return built.dcl_kv_write(ctx.ptr, ctypes.byref(dcl.KvCacheDesc(**d)), P, P, 128, P, 1)

        for kw, words in ((dict(format=3), "format"), (dict(format=5), "format"), (dict(k_exp_dev=None), "scales"), (dict(v_exp_dev=None), "scales"),
                          (dict(v_exp_dev=P + 4), "aligned"), (dict(head_dim=32), "head_dim")):
            refused(write(**kw), words)
