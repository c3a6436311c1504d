"""Refusals of the serving calls (CPU only): what the binding refuses before a call, and what the C
ABI refuses before it touches a device."""
import ctypes

import numpy as np
import pytest
import torch

import paper_2607_20467_gb300 as dcl


class FakeCuda:
    """A CUDA tensor's shape, strides and element size."""

    is_cuda = True

    def __init__(self, shape, itemsize, stride=None, ptr=0x7000_0000):
        self.shape, self.itemsize, self.dtype, self.ptr = tuple(shape), itemsize, f"{itemsize}-byte", ptr
        dense = [1]
        for s in reversed(self.shape[1:]):
            dense.insert(0, dense[0] * s)
        self.dense = tuple(dense) if self.shape else ()
        self.strides = tuple(stride) if stride else self.dense

    def element_size(self):
        return self.itemsize

    def numel(self):
        return int(np.prod(self.shape))

    def stride(self):
        return self.strides

    def is_contiguous(self):
        return self.strides == self.dense

    def data_ptr(self):
        return self.ptr


class Recorder:
    def __init__(self):
        self.calls = []

    def __getattr__(self, name):
        def fn(*args):
            self.calls.append((name, args))
            return 0
        return fn


def _context():
    ctx = object.__new__(dcl.Context)
    ctx._L, ctx.ptr, ctx.shape = Recorder(), None, None
    return ctx


def _cache(pages=4, heads=2, page_len=16, hd=64, fp8=True):
    size = 1 if fp8 else 2
    t = lambda: FakeCuda((pages, heads, page_len, hd), size)
    e = lambda: FakeCuda((pages, heads, page_len), 1) if fp8 else None
    return dcl.KvCache(t(), t(), e(), e())


def test_cache_takes_only_matching_tensors():
    k, e = FakeCuda((4, 2, 16, 64), 1), FakeCuda((4, 2, 16), 1)
    with pytest.raises(ValueError, match="k_exp"):
        dcl.KvCache(k, k)
    with pytest.raises(ValueError, match="no exponents"):
        dcl.KvCache(FakeCuda((4, 2, 16, 64), 2), FakeCuda((4, 2, 16, 64), 2), e, e)
    with pytest.raises(ValueError, match="differ"):
        dcl.KvCache(k, FakeCuda((4, 2, 32, 64), 1), e, e)
    with pytest.raises(ValueError, match="at least"):
        dcl.KvCache(k, k, FakeCuda((3, 2, 16), 1), e)
    with pytest.raises(TypeError):
        dcl.KvCache(k, k, FakeCuda((4, 2, 16), 4), e)
    with pytest.raises(ValueError, match="device buffer"):
        dcl.KvCache(torch.zeros(4, 2, 16, 64, dtype=torch.uint8), k, e, e)
    with pytest.raises(ValueError, match="expected"):
        dcl.KvCache(FakeCuda((4, 16, 64), 1), FakeCuda((4, 16, 64), 1), e, e)


def test_calls_refuse_what_a_kernel_would_read_past():
    ctx, cache = _context(), _cache()
    rows, slots = FakeCuda((5, 2, 64), 2), FakeCuda((5,), 4)
    for bad in (FakeCuda((5, 3, 64), 2), FakeCuda((5, 2, 32), 2), FakeCuda((5, 2, 64), 2, (128, 1, 2)),
                torch.zeros(5, 2, 64, dtype=torch.bfloat16), FakeCuda((5, 2, 64), 2, (64, 64, 1))):
        with pytest.raises(ValueError):
            ctx.kv_write(cache, bad, rows, slots)
        with pytest.raises(ValueError):
            ctx.kv_read(cache, slots, rows, bad)
    with pytest.raises(ValueError, match="at least 5"):
        ctx.kv_write(cache, rows, rows, FakeCuda((4,), 4))
    with pytest.raises(ValueError, match="row stride"):
        ctx.kv_write(cache, rows, FakeCuda((5, 2, 64), 2, (256, 64, 1)), slots)
    with pytest.raises(TypeError):
        ctx.kv_write(cache, rows, rows, FakeCuda((5,), 8))
    q, out = FakeCuda((3, 4, 64), 2), FakeCuda((3, 4, 64), 2)
    table, lens, starts = FakeCuda((2, 7), 4), FakeCuda((2,), 4), FakeCuda((3,), 4)
    with pytest.raises(ValueError, match="head_dim"):
        ctx.kv_attention(cache, FakeCuda((3, 4, 128), 2), starts, table, lens, out, max_new=1)
    with pytest.raises(ValueError, match="q_start"):
        ctx.kv_attention(cache, q, FakeCuda((2,), 4), table, lens, out, max_new=1)
    with pytest.raises(ValueError, match="seq_len"):
        ctx.kv_attention(cache, q, starts, table, FakeCuda((1,), 4), out, max_new=1)
    with pytest.raises(ValueError, match="contiguous"):
        ctx.kv_attention(cache, q, starts, FakeCuda((2, 7), 4, (14, 1)), lens, out, max_new=1)
    with pytest.raises(ValueError, match="lse"):
        ctx.kv_attention(cache, q, starts, table, lens, out, max_new=1, lse=FakeCuda((11,), 4))
    z, token = FakeCuda((3, 100), 2), FakeCuda((3,), 4)
    with pytest.raises(TypeError):
        ctx.sample(FakeCuda((3, 100), 4), token)
    with pytest.raises(ValueError):
        ctx.sample(z, FakeCuda((2,), 4))
    with pytest.raises(ValueError):
        ctx.sample(z, token, noise=FakeCuda((3, 99), 4))
    with pytest.raises(ValueError):
        ctx.sample(z, token, top_p=FakeCuda((2,), 4))
    with pytest.raises(ValueError):
        ctx.sample(FakeCuda((3, 100), 2, (100, 2)), token)
    assert ctx._L.calls == []


def test_calls_pass_strides_on():
    ctx, cache = _context(), _cache()
    rows = FakeCuda((5, 2, 64), 2, (512, 64, 1))
    ctx.kv_write(cache, rows, rows, FakeCuda((5,), 4))
    ctx.sample(FakeCuda((3, 100), 2, (107, 1)), FakeCuda((3,), 4), noise=FakeCuda((3, 100), 4, (200, 1)))
    (w, wa), (s, sa) = ctx._L.calls
    assert w == "dcl_kv_write" and wa[4] == 512 and wa[6] == 5
    assert s == "dcl_sample" and sa[2] == 107 and sa[4] == 200 and sa[5:7] == (3, 100)


@pytest.fixture(scope="module")
def built():
    import __graft_entry__
    __graft_entry__.build()
    return dcl.lib()


def test_null_context_is_rejected(built):
    n = dcl.DCL_ERR_INVALID_ARG
    assert built.dcl_kv_write(None, None, None, None, 0, None, 0) == n
    assert built.dcl_kv_read(None, None, None, 0, None, None, 0) == n
    assert built.dcl_kv_attention(None, None, None, 0, None, None, 0, None, 0, 0, 0, 0, 0, 0.0, None, None) == n
    assert built.dcl_sample(None, None, 0, None, 0, 0, 0, None, None, None, None, None, None, None) == n
    assert built.dcl_synchronise(None) == n


@pytest.mark.gpu
def test_the_abi_refuses_bad_arguments(built):
    """Every refusal is a status with a message, decided on the host (no pointer is followed)."""
    with dcl.Context(None, 1, 1) as ctx:
        P = 0x7000_0000  # never dereferenced: each call is refused

        def cache(**kw):
            d = dict(n_pages=4, page_len=16, n_kv_heads=2, head_dim=64, format=1, k_dev=P, v_dev=P, k_exp_dev=P,
                     v_exp_dev=P)
            d.update(kw)
            return ctypes.byref(dcl.KvCacheDesc(**d))

        def refused(st, words):
            assert st == dcl.DCL_ERR_INVALID_ARG
            assert words in built.dcl_last_error(ctx.ptr).decode()

        def write(c=None, k=P, v=P, stride=128, slots=P, n=1):
            return built.dcl_kv_write(ctx.ptr, c if c is not None else cache(), k, v, stride, slots, n)

        for kw, words in ((dict(format=2), "format"), (dict(page_len=24), "page_len"), (dict(page_len=8), "page_len"),
                          (dict(page_len=512), "page_len"), (dict(head_dim=96), "head_dim"),
                          (dict(n_kv_heads=0), "n_kv_heads"), (dict(n_pages=0), "n_pages"),
                          (dict(n_pages=1 << 27), "2^31"), (dict(k_exp_dev=None), "exponents"),
                          (dict(k_dev=None), "NULL"), (dict(v_dev=P + 8), "aligned")):
            refused(write(cache(**kw)), words)
        for kw, words in ((dict(k=None), "NULL"), (dict(slots=None), "NULL"), (dict(n=-1), "n must"),
                          (dict(stride=127), "row_stride"), (dict(stride=132), "row_stride"), (dict(v=P + 2), "aligned")):
            refused(write(**kw), words)

        def attention(c=None, q=P, qs=256, starts=P, table=P, pages=3, lens=P, batch=2, n_q=2, new=1, heads=4,
                      causal=0, scale=0.0, out=P):
            return built.dcl_kv_attention(ctx.ptr, c if c is not None else cache(), q, qs, starts, table, pages, lens,
                                          batch, n_q, new, heads, causal, scale, out, None)

        for kw, words in ((dict(heads=3), "n_heads"), (dict(batch=-1), "batch"), (dict(causal=2), "causal"),
                          (dict(q=None), "NULL"), (dict(out=None), "NULL"), (dict(pages=0), "max_pages"),
                          (dict(new=0), "max_new"), (dict(qs=255), "q_stride"), (dict(qs=260), "q_stride"),
                          (dict(q=P + 2), "aligned"), (dict(scale=-1.0), "scale"), (dict(scale=float("nan")), "scale")):
            refused(attention(**kw), words)
        assert attention(batch=0) == dcl.DCL_OK and attention(n_q=0) == dcl.DCL_OK

        def sample(z=P, zs=100, g=None, gs=0, rows=1, V=100, token=P):
            return built.dcl_sample(ctx.ptr, z, zs, g, gs, rows, V, None, None, None, None, token, None, None)

        for kw, words in ((dict(z=None), "NULL"), (dict(token=None), "NULL"), (dict(V=0), "V"), (dict(zs=99), "strides"),
                          (dict(g=P, gs=99), "strides"), (dict(rows=-1), "rows")):
            refused(sample(**kw), words)
        assert sample(rows=0) == dcl.DCL_OK
