"""The serving calls refuse tensors whose elements have the right size and another meaning (CPU only)."""
import pytest
import torch

import paper_2607_20467_gb300 as dcl


class OnDevice:
    """A CPU tensor that says it is a CUDA tensor (its data is never looked at)."""

    is_cuda = True

    def __init__(self, *shape, dtype):
        self.t = torch.empty(shape, dtype=dtype)

    def __getattr__(self, name):
        return getattr(self.t, name)


class Recorder:
    def __init__(self):
        self.calls = []

    def __getattr__(self, name):
        def fn(*args):
            self.calls.append(name)
            return 0
        return fn


BF, F16, F32, I32, U8, I8 = torch.bfloat16, torch.float16, torch.float32, torch.int32, torch.uint8, torch.int8


@pytest.fixture
def ctx():
    c = object.__new__(dcl.Context)
    c._L, c.ptr, c.shape = Recorder(), None, None
    return c


def _cache(k=U8, v=U8, ke=I8, ve=I8, fp8=True):
    e = lambda t: OnDevice(4, 2, 16, dtype=t) if fp8 else None
    return dcl.KvCache(OnDevice(4, 2, 16, 64, dtype=k), OnDevice(4, 2, 16, 64, dtype=v), e(ke), e(ve))


def test_caches():
    for t in (U8, I8, torch.float8_e4m3fn):
        _cache(t, t)
    _cache(BF, BF, fp8=False)
    _cache(torch.int16, torch.int16, fp8=False)  # (bit patterns)
    for kw in (dict(k=torch.float8_e5m2), dict(v=torch.float8_e5m2), dict(v=torch.bool), dict(ke=torch.bool),
               dict(ve=torch.float8_e4m3fn), dict(k=F16, v=F16, fp8=False), dict(k=BF, v=F16, fp8=False)):
        with pytest.raises(TypeError):
            _cache(**kw)


def test_rows_and_slots(ctx):
    cache = _cache()
    good, slots = OnDevice(5, 2, 64, dtype=BF), OnDevice(5, dtype=I32)
    for k, v, s in ((OnDevice(5, 2, 64, dtype=F16), good, slots), (good, OnDevice(5, 2, 64, dtype=F16), slots),
                    (good, good, OnDevice(5, dtype=F32))):
        with pytest.raises(TypeError):
            ctx.kv_write(cache, k, v, s)
        with pytest.raises(TypeError):
            ctx.kv_read(cache, s, k, v)
    assert ctx._L.calls == []
    ctx.kv_write(cache, good, good, slots)
    ctx.kv_read(cache, slots, good, good)
    assert ctx._L.calls == ["dcl_kv_write", "dcl_kv_read"]


def test_attention(ctx):
    cache = _cache()
    right = dict(q=BF, q_start=I32, page_table=I32, seq_len=I32, out=BF, lse=F32)
    shape = dict(q=(3, 4, 64), q_start=(3,), page_table=(2, 7), seq_len=(2,), out=(3, 4, 64), lse=(3, 4))
    wrong = dict(q=F16, q_start=F32, page_table=F32, seq_len=F32, out=F16, lse=I32)
    make = lambda types: {n: OnDevice(*shape[n], dtype=t) for n, t in types.items()}
    for name, t in wrong.items():
        with pytest.raises(TypeError, match=name):
            ctx.kv_attention(cache, max_new=1, **make({**right, name: t}))
    assert ctx._L.calls == []
    ctx.kv_attention(cache, max_new=1, **make(right))
    assert ctx._L.calls == ["dcl_kv_attention"]


def test_sampling(ctx):
    right = dict(logits=BF, token=I32, noise=F32, temperature=F32, top_k=I32, top_p=F32, min_p=F32, prob=F32, conf=F32)
    wrong = dict(logits=F16, token=F32, noise=I32, temperature=I32, top_k=F32, top_p=I32, min_p=I32, prob=I32, conf=I32)
    make = lambda types: {n: OnDevice(*((3, 100) if n in ("logits", "noise") else (3,)), dtype=t) for n, t in types.items()}
    for name, t in wrong.items():
        with pytest.raises(TypeError, match=name):
            ctx.sample(**make({**right, name: t}))
    assert ctx._L.calls == []
    ctx.sample(**make(right))
    assert ctx._L.calls == ["dcl_sample"]
