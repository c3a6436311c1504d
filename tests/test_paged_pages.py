"""The paged decoding example gives its pages back, also where it does not come to an end (CPU only)."""
import os
import sys

import numpy as np
import pytest

sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))
import paged_decode  # noqa: E402


def _model(n_pages):
    model = object.__new__(paged_decode.PagedModel)
    model.ctx, model.shape, model.page_len, model.free = None, None, 16, list(range(n_pages))
    return model


def test_too_few_pages_for_the_last_sequence():
    model = _model(5)
    with pytest.raises(MemoryError):
        paged_decode.generate(model, [np.zeros(20, np.int32)] * 3, 12)  # two pages each
    assert sorted(model.free) == list(range(5))


def test_a_step_that_fails(monkeypatch):
    model = _model(8)

    def fails(*args, **kw):
        raise RuntimeError("a step failed")
    monkeypatch.setattr(paged_decode.torch, "tensor", fails)
    monkeypatch.setattr(paged_decode.torch, "Generator", fails)
    with pytest.raises(RuntimeError, match="a step failed"):
        paged_decode.generate(model, [np.zeros(20, np.int32)] * 3, 12)
    assert sorted(model.free) == list(range(8))
