"""dcl_kv_attention of more sequences than a lane keeps while it looks for its CTA's part (32 or 128, by kernel), in
every format and by every kernel, against the references of the formats' tests and by their tolerances."""
import numpy as np
import pytest

import test_gpu_kv_attention as wide_formats
import test_gpu_q4_attention as q4
from test_gpu_kv_attention import ops  # noqa: F401 (a fixture)

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("fmt", ["bf16", "fp8", "q4"])
@pytest.mark.parametrize("batch", [32, 33, 100, 129, 300])
@pytest.mark.parametrize("max_new,wide", [(1, 0), (6, 0), (16, 0), (40, 20000)])  # (2 rows of a kv head each: four kernels)
def test_more_sequences_than_a_lane_keeps(ops, fmt, batch, max_new, wide):  # noqa: F811
    rng = np.random.default_rng(batch + max_new)
    lens = rng.integers(0, 60, batch)
    lens[rng.integers(0, batch, 3)] = (700, 300, 129)
    news = np.minimum(rng.integers(0, 3, batch), max_new)
    news[rng.integers(0, batch, 2)] = max_new
    args = (ops, rng, lens.tolist(), news.tolist(), 2, 1, 64, 16)
    kw = dict(max_new=max_new, wide=wide)
    if fmt == "q4":
        q4._check(*args, causal=bool(batch & 1), **kw)
    else:
        wide_formats._check(*args, fmt == "fp8", **kw)
