"""Which format a cache is taken for, by its tensors (CPU only)."""
import pytest

import paper_2607_20467_gb300 as dcl
from test_serving_args import FakeCuda


def test_exponents_may_be_raw_addresses():
    codes = FakeCuda((4, 2, 16, 64), 1)
    cache = dcl.KvCache(codes, codes, 0x7000_0000, 0x7000_1000)
    assert (cache.format, cache.head_dim) == (dcl.DCL_KV_FP8, 64)
    assert (cache.desc.k_exp_dev, cache.desc.v_exp_dev) == (0x7000_0000, 0x7000_1000)


def test_scales_are_no_raw_address():
    codes, scales = FakeCuda((4, 2, 16, 32), 1), FakeCuda((4, 2, 16, 2), 1)
    with pytest.raises(ValueError, match="scales expected"):
        dcl.KvCache(codes, codes, scales, 0x7000_0000)
