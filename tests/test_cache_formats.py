"""Which format a cache is taken for, by its tensors (CPU only)."""
import numpy as np
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


@pytest.mark.parametrize("bytes_", [32, 64])
def test_scales_in_another_shape_are_not_taken_for_exponents(bytes_):
    """4-bit codes have as many bytes as FP8 codes of half the head_dim; their scales, flattened, would pass as
    exponents of such a cache."""
    n = bytes_ // 16
    codes, exps = FakeCuda((4, 2, 16, bytes_), 1), FakeCuda((4, 2, 16), 1)
    for flat in (FakeCuda((4, 2, 16 * n), 1), FakeCuda((4 * 2 * 16 * n,), 1), FakeCuda((4, 2, n, 16), 1)):
        for pair in ((flat, flat), (exps, flat), (flat, exps)):
            with pytest.raises(ValueError, match="scales"):
                dcl.KvCache(codes, codes, *pair)


def test_exponents_of_other_shapes_are():
    codes = FakeCuda((4, 2, 16, 64), 1)
    for exps in (FakeCuda((4, 2, 16), 1), FakeCuda((128,), 1), FakeCuda((4, 2, 16, 1), 1), FakeCuda((200,), 1)):
        assert dcl.KvCache(codes, codes, exps, exps).format == dcl.DCL_KV_FP8
    codes, exps = FakeCuda((4, 2, 16, 128), 1), FakeCuda((4 * 2 * 16 * 8,), 1)  # (no 4-bit cache has 256 components)
    assert dcl.KvCache(codes, codes, exps, exps).format == dcl.DCL_KV_FP8
    codes = FakeCuda((4, 2, 16, 64), 1)
    codes.dtype = "torch.float8_e4m3fn"  # (which says what it is)
    assert dcl.KvCache(codes, codes, FakeCuda((512,), 1), FakeCuda((512,), 1)).format == dcl.DCL_KV_FP8


@pytest.mark.parametrize("bytes_", [32, 64, 128])
def test_host_arrays_are_no_exponents(bytes_):
    codes = FakeCuda((4, 2, 16, bytes_), 1)
    for exps in (np.zeros((4, 2, 16), np.int8), np.zeros((4, 2, 16, bytes_ // 16), np.uint8)):
        with pytest.raises(ValueError):
            dcl.KvCache(codes, codes, exps, exps)
