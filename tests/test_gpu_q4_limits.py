"""dcl_kv_attention over a 4-bit cache where rows see nothing, against the reference and by the tolerance of
test_gpu_q4_attention."""
import numpy as np
import pytest

import test_gpu_q4_attention as att
from test_gpu_q4_attention import ops  # noqa: F401 (a fixture)

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("heads,kv,hd", [(4, 4, 64), (7, 1, 128), (8, 1, 64)])
@pytest.mark.parametrize("page_len", [16, 64])
@pytest.mark.parametrize("lens,news", [([0], [20]), ([3], [20]), ([3, 500, 0], [20, 2, 9]), ([300], [400])])
def test_causal_rows_before_the_first_position(ops, lens, news, page_len, heads, kv, hd):  # noqa: F811
    """Sequences with more rows than positions, and more than max_new says (the kernel for up to 8 rows takes them
    in passes): the first rows stand before position 0, see nothing, and no page is looked up for them."""
    att._check(ops, np.random.default_rng(sum(lens) + hd), lens, news, heads, kv, hd, page_len, causal=True, max_new=1)


@pytest.mark.parametrize("lens,new", [([2, 0], 8), ([1], 4)])
def test_causal_rows_before_the_first_position_within_max_new(ops, lens, new):  # noqa: F811
    att._check(ops, np.random.default_rng(new), lens, [new] * len(lens), 2, 2, 128, 32, causal=True)
