"""dcl_kv_plan of more sequences than one block keeps in shared memory (2048), and of the largest pages: the steps of
test_gpu_kv_plan."""
import pytest

import test_gpu_kv_plan as plan
from test_gpu_kv_plan import ops  # noqa: F401 (a fixture)

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("batch,page_len,width,n_pages", [
    (2047, 16, 3, 4000), (2048, 32, 4, 5000), (2049, 16, 4, 5000), (5000, 64, 3, 9000), (40, 256, 5, 110), (256, 16, 4, 600), (257, 16, 4, 600)])
def test_steps_of_growing_shrinking_and_ending_sequences(ops, batch, page_len, width, n_pages):  # noqa: F811
    plan.test_steps_of_growing_shrinking_and_ending_sequences(ops, batch, page_len, width, n_pages)


@pytest.mark.parametrize("batch,rows", [(256, 4096), (256, 4097), (257, 4000), (2048, 9000), (2049, 9000), (5000, 12000)])
def test_lengths_that_take_the_place_of_the_starts(ops, batch, rows):  # noqa: F811
    plan.test_lengths_that_take_the_place_of_the_starts(ops, batch, rows)
