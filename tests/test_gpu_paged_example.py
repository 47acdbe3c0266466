"""The serving loop of examples/paged_serving.py: all five calls of the paged cache in
one batch after the other."""
import importlib.util
import os

import pytest
import torch

pytestmark = pytest.mark.gpu

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def example():
    spec = importlib.util.spec_from_file_location("paged_serving", os.path.join(ROOT, "examples", "paged_serving.py"))
    m = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(m)
    return m


# fp32: two layers of sums over up to 280 keys and 512 columns, each off by less than 1e-5 of
# its terms.  16 bits: the projections round their results to half a unit (2^-8, 2^-11), five
# times a layer, and the residual keeps the state larger than what is added.
@pytest.mark.parametrize("dtype,tol", [(torch.float32, 1e-4), (torch.bfloat16, 0.04), (torch.float16, 0.005)])
def test_serving_loop_gives_the_whole_sequence_run(gpu, dtype, tol):
    tokens, steps, worst = example().serve(requests=9, check=True, dtype=dtype)
    assert tokens > 500 and steps > 20
    assert worst < tol


def test_sparse_serving_over_all_pages_is_the_dense_one(gpu):
    """Enough pages per token that every one is selected: the same states."""
    tokens, steps, worst = example().serve(requests=6, sparse=20, check=True, dtype=torch.float32)
    assert worst < 1e-4


def test_sparse_serving_runs_over_a_few_pages(gpu):
    tokens, steps, worst = example().serve(requests=6, sparse=4)
    assert worst is None and tokens > 300
