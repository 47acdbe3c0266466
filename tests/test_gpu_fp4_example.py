"""The serving loop of examples/paged_serving.py over a cache in 4 bits, and with answers that share a prompt's pages."""
import pytest
import torch

from tests.test_gpu_paged_example import example

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16, torch.float32])
@pytest.mark.parametrize("answers", [1, 3])
def test_serving_from_four_bits(gpu, dtype, answers):
    tokens, steps, worst = example().serve(requests=6, dtype=dtype, answers=answers, four_bits=True)
    assert worst is None and tokens > 300 and steps > 10


def test_answers_that_share_a_prompt(gpu):
    """Each answer ends in the state of its whole sequence: two layers of fp32 sums, each off by less than 1e-5."""
    alone = example().serve(requests=6, check=True, dtype=torch.float32)
    tokens, steps, worst = example().serve(requests=6, check=True, dtype=torch.float32, answers=4)
    assert worst < 1e-4 and tokens > alone[0]


def test_shared_answers_over_selected_pages(gpu):
    """Summaries go with the pages: with every page selected, the dense states."""
    tokens, steps, worst = example().serve(requests=4, sparse=20, check=True, dtype=torch.float32, answers=3)
    assert worst < 1e-4


def test_no_selection_in_four_bits():
    with pytest.raises(ValueError):
        example().serve(sparse=4, four_bits=True)
