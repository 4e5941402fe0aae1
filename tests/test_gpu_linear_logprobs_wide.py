"""Weight gradients on wide tiles, and hidden states' gradients on wide tiles over several pieces of the vocabulary: the sizes that take them, which
tests/sanitize/plan_checks.cpp holds to."""
import pytest
import torch

from _tokens import TYPES
from test_gpu_linear_logprobs import backward

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def B():
    from paper_1805_10032_amd import binding
    binding.load_library()
    yield binding
    torch.cuda.empty_cache()


@pytest.mark.parametrize("ty", TYPES)
@pytest.mark.parametrize("rows,vocab,width,offsets,pad,entropy", [
    (2100, 12600, 1000, [0, 1030, 2095], 0, False),     # two groups, odd remainders of the tokens, the weights and the vocabulary
    (2100, 12600, 1000, [5, 2100, 2100], 3, True),      # packed copies; one group holds everything
    (2101, 25090, 1024, None, 0, False),                # rows of gradients on memory lines: past the caches
    (8200, 8500, 1544, [0, 4100, 8190], 0, False),      # two pieces of the vocabulary, wide tiles of everything
])
def test_backward_on_wide_tiles(B, rows, vocab, width, offsets, pad, entropy, ty):
    """Each gradient against float64; then, bit for bit, alone and without the bias's."""
    backward(B, rows, vocab, width, ty, offsets, entropy, pad_w=pad, seed=13)
