"""Log probabilities without logits at the corners of their documented sizes."""
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


@pytest.mark.parametrize("rows,vocab", [(65281, 1 << 24), (1500, (1 << 24) - 255), (70000, 300000)])
def test_the_most_tiles(B, rows, vocab):
    """Weights that are read as they stand, whose rows are all alike: every logit of a token is the same whole number and every probability 1 / vocab.  Sums
    of `vocab` ones are whole numbers up to 2^24, exact; the logarithm and two differences are off by less than 2^-20 of 1 + log vocab."""
    width = 8
    h = torch.zeros(rows, width, dtype=torch.bfloat16, device="cuda")
    h[:, 0] = 1.0
    w = torch.zeros(vocab, width, dtype=torch.bfloat16, device="cuda")
    w[:, 0] = 2.0
    labels = (torch.arange(rows, device="cuda") * 257 % vocab).int()
    labels[::3] = vocab - 1
    labels[5] = -1
    logp, entropy, stats = B.zeno_linear_logprobs(h, w, None, labels, want_entropy=True, want_stats=True)
    size = torch.tensor(float(vocab), dtype=torch.float64).log().item()
    near = 2.0 ** -20 * (1 + size)
    assert logp[5] == 0
    logp[5] = -size
    assert (logp + size).abs().max() <= near and (entropy - size).abs().max() <= near and (stats[:, 0] == 2).all()


@pytest.mark.parametrize("ty", TYPES)
@pytest.mark.parametrize("rows,offsets", [(5, None), (70, [0, 30, 69]), (300, None)])
def test_weights_that_are_packed_in_pieces(B, rows, offsets, ty):
    """More weights than are packed at a time in one piece of dz: few tokens, and tiles."""
    backward(B, rows, 10000, 8191, ty, offsets, False, seed=21)
