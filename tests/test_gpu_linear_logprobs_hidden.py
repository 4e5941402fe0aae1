"""Gradients of the hidden states where the weights' rows share a component: dz sums to nearly nothing over the vocabulary, so the component cancels in
dz W, and what is left shows how many bits dz is held in.

Bounds.  `e`: dz in float32 (Reference.grad).  dz in 16-bit types is two planes of them, the second of what the first has left: off by at most
half_step^2 of itself, and by 2^-38 of the group's largest gradient where fp16's steps end; in float32 three bf16 pieces, below 2^-24.  A sum of n products
in float32 is off by n EPS of its terms' magnitudes; two planes make 2 n of them.  Then one rounding to the type.  The states' and weights' sums of 16
products keep `e` two orders below a single plane's error."""
import pytest
import torch

from _tokens import EPS, TYPES, half_step, smallest_half
from test_gpu_linear_logprobs import Reference, inside

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def B():
    from paper_1805_10032_amd import binding
    binding.load_library()
    return binding


@pytest.mark.parametrize("ty", TYPES)
@pytest.mark.parametrize("which", ["label", "entropy", "both"])
@pytest.mark.parametrize("rows,vocab,width,offsets", [
    (40, 50, 16, None),                        # few tokens
    (300, 50, 16, [0, 100, 100, 297]),         # tiles of 128, several groups
    (300, 140, 24, None),
    (129, 33, 9, [3, 129]),                    # packed copies
    (8200, 70, 1544, None),                    # wide tiles of hidden states
])
def test_weights_that_share_a_component(B, rows, vocab, width, offsets, which, ty):
    dtype = TYPES[ty]
    gen = torch.Generator(device="cuda").manual_seed(rows + vocab)
    rand = lambda *s: torch.randn(s, generator=gen, device="cuda", dtype=torch.float64)
    shared = 10.0 * rand(1, width)
    w = ((rand(vocab, width) + shared) / 16).to(dtype)
    # states across the shared component, so that logits are small; the first sixteen columns alone hold them
    h = rand(rows, width)
    h[:, 16:] = 0
    across = shared.clone()
    across[:, 16:] = 0
    h = (h - (h @ across.t()) / (across @ across.t()) * across).to(dtype)
    labels = torch.randint(0, vocab, (rows,), generator=gen, device="cuda", dtype=torch.int32)
    labels[2] = -1
    g = -(1 + 0.1 * torch.randn(rows, generator=gen, device="cuda")) if which != "entropy" else None
    q = -(1 + 0.1 * torch.randn(rows, generator=gen, device="cuda")) if which != "label" else None
    ref = Reference(h, w, None, labels)
    _, entropy, stats = B.zeno_linear_logprobs(h, w, None, labels, want_entropy=True, want_stats=True)
    off = offsets or [0, rows]
    groups = None if offsets is None else torch.tensor(offsets, dtype=torch.int32, device="cuda")
    dh, _, _ = B.zeno_linear_logprobs_backward(h, w, None, stats, labels=labels if g is not None else None, grad_logp=g,
                                               entropy=entropy if q is not None else None, grad_entropy=q, groups=groups, want_weight=False,
                                               want_bias=False)
    dz, e = ref.grad(g, q)
    held = 2.0 ** -24 if ty == "fp32" else half_step(dtype) ** 2
    least = 0.0 if ty == "fp32" else 2.0 ** -38 * float(((g.abs() if g is not None else 0) + (22 * q.abs() if q is not None else 0)).max())
    want, size = dz @ ref.W, dz.abs() @ ref.W.abs()
    bound = e @ ref.W.abs() + held * size + least * ref.W.abs().sum(0) + (6 if ty == "fp32" else 2) * (vocab + 40) * EPS * size
    bound = bound * 1.01 + half_step(dtype) * (want.abs() + bound) + smallest_half(dtype)
    lo, hi = off[0], off[-1]
    inside(dh[lo:hi], want[lo:hi], bound[lo:hi], "dh")
    assert (dh[:lo] == 0).all() and (dh[hi:] == 0).all()
    # No further from 64 bits than the rounded exact result, but for a tenth: half_step^2 is 1 / 256 of a rounding or less, and ten times that (what is
    # left of the shared component) 1 / 25, which adds 1 / 1250 to a root of squares; float32's own errors lie below both.
    rounded = (want[lo:hi].to(dtype).double() - want[lo:hi]).norm()
    if ty != "fp32" and which != "entropy":
        assert (dh[lo:hi].double() - want[lo:hi]).norm() <= 1.1 * rounded


@pytest.mark.parametrize("ty", ["bf16", "fp16"])
def test_pieces_of_the_vocabulary_that_share_a_component(B, ty):
    """The same over several pieces of the vocabulary and wide tiles of hidden states, whose sums are added in memory."""
    rows, vocab, width, dtype = 8200, 8500, 1544, TYPES[ty]
    gen = torch.Generator(device="cuda").manual_seed(7)
    rand = lambda *s: torch.randn(s, generator=gen, device="cuda")
    shared = 10.0 * rand(1, width)
    w = ((rand(vocab, width) + shared) / 16).to(dtype)
    h = rand(rows, width)
    h[:, 16:] = 0
    across = shared.clone()
    across[:, 16:] = 0
    h = (h - (h @ across.t()) / (across @ across.t()) * across).to(dtype)
    labels = torch.randint(0, vocab, (rows,), generator=gen, device="cuda", dtype=torch.int32)
    g = torch.full((rows,), -1.0, device="cuda")
    _, _, stats = B.zeno_linear_logprobs(h, w, None, labels, want_stats=True)
    dh, _, _ = B.zeno_linear_logprobs_backward(h, w, None, stats, labels=labels, grad_logp=g, want_weight=False, want_bias=False)
    ref = Reference(h, w, None, labels)
    dz, e = ref.grad(g, None)
    want, size = dz @ ref.W, dz.abs() @ ref.W.abs()
    bound = e @ ref.W.abs() + half_step(dtype) ** 2 * size + 2.0 ** -38 * ref.W.abs().sum(0) + 2 * (vocab + 40) * EPS * size
    inside(dh, want, bound * 1.01 + half_step(dtype) * (want.abs() + bound) + smallest_half(dtype), "dh")
    assert (dh.double() - want).norm() <= 1.1 * (want.to(dtype).double() - want).norm()
