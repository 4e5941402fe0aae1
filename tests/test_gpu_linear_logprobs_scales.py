"""Gradients of any size that float32 holds, in each group its own: 2^120 in one and 2^-100 in the next come out as accurate as 1 does.

Bounds are those of ordinary gradients (test_gpu_linear_logprobs.py), scaled: dz in float32 is off by `e`; in 16-bit types its pieces by 2^-22 of it (weights) or
half_step^2 (hidden states) and 2^-38 of the group's largest gradient."""
import pytest
import torch

from _tokens import EPS, TYPES, half_step, smallest_half
from test_gpu_linear_logprobs import Reference, inside, problem

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def B():
    from paper_1805_10032_amd import binding
    binding.load_library()
    return binding


def check(B, rows, vocab, width, ty, offsets, powers, g, q, h_power=0):
    dtype = TYPES[ty]
    h, w, b, labels = problem(rows, vocab, width, dtype, 17, spread=1.0)
    h = (h.float() * 2.0 ** h_power).to(dtype)
    w = (w.float() * 2.0 ** -h_power).to(dtype)
    ref = Reference(h, w, b, labels)
    group = torch.bucketize(torch.arange(rows, device="cuda"), torch.tensor(offsets[1:], device="cuda"), right=True).clamp(max=len(powers) - 1)
    factor = 2.0 ** torch.tensor(powers, dtype=torch.float64, device="cuda")[group]
    one = [None if t is None else t.double() for t in (g, q)]
    G, Q = (None if t is None else (t * factor).float() for t in one)
    # the powers of two scale everything exactly, so the bounds of the ordinary gradients do too
    dz, e = ref.grad(g, q)
    largest = sum(t.abs() * f for t, f in ((g, 1), (q, 22)) if t is not None)
    _, entropy, stats = B.zeno_linear_logprobs(h, w, b, labels, want_entropy=True, want_stats=True)
    dh, dw, db = B.zeno_linear_logprobs_backward(h, w, b, stats, labels=labels if g is not None else None, grad_logp=G,
                                                 entropy=entropy if q is not None else None, grad_entropy=Q,
                                                 groups=torch.tensor(offsets, dtype=torch.int32, device="cuda"))
    planes = 2.0 ** -24 if ty == "fp32" else 2.0 ** -22
    for i, power in enumerate(powers):
        part = slice(offsets[i], offsets[i + 1])
        tokens, scale = offsets[i + 1] - offsets[i], 2.0 ** power
        least = 0.0 if ty == "fp32" else 2.0 ** -38 * float(largest[part].max())
        d, de, H = dz[part], e[part] + planes * dz[part].abs() + least, ref.H[part]
        inexact = 2.0 ** -39 * ref.H[part].abs().amax(0) if ty == "bf16" else 0.0
        bound = de.t() @ H.abs() + d.abs().sum(0)[:, None] * inexact + (2 * tokens + 12) * EPS * (d.abs().t() @ H.abs())
        want = d.t() @ H
        # (2^-126: the smallest normal number)
        inside(dw[i].view(vocab, width).double() / scale, want, bound * 1.01 + EPS * want.abs() + 2.0 ** (-126 - power), f"dweight {power}")
        inside(db[i].double() / scale, d.sum(0), (de.sum(0) + (3 * tokens + 16) * EPS * d.abs().sum(0)) * 1.01 + 2.0 ** (-126 - power), f"dbias {power}")
        if ty == "fp16":
            continue       # (the type has no such numbers)
        held = planes if ty == "fp32" else half_step(dtype) ** 2
        W, want = ref.W.abs(), d @ ref.W
        bound = (e[part] + held * d.abs() + least) @ W + 6 * (vocab + 40) * EPS * (d.abs() @ W)
        bound = bound * 1.01 + half_step(dtype) * (want.abs() + bound) + 2.0 ** (-126 - power)
        # what lies beyond the type (2^80 times weights of 2^60: 2^140) has no finite value: an infinity, or NaN where terms beyond it have both signs
        beyond = (want.abs() - bound) * scale >= 2.0 ** 128
        assert not dh[part][beyond].isfinite().any()
        inside(torch.where(beyond, want, dh[part].double() / scale), want, bound, f"dhidden {power}")


@pytest.mark.parametrize("ty", TYPES)
@pytest.mark.parametrize("rows,vocab,width", [(40, 90, 24), (300, 90, 24), (300, 260, 33)])
def test_large_and_small_gradients_of_groups(B, rows, vocab, width, ty):
    gen = torch.Generator(device="cuda").manual_seed(rows)
    rand = lambda: torch.rand(rows, generator=gen, device="cuda")
    off = [0, rows // 4, rows // 2, 3 * rows // 4, rows]
    check(B, rows, vocab, width, ty, off, [120, -100, 0, 114], -0.5 - 0.5 * rand(), None)
    check(B, rows, vocab, width, ty, off, [116, -96, 100, -86], -0.5 - 0.5 * rand(), 0.1 * rand())


@pytest.mark.parametrize("ty", TYPES)
def test_hidden_states_beside_large_gradients(B, ty):
    """Columns that are scaled up or down too: the two powers together may leave float32's range, their product does not."""
    rows, vocab, width = 70, 33, 16
    off = [0, 20, 40, 70]
    gen = torch.Generator(device="cuda").manual_seed(4)
    g = -0.5 - 0.5 * torch.rand(rows, generator=gen, device="cuda")
    for power in (-10, 8) if ty == "fp16" else (-60, -10, 40):
        # (dweight goes with g h: 2^117 2^8, 2^-60 2^-60, 2^80 2^40 at most; sums of 30 terms stay below 2^127)
        check(B, rows, vocab, width, ty, off, [80, -60, 117 if power < 10 else 70], g, None, power)


@pytest.mark.parametrize("ty", TYPES)
def test_gradients_of_the_entropy_near_the_largest_number(B, ty):
    """22 times them leaves float32; dz, p (log p + H) times them, does not, nor do sums of six tokens (six times p |log p + H| < 1/4 and |h| < 5: below 2^3)."""
    rows, vocab, width = 12, 200, 16
    q = torch.full((rows,), 0.75, device="cuda")
    check(B, rows, vocab, width, ty, [0, 6, 12], [124, -70], None, q)


@pytest.mark.parametrize("rows,vocab,width", [(40, 90, 24), (300, 90, 24)])
def test_small_and_large_gradients_of_one_group_in_float32(B, rows, vocab, width):
    """A token's gradient does not depend on another's: a power of two scales a row of dhidden exactly, 2^-80 beside 2^80 (all terms and sums of both
    stay normal but for those below 2^-40 of the largest)."""
    h, w, b, labels = problem(rows, vocab, width, torch.float32, 23, spread=1.0)
    gen = torch.Generator(device="cuda").manual_seed(2)
    g = -0.5 - 0.5 * torch.rand(rows, generator=gen, device="cuda")
    q = 0.1 * torch.rand(rows, generator=gen, device="cuda")
    _, entropy, stats = B.zeno_linear_logprobs(h, w, b, labels, want_entropy=True, want_stats=True)
    factor = torch.where(torch.arange(rows, device="cuda") % 2 == 0, 2.0 ** 80, 2.0 ** -80)

    def dhidden(g, q):
        return B.zeno_linear_logprobs_backward(h, w, b, stats, labels=labels, grad_logp=g, entropy=entropy, grad_entropy=q, want_weight=False,
                                               want_bias=False)[0]
    plain, far = dhidden(g, q), dhidden(g * factor, q * factor)
    assert (far.double() / factor[:, None].double() - plain.double()).abs().max() <= 2.0 ** -40 * vocab
