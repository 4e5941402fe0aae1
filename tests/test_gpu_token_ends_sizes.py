"""Embedding and log probabilities without logits at the ends of their ranges: rows far apart, offsets past 2^31, more workgroups than a
dimension of a launch holds, the widest rows, the largest vocabulary, the most tokens and groups.  What such a call gives has to be, bit for bit, what
the same rows give close together, or sums of small whole numbers, which float32 holds exactly."""
import pytest
import torch

pytestmark = pytest.mark.gpu
TYPES = {"fp32": torch.float32, "bf16": torch.bfloat16, "fp16": torch.float16}


@pytest.fixture(scope="module")
def B():
    from paper_1805_10032_amd import binding
    binding.load_library()
    yield binding
    torch.cuda.empty_cache()


def far(x, pitch):
    """The same rows `pitch` elements apart, in memory that is not cleared."""
    out = torch.empty((x.shape[0] - 1) * pitch + x.shape[1], dtype=x.dtype, device="cuda").as_strided(x.shape, (pitch, 1))
    out.copy_(x)
    return out


@pytest.mark.parametrize("rows,width", [(2049, 1 << 24), (8192, (1 << 22) + 64)])
def test_lookup_of_more_workgroups_than_a_dimension_holds(B, rows, width):
    table = torch.randint(-100, 100, (3, width), device="cuda").bfloat16()
    ids = torch.arange(rows, device="cuda", dtype=torch.int32) % 4 - 1
    out = torch.empty(rows, width, dtype=torch.bfloat16, device="cuda")
    B.zeno_embedding(ids, table, out=out)
    for i in range(4):
        want = torch.zeros_like(table[0]) if i == 0 else table[i - 1]
        for part in range(i, rows, 4 * 64):
            assert (out[part:part + 4 * 64:4] == want).all(), (i, part)
    del out
    torch.cuda.empty_cache()


def test_gradient_without_rows_of_a_large_table(B):
    vocab, width = 1 << 20, (1 << 15) + 1
    G = torch.full((1, vocab * width), 9.0, device="cuda")
    B.zeno_embedding_backward(torch.empty(0, width, device="cuda"), torch.empty(0, dtype=torch.int32, device="cuda"), vocab, dtable=G)
    for part in G[0].split(1 << 30):
        assert not part.any()
    del G, part
    torch.cuda.empty_cache()


@pytest.mark.parametrize("ty", TYPES)
@pytest.mark.parametrize("rows", [5, 70, 300])
def test_linear_rows_far_apart(B, rows, ty):
    vocab, width = 700, 40
    gen = torch.Generator(device="cuda").manual_seed(rows)
    rand = lambda *s: torch.randn(s, generator=gen, device="cuda")
    h, w, b = rand(rows, width).to(TYPES[ty]), (rand(vocab, width) * 0.3).to(TYPES[ty]), rand(vocab)
    labels = torch.randint(0, vocab, (rows,), generator=gen, device="cuda", dtype=torch.int32)
    g, q = rand(rows), rand(rows)
    groups = torch.tensor([0, rows // 2, rows - 1], dtype=torch.int32, device="cuda")
    h2, w2 = far(h, (1 << 31) // rows + 9), far(w, (1 << 31) // vocab + 16)
    one, two = (B.zeno_linear_logprobs(x, y, b, labels, want_entropy=True, want_stats=True) for x, y in ((h, w), (h2, w2)))
    assert all(torch.equal(x, y) for x, y in zip(one, two))
    n = vocab * width
    G = torch.zeros(2, n + vocab, device="cuda")
    G2 = far(G, (1 << 31) + 5)
    dh, _, _ = B.zeno_linear_logprobs_backward(h, w, b, one[2], labels=labels, grad_logp=g, entropy=one[1], grad_entropy=q, groups=groups,
                                               dweight=G[:, :n], dbias=G[:, n:])
    dh2 = far(torch.zeros_like(dh), (1 << 31) // rows + 3)
    B.zeno_linear_logprobs_backward(h2, w2, b, two[2], labels=labels, grad_logp=g, entropy=two[1], grad_entropy=q, groups=groups, dhidden=dh2,
                                    dweight=G2[:, :n], dbias=G2[:, n:])
    assert torch.equal(dh, dh2) and torch.equal(G, G2)


@pytest.mark.parametrize("ty", TYPES)
@pytest.mark.parametrize("rows,vocab,width", [(70, 300, 1 << 16), (3, 40, 1 << 16), (3, 1 << 24, 3), (300, 1 << 21, 9), (1 << 22, 5, 2), (130, 1 << 17, 1 << 15)])
def test_linear_of_equal_logits(B, rows, vocab, width, ty):
    """Weights whose rows are all alike: every logit of a token is the same whole number, and every probability 1 / vocab.  dz is -1 / vocab but for the
    label's, dW of a column of ones its sum over the tokens."""
    h = torch.zeros(rows, width, dtype=TYPES[ty], device="cuda")
    h[:, 0] = 1.0
    h[:, -1] = 1.0
    w = torch.zeros(vocab, width, dtype=TYPES[ty], device="cuda")
    w[:, -1] = 2.0
    labels = (torch.arange(rows, device="cuda") % vocab).int()
    labels[0] = vocab - 1
    logp, entropy, stats = B.zeno_linear_logprobs(h, w, None, labels, want_entropy=True, want_stats=True)
    size = torch.tensor(float(vocab), dtype=torch.float64).log().item()
    near = 2.0 ** -20 * (1 + size)   # sums of `vocab` ones: whole numbers below 2^24, exact; the logarithm and two differences
    assert (logp + size).abs().max() <= near and (entropy - size).abs().max() <= near
    assert (stats[:, 0] == 2).all()
    g = torch.full((rows,), -1.0, device="cuda")
    small = vocab * width <= 1 << 31
    dh, dw, db = B.zeno_linear_logprobs_backward(h, w, None, stats, labels=labels, grad_logp=g, want_weight=small)
    # dh: all of dz times 2, which cancels: what is left are 1 / vocab's rounding, vocab times, and those of the additions
    half = {"fp32": 2.0 ** -22, "bf16": 2.0 ** -8, "fp16": 2.0 ** -11}[ty]
    assert dh[:, -1].float().abs().max() <= 4 * (half + near + (vocab / 8 + 600) * 2.0 ** -24) and (dh[:, 1:-1] == 0).all()
    hits = torch.bincount(labels.long(), minlength=vocab).double()
    want = rows / vocab - hits
    bound = (rows / vocab + hits) * (near + rows * 2.0 ** -24 + 2.0 ** -21) + rows * 2.0 ** -38
    assert ((db[0].double() - want).abs() <= bound).all()
    if small:
        table = dw.view(vocab, width)
        assert ((table[:, 0].double() - want).abs() <= bound).all() and torch.equal(table[:, 0], table[:, -1]) and (table[:, 1:-1] == 0).all()
    del w, h, dw
    torch.cuda.empty_cache()


def test_the_most_groups(B):
    rows, vocab, width, m = 3000, 40, 24, 1024
    gen = torch.Generator(device="cuda").manual_seed(2)
    cuts = torch.randint(0, rows + 1, (m + 1,), generator=gen, device="cuda").sort()[0].int()
    h, w = torch.randn(rows, width, generator=gen, device="cuda").bfloat16(), torch.randn(vocab, width, generator=gen, device="cuda").bfloat16()
    labels = torch.randint(0, vocab, (rows,), generator=gen, device="cuda", dtype=torch.int32)
    g = torch.full((rows,), -1.0, device="cuda")
    _, _, stats = B.zeno_linear_logprobs(h, w, None, labels, want_stats=True)
    dh, dw, db = B.zeno_linear_logprobs_backward(h, w, None, stats, labels=labels, grad_logp=g, groups=cuts)
    z = h.double() @ w.double().t()
    dz = torch.softmax(z, 1)
    dz[torch.arange(rows, device="cuda"), labels.long()] -= 1
    inside = torch.zeros(rows, dtype=torch.bool, device="cuda")
    inside[int(cuts[0]):int(cuts[-1])] = True
    worker = torch.bucketize(torch.arange(rows, device="cuda"), cuts[1:].long(), right=True).clamp(max=m - 1)
    # a logit has width + 8 roundings of sum |h w| < 60: its probability is off by less than 2^-12 of itself; 2^-22 where one that is nearly 1 is missing
    # in a sum near 1, for the pieces of dz and for the sums
    for got, factor in ((dw.view(m, vocab, width), h.double()[:, None, :]), (db[:, :, None], torch.ones(rows, 1, 1, dtype=torch.float64, device="cuda"))):
        factor = factor * inside[:, None, None]
        want = torch.zeros(got.shape, dtype=torch.float64, device="cuda").index_add_(0, worker, dz[:, :, None] * factor)
        bound = torch.zeros_like(want).index_add_(0, worker, (dz.abs()[:, :, None] + 2.0 ** -10) * factor.abs()) * 2.0 ** -12
        assert ((got.double() - want).abs() <= bound).all()
    assert (dh[~inside] == 0).all()
