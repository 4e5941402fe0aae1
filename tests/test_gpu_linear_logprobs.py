"""Log probabilities straight from hidden states, and their gradients per worker, against float64.

Bounds count roundings.  A logit is a sum of `width` exact products (float32 operands: of six piece products, what is left out is below 4 EPS
of a product) in float32, so it is off by at most (width + 8) EPS sum |h w| and the bias's addition.  The logarithm of the sum of exponentials moves by
no more than the p-weighted mean of that, and adds a chain of at most 256 + slices additions and the exponentials' own errors (a product rounded to float32, 2 EPS |d|, and
an instruction that is right to 2^-22).  dz is p (..): p's relative error is that of its logarithm.  Gradients add the rounding of dz to its pieces and
float32 sums."""
import numpy as np
import pytest
import torch

from _tokens import EPS, TYPES, around, half_step, smallest_half, strided

pytestmark = pytest.mark.gpu
EXP = 2.0 ** -22


@pytest.fixture(scope="module")
def B():
    from paper_1805_10032_amd import binding
    binding.load_library()
    return binding


def problem(rows, vocab, width, dtype, seed=0, pad_h=0, pad_w=0, offset=0, masked=0.0, bias=True, spread=2.0):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    rand = lambda *s: torch.randn(s, generator=gen, device="cuda", dtype=torch.float64)
    h, h_buf = strided(rand(rows, width), dtype, width + pad_h, offset)
    w, w_buf = strided(rand(vocab, width) * (spread / width ** 0.5), dtype, width + pad_w, offset)
    b = rand(vocab).float() if bias else None
    labels = torch.randint(0, vocab, (rows,), generator=gen, device="cuda", dtype=torch.int32)
    if masked and vocab > 1:
        ban = torch.rand(vocab, generator=gen, device="cuda") < masked
        ban[0] = False
        b = torch.zeros(vocab, device="cuda") if b is None else b
        b[ban] = float("-inf")
        labels[ban[labels.long()]] = 0
    if rows > 5:
        labels[3] = -1
    return h, w, b, labels


class Reference:
    """Everything in float64 on the same inputs, with bounds."""

    def __init__(self, h, w, b, labels):
        H, W = h.double(), w.double()
        self.H, self.W = H, W
        width, vocab = H.shape[1], W.shape[0]
        z = H @ W.t()
        ez = (width + 8) * EPS * (H.abs() @ W.abs().t())
        if b is not None:
            z = z + b.double()
        ez = ez + EPS * torch.where(z.isfinite(), z.abs(), torch.zeros_like(z))
        M = z.amax(1, keepdim=True)
        self.empty = (M == -float("inf"))[:, 0]
        M = torch.where(M.isfinite(), M, torch.zeros_like(M))
        d = z - M
        e = torch.exp(d)
        s = e.sum(1, keepdim=True)
        s = torch.where(s > 0, s, torch.ones_like(s))
        self.lse = torch.log(s)
        self.lp = d - self.lse
        self.p = e / s
        flat = torch.where(self.p > 0, self.lp, torch.zeros_like(z))
        dd = torch.where(self.p > 0, d, torch.zeros_like(d)).abs()
        self.entropy = -(self.p * flat).sum(1)
        chain = (256 + vocab / 64 + 24) * EPS
        self.e_lse = (self.p * (ez + 2 * dd * EPS + EXP)).sum(1, keepdim=True) + chain
        scale = torch.where(d.isfinite(), d.abs(), torch.zeros_like(d)) + self.lse.abs() + M.abs()
        self.e_lp = ez + self.e_lse + 4 * EPS * scale
        lph = (flat + self.entropy[:, None]).abs()
        # the entropy's derivative along z is -p (log p + H); its two sums of `chain` additions, their quotient and difference
        self.e_ent = (self.p * lph * (ez + 2 * dd * EPS + EXP)).sum(1) + 2 * chain * ((self.p * dd).sum(1) + self.lse[:, 0].abs()) + 8 * EPS * (1 + self.lse[:, 0].abs())
        self.flat = flat
        self.y = labels.long()
        self.ok = (self.y >= 0) & (self.y < vocab)
        yc = self.y.clamp(0, vocab - 1)[:, None]
        self.logp = torch.where(self.ok, self.lp.gather(1, yc)[:, 0], torch.zeros_like(self.lse[:, 0]))
        self.e_logp = torch.where(self.ok, self.e_lp.gather(1, yc)[:, 0], torch.zeros_like(self.lse[:, 0]))

    def grad(self, g, q):
        rows, vocab = self.p.shape
        G = torch.zeros(rows, 1, dtype=torch.float64, device=self.p.device) if g is None else torch.where(self.ok, g.double(), torch.zeros_like(g.double()))[:, None]
        Q = torch.zeros_like(G) if q is None else q.double()[:, None]
        inner = G + Q * (self.flat + self.entropy[:, None])
        size = G.abs() + Q.abs() * (self.flat.abs() + self.entropy[:, None])
        dz = -self.p * inner
        one = torch.zeros_like(dz)
        one[torch.arange(rows, device=dz.device)[self.ok], self.y[self.ok]] = 1.0
        dz = dz + one * G
        rel = self.e_lp + 2 * self.flat.abs() * EPS + EXP + 4 * EPS
        rel = torch.where(self.p > 0, rel, torch.zeros_like(rel))
        e = self.p * (rel * inner.abs() + 6 * EPS * size + Q.abs() * (self.e_lp.where(self.p > 0, torch.zeros_like(rel)) + self.e_ent[:, None])) + 4 * EPS * (dz.abs() + one * G.abs()) + 2.0 ** -120
        return dz, e


def inside(got, ref, bound, what):
    err = (got.double() - ref).abs()
    bad = ~(err <= bound)
    assert not bad.any(), (what, float(err.max()), float((err / bound).nan_to_num(posinf=1e30).max()), bad.nonzero()[:5].tolist())


SIZES = [
    # rows, vocab, width, pads of h and w, offset
    (1, 1, 1, 0, 0, 0), (1, 2, 3, 1, 2, 1), (3, 5, 8, 0, 0, 0), (2, 33, 16, 8, 8, 8), (17, 129, 40, 0, 0, 0), (31, 127, 31, 1, 0, 1),
    (33, 1000, 65, 0, 3, 2), (128, 128, 64, 0, 0, 0), (129, 257, 72, 8, 16, 0), (130, 300, 96, 1, 1, 0), (1, 5000, 256, 0, 0, 0),
    (255, 700, 513, 0, 0, 1), (64, 4100, 104, 0, 0, 0), (257, 255, 33, 7, 0, 3), (5, 20000, 128, 0, 0, 0), (600, 10, 24, 0, 0, 0),
]


@pytest.mark.parametrize("ty", TYPES)
@pytest.mark.parametrize("rows,vocab,width,pad_h,pad_w,offset", SIZES)
@pytest.mark.parametrize("masked", [0.0, 0.4])
def test_forward(B, rows, vocab, width, pad_h, pad_w, offset, ty, masked):
    h, w, b, labels = problem(rows, vocab, width, TYPES[ty], rows + vocab, pad_h, pad_w, offset, masked, bias=vocab % 2 == 1)
    ref = Reference(h, w, b, labels)
    logp, entropy, stats = B.zeno_linear_logprobs(h, w, b, labels, want_entropy=True, want_stats=True)
    inside(logp, ref.logp, ref.e_logp, "logp")
    inside(entropy, ref.entropy, ref.e_ent, "entropy")
    again = B.zeno_linear_logprobs(h, w, b, labels, want_entropy=True, want_stats=True)
    assert all(torch.equal(x, y) for x, y in zip((logp, entropy, stats), again))
    only, none, nothing = B.zeno_linear_logprobs(h, w, b, labels)
    assert torch.equal(only, logp) and none is None and nothing is None
    a, ent, st = B.zeno_linear_logprobs(h, w, b, want_entropy=True)
    assert a is None and torch.equal(ent, entropy) and st is None


def backward(B, rows, vocab, width, ty, offsets, entropy_too, *, pad_h=0, pad_w=0, offset=0, masked=0.0, seed=1, grad=True):
    dtype = TYPES[ty]
    h, w, b, labels = problem(rows, vocab, width, dtype, seed, pad_h, pad_w, offset, masked)
    ref = Reference(h, w, b, labels)
    gen = torch.Generator(device="cuda").manual_seed(seed + 7)
    g = -(1 + 0.1 * torch.randn(rows, generator=gen, device="cuda")) / rows if grad else None
    q = -0.1 * torch.rand(rows, generator=gen, device="cuda") / rows if entropy_too else None
    _, entropy, stats = B.zeno_linear_logprobs(h, w, b, labels, want_entropy=True, want_stats=True)
    off = offsets or [0, rows]
    m = len(off) - 1
    groups = None if offsets is None else torch.tensor(offsets, dtype=torch.int32, device="cuda")
    n = vocab * width
    G, buf = strided(torch.full((m, n + vocab), 3.0), torch.float32, n + vocab + 5, 3)
    before = around(G, buf)
    dh, dh_buf = strided(torch.full((rows, width), 5.0), dtype, width + pad_h, offset)
    dh_before = around(dh, dh_buf)
    B.zeno_linear_logprobs_backward(h, w, b, stats, labels=labels if grad else None, grad_logp=g, entropy=entropy if entropy_too else None,
                                    grad_entropy=q, groups=groups, dhidden=dh, dweight=G[:, :n], dbias=G[:, n:])
    dz, e = ref.grad(g, q)
    planes = 2.0 ** -24 if ty == "fp32" else 2.0 ** -22
    first = {"fp32": 2.0 ** -24, "bf16": 2.0 ** -8, "fp16": 2.0 ** -11}[ty]
    least = 0.0
    if ty != "fp32":
        least = 2.0 ** -38 * float(((g.abs() if grad else 0) + (22 * q.abs() if q is not None else 0)).max())
    lo, hi = off[0], off[-1]
    W, H = ref.W, ref.H
    want = dz @ W
    bound = (e + first * dz.abs() + least * 2) @ W.abs() + (vocab + 40) * EPS * (dz.abs() @ W.abs())
    bound = bound * 1.01 + half_step(dtype) * (want.abs() + bound) + smallest_half(dtype)
    inside(dh[lo:hi], want[lo:hi], bound[lo:hi], "dh")
    assert (dh[:lo] == 5).all() and (dh[hi:] == 5).all()
    for i in range(m):
        part = slice(off[i], off[i + 1])
        tokens = off[i + 1] - off[i]
        d, de = dz[part], e[part] + planes * dz[part].abs() + least
        want = d.t() @ H[part]
        inexact = 2.0 ** -39 * H.abs().amax(0) if ty == "bf16" and rows else 0.0   # hidden states in fp16, columns scaled
        bound = de.t() @ H[part].abs() + d.abs().sum(0)[:, None] * inexact + (2 * tokens + 12) * EPS * (d.abs().t() @ H[part].abs())
        inside(G[i, :n].view(vocab, width), want, bound * 1.01 + EPS * want.abs() + 2.0 ** -120, f"dweight {i}")
        inside(G[i, n:], d.sum(0), (de.sum(0) + (3 * tokens + 16) * EPS * d.abs().sum(0)) * 1.01 + 2.0 ** -120, f"dbias {i}")
    assert torch.equal(before.isnan(), around(G, buf).isnan()) and torch.equal(dh_before.isnan(), around(dh, dh_buf).isnan())
    # equal bits, outputs one at a time
    kw = dict(labels=labels if grad else None, grad_logp=g, entropy=entropy if entropy_too else None, grad_entropy=q, groups=groups)
    a, none, nothing = B.zeno_linear_logprobs_backward(h, w, b, stats, want_weight=False, want_bias=False, **kw)
    assert torch.equal(a[lo:hi], dh[lo:hi]) and (a[:lo] == 0).all() and none is None and nothing is None
    _, a, _ = B.zeno_linear_logprobs_backward(h, w, b, stats, want_hidden=False, want_bias=False, **kw)
    assert torch.equal(a, G[:, :n])
    _, _, a = B.zeno_linear_logprobs_backward(h, w, b, stats, want_hidden=False, want_weight=False, **kw)
    assert torch.equal(a, G[:, n:])


BACK = [
    (1, 1, 1, None, 0, 0, 0), (1, 3, 2, [0, 1], 1, 0, 1), (4, 7, 8, [0, 2, 2, 4], 0, 0, 0), (9, 40, 16, [1, 3, 8], 0, 0, 0),
    (40, 130, 33, [0, 1, 39, 40], 0, 1, 0), (130, 129, 64, None, 0, 0, 0), (100, 1000, 72, [0, 50, 100], 0, 0, 0), (257, 300, 136, [5, 70, 200, 250], 8, 8, 0),
    (33, 2500, 24, [0, 33], 0, 0, 0), (300, 17, 300, [0, 150, 300], 3, 2, 1), (700, 64, 8, None, 0, 0, 0),
]


@pytest.mark.parametrize("ty", TYPES)
@pytest.mark.parametrize("rows,vocab,width,offsets,pad_h,pad_w,offset", BACK)
def test_backward(B, rows, vocab, width, offsets, pad_h, pad_w, offset, ty):
    backward(B, rows, vocab, width, ty, offsets, rows % 2 == 0, pad_h=pad_h, pad_w=pad_w, offset=offset, masked=0.3 if vocab > 100 else 0.0)


@pytest.mark.parametrize("ty", TYPES)
def test_backward_of_the_entropy_alone(B, ty):
    backward(B, 50, 90, 24, ty, [0, 20, 50], True, grad=False)


@pytest.mark.parametrize("ty", TYPES)
@pytest.mark.parametrize("rows,vocab,width,offsets", [
    (2000, 6400, 512, [0, 500, 900, 1500, 1990]),       # wide tiles of logits and of weights
    (8200, 500, 1544, [0, 8200]),                       # wide tiles of hidden states
    (40000, 4000, 16, [0, 20000, 39999]),               # the vocabulary in pieces
])
def test_backward_large(B, rows, vocab, width, offsets, ty):
    backward(B, rows, vocab, width, ty, offsets, False, seed=3)


@pytest.mark.parametrize("ty", TYPES)
@pytest.mark.parametrize("rows,vocab,width,pad", [(70000, 300, 8, 0), (2050, 6500, 200, 0), (2, 33000, 2047, 0), (300, 40000, 1720, 1)])
def test_forward_large(B, rows, vocab, width, pad, ty):
    """Tokens in blocks, wide tiles, weights packed in pieces."""
    h, w, b, labels = problem(rows, vocab, width, TYPES[ty], 5, 0, pad, 0)
    ref = Reference(h, w, b, labels)
    logp, entropy, _ = B.zeno_linear_logprobs(h, w, b, labels, want_entropy=True)
    inside(logp, ref.logp, ref.e_logp, "logp")
    inside(entropy, ref.entropy, ref.e_ent, "entropy")


@pytest.mark.parametrize("ty", TYPES)
@pytest.mark.parametrize("rows", [5, 300])
def test_tokens_without_a_distribution(B, rows, ty):
    """Masks that leave nothing, masks of the lowest values, infinities and NaN."""
    vocab, width = 300, 40
    h, w, b, labels = problem(rows, vocab, width, TYPES[ty], 2, bias=False)
    nothing = torch.full((vocab,), float("-inf"), device="cuda")
    g = torch.full((rows,), -1.0 / rows, device="cuda")
    labels[:] = 7
    labels[1], labels[2] = -1, vocab
    logp, entropy, stats = B.zeno_linear_logprobs(h, w, nothing, labels, want_entropy=True, want_stats=True)
    assert logp[1] == 0 and logp[2].isnan() and (logp[3:] == -float("inf")).all() and logp[0] == -float("inf")
    assert (entropy == 0).all() and (stats[:, 0] == -float("inf")).all() and (stats[:, 1] == 0).all()
    labels[2] = 7
    grads = B.zeno_linear_logprobs_backward(h, w, nothing, stats, labels=labels, grad_logp=g, entropy=entropy, grad_entropy=g)
    assert all((x == 0).all() for x in grads)
    # the lowest finite values do what -inf does, in any number
    for low in (-1e30, torch.finfo(torch.float32).min):
        few = torch.full((vocab,), float(low), device="cuda")
        few[5] = few[7] = 0.0
        gone = few.clone()
        gone[few < 0] = float("-inf")
        a = B.zeno_linear_logprobs(h, w, few, labels, want_entropy=True, want_stats=True)
        c = B.zeno_linear_logprobs(h, w, gone, labels, want_entropy=True, want_stats=True)
        assert all(torch.equal(x, y) for x, y in zip(a, c))
        x = B.zeno_linear_logprobs_backward(h, w, few, a[2], labels=labels, grad_logp=g, entropy=a[1], grad_entropy=g)
        y = B.zeno_linear_logprobs_backward(h, w, gone, c[2], labels=labels, grad_logp=g, entropy=c[1], grad_entropy=g)
        assert all(torch.equal(i, j) for i, j in zip(x, y)) and all(i.isfinite().all() for i in x)
    # a NaN or an infinity among the tokens' states stays in their rows
    clean = B.zeno_linear_logprobs(h, w, None, labels, want_entropy=True, want_stats=True)
    bad = h.clone()
    bad[0, 3] = float("nan")
    bad[4, 0] = float("inf")
    logp, entropy, stats = B.zeno_linear_logprobs(bad, w, None, labels, want_entropy=True, want_stats=True)
    keep = torch.ones(rows, dtype=torch.bool, device="cuda")
    keep[[0, 4]] = False
    assert logp[0].isnan() and logp[4].isnan() and entropy[0].isnan() and entropy[4].isnan()
    assert torch.equal(logp[keep], clean[0][keep]) and torch.equal(entropy[keep], clean[1][keep])
    groups = torch.tensor([0, 1, 4, 5, rows], dtype=torch.int32, device="cuda")
    dh, dw, db = B.zeno_linear_logprobs_backward(bad, w, None, stats, labels=labels, grad_logp=g, groups=groups)
    assert dh[0].isnan().all() and dh[4].isnan().all() and dh[keep].isfinite().all()
    assert db[0].isnan().all() and db[1].isfinite().all() and db[2].isnan().all() and dw[1].isfinite().all() and dw[3].isfinite().all() and db[3].isfinite().all()
    # a label that is none
    labels[2] = vocab + 5
    dh, dw, db = B.zeno_linear_logprobs_backward(h, w, None, clean[2], labels=labels, grad_logp=g, groups=groups)
    assert dh[2].isnan().all() and dh[:2].isfinite().all() and dh[3:].isfinite().all() and db[0].isfinite().all()


def test_gradients_against_differences(B):
    """f = sum(g logp) + sum(q entropy) in float32, moved in directions of its inputs: the central difference is off by the function's own
    bound over the step and by a third derivative's share, h^2 |f'''| / 6 with |f'''| <= 8 (sum |g| + |q|) |dz|^3 for moves of logits |dz|."""
    rows, vocab, width = 24, 50, 20
    h, w, b, labels = problem(rows, vocab, width, torch.float32, 11, spread=1.0)
    gen = torch.Generator(device="cuda").manual_seed(3)
    g = -torch.rand(rows, generator=gen, device="cuda")
    q = 0.2 * torch.rand(rows, generator=gen, device="cuda")
    _, entropy, stats = B.zeno_linear_logprobs(h, w, b, labels, want_entropy=True, want_stats=True)
    grads = B.zeno_linear_logprobs_backward(h, w, b, stats, labels=labels, grad_logp=g, entropy=entropy, grad_entropy=q)

    def f(h, w, b):
        logp, entropy, _ = B.zeno_linear_logprobs(h, w, b, labels, want_entropy=True)
        ref = Reference(h, w, b, labels)
        error = (g.double().abs() * ref.e_logp + q.double().abs() * ref.e_ent).sum()
        return float((g.double() * logp.double()).sum() + (q.double() * entropy.double()).sum()), float(error)

    step = 2.0 ** -6
    for which, grad in enumerate((grads[0], grads[1].view(vocab, width), grads[2][0])):
        for seed in range(3):
            inputs = [h, w, b]
            u = torch.randn(inputs[which].shape, generator=gen, device="cuda")
            u = u / u.abs().max() * (0.2 if which == 1 else 1.0)
            up, down = list(inputs), list(inputs)
            up[which], down[which] = inputs[which] + step * u, inputs[which] - step * u
            (a, ea), (c, ec) = f(*up), f(*down)
            side = u.double().abs()
            dz = float((side @ w.double().abs().t() if which == 0 else h.double().abs() @ side.t() if which == 1 else side).max())
            # (inputs are rounded when they are moved: EPS of them, through the gradient)
            moved = float((grad.double().abs() * inputs[which].double().abs()).sum()) * 2 * EPS
            bound = (ea + ec + moved) / (2 * step) + step ** 2 / 6 * 8 * float((g.abs() + q.abs() * 5).sum()) * dz ** 3
            got = float((grad.double() * u.double()).sum())
            assert abs((a - c) / (2 * step) - got) <= bound + 1e-5 * abs(got), (which, (a - c) / (2 * step), got, bound)


@pytest.mark.parametrize("ty", TYPES)
def test_in_place(B, ty):
    h, w, b, labels = problem(100, 200, 48, TYPES[ty], 4)
    g = torch.full((100,), -0.01, device="cuda")
    _, _, stats = B.zeno_linear_logprobs(h, w, b, labels, want_stats=True)
    dh, dw, db = B.zeno_linear_logprobs_backward(h, w, b, stats, labels=labels, grad_logp=g)
    mine = h.clone()
    out, dw2, db2 = B.zeno_linear_logprobs_backward(mine, w, b, stats, labels=labels, grad_logp=g, dhidden=mine)
    assert out is mine and torch.equal(mine, dh) and torch.equal(dw, dw2) and torch.equal(db, db2)


def test_without_rows(B):
    h, w = torch.empty(0, 24, device="cuda"), torch.randn(30, 24, device="cuda")
    i32 = dict(dtype=torch.int32, device="cuda")
    logp, entropy, stats = B.zeno_linear_logprobs(h, w, None, torch.empty(0, **i32), want_entropy=True, want_stats=True)
    assert logp.numel() == entropy.numel() == stats.numel() == 0
    dh, dw, db = B.zeno_linear_logprobs_backward(h, w, None, stats, labels=torch.empty(0, **i32), grad_logp=logp, groups=torch.zeros(4, **i32),
                                                 dweight=torch.full((3, 720), 9.0, device="cuda"), dbias=torch.full((3, 30), 9.0, device="cuda"))
    assert dh.shape == (0, 24) and (dw == 0).all() and (db == 0).all()


def test_broken_offsets_stay_inside(B):
    h, w, b, labels = problem(90, 70, 24, torch.bfloat16, 6)
    g = torch.full((90,), -0.1, device="cuda")
    _, _, stats = B.zeno_linear_logprobs(h, w, b, labels, want_stats=True)
    n = 70 * 24
    G, buf = strided(torch.zeros(3, n + 70), torch.float32, n + 100, 9)
    before = around(G, buf)
    for bad in ([5, 3, 2, 90], [-4, 10, 1 << 30, 20], [1 << 30, 1 << 30, -1, 7]):
        B.zeno_linear_logprobs_backward(h, w, b, stats, labels=labels, grad_logp=g, groups=torch.tensor(bad, dtype=torch.int32, device="cuda"),
                                        dweight=G[:, :n], dbias=G[:, n:])
    torch.cuda.synchronize()
    assert torch.equal(before.isnan(), around(G, buf).isnan())


@pytest.mark.parametrize("ty", TYPES)
def test_captured(B, ty):
    """Both passes captured, with a workspace each, replayed with other inputs and eager work between the replays."""
    rows, vocab, width = 150, 500, 64
    h, w, b, labels = problem(rows, vocab, width, TYPES[ty], 8)
    g = torch.full((rows,), -0.1, device="cuda")
    groups = torch.tensor([0, 60, 150], dtype=torch.int32, device="cuda")
    out = [torch.empty(rows, device="cuda"), torch.empty(rows, 2, device="cuda"), torch.empty_like(h), torch.empty(2, vocab * width, device="cuda"),
           torch.empty(2, vocab, device="cuda")]
    ws = B.alloc_linear_logprobs_workspace(rows, vocab, width, h.dtype), B.alloc_linear_logprobs_backward_workspace(rows, vocab, width, h.dtype, 2)

    def call(out, ws):
        B.zeno_linear_logprobs(h, w, b, labels, logp=out[0], stats=out[1], workspace=ws[0])
        B.zeno_linear_logprobs_backward(h, w, b, out[1], labels=labels, grad_logp=g, groups=groups, dhidden=out[2], dweight=out[3], dbias=out[4],
                                        workspace=ws[1])

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        call(out, ws)
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call(out, ws)
    for i in range(4):
        h.normal_()
        g.uniform_(-1, 0)
        for t in out:
            t.fill_(float("nan"))
        graph.replay()
        torch.cuda.synchronize()
        eager = [torch.full_like(t, float("nan")) for t in out]
        call(eager, [torch.empty_like(x) for x in ws])
        assert all(torch.equal(x, y) for x, y in zip(out, eager))


@pytest.mark.parametrize("ty", TYPES)
@pytest.mark.parametrize("rows,vocab,width", [(40, 300, 64), (600, 700, 136)])
def test_one_groups_values_do_not_show_in_anothers_gradients(B, rows, vocab, width, ty):
    """Bit for bit, however large the gradients and hidden states of another group, or of rows that belong to nobody, are."""
    h, w, b, labels = problem(rows, vocab, width, TYPES[ty], 5)
    offsets = [3, rows // 3, rows // 3, rows // 2 + 1, rows - 4]
    off = torch.tensor(offsets, dtype=torch.int32, device="cuda")
    g = torch.randn(rows, device="cuda")
    q = torch.randn(rows, device="cuda")

    def gradients(h, g, q):
        _, entropy, stats = B.zeno_linear_logprobs(h, w, b, labels, want_entropy=True, want_stats=True)
        G = torch.full((4, vocab * width + vocab), 3.0, device="cuda")
        dh = torch.full_like(h, 5.0)
        B.zeno_linear_logprobs_backward(h, w, b, stats, labels=labels, grad_logp=g, entropy=entropy, grad_entropy=q, groups=off, dhidden=dh,
                                        dweight=G[:, :vocab * width], dbias=G[:, vocab * width:])
        return G, dh
    G, dh = gradients(h, g, q)
    other = torch.ones(rows, dtype=torch.bool, device="cuda")
    other[offsets[2]:offsets[3]] = False
    for factor, gradient in ((2.0 ** 10, 2.0 ** 40), (1.0, float("inf")), (float("nan"), float("nan"))):
        h2, g2, q2 = h.clone(), g.clone(), q.clone()
        h2[other] *= factor
        g2[other] *= gradient
        q2[other] *= gradient
        G2, dh2 = gradients(h2, g2, q2)
        assert torch.equal(G2[2], G[2]), (factor, gradient)
        assert torch.equal(dh2[~other], dh[~other]), (factor, gradient)
        assert (G2[1] == 0).all() and torch.equal(dh2[:3], dh[:3]) and torch.equal(dh2[-4:], dh[-4:])


@pytest.mark.parametrize("ty", TYPES)
@pytest.mark.parametrize("rows,vocab,width,offsets", [
    (1024, 3, 5, None), (14000, 11, 19, None), (5000, 140, 130, [0, 3, 3, 4990]), (3100, 200, 33, [40, 1600, 3100]), (40000, 3500, 2, None),
])
def test_weight_gradients_of_many_tokens_and_few_weights(B, rows, vocab, width, offsets, ty):
    """A group's tokens in parts, more of them than it has tokens too."""
    backward(B, rows, vocab, width, ty, offsets, True, seed=9)
