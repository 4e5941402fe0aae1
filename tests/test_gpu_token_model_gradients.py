"""The gradients of TokenModel, operator by operator: each is compared in float64 with what its own inputs give, so that no bound has to
cover the layers before it, and every block of G with the sums that belong there."""
import numpy as np
import pytest
import torch

from tests import _tokens as T
from tests.test_gpu_token_model import setup

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def B():
    from paper_1805_10032_amd import binding
    binding.load_library()
    return binding


def numbers(t):
    return t.double().cpu().numpy()


class Recorded:
    """What the operators were called with and gave during one call of TokenModel.gradients, the last layer first."""

    def __init__(self, monkeypatch, B):
        self.weight, self.norm, self.loss = [], [], []
        weight, norm, loss = B.zeno_weight_gradient, B.zeno_layer_norm_backward, B.zeno_logprobs_backward

        def zeno_logprobs_backward(logits, stats, **kw):
            z = logits.clone()
            out = loss(logits, stats, **kw)
            self.loss.append((z, kw["grad_logp"].clone(), out.clone()))
            return out

        def zeno_weight_gradient(dy, ckpt, **kw):
            self.weight.append((dy.clone(), B.zeno_checkpoint_values(ckpt)))
            return weight(dy, ckpt, **kw)

        def zeno_layer_norm_backward(dy, x, mean, rstd, scale, **kw):
            before = dy.clone()
            out = norm(dy, x, mean, rstd, scale, **kw)
            self.norm.append((before, B.zeno_checkpoint_values(x), mean.clone(), rstd.clone(), None if out[0] is None else out[0].clone()))
            return out

        monkeypatch.setattr(B, "zeno_logprobs_backward", zeno_logprobs_backward)
        monkeypatch.setattr(B, "zeno_weight_gradient", zeno_weight_gradient)
        monkeypatch.setattr(B, "zeno_layer_norm_backward", zeno_layer_norm_backward)


def inside(got, want, tol, what):
    err = np.abs(got - want)
    assert (err <= tol).all(), (what, np.argwhere(~(err <= tol))[:4].tolist(), err.max())
    # the bound means something: zeros do not pass it
    assert not (np.abs(want) <= tol).all(), what


@pytest.mark.parametrize("dtype", list(T.TYPES.values()))
@pytest.mark.parametrize("widths", [[24, 11], [40, 33, 70], [64, 130, 96, 300]])
def test_every_block_of_G(B, monkeypatch, widths, dtype):
    tokens, m = 150, 5
    model, x, hidden, labels, off = setup(widths, tokens, m, dtype)
    groups = torch.tensor(off, dtype=torch.int32, device="cuda")
    G = torch.full((m, model.num_params), 9.0, device="cuda")
    seen = Recorded(monkeypatch, B)
    model.gradients(x, hidden, labels, groups, G)
    torch.cuda.synchronize()
    half, small, layers = T.half_step(dtype), T.smallest_half(dtype), len(widths) - 1
    lab, G, x = labels.cpu().numpy(), numbers(G), numbers(x)
    lo, hi = off[0], off[-1]
    counted = [max(1, int((lab[p:q] >= 0).sum())) for p, q in zip(off, off[1:])]
    # fp16 keeps the tokens' gradients loss_scale times as large as those of their own loss; otherwise they are those of the mean
    unit = np.array([model.loss_scale * n if dtype == torch.float16 else 1.0 for n in counted])
    per_token = np.zeros(tokens)
    for (p, q), n, u in zip(zip(off, off[1:]), counted, unit):
        per_token[p:q] = u / n
    # the loss: p and 1 - p come from float32 statistics of at most 300 values and exponentials, 64 roundings in all
    z, g, dz = (numbers(t) for t in seen.loss[0])
    assert np.abs(g + per_token)[lo:hi].max() <= 2 * T.EPS * per_token.max()
    e = np.exp(z - z.max(1, keepdims=True))
    prob = e / e.sum(1, keepdims=True)
    want = prob.copy()
    want[np.arange(tokens), np.maximum(lab, 0)] -= 1
    want *= ((lab >= 0) * per_token)[:, None]
    mag = (prob + (want < 0)) * per_token[:, None]
    inside(dz[lo:hi], want[lo:hi], (64 * T.EPS * mag + half * np.abs(want) * (1 + 2 ** -6) + small)[lo:hi], "dlogits")
    for layer in reversed(range(layers)):
        width, out = widths[layer], widths[layer + 1]
        blocks = [(at, n) for at, n in model.offsets[layer]]
        dz, y = (numbers(t) for t in seen.weight[layers - 1 - layer])
        dy, h, mean, rstd, dx = [None if t is None else numbers(t) for t in seen.norm[layers - 1 - layer]]
        nw, nb, w, b = [G[:, at:at + n] for at, n in blocks]
        if layer < layers - 1:
            assert np.array_equal(dz[lo:hi], below[lo:hi])
        # the product with the weights is the library's: a float32 sum of `out` terms, at most as many roundings of the sum of |terms|, and
        # its partial sums may be rounded to the type as well as the result
        wt = numbers(torch.tensor(x[blocks[2][0]:sum(blocks[2])]).float().view(out, width).to(dtype))
        inside(dy[lo:hi], (dz @ wt)[lo:hi], ((4 * half + out * T.EPS) * (np.abs(dz) @ np.abs(wt)) + small)[lo:hi], ("dy", layer))
        xh = (h - mean[:, None]) * rstd[:, None]
        scale = x[blocks[0][0]:sum(blocks[0])]
        for i, (p, q) in enumerate(zip(off, off[1:])):
            # sums of q - p terms in float32 (three exact pieces a term at most), xh and the division by `unit` included
            k = (3 * (q - p) + 24) * 2 * T.EPS
            sums = [(nw, (dy[p:q] * xh[p:q]).sum(0), np.abs(dy[p:q] * xh[p:q]).sum(0)), (nb, dy[p:q].sum(0), np.abs(dy[p:q]).sum(0)),
                    (w, (dz[p:q].T @ y[p:q]).ravel(), (np.abs(dz[p:q]).T @ np.abs(y[p:q])).ravel()),
                    (b, dz[p:q].sum(0), np.abs(dz[p:q]).sum(0))]
            for name, (got, sum_, mag) in zip(("norm weight", "norm bias", "weight", "bias"), sums):
                if p == q or not (lab[p:q] >= 0).any():
                    assert not got[i].any()
                else:
                    inside(got[i] * unit[i], sum_, k * mag + 1e-30, (name, layer, i))
        if layer == 0:
            assert dx is None
            continue
        a = dy * scale
        c1, c2 = a.mean(1, keepdims=True), (a * xh).mean(1, keepdims=True)
        k = width + 24
        tol = rstd[:, None] * ((k * T.EPS) * (np.abs(a).mean(1, keepdims=True) + np.abs(xh) * np.abs(a * xh).mean(1, keepdims=True))
                               + 5 * T.EPS * (np.abs(a) + np.abs(c1) + np.abs(xh * c2)))
        want = rstd[:, None] * (a - c1 - xh * c2)
        tol = tol + (np.abs(want) + tol) * half + small
        inside(dx[lo:hi], want[lo:hi], tol[lo:hi], ("dx", layer))
        for wrong in (want + rstd[:, None] * c1, want + rstd[:, None] * xh * c2):      # a term left out would be noticed
            assert not (np.abs(dx - wrong) <= tol)[lo:hi].all()
        below = dx


@pytest.mark.parametrize("dtype", list(T.TYPES.values()))
def test_a_large_vocabulary_and_many_tokens(B, dtype):
    """Probabilities over the number of tokens are far below fp16's smallest value: what the tokens push down has to stay in the
    gradient.  The last layer's blocks against float64 sums from the model's own logits."""
    width, vocab, tokens, m = 48, 32000, 6000, 2
    model, x, hidden, labels, _ = setup([width, vocab], tokens, m, dtype, seed=9)
    off = [0, 2500, tokens]
    G = torch.empty(m, model.num_params, device="cuda")
    logits, kept = model.forward(x, hidden, keep=True)
    y = B.zeno_checkpoint_values(kept[0][3]).double()
    model.gradients(x, hidden, labels, torch.tensor(off, dtype=torch.int32, device="cuda"), G)
    half = T.half_step(dtype)
    # fp16 subnormals are 2^-24 apart; with a scale of 64 that is 2^-30 of a token's own loss
    floor = {torch.float16: 2.0 ** -31}.get(dtype, 2.0 ** -126)
    for i, (p, q) in enumerate(zip(off, off[1:])):
        keep = labels[p:q] >= 0
        n = int(keep.sum())
        dz = torch.softmax(logits[p:q].double(), 1)
        prob = dz.clone()
        dz[torch.arange(q - p, device="cuda"), labels[p:q].long().clamp(min=0)] -= 1
        prob[torch.arange(q - p, device="cuda"), labels[p:q].long().clamp(min=0)] += 1
        dz, prob = dz[keep] / n, prob[keep] / n
        # an entry: half a step, and 512 float32 roundings of the statistics (sums of 32000 values over 64 lanes or more)
        err = half * dz.abs() + 512 * T.EPS * prob + floor / n
        a = y[p:q][keep]
        sums = (3 * (q - p) + 24) * 2 * T.EPS
        at, size = model.offsets[0][2]
        got = G[i, at:at + size].view(vocab, width).double()
        want = dz.t().contiguous() @ a
        tol = err.t().contiguous() @ a.abs() + sums * (dz.abs().t().contiguous() @ a.abs())
        assert ((got - want).abs() <= tol).all(), ("weight", i, float(((got - want).abs() / tol).max()))
        at, size = model.offsets[0][3]
        got, want, tol = G[i, at:at + size].double(), dz.sum(0), err.sum(0) + sums * dz.abs().sum(0)
        assert ((got - want).abs() <= tol).all(), ("bias", i, float(((got - want).abs() / tol).max()))
        assert not (want.abs() <= tol).any()


def test_candidates_of_another_size_are_refused(B):
    """A single column would otherwise be added to every parameter."""
    model, x, hidden, labels, _ = setup([16, 9], 30, 2, torch.float32)
    for d in (1, model.num_params - 1):
        with pytest.raises(ValueError):
            model.scores(x, torch.zeros(3, d, device="cuda"), hidden, labels, 0.1, 1e-3)


@pytest.mark.parametrize("dtype", list(T.TYPES.values()))
def test_another_default_type(B, dtype):
    model, x, hidden, labels, off = setup([16, 9], 30, 2, dtype)
    groups = torch.tensor(off, dtype=torch.int32, device="cuda")
    G, again = torch.empty(2, model.num_params, device="cuda"), torch.empty(2, model.num_params, device="cuda")
    model.gradients(x, hidden, labels, groups, G)
    scores = model.scores(x, G, hidden, labels, 0.1, 1e-3)
    torch.set_default_dtype(torch.float64)
    try:
        model.gradients(x, hidden, labels, groups, again)
        assert torch.equal(G, again) and torch.equal(scores, model.scores(x, G, hidden, labels, 0.1, 1e-3))
    finally:
        torch.set_default_dtype(torch.float32)


@pytest.mark.parametrize("dtype", list(T.TYPES.values()))
def test_no_tokens(B, dtype):
    """A batch without tokens: every worker sends zeros; each output by itself is empty."""
    model, x, _, _, _ = setup([16, 9], 30, 2, dtype)
    hidden, labels = torch.empty(0, 16, dtype=dtype, device="cuda"), torch.empty(0, dtype=torch.int32, device="cuda")
    G = torch.full((3, model.num_params), 7.0, device="cuda")
    logp = model.gradients(x, hidden, labels, torch.zeros(4, dtype=torch.int32, device="cuda"), G)
    assert logp.shape == (0,) and not G.any()
    assert B.zeno_logprobs(hidden, labels)[0].shape == (0,)
    assert B.zeno_logprobs(hidden, want_entropy=True)[1].shape == (0,) and B.zeno_logprobs(hidden, want_stats=True)[2].shape == (0, 2)
    w = torch.ones(16, device="cuda")
    y, mean, rstd, ck = B.zeno_layer_norm(hidden, w, want_checkpoint=True)
    for src in (hidden, ck):
        dx, dw, db = B.zeno_layer_norm_backward(hidden, src, mean, rstd, w, want_weight=False, want_bias=False)
        assert dx.shape == (0, 16) and dw is None and db is None


@pytest.mark.parametrize("dtype", list(T.TYPES.values()))
def test_captured_and_replayed(B, dtype):
    """An iteration's gradients and scores in a graph, replayed on other tokens with eager work between."""
    n, m = 700, 5
    model, x, _, _, _ = setup([96, 160, 1000], 30, 2, dtype)
    hidden, labels = torch.randn(n, 96, device="cuda").to(dtype), torch.zeros(n, dtype=torch.int32, device="cuda")
    groups = torch.tensor([0, 100, 100, 300, 600, 690], dtype=torch.int32, device="cuda")
    G, out = torch.empty(m, model.num_params, device="cuda"), {}

    def run():
        out["logp"] = model.gradients(x, hidden, labels, groups, G)
        out["scores"] = model.scores(x, G, hidden[:64], labels[:64], 0.1, 1e-3)

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        run()
    torch.cuda.current_stream().wait_stream(side)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        run()
    captured = dict(out)
    gen = torch.Generator(device="cuda").manual_seed(4)
    for _ in range(4):
        hidden.copy_(torch.randn(n, 96, generator=gen, device="cuda"))
        labels.copy_(torch.randint(-1, 1000, (n,), generator=gen, device="cuda"))
        run()
        torch.cuda.synchronize()
        want = G.clone(), out["logp"].clone(), out["scores"].clone()
        G.fill_(float("nan"))
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(want, (G, captured["logp"], captured["scores"])))
        assert all(torch.isfinite(t).all() for t in want) and G[0].any() and not G[1].any()
