"""The operators at both ends of a model together, as an iteration of Algorithm 1 uses them: tokens in, workers' gradients into rows of G, scores,
selection and update; streams and graphs."""
import numpy as np
import pytest
import torch

from tests import _tokens as T

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def B():
    from paper_1805_10032_amd import binding
    binding.load_library()
    return binding


def setup(widths, inputs, tokens, m, dtype, seed=0, **kw):
    from paper_1805_10032_amd.token_model import TokenModel
    model = TokenModel(widths, dtype, inputs=inputs, keep_logits=False, **kw)
    g = torch.Generator().manual_seed(seed)
    x = model.init(seed)
    x += 0.05 * torch.randn(model.num_params, generator=g).cuda()
    ids = torch.randint(0, inputs, (tokens,), generator=g, dtype=torch.int32)
    ids[5] = -1
    labels = torch.randint(0, widths[-1], (tokens,), generator=g, dtype=torch.int32)
    labels[::7] = -1
    off = sorted(torch.randint(0, tokens - 2, (m - 2,), generator=g).tolist())
    off = [1, 1, *off, tokens - 2]                      # a worker without tokens, tokens of nobody
    return model, x, ids.cuda(), labels.cuda(), torch.tensor(off, dtype=torch.int32, device="cuda"), off


@pytest.mark.parametrize("tied", [False, True])
@pytest.mark.parametrize("width,vocab,tokens", [(24, 40, 150), (72, 300, 400), (33, 129, 90)])
def test_gradients_in_float32(B, width, vocab, tokens, tied):
    """Lookup, norm and last layer against the formulas in float64, with the norm's input as its checkpoint holds it in its place of the
    backward pass (that is the operator's definition).  Every value passes through four sums of at most `longest` terms (width, vocabulary, tokens) in
    float32, each off by longest EPS of its terms' magnitudes, which are carried along."""
    m = 4
    model, x, ids, labels, groups, off = setup([width, vocab], vocab, tokens, m, torch.float32, tied=tied)
    wide = torch.full((m, model.num_params + 3), 9.0, device="cuda")
    G = wide[:, 1:1 + model.num_params]
    logp = model.gradients(x, ids, labels, groups, G)
    torch.cuda.synchronize()
    assert (wide[:, 0] == 9).all() and (wide[:, 1 + model.num_params:] == 9).all()
    X, y, i = x.double().cpu().numpy(), labels.cpu().numpy(), ids.cpu().numpy()
    E = X[:vocab * width].reshape(vocab, width)
    nw, nb, w, b = [X[at:at + n] for at, n in model.offsets[0]]
    W = w.reshape(vocab, width)
    s = np.float64(np.float32(model.scale))
    h = np.where((i >= 0)[:, None], E[np.maximum(i, 0)] * s, 0.0)
    out, mean, rstd, _ = T.layer_norm(h, nw, nb, model.eps)
    z = out @ W.T + b
    lp = z - z.max(1, keepdims=True)
    lp -= np.log(np.exp(lp).sum(1, keepdims=True))
    p = np.exp(lp)
    longest = max(width, vocab, tokens) + 64
    unit = longest * T.EPS
    size_z = np.abs(out) @ np.abs(W).T + np.abs(b)
    # (rstd of the row of zeros is 1 / sqrt(eps); its errors are relative like the others')
    e_z = 4 * unit * size_z
    got_lp = logp.double().cpu().numpy()
    want_lp = np.where(y >= 0, lp[np.arange(tokens), np.maximum(y, 0)], 0.0)
    assert (np.abs(got_lp - want_lp) <= 2 * e_z.max(1) + 40 * T.EPS * (np.abs(lp).max(1) + np.abs(z).max(1))).all()
    h32 = np.float32(h).astype(np.float64)
    kept = T.checkpoint_values(*T.checkpoint(h32), width)
    G64 = G.double().cpu().numpy()
    for g in range(m):
        rows = np.arange(off[g], off[g + 1])
        n = max(1, (y[rows] >= 0).sum())
        one = np.zeros((len(rows), vocab))
        counted = y[rows] >= 0
        one[np.arange(len(rows))[counted], y[rows][counted]] = 1.0
        dz = (p[rows] - one) * counted[:, None] / n
        e_dz = (p[rows] * (2 * e_z[rows] + 2 * e_z[rows].max(1, keepdims=True) + 60 * T.EPS * (1 + np.abs(lp[rows]))) + 8 * T.EPS * one) * counted[:, None] / n
        dW, e_dW = dz.T @ out[rows], e_dz.T @ np.abs(out[rows]) + 4 * unit * (np.abs(dz).T @ np.abs(out[rows]))
        db, e_db = dz.sum(0), e_dz.sum(0) + 2 * unit * np.abs(dz).sum(0)
        dy = dz @ W
        e_dy = e_dz @ np.abs(W) + 2 * unit * (np.abs(dz) @ np.abs(W))
        xh = (kept[rows] - mean[rows][:, None]) * rstd[rows][:, None]
        a, e_a = dy * nw, e_dy * np.abs(nw) + 2 * T.EPS * np.abs(dy * nw)
        c1, c2 = a.mean(1, keepdims=True), (a * xh).mean(1, keepdims=True)
        dx = rstd[rows][:, None] * (a - c1 - xh * c2)
        size = np.abs(a) + np.abs(a).mean(1, keepdims=True) + np.abs(xh) * np.abs(a * xh).mean(1, keepdims=True)
        e_size = e_a + e_a.mean(1, keepdims=True) + np.abs(xh) * (e_a * np.abs(xh)).mean(1, keepdims=True)
        e_dx = rstd[rows][:, None] * (e_size + 6 * unit * size)
        dE, e_dE = np.zeros((vocab, width)), np.zeros((vocab, width))
        known = i[rows] >= 0
        np.add.at(dE, i[rows][known], s * dx[known])
        np.add.at(e_dE, i[rows][known], s * (e_dx[known] + unit * np.abs(dx[known])))
        got = {k: G64[g][at:at + n_] for k, (at, n_) in zip(("nw", "nb", "w", "b"), model.offsets[0])}
        table = G64[g][:vocab * width].reshape(vocab, width)
        want_dnw, e_dnw = (dy * xh).sum(0), (e_dy * np.abs(xh)).sum(0) + 6 * unit * np.abs(dy * xh).sum(0)
        checks = [(got["b"], db, e_db), (got["nw"], want_dnw, e_dnw), (got["nb"], dy.sum(0), e_dy.sum(0) + 2 * unit * np.abs(dy).sum(0))]
        if tied:
            checks.append((table, dE + dW, e_dE + e_dW + 2 * T.EPS * (np.abs(dE) + np.abs(dW))))
        else:
            checks += [(table, dE, e_dE), (got["w"].reshape(vocab, width), dW, e_dW)]
        for k, (have, want, e) in enumerate(checks):
            assert (np.abs(have - want) <= e * 1.1 + 1e-30).all(), (g, k, np.abs(have - want).max(), (np.abs(have - want) / (e + 1e-30)).max())


@pytest.mark.parametrize("dtype", T.TYPES)
def test_the_model_is_its_operators(B, dtype):
    """Two layers, in every type: the same calls by hand give the same bits."""
    ty = T.TYPES[dtype]
    model, x, ids, labels, groups, off = setup([40, 72, 90], 55, 200, 4, ty)
    G = torch.zeros(4, model.num_params, device="cuda")
    logp = model.gradients(x, ids, labels, groups, G)
    table, (first, last) = x[:55 * 40].view(55, 40), model._views(x)
    h0 = B.zeno_embedding(ids, table, ty, scale=model.scale)
    y0, mean0, rstd0, c0 = B.zeno_layer_norm(h0, first[0], first[1], model.eps, want_checkpoint=True)
    w0 = first[2].view(72, 40).to(ty)
    h1 = torch.addmm(first[3].to(ty), y0, w0.t())
    y1, mean1, rstd1, c1 = B.zeno_layer_norm(h1, last[0], last[1], model.eps, want_checkpoint=True)
    w1 = last[2].view(90, 72).to(ty)
    mine, _, stats = B.zeno_linear_logprobs(y1, w1, last[3], labels, want_stats=True)
    assert torch.equal(mine, logp)
    n = [max(1, int((labels[p:q] >= 0).sum())) for p, q in zip(off, off[1:])]
    worker = [min(3, sum(t >= q for q in off[1:])) for t in range(200)]
    grad = torch.full((200,), -model.loss_scale, device="cuda") if dtype == "fp16" else torch.tensor([-1.0 / n[g] for g in worker], device="cuda")
    dy, dw1, db1 = B.zeno_linear_logprobs_backward(y1, w1, last[3], stats, labels=labels, grad_logp=grad, groups=groups)
    d1, dnw1, dnb1 = B.zeno_layer_norm_backward(dy, c1, mean1, rstd1, last[0], groups=groups)
    # (rows of nobody: the model's norm writes in place and leaves what it found)
    d1[:off[0]], d1[off[-1]:] = dy[:off[0]], dy[off[-1]:]
    dw0, db0 = B.zeno_weight_gradient(d1, B.zeno_checkpoint(y0), groups=groups)
    dy0 = torch.mm(d1, w0)
    d0, dnw0, dnb0 = B.zeno_layer_norm_backward(dy0, c0, mean0, rstd0, first[0], groups=groups)
    dE = B.zeno_embedding_backward(d0, ids, 55, scale=model.scale, groups=groups)
    want = torch.cat([dE, dnw0, dnb0, dw0, db0, dnw1, dnb1, dw1, db1], 1)
    if dtype == "fp16":
        want *= (1.0 / (model.loss_scale * torch.tensor(n, device="cuda"))).float()[:, None]
    assert torch.equal(want, G)


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
def test_a_tied_table_has_both_gradients(B, dtype):
    """The gradient of a tied table is the sum of what it would be as two blocks, rounded once more."""
    ty, vocab, width = T.TYPES[dtype], 70, 24
    both, x2, ids, labels, groups, off = setup([width, vocab], vocab, 120, 4, ty)
    from paper_1805_10032_amd.token_model import TokenModel
    tied = TokenModel([width, vocab], ty, inputs=vocab, tied=True, keep_logits=False)
    n = vocab * width
    at = both.offsets[0][2][0]
    x2[at:at + n] = x2[:n]
    x1 = torch.cat([x2[:n + 2 * width], x2[at + n:]])
    assert x1.numel() == tied.num_params
    G2, G1 = torch.zeros(4, both.num_params, device="cuda"), torch.zeros(4, tied.num_params, device="cuda")
    assert torch.equal(both.gradients(x2, ids, labels, groups, G2), tied.gradients(x1, ids, labels, groups, G1))
    assert torch.equal(G1[:, :n], G2[:, :n] + G2[:, at:at + n])
    assert torch.equal(G1[:, n:n + 2 * width], G2[:, n:n + 2 * width]) and torch.equal(G1[:, n + 2 * width:], G2[:, at + n:])


def test_an_iteration(B):
    """Gradients, scores, selection and update of a model that takes tokens and keeps no logits."""
    gamma, rho, b = 0.1, 1e-3, 1
    model, x, ids, labels, groups, off = setup([24, 60], 80, 150, 5, torch.float32)
    G = torch.zeros(5, model.num_params, device="cuda")
    model.gradients(x, ids, labels, groups, G)
    G[3] *= -4.0
    s = model.scores(x, G, ids, labels, gamma, rho)
    counted = (labels >= 0)
    want = []
    for i in range(5):
        gain = (model.logprobs(x - gamma * G[i], ids, labels).double() - model.logprobs(x, ids, labels).double())[counted].mean()
        want.append(float(gain - rho * (G[i].double() ** 2).sum()))
    want = np.array(want)
    # (x - gamma G is formed by one rounding here and in scores(): torch.add's alpha; logits move by EPS of x through `width` terms)
    tol = 1e-5
    assert np.abs(s.double().cpu().numpy() - want).max() <= tol * (1 + np.abs(want).max())
    x_next, _, sel = B.zeno_aggregate_update(G, s, b, gamma, x)
    assert 3 not in sel.tolist()
    mean = G[sel.long()].double().mean(0)
    assert (x_next.double() - (x.double() - gamma * mean)).abs().max() <= 2 * T.EPS * float(x.abs().max() + gamma * mean.abs().max())


def test_two_streams(B):
    """Calls that overlap in time, each with its workspace."""
    torch.manual_seed(0)
    inputs = []
    for k, rows in enumerate((700, 300)):
        h, w = torch.randn(rows, 128, device="cuda").bfloat16(), (torch.randn(3000, 128, device="cuda") * 0.1).bfloat16()
        labels = torch.randint(0, 3000, (rows,), device="cuda", dtype=torch.int32)
        inputs.append((h, w, labels, torch.full((rows,), -1.0 / rows, device="cuda")))

    def call(h, w, labels, g):
        logp, _, stats = B.zeno_linear_logprobs(h, w, None, labels, want_stats=True)
        dh, dw, db = B.zeno_linear_logprobs_backward(h, w, None, stats, labels=labels, grad_logp=g)
        return logp, dh, dw, db, B.zeno_embedding_backward(dh, labels, 3000, dtable=dw, accumulate=True)

    alone = [[t.clone() for t in call(*i)] for i in inputs]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    for _ in range(5):
        got = []
        for st, i in zip(streams, inputs):
            with torch.cuda.stream(st):
                got.append(call(*i))
        torch.cuda.synchronize()
        for a, c in zip(alone, got):
            assert all(torch.equal(x, y) for x, y in zip(a, c))


def test_two_graphs(B):
    """Two captured iterations, each with the workspaces of its own pool, replayed in turn with eager work between."""
    torch.manual_seed(1)
    rows, vocab, width = 260, 900, 64
    sets = []
    for k in range(2):
        ids = torch.randint(0, vocab, (rows,), device="cuda", dtype=torch.int32)
        table = torch.randn(vocab, width, device="cuda") * 0.1
        sets.append(dict(ids=ids, labels=ids.roll(1).contiguous(), table=table, g=torch.full((rows,), -1.0 / rows, device="cuda")))

    def call(s):
        h = B.zeno_embedding(s["ids"], s["table"], torch.bfloat16, scale=8.0)
        w = s["table"].bfloat16()
        logp, _, stats = B.zeno_linear_logprobs(h, w, None, s["labels"], want_stats=True)
        dh, dw, _ = B.zeno_linear_logprobs_backward(h, w, None, stats, labels=s["labels"], grad_logp=s["g"], want_bias=False)
        return logp, B.zeno_embedding_backward(dh, s["ids"], vocab, scale=8.0, dtable=dw, accumulate=True)

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        for s in sets:
            call(s)
    torch.cuda.current_stream().wait_stream(side)
    graphs, outs = [], []
    for s in sets:
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            outs.append(call(s))
        graphs.append(graph)
    for i in range(4):
        for s in sets:
            s["table"].normal_(std=0.1)
            s["ids"].random_(0, vocab)
        for graph in graphs:
            graph.replay()
        torch.cuda.synchronize()
        for s, out in zip(sets, outs):
            eager = call(s)
            torch.cuda.synchronize()
            assert all(torch.equal(x, y) for x, y in zip(out, eager))
