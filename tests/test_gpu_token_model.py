"""The operators together, as an iteration of Algorithm 1 uses them: workers' gradients into rows of G, scores, selection and update."""
import numpy as np
import pytest
import torch

from tests import _tokens as T
from tests._util import check_selection

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def B():
    from paper_1805_10032_amd import binding
    binding.load_library()
    return binding


def setup(widths, tokens, m, dtype, seed=0):
    from paper_1805_10032_amd.token_model import TokenModel
    model = TokenModel(widths, dtype)
    g = torch.Generator().manual_seed(seed)
    x = model.init(seed)
    x += 0.05 * torch.randn(model.num_params, generator=g).cuda()
    hidden = torch.randn(tokens, widths[0], generator=g).to(dtype).cuda()
    labels = torch.randint(0, widths[-1], (tokens,), generator=g, dtype=torch.int32)
    labels[::7] = -1
    cuts = sorted(torch.randint(0, tokens, (m - 1,), generator=g).tolist())
    off = [0, *cuts, tokens - 2]
    off[1] = off[0]                                     # a worker without tokens
    off = sorted(min(v, tokens - 2) for v in off)
    return model, x, hidden, labels.cuda(), off


def views(model, v):
    out = []
    for parts, width, o in zip(model.offsets, model.widths, model.widths[1:]):
        nw, nb, w, b = [v[at:at + n] for at, n in parts]
        out.append((nw, nb, w.reshape(o, width), b))
    return out


def forward64(model, x, hidden):
    h, saved = hidden, []
    for nw, nb, w, b in views(model, x):
        y, mean, rstd, xh = T.layer_norm(h, nw, nb, model.eps)
        saved.append((h, y, mean, rstd))
        h = y @ w.T + b
    return h, saved


def logp64(z, labels):
    M = z.max(1, keepdims=True)
    lp = z - M - np.log(np.exp(z - M).sum(1, keepdims=True))
    return np.where(labels >= 0, lp[np.arange(len(labels)), np.maximum(labels, 0)], 0.0), np.exp(lp)


@pytest.mark.parametrize("widths", [[24, 11], [40, 33, 70], [64, 130, 96, 300]])
def test_gradients_in_float32(B, widths):
    """All workers' gradients against the formulas in float64, with the activations that the checkpoints hold in their places of
    the backward pass (they are the operators' definition)."""
    tokens, m = 150, 5
    model, x, hidden, labels, off = setup(widths, tokens, m, torch.float32)
    groups = torch.tensor(off, dtype=torch.int32, device="cuda")
    wide = torch.full((m, model.num_params + 3), 9.0, device="cuda")
    G = wide[:, 1:1 + model.num_params]
    logp = model.gradients(x, hidden, labels, groups, G)
    _, kept = model.forward(x, hidden, keep=True)
    torch.cuda.synchronize()
    assert (wide[:, 0] == 9).all() and (wide[:, 1 + model.num_params:] == 9).all()
    x64, h64, lab = x.double().cpu().numpy(), hidden.double().cpu().numpy(), labels.cpu().numpy()
    z, saved = forward64(model, x64, h64)
    lp, p = logp64(z, lab)
    n_layers, widest = len(widths) - 1, max(widths)
    # a layer's output is off by (width + 16) EPS of the sum of |terms|; the errors of the layers before are passed on by factors of
    # about one.  Activations and logits here are below 8.
    act = n_layers * (widest + 32) * T.EPS * 8
    assert np.abs(logp.double().cpu().numpy() - lp).max() <= 4 * act
    got = G.double().cpu().numpy()
    want, mag = np.zeros_like(got), np.zeros_like(got)
    for i, (a, b) in enumerate(zip(off, off[1:])):
        n = max(1, int((lab[a:b] >= 0).sum()))
        dz = p[a:b].copy()
        dz[np.arange(b - a), np.maximum(lab[a:b], 0)] -= 1
        dz *= (lab[a:b] >= 0)[:, None] / n
        wv, mv = views(model, want[i]), views(model, mag[i])
        for layer in reversed(range(n_layers)):
            nw, nb, w, bias = views(model, x64)[layer]
            ckpt_h, mean, rstd, ckpt_y, _ = kept[layer]
            h_kept = B.zeno_checkpoint_values(ckpt_h).double().cpu().numpy()[a:b]
            y_kept = B.zeno_checkpoint_values(ckpt_y).double().cpu().numpy()[a:b]
            mu, r = mean.double().cpu().numpy()[a:b], rstd.double().cpu().numpy()[a:b]
            xh = (h_kept - mu[:, None]) * r[:, None]
            wv[layer][2][:] = dz.T @ y_kept
            wv[layer][3][:] = dz.sum(0)
            mv[layer][2][:] = np.abs(dz).T @ np.abs(y_kept)
            mv[layer][3][:] = np.abs(dz).sum(0)
            dy = dz @ w
            size = np.abs(dz) @ np.abs(w)
            wv[layer][0][:] = (dy * xh).sum(0)
            wv[layer][1][:] = dy.sum(0)
            mv[layer][0][:] = (size * np.abs(xh)).sum(0)
            mv[layer][1][:] = size.sum(0)
            t = dy * nw
            dz = r[:, None] * (t - t.mean(1, keepdims=True) - xh * (t * xh).mean(1, keepdims=True))
    # every factor of a term is off by about `act` of its size, the sums by (tokens + widest) EPS; norms and products multiply the sizes
    # of the terms by at most about 30 from layer to layer
    tol = (8 * act + (tokens + widest + 64) * 2 * T.EPS) * (mag + 30 * mag.max(1, keepdims=True) * (n_layers > 1)) + 1e-12
    assert (np.abs(got - want) <= tol).all(), np.abs(got - want).max()
    assert not got[0].any()


def test_gradients_against_differences(B):
    """The slope of the mean loss along the gradient, from central differences of the float64 definition: with 8-bit activations each
    term of the gradient is off by at most 2^-4 of itself, its activation's rounding, in every layer."""
    model, x, hidden, labels, _ = setup([24, 16, 40], 120, 1, torch.float32, seed=3)
    G = torch.empty(1, model.num_params, device="cuda")
    model.gradients(x, hidden, labels, torch.tensor([0, 120], dtype=torch.int32, device="cuda"), G)
    x64, h64, lab = x.double().cpu().numpy(), hidden.double().cpu().numpy(), labels.cpu().numpy()
    u = G[0].double().cpu().numpy()

    def loss(v):
        z, _ = forward64(model, v, h64)
        return -logp64(z, lab)[0].sum() / (lab >= 0).sum()

    step = 1e-4 / np.linalg.norm(u)
    slope = (loss(x64 + step * u) - loss(x64 - step * u)) / (2 * step)
    assert abs(slope / (u @ u) - 1) <= 2 * 2.0 ** -4


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16, torch.float16])
def test_an_iteration(B, dtype):
    """Eight workers, three of them faulty: gradients, scores, selection, average and update."""
    from paper_1805_10032_amd.token_model import token_worker_gradients
    m, b, gamma, rho = 8, 3, 0.5, 1e-3
    model, x, hidden, labels, _ = setup([48, 64, 90], 400, m, dtype, seed=5)
    off = [50 * i for i in range(m + 1)]
    groups = torch.tensor(off, dtype=torch.int32, device="cuda")
    server_h, server_l = hidden[:64].clone(), labels[:64].clone()
    for attack in ("none", "sign_flip", "bit_flip", "label_flip"):
        G = B.alloc_candidates(m, model.num_params)
        token_worker_gradients(model, G, x, hidden, labels, groups, [1, 4, 6], attack)
        scores = model.scores(x, G, server_h, server_l, gamma, rho)
        x_next, out, sel = B.zeno_aggregate_update(G, scores, b, gamma, x)
        torch.cuda.synchronize()
        assert torch.isfinite(G).all() and torch.isfinite(x_next).all()
        # the score's definition in float64 on the log probabilities that the model gives
        lx = model.logprobs(x, server_h, server_l).double().cpu().numpy()
        keep = server_l.cpu().numpy() >= 0
        want, scale = np.zeros(m), np.zeros(m)
        for i in range(m):
            li = model.logprobs(torch.add(x, G[i], alpha=-gamma), server_h, server_l).double().cpu().numpy()
            gain, pen = (li - lx)[keep].mean(), rho * float((G[i].double() ** 2).sum())
            want[i], scale[i] = gain - pen, abs(gain) + pen
        assert (np.abs(scores.double().cpu().numpy() - want) <= 2.0 ** -23 * scale + 1e-12).all()
        check_selection(sel.cpu().numpy(), want, b, 2.0 ** -22, scale)
        chosen = G[sel.long()].double().mean(0)
        assert ((x_next.double() - (x.double() - float(np.float32(gamma)) * chosen)).abs() <= 2.0 ** -23 * (x.double().abs() + 1)).all()
        if attack == "bit_flip":
            assert torch.equal(G[1], G[4]) and torch.equal(G[1], G[6])


def test_scores_in_float32(B):
    model, x, hidden, labels, off = setup([32, 50], 100, 4, torch.float32, seed=7)
    G = torch.randn(4, model.num_params, device="cuda") * 0.02
    s = model.scores(x, G, hidden, labels, 0.3, 1e-2).double().cpu().numpy()
    x64, h64, lab, G64 = x.double().cpu().numpy(), hidden.double().cpu().numpy(), labels.cpu().numpy(), G.double().cpu().numpy()
    n = (lab >= 0).sum()
    base = logp64(forward64(model, x64, h64)[0], lab)[0].sum() / n
    for i in range(4):
        moved = logp64(forward64(model, x64 - 0.3 * G64[i], h64)[0], lab)[0].sum() / n
        # log probabilities below 8, their errors as above; the moved parameters are rounded to float32
        assert abs(s[i] - (moved - base - 1e-2 * (G64[i] ** 2).sum())) <= 2 * (50 + 64) * T.EPS * 8 * 4


def test_refusals(B):
    from paper_1805_10032_amd.token_model import TokenModel, token_worker_gradients
    with pytest.raises(ValueError):
        TokenModel([5])
    with pytest.raises(ValueError):
        TokenModel([5, 4], torch.float64)
    model, x, hidden, labels, off = setup([16, 9], 30, 2, torch.float32)
    with pytest.raises(ValueError):
        model.gradients(x, hidden, labels, torch.tensor(off, dtype=torch.int32, device="cuda"), torch.empty(3, model.num_params, device="cuda"))
    with pytest.raises(ValueError):
        token_worker_gradients(model, torch.empty(2, model.num_params, device="cuda"), x, hidden, labels,
                               torch.tensor(off, dtype=torch.int32, device="cuda"), [0], "noise")
