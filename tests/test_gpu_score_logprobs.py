"""Definition 2 from log probabilities against the definition in float64."""
import numpy as np
import pytest
import torch

from paper_1805_10032_amd import workloads as WL

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def B():
    from paper_1805_10032_amd import binding
    binding.load_library()
    return binding


@pytest.mark.parametrize("m,d,n,align", [(1, 1, 1, 1), (3, 5, 2, 1), (20, 4097, 64, 1), (7, 100003, 300, 32), (1024, 33, 5, 1), (2, 3000001, 1000, 4)])
def test_scores(B, m, d, n, align):
    g = torch.Generator().manual_seed(m + d)
    G = WL._alloc_rows(m, d, align, "cuda")
    G.copy_(torch.randn(m, d, generator=g))
    lx = -torch.rand(n, generator=g) * 5
    buf = torch.full((m, n + 3), float("nan"), device="cuda")
    lc = buf[:, :n]
    lc.copy_(lx + 0.1 * torch.randn(m, n, generator=g))
    labels = torch.randint(-1, 3, (n,), generator=g, dtype=torch.int32)
    for lab in (None, labels, torch.full((n,), -1, dtype=torch.int32)):
        for rho in (0.0, 1e-3):
            got = B.zeno_score_logprobs(G, lx.cuda(), lc, rho, labels=None if lab is None else lab.cuda()).double().cpu().numpy()
            keep = np.ones(n, bool) if lab is None else lab.numpy() != -1
            diff = (lc.double().cpu().numpy() - lx.double().numpy())[:, keep]
            gain = diff.mean(1) if keep.any() else np.zeros(m)
            norm = (G.double().cpu().numpy() ** 2).sum(1)
            want = gain - rho * norm
            # float64 sums, rho as the float32 it is passed as, one rounding to float32
            tol = 2.0 ** -24 * np.abs(want) + 2.0 ** -24 * rho * norm + (d + n) * 2.0 ** -53 * (np.abs(diff).mean(1) if keep.any() else 0 + rho * norm)
            assert (np.abs(got - want) <= tol).all(), (lab is None, rho, np.abs(got - want).max())


def test_values_that_are_not_finite(B):
    G = torch.ones(6, 50, device="cuda")
    G[1, 3] = float("inf")
    G[2, 4] = float("nan")
    G[3, :] = 3e38
    lx = torch.full((4,), -1.0, device="cuda")
    lc = torch.full((6, 4), -0.5, device="cuda")
    lc[4, 1] = float("-inf")
    lc[5, 2] = float("nan")
    s = B.zeno_score_logprobs(G, lx, lc, 0.5).cpu().numpy()
    assert s[0] == 0.5 - 25.0 and s[1] == -np.inf and np.isnan(s[2]) and s[3] == -np.inf and s[4] == -np.inf and np.isnan(s[5])
    out, sel = B.zeno_aggregate(G, torch.tensor(s, device="cuda"), 5)
    assert sel.tolist() == [0]
