"""Gradients of a linear layer's weights from 8-bit activations, per worker, against float64 sums of the same values."""
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


def check(B, rows, out, width, ty, offsets=None, seed=1, pitch=None, shift=0, edit=None, G_extra=(0, 0)):
    g = torch.Generator().manual_seed(seed)
    a = torch.randn(rows, width, generator=g) * torch.exp(0.7 * torch.randn(width, generator=g))
    dy = torch.randn(rows, out, generator=g)
    if edit is not None:
        edit(a, dy)
    dy, _ = T.strided(dy, T.TYPES[ty], pitch or out, shift)
    ck = B.zeno_checkpoint(a.cuda())
    off = [0, rows] if offsets is None else offsets
    m = len(off) - 1
    groups = None if offsets is None else torch.tensor(off, dtype=torch.int32, device="cuda")
    n = out * width
    before, behind = G_extra
    G = torch.full((m, before + n + out + behind), 7.0, device="cuda")
    dw, db = B.zeno_weight_gradient(dy, ck, groups=groups, dweight=G[:, before:before + n], dbias=G[:, before + n:before + n + out])
    torch.cuda.synchronize()
    a64, d64 = B.zeno_checkpoint_values(ck).double().cpu().numpy(), dy.double().cpu().numpy()
    for i, (p, q) in enumerate(zip(off, off[1:])):
        with np.errstate(invalid="ignore"):
            want, mag = d64[p:q].T @ a64[p:q], np.abs(d64[p:q]).T @ np.abs(a64[p:q])
            # exact products (float32's three pieces leave at most 2^-24 of dy out); every addition rounds a sum by at most
            # 2^-23 of it (the matrix instruction's own rounding included), and three pieces are three additions a token
            pieces = {"fp32": 3, "bf16": 1, "fp16": 2}[ty]
            tol = (pieces * (q - p) + 8) * 2 * T.EPS * mag + 1e-37
            got = dw[i].double().cpu().numpy().reshape(out, width)
            ok = (np.abs(got - want) <= tol) | (got == want) | (np.isnan(got) & np.isnan(want))
            assert ok.all(), (i, np.argwhere(~ok)[:5], got[~ok][:5], want[~ok][:5])
            wb, mb = d64[p:q].sum(0), np.abs(d64[p:q]).sum(0)
            gb = db[i].double().cpu().numpy()
            ok = (np.abs(gb - wb) <= (q - p + 8) * T.EPS * mb + 1e-37) | (gb == wb) | (np.isnan(gb) & np.isnan(wb))
            assert ok.all(), ("bias", i, np.argwhere(~ok)[:5])
    assert (G[:, :before] == 7).all() and (G[:, before + n + out:] == 7).all()
    return G


SHAPES = [(1, 1, 1), (2, 3, 5), (31, 10, 33), (33, 128, 128), (64, 129, 127), (100, 257, 300), (77, 64, 1001), (600, 10, 40), (40, 513, 96)]


@pytest.mark.parametrize("ty", ["fp32", "bf16", "fp16"])
@pytest.mark.parametrize("rows,out,width", SHAPES)
def test_one_group(B, rows, out, width, ty):
    check(B, rows, out, width, ty)
    check(B, rows, out, width, ty, pitch=out + 3, shift=5, seed=2)


@pytest.mark.parametrize("ty", ["fp32", "bf16", "fp16"])
@pytest.mark.parametrize("rows,out,width", [(200, 40, 70), (900, 130, 260), (3000, 7, 33)])
def test_groups(B, rows, out, width, ty):
    off = [2, 2, 3, rows // 4, rows // 4 + 31, rows // 2, rows - 7, rows - 7]
    G = check(B, rows, out, width, ty, off, G_extra=(3, 2))
    n = out * width + out
    assert not G[0, 3:3 + n].any() and not G[-1, 3:3 + n].any()
    assert torch.equal(G, check(B, rows, out, width, ty, off, G_extra=(3, 2)))       # the same bits every time


@pytest.mark.parametrize("ty", ["fp32", "bf16", "fp16"])
@pytest.mark.parametrize("out", [1, 4, 5, 8, 9, 12, 13, 16, 17, 24, 25, 32, 33])
def test_few_outputs(B, out, ty):
    """Every number of outputs that has a variant of its own, widths on both sides of a workgroup's columns, tokens of one wave, of
    several, and of several workgroups."""
    check(B, 700, out, 530, ty, [1, 1, 34, 300, 699], G_extra=(1, 1))
    check(B, 3001, out, 255, ty, pitch=out + 1, shift=1)
    check(B, 9, out, 4, ty)


def test_long_sums(B):
    """Tokens cut into pieces that several workgroups sum."""
    check(B, 20000, 10, 100, "fp32")
    check(B, 9001, 200, 140, "bf16", [0, 4000, 4000, 9001])
    check(B, 5000, 10, 30, "fp16", [0, 5, 5000])


@pytest.mark.parametrize("ty", ["fp32", "bf16", "fp16"])
@pytest.mark.parametrize("m,out,width", [(64, 300, 257), (256, 129, 200), (70, 264, 500)])
def test_wide_tiles(B, m, out, width, ty):
    """Enough output for the wide tiles: ragged groups, empty ones and ones of a single token, widths that end inside a tile."""
    g = torch.Generator().manual_seed(m)
    sizes = torch.randint(0, 180, (m,), generator=g)
    sizes[:4] = torch.tensor([0, 1, 32, 33])
    off = [0, *torch.cumsum(sizes, 0).tolist()]
    rows = max(off[-1] + 3, 64 * m)
    check(B, rows, out, width, ty, off, G_extra=(1, 2))
    check(B, rows, out, width, ty, off, pitch=out + 1, shift=3)


@pytest.mark.parametrize("ty", ["fp32", "bf16", "fp16"])
def test_values_that_are_not_finite(B, ty):
    """An infinity in dy meets ordinary activations and zeros; a NaN among the activations; they reach their row or column only."""
    def edit(a, dy):
        dy[3, 2] = float("inf")
        a[3, 4] = 0.0
        a[5, 6] = float("nan")
        dy[7, 1] = float("-inf")
        a[7, :] = a[7, :].abs() + 0.5
    check(B, 50, 40, 70, ty, edit=edit)


def test_floats_at_the_ends_of_the_range(B):
    def edit(a, dy):
        dy[0, 0] = 3.4e38
        a[0, :] = 0.25
        dy[1:, 0] = 0.0
        dy[:, 1] *= 1e-20
        dy[:, 2] *= 1e30
        a[:, 5] *= 1e-6
    check(B, 40, 8, 40, "fp32", edit=edit)


def test_no_rows_and_no_bias(B):
    ck = B.zeno_checkpoint(torch.empty(0, 40, device="cuda"))
    dw, db = B.zeno_weight_gradient(torch.empty(0, 9, device="cuda"), ck, groups=torch.zeros(3, dtype=torch.int32, device="cuda"))
    assert dw.shape == (2, 360) and not dw.any() and not db.any()
    x, dy = torch.randn(30, 40, device="cuda"), torch.randn(30, 9, device="cuda")
    ck = B.zeno_checkpoint(x)
    dw, db = B.zeno_weight_gradient(dy, ck)
    only, none = B.zeno_weight_gradient(dy, ck, want_bias=False)
    assert none is None and torch.equal(only, dw)


@pytest.mark.parametrize("out", [3, 40, 300])
def test_every_nan_stays_one(B, out):
    """A float32 NaN whose payload lies in the lower half: its leading bits alone are those of an infinity."""
    dy = torch.ones(70, out)
    dy[5, 2] = torch.tensor([0x7f800001], dtype=torch.int32).view(torch.float32)
    dy = dy.cuda()
    dw, db = B.zeno_weight_gradient(dy, B.zeno_checkpoint(torch.ones(70, 300, device="cuda")))
    dw = dw.reshape(out, 300)
    assert torch.isnan(dw[2]).all() and torch.isnan(db[0, 2])
    keep = [o for o in range(out) if o != 2]
    assert (dw[keep] == 70).all() and (db[0, keep] == 70).all()


def whole_sums(B, rows, out, width, ty, off, pitch=None, before=0):
    """Small whole numbers, whose sums float32 holds exactly, and a workspace that held NaN."""
    g = torch.Generator().manual_seed(rows + out + width)
    dy, a = (torch.randint(-2, 3, (rows, n), generator=g).float() for n in (out, width))
    dy, _ = T.strided(dy, T.TYPES[ty], pitch or out, before)
    a = a.cuda()
    m, n = len(off) - 1, out * width
    G = torch.full((m, before + n + out + 1), 7.0, device="cuda")
    ws = B.alloc_weight_gradient_workspace(rows, out, width, m).fill_(255)
    B.zeno_weight_gradient(dy, B.zeno_checkpoint(a), groups=torch.tensor(off, dtype=torch.int32, device="cuda"), dweight=G[:, before:before + n],
                           dbias=G[:, before + n:before + n + out], workspace=ws)
    for i, (p, q) in enumerate(zip(off, off[1:])):
        d = dy[p:q].float()
        assert torch.equal(G[i, before:before + n].view(out, width), d.t().contiguous() @ a[p:q]), i
        assert torch.equal(G[i, before + n:before + n + out], d.sum(0)), i
    assert (G[:, :before] == 7).all() and (G[:, -1] == 7).all()
    return ws.numel()


@pytest.mark.parametrize("ty", ["fp32", "bf16", "fp16"])
@pytest.mark.parametrize("rows,out,width,off", [
    (16500, 4096, 1024, [3, 16490]), (16500, 4096, 1024, [0, 16500]), (9000, 2048, 2048, [0, 4000, 9000]),
    (8300, 4093, 1025, [1, 8299]), (16400, 1000, 1000, [0, 5, 16400]), (17000, 521, 2050, [0, 0, 16993]), (17000, 300, 4095, [2, 35, 17000])])
def test_wide_tiles_of_cut_tokens(B, rows, out, width, off, ty):
    """Wide tiles whose tokens several workgroups share: ragged and empty groups, groups shorter than a piece, outputs that are no
    multiple of eight and widths that end inside a tile."""
    m = len(off) - 1
    wide = -(-out // 256) * -(-width // 256) * m
    assert out > 128 and width > 128 and wide < 256 and rows // m >= 1024 * ((255 + wide) // wide)      # what leads to this plan
    used = whole_sums(B, rows, out, width, ty, off, pitch=out + 3 if out % 8 else out, before=1 if out % 8 else 0)
    assert used >= 4 * m * ((255 + wide) // wide) * (out * width + out)


@pytest.mark.parametrize("ty", ["fp32", "bf16", "fp16"])
@pytest.mark.parametrize("rows,out,width,off", [(9000, 200, 140, [0, 9000]), (5000, 129, 1000, [0, 8, 4990]), (12000, 12, 600, [5, 5, 12000])])
def test_other_plans_of_cut_tokens(B, rows, out, width, off, ty):
    used = whole_sums(B, rows, out, width, ty, off)
    assert used > 256
