"""Layer norm, its backward pass with the gradients of several workers' weights, and both with a checkpoint in 8 bits."""
import numpy as np
import pytest
import torch

from tests import _tokens as T

pytestmark = pytest.mark.gpu
EPS_NORM = 1e-5


@pytest.fixture(scope="module")
def B():
    from paper_1805_10032_amd import binding
    binding.load_library()
    return binding


def chain(width, per_load):
    """Longest chain of additions over a row: a thread's values (32 at most, or the long kernel's share of 1024 threads), the wave's
    six steps, sixteen waves."""
    return max(32, int(np.ceil(width / (1024 * per_load))) * per_load) + 6 + 16


def make(rows, width, ty, seed, pitch=None, offset=0, shift=0.1):
    g = torch.Generator().manual_seed(seed)
    x = torch.randn(rows, width, generator=g) * torch.exp(0.5 * torch.randn(width, generator=g)) + shift
    x, buf = T.strided(x, T.TYPES[ty], pitch, offset)
    weight = (1 + 0.2 * torch.randn(width + 1, generator=g)).cuda()[1:]       # 4-byte aligned only
    bias = (0.3 * torch.randn(width + 3, generator=g)).cuda()[3:]
    return x, buf, weight, bias, g


def check_forward(B, x, weight, bias, ckpt=False, y=None):
    rows, width = x.shape
    k = chain(width, 16 // x.element_size())
    got, mean, rstd, kept = B.zeno_layer_norm(x, weight, bias, EPS_NORM, want_checkpoint=ckpt, y=y)
    torch.cuda.synchronize()
    x64, w64 = x.double().cpu().numpy(), weight.double().cpu().numpy()
    b64 = None if bias is None else bias.double().cpu().numpy()
    want, m64, r64, xh = T.layer_norm(x64, w64, b64, EPS_NORM)
    dev = np.abs(x64 - m64[:, None])
    e_mean = (k + 2) * T.EPS * np.abs(x64).mean(1) + 1e-45
    var = 1 / r64 ** 2
    # the variance: rounded differences, their squares summed, the mean's error squared
    e_rstd = 0.5 * ((k + 6) * T.EPS + (e_mean ** 2 + 2 * T.EPS * e_mean * dev.mean(1)) / var) + 4 * T.EPS
    assert (np.abs(mean.cpu().numpy() - m64) <= e_mean).all()
    assert (np.abs(rstd.cpu().numpy() / r64 - 1) <= e_rstd).all()
    tol = np.abs(w64) * r64[:, None] * (e_mean[:, None] + T.EPS * dev) + np.abs(xh * w64) * (e_rstd[:, None] + 3 * T.EPS)
    tol = tol + T.EPS * np.abs(want) + (np.abs(want) + tol) * T.half_step(x.dtype) + T.smallest_half(x.dtype)
    err = np.abs(got.double().cpu().numpy() - want)
    assert (err <= tol).all(), (np.argwhere(err > tol)[:5], err.max())
    if ckpt:
        alone = B.zeno_checkpoint(x)
        assert torch.equal(kept.values, alone.values) and torch.equal(kept.scales, alone.scales)
    return got, mean, rstd, kept


SHAPES = [  # rows, width, type, extra pitch, offset
    (1, 1, "fp32", 0, 0), (2, 2, "bf16", 1, 1), (5, 31, "fp32", 0, 0), (3, 33, "fp16", 0, 3), (9, 256, "fp32", 0, 0),
    (4, 257, "bf16", 0, 0), (66, 512, "bf16", 0, 0), (17, 1001, "fp32", 0, 1), (6, 2048, "bf16", 8, 0), (5, 2050, "fp16", 0, 0),
    (3, 4096, "bf16", 0, 0), (4, 4097, "fp32", 1, 0), (2, 8192, "bf16", 0, 0), (3, 8193, "fp16", 0, 0), (2, 16384, "fp32", 0, 0),
    (2, 16390, "fp32", 0, 2), (2, 32768, "bf16", 0, 0), (2, 40001, "bf16", 0, 0), (3, 33000, "fp32", 0, 0),
]


@pytest.mark.parametrize("rows,width,ty,extra,offset", SHAPES)
def test_forward(B, rows, width, ty, extra, offset):
    x, _, weight, bias, _ = make(rows, width, ty, rows + width, width + extra, offset)
    check_forward(B, x, weight, bias)
    check_forward(B, x, weight, None, ckpt=True)


def test_more_rows_than_the_chip_holds(B):
    for rows, width, ty in ((9001, 40, "bf16"), (3000, 2300, "bf16"), (700, 9000, "fp32")):
        x, _, weight, bias, _ = make(rows, width, ty, 5)
        check_forward(B, x, weight, bias, ckpt=True)


def test_large_offset_and_constant_rows(B):
    """A mean far larger than the deviation is subtracted before squaring; a row of equal values comes out as the bias."""
    x, _, weight, bias, _ = make(6, 700, "fp32", 6, shift=1000.0)
    check_forward(B, x, weight, bias)
    x[2, :] = 3.0
    y, mean, rstd, _ = B.zeno_layer_norm(x, weight, bias, EPS_NORM)
    assert abs(float(mean[2]) - 3.0) <= 700 * T.EPS * 3 and (y[2] - bias).abs().max() <= 700 * T.EPS * 3 / EPS_NORM ** 0.5 * weight.abs().max()


def test_rows_that_are_not_finite_stay_alone(B):
    for width in (100, 3000, 40000):
        x, _, weight, bias, _ = make(4, width, "fp32", 7)
        clean = B.zeno_layer_norm(x, weight, bias, EPS_NORM)[0].clone()
        x[1, 5] = float("nan")
        x[2, 7] = float("inf")
        y, mean, rstd, _ = B.zeno_layer_norm(x, weight, bias, EPS_NORM)
        assert torch.isnan(y[1]).all() and torch.isnan(y[2]).all()
        assert torch.equal(y[0], clean[0]) and torch.equal(y[3], clean[3])


def check_backward(B, x, weight, offsets, ckpt, seed=8, dy=None, dx=None, G=None, **want):
    rows, width = x.shape
    g = torch.Generator().manual_seed(seed)
    if dy is None:
        dy = torch.randn(rows, width, generator=g).to(x.dtype).cuda()
    _, mean, rstd, kept = B.zeno_layer_norm(x, weight, None, EPS_NORM, want_checkpoint=ckpt)
    groups = None if offsets is None else torch.tensor(offsets, dtype=torch.int32, device="cuda")
    off = [0, rows] if offsets is None else offsets
    m = len(off) - 1
    dw = db = None
    if G is not None:
        dw, db = G[:, 1:1 + width], G[:, 1 + width:1 + 2 * width]
    dy64 = dy.double().cpu().numpy()
    dx, dw, db = B.zeno_layer_norm_backward(dy, kept if ckpt else x, mean, rstd, weight, groups=groups, dx=dx, dweight=dw, dbias=db, **want)
    torch.cuda.synchronize()
    x64 = (B.zeno_checkpoint_values(kept) if ckpt else x).double().cpu().numpy()
    w64, m64, r64 = weight.double().cpu().numpy(), mean.double().cpu().numpy(), rstd.double().cpu().numpy()
    xh = (x64 - m64[:, None]) * r64[:, None]
    want_dx, want_dw, want_db, c1, c2 = T.layer_norm_grad(dy64, xh, r64, w64, off)
    a = np.abs(dy64 * w64)
    k = chain(width, 16 // x.element_size())
    if dx is not None:
        e_c1, e_c2 = (k + 3) * T.EPS * a.mean(1, keepdims=True), (k + 6) * T.EPS * (a * np.abs(xh)).mean(1, keepdims=True)
        tol = r64[:, None] * (e_c1 + np.abs(xh) * e_c2 + 5 * T.EPS * (a + np.abs(c1) + np.abs(xh * c2)))
        tol = tol + (np.abs(want_dx) + tol) * T.half_step(x.dtype) + T.smallest_half(x.dtype)
        err = np.abs(dx.double().cpu().numpy() - want_dx)[off[0]:off[-1]]
        assert (err <= tol[off[0]:off[-1]]).all(), (np.argwhere(err > tol[off[0]:off[-1]])[:5], err.max())
    for i, (p, q) in enumerate(zip(off, off[1:])):
        n = q - p + 8      # additions of the longest chain over the rows, however they are cut; xh has two roundings, the product one
        if dw is not None:
            tol = (n + 4) * T.EPS * np.abs(dy64[p:q] * xh[p:q]).sum(0) + 1e-40
            err = np.abs(dw[i].double().cpu().numpy() - want_dw[i])
            assert (err <= tol).all(), ("dweight", i, np.argwhere(err > tol)[:5], err.max())
        if db is not None:
            tol = n * T.EPS * np.abs(dy64[p:q]).sum(0) + 1e-40
            err = np.abs(db[i].double().cpu().numpy() - want_db[i])
            assert (err <= tol).all(), ("dbias", i, np.argwhere(err > tol)[:5], err.max())
    return dx, dw, db


@pytest.mark.parametrize("ckpt", [False, True])
@pytest.mark.parametrize("rows,width,ty,extra,offset", SHAPES)
def test_backward(B, rows, width, ty, extra, offset, ckpt):
    x, _, weight, _, _ = make(rows, width, ty, rows + width, width + extra, offset)
    check_backward(B, x, weight, None, ckpt)


@pytest.mark.parametrize("ckpt", [False, True])
@pytest.mark.parametrize("rows,width,ty", [(300, 70, "fp32"), (1500, 600, "bf16"), (700, 2304, "fp16"), (90, 9001, "fp32"), (70, 40000, "bf16")])
def test_groups(B, rows, width, ty, ckpt):
    """Ragged groups, empty ones, groups of one row, rows that belong to nobody in front and behind; the gradients go into
    columns of rows of G with an odd pitch, and nothing else of G or of dx changes."""
    x, _, weight, _, g = make(rows, width, ty, rows)
    off = [3, 3, 4, rows // 3, rows // 3, rows // 2 + 1, rows - 5, rows - 5]
    m = len(off) - 1
    G = torch.full((m, 2 * width + 6), 7.0, device="cuda")
    dx = torch.full((rows, width), 5.0, device="cuda", dtype=x.dtype)
    dx, dw, db = check_backward(B, x, weight, off, ckpt, dx=dx, G=G)
    assert not G[0, 1:1 + 2 * width].any() and not G[m - 1, 1:1 + 2 * width].any()
    assert (G[:, 0] == 7).all() and (G[:, 1 + 2 * width:] == 7).all()
    assert (dx[:3] == 5).all() and (dx[rows - 5:] == 5).all()
    again = check_backward(B, x, weight, off, ckpt)
    assert torch.equal(again[1], dw) and torch.equal(again[2], db)      # the same bits every time


@pytest.mark.parametrize("ckpt", [False, True])
@pytest.mark.parametrize("rows,width,ty,extra,offset", [
    (1100, 4100, "fp32", 0, 0), (1500, 4099, "bf16", 1, 1), (1030, 6144, "bf16", 0, 0), (530, 8192, "fp32", 0, 0),
    (600, 8200, "bf16", 0, 0), (580, 12001, "fp16", 0, 3), (300, 16384, "bf16", 8, 0), (520, 12288, "fp32", 0, 0),
    (270, 16383, "fp32", 2, 1)])
def test_wide_rows(B, rows, width, ty, extra, offset, ckpt):
    """Several rows a workgroup at every number of waves and pieces a row, with groups that end inside a chunk, also in place."""
    x, _, weight, bias, g = make(rows, width, ty, rows + width, width + extra, offset)
    check_forward(B, x, weight, bias, ckpt=ckpt)
    off = [1, rows // 2, rows // 2, rows // 2 + 2, rows]
    dy = torch.randn(rows, width, generator=g).to(x.dtype).cuda()
    dx, dw, db = check_backward(B, x, weight, off, ckpt, dy=dy)
    inplace = check_backward(B, x, weight, off, ckpt, dy=dy, dx=dy)
    assert inplace[0] is dy and torch.equal(dy[1:], dx[1:]) and torch.equal(inplace[1], dw) and torch.equal(inplace[2], db)


def test_many_groups(B):
    rows, m = 2000, 1024
    x, _, weight, _, g = make(rows, 65, "fp32", 9)
    cuts = torch.sort(torch.randint(0, rows + 1, (m + 1,), generator=g)).values.tolist()
    check_backward(B, x, weight, cuts, False)


def test_outputs_alone_and_in_place(B):
    for width in (300, 5000, 40000):
        x, _, weight, _, g = make(40, width, "bf16", 10)
        off = [0, 17, 40]
        dy = torch.randn(40, width, generator=g).bfloat16().cuda()
        dx, dw, db = check_backward(B, x, weight, off, False, dy=dy)
        only = check_backward(B, x, weight, off, False, dy=dy, want_weight=False, want_bias=False)
        assert only[1] is None and torch.equal(only[0], dx)
        only = check_backward(B, x, weight, off, False, dy=dy, want_dx=False, want_bias=False)
        assert only[0] is None and torch.equal(only[1], dw)
        only = check_backward(B, x, weight, off, False, dy=dy, want_dx=False, want_weight=False)
        assert torch.equal(only[2], db)
        inplace = check_backward(B, x, weight, off, False, dy=dy, dx=dy)
        assert inplace[0] is dy and torch.equal(dy, dx)


def test_no_rows(B):
    x = torch.empty(0, 40, device="cuda")
    w = torch.ones(40, device="cuda")
    y, mean, rstd, ck = B.zeno_layer_norm(x, w, want_checkpoint=True)
    groups = torch.zeros(4, dtype=torch.int32, device="cuda")
    dx, dw, db = B.zeno_layer_norm_backward(x, ck, mean, rstd, w, groups=groups)
    assert dx.shape == (0, 40) and dw.shape == (3, 40) and not dw.any() and not db.any()


def test_gradient_against_differences(B):
    """Central differences of sum(dy y) in float64 of the definition."""
    x, _, weight, bias, g = make(3, 9, "fp32", 12)
    dy = torch.randn(3, 9, generator=g).cuda()
    _, mean, rstd, _ = B.zeno_layer_norm(x, weight, bias, EPS_NORM)
    dx, dw, db = B.zeno_layer_norm_backward(dy, x, mean, rstd, weight)
    x64, w64, b64, d64 = (t.double().cpu().numpy() for t in (x, weight, bias, dy))
    value = lambda xx, ww, bb: (d64 * T.layer_norm(xx, ww, bb, EPS_NORM)[0]).sum()
    step = 1e-5

    def slope(args, which, at):
        ends = []
        for sign in (1, -1):
            a = [v.copy() for v in args]
            a[which][at] += sign * step
            ends.append(value(*a))
        return (ends[0] - ends[1]) / (2 * step)

    args = (x64, w64, b64)
    # third derivatives of at most about 1e3 times step^2 / 6, rounding 2^-52 |value| / step, and the kernel's float32 (values below 20)
    tol = 1e3 * step ** 2 + 1e-8 + 20 * 64 * T.EPS
    for r in range(3):
        for j in range(9):
            assert abs(slope(args, 0, (r, j)) - float(dx[r, j])) <= tol
    for j in range(9):
        assert abs(slope(args, 1, j) - float(dw[0, j])) <= tol and abs(slope(args, 2, j) - float(db[0, j])) <= tol


@pytest.mark.parametrize("ckpt", [False, True])
@pytest.mark.parametrize("width,ty", [(1, "fp32"), (32, "fp32"), (100, "bf16"), (1001, "fp32"), (2050, "bf16"), (6144, "bf16"), (9001, "fp32"),
                                      (20000, "fp32"), (40001, "bf16")])
def test_what_lies_behind_a_row_has_no_weight(B, width, ty, ckpt):
    """Equal values of a size whose product with rstd is out of range: xh is 0 in every column, so dx = rstd (a - mean(a)).  Lanes
    behind the row's end must not bring in an infinity."""
    rows, big, r = 3, 2.0 ** 110, 2.0 ** 20
    g = torch.Generator().manual_seed(width)
    x = torch.full((rows, width), big, dtype=T.TYPES[ty], device="cuda")
    dy = torch.randn(rows, width, generator=g).to(T.TYPES[ty]).cuda()
    w = (1 + 0.2 * torch.randn(width, generator=g)).cuda()
    mean, rstd = torch.full((rows,), big, device="cuda"), torch.full((rows,), r, device="cuda")
    dx, dw, db = B.zeno_layer_norm_backward(dy, B.zeno_checkpoint(x) if ckpt else x, mean, rstd, w)
    d64 = dy.double().cpu().numpy()
    a = d64 * w.double().cpu().numpy()
    want = r * (a - a.mean(1, keepdims=True))
    tol = r * ((chain(width, 16 // x.element_size()) + 3) * T.EPS * np.abs(a).mean(1, keepdims=True) + 5 * T.EPS * np.abs(a))
    tol = tol + (np.abs(want) + tol) * T.half_step(x.dtype)
    assert (np.abs(dx.double().cpu().numpy() - want) <= tol).all()
    assert not dw.any()
    assert (np.abs(db[0].double().cpu().numpy() - d64.sum(0)) <= (rows + 8) * T.EPS * np.abs(d64).sum(0)).all()


@pytest.mark.parametrize("ckpt", [False, True])
@pytest.mark.parametrize("width", [100, 3000, 9001, 20000])
def test_variance_out_of_range(B, width, ckpt):
    """One value of 1e38: rstd is 0 in float32, so xh and dx are 0, whatever dy is."""
    x, _, weight, _, g = make(3, width, "fp32", 14)
    x[1, 5] = 1e38
    dy = torch.randn(3, width, generator=g).cuda()
    dy[1] *= 1000
    _, mean, rstd, kept = B.zeno_layer_norm(x, weight, None, EPS_NORM, want_checkpoint=True)
    assert float(rstd[1]) == 0
    dx, dw, _ = B.zeno_layer_norm_backward(dy, kept if ckpt else x, mean, rstd, weight, groups=torch.tensor([0, 1, 2, 3], dtype=torch.int32, device="cuda"))
    assert not dx[1].any() and not dw[1].any() and torch.isfinite(dx).all() and dx[0].any() and dx[2].any()


@pytest.mark.parametrize("ckpt", [False, True])
@pytest.mark.parametrize("rows,width,ty", [(1300, 257, "fp32"), (700, 512, "fp32"), (900, 513, "fp32"), (1100, 1025, "fp32"), (600, 2048, "fp32"),
                                           (530, 2051, "fp32"), (520, 4096, "fp32"), (1200, 513, "bf16"), (800, 1025, "fp16"), (520, 8193, "bf16")])
def test_every_shape_of_rows(B, rows, width, ty, ckpt):
    """Both ends of every number of waves and pieces that a row may take, several rows a workgroup, ragged groups, also in place."""
    x, _, weight, bias, g = make(rows, width, ty, rows + width)
    check_forward(B, x, weight, bias, ckpt=ckpt)
    off = [0, 7, 7, rows // 2 + 1, rows - 1]
    dy = torch.randn(rows, width, generator=g).to(x.dtype).cuda()
    dx, dw, db = check_backward(B, x, weight, off, ckpt, dy=dy)
    inplace = check_backward(B, x, weight, off, ckpt, dy=dy, dx=dy)
    assert inplace[0] is dy and torch.equal(dy[:-1], dx[:-1]) and torch.equal(inplace[1], dw) and torch.equal(inplace[2], db)
