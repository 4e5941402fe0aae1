"""Activations in 8 bits against the definition, code for code."""
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


def same_codes(got, want):
    """NaN has two codes (a sign); all others are equal bit for bit."""
    nan = ((got & 127) == 127) & ((want & 127) == 127)
    return np.array_equal(np.where(nan, 127, got), np.where(nan, 127, want))


def check(B, x):
    rows, width = x.shape
    ck = B.zeno_checkpoint(x)
    codes, scales = T.checkpoint(x.double().cpu().numpy())
    assert np.array_equal(ck.scales.cpu().numpy(), scales)
    assert same_codes(ck.values.cpu().numpy(), codes)
    want = T.checkpoint_values(codes, scales, width)
    for ty in T.TYPES.values():
        got = B.zeno_checkpoint_values(ck, ty).double().cpu().numpy()
        top = torch.finfo(ty).max
        exact = np.clip(want, -top, top)
        if ty == torch.float32 or ty == torch.bfloat16:
            # a product below the smallest normal float32 may be a subnormal or its flush
            ok = (got == exact) | (np.isnan(got) & np.isnan(exact)) | ((np.abs(exact) < 2.0 ** -126) & (np.abs(got - exact) <= 2.0 ** -126))
        else:
            ok = (np.abs(got - exact) <= np.abs(exact) * 2.0 ** -11 + 2.0 ** -25) | (np.isnan(got) & np.isnan(exact))
        assert ok.all(), (ty, np.argwhere(~ok)[:5])
    return ck


@pytest.mark.parametrize("ty", ["fp32", "bf16", "fp16"])
@pytest.mark.parametrize("rows,width,extra,offset", [(1, 1, 0, 0), (3, 31, 0, 1), (2, 32, 1, 0), (5, 33, 0, 3), (7, 100, 5, 7),
                                                     (4, 256, 0, 0), (3, 1001, 0, 0), (2, 4096, 0, 0), (1, 20011, 0, 0)])
def test_values(B, rows, width, ty, extra, offset):
    g = torch.Generator().manual_seed(rows + width)
    x = torch.randn(rows, width, generator=g) * torch.exp(2 * torch.randn(width, generator=g))
    view, buf = T.strided(x, T.TYPES[ty], width + extra, offset)
    check(B, view)


@pytest.mark.parametrize("ty", ["fp32", "bf16", "fp16"])
def test_borders(B, ty):
    """Ties between neighbours, blocks of zeros, scales on both sides of a power of two, the smallest and largest values,
    infinities and NaN beside ordinary values."""
    dt = T.TYPES[ty]
    fin = torch.finfo(dt)
    rows = []
    for top in (448.0, 449.0, 512.0, 1.75, 1.7578125, 2.0, 1.0):
        r = torch.zeros(96)
        r[0] = top
        r[1:9] = torch.tensor([17.0, 18.0, 19.0, 1.0625, 1.1875, -1.0625, 0.0009765625, -0.0])
        r[32:40] = torch.tensor([fin.tiny, -fin.tiny, fin.smallest_normal * 3, 0, 0, 0, 0, 0])
        rows.append(r)
    r = torch.zeros(96)
    r[0], r[1], r[2], r[3], r[40] = fin.max, -fin.max, fin.max / 2, 1.0, float("inf")
    r[41], r[42], r[43], r[70] = 3.0, float("-inf"), float("nan"), float("nan")
    rows.append(r)
    r = torch.full((96,), float("inf"))
    rows.append(r)
    r = torch.full((96,), float(fin.smallest_normal) / 4)      # subnormals of the type
    rows.append(r)
    x = torch.stack(rows).to(dt).cuda()
    check(B, x)


def test_scales_of_every_power(B):
    k = torch.arange(-149, 128, dtype=torch.float64)
    x = torch.zeros(len(k), 32, dtype=torch.float64)
    x[:, 0] = 2.0 ** k
    x[:, 1] = 2.0 ** k * 0.6
    x[:, 2] = -(2.0 ** k) * 0.013
    check(B, x.float().cuda())


def test_rows_can_be_taken_out(B):
    x = torch.randn(10, 77, device="cuda")
    ck = check(B, x)
    part = B.Checkpoint(ck.values[3:7], ck.scales[3:7], 77)
    assert torch.equal(B.zeno_checkpoint_values(part), B.zeno_checkpoint_values(ck)[3:7])


def test_no_rows_and_what_lies_around(B):
    ck = B.zeno_checkpoint(torch.empty(0, 50, device="cuda"))
    assert ck.values.shape == (0, 64) and B.zeno_checkpoint_values(ck).shape == (0, 50)
    x = torch.randn(4, 45, device="cuda")
    ck = B.zeno_checkpoint(x)
    out, buf = T.strided(torch.zeros(4, 45), torch.bfloat16, 47, 3)
    B.zeno_checkpoint_values(ck, out=out)
    assert torch.equal(out, B.zeno_checkpoint_values(ck, torch.bfloat16)) and torch.isnan(T.around(out, buf)).all()


def test_every_code_and_scale(B):
    """The way back of all 256 codes at all 248 scales: exact in float32, and in bf16 but for what lies below its smallest steps (2^-133)."""
    codes = np.tile(np.arange(256, dtype=np.uint8), (248, 1))
    scales = np.tile(np.arange(248, dtype=np.uint8)[:, None], (1, 8))
    ck = B.Checkpoint(torch.from_numpy(codes).cuda(), torch.from_numpy(scales).cuda(), 256)
    want = T.checkpoint_values(codes, scales, 256)
    for ty in (torch.float32, torch.bfloat16):
        top = torch.finfo(ty).max
        exact = np.clip(want, -top, top)
        got = B.zeno_checkpoint_values(ck, ty).double().cpu().numpy()
        same = (got == exact) | (np.isnan(got) & np.isnan(exact))
        if ty == torch.bfloat16:
            assert (np.abs(got - exact)[:3][~same[:3]] <= 2.0 ** -134).all()
            same = same[3:]
        assert same.all(), (ty, np.argwhere(~same)[:5])
