"""The operators for models that answer with tokens at the ends of their ranges: rows far apart, offsets past 2^31, more rows than a
launch has workgroups, the most groups.  What such a call gives has to be, bit for bit, what the same rows give close together, or sums
of small whole numbers, which float32 holds exactly."""
import math

import pytest
import torch

pytestmark = pytest.mark.gpu
TYPES = {"fp32": torch.float32, "bf16": torch.bfloat16, "fp16": torch.float16}


@pytest.fixture(scope="module")
def B():
    from paper_1805_10032_amd import binding
    binding.load_library()
    return binding


def far(x, pitch):
    """The same rows `pitch` elements apart, in memory that is not cleared."""
    buf = torch.empty((x.shape[0] - 1) * pitch + x.shape[1], dtype=x.dtype, device="cuda")
    out = buf.as_strided(x.shape, (pitch, 1))
    out.copy_(x)
    return out


def whole(shape, gen, most=2):
    return torch.randint(-most, most + 1, shape, generator=gen).float()


@pytest.mark.parametrize("ty", list(TYPES))
@pytest.mark.parametrize("vocab", [10, 300, 9000])
def test_logits_far_apart(B, vocab, ty):
    g = torch.Generator().manual_seed(vocab)
    z = torch.randn(7, vocab, generator=g).to(TYPES[ty]).cuda()
    lab = torch.randint(0, vocab, (7,), generator=g, dtype=torch.int32).cuda()
    z2 = far(z, (1 << 29) + 1)
    one, two = (B.zeno_logprobs(q, lab, top=3, want_entropy=True, want_stats=True) for q in (z, z2))
    for a, b in zip(one, two):
        assert torch.equal(a, b)
    h = torch.randn(7, generator=g).cuda()
    d = B.zeno_logprobs_backward(z, one[2], labels=lab, grad_logp=h, entropy=one[1], grad_entropy=h)
    d2 = B.zeno_logprobs_backward(z2, one[2], labels=lab, grad_logp=h, entropy=one[1], grad_entropy=h, out=z2)
    assert torch.equal(d, d2)


@pytest.mark.parametrize("ty", list(TYPES))
@pytest.mark.parametrize("width", [33, 4100, 17000])
def test_activations_far_apart(B, width, ty):
    g = torch.Generator().manual_seed(width)
    x, dy = (torch.randn(7, width, generator=g).to(TYPES[ty]).cuda() for _ in range(2))
    w, b = torch.randn(width, generator=g).cuda(), torch.randn(width, generator=g).cuda()
    x2, dy2 = far(x, (1 << 29) + 3), far(dy, (1 << 29) + 5)
    y, mean, rstd, ck = B.zeno_layer_norm(x, w, b, want_checkpoint=True)
    y2, mean2, rstd2, ck2 = B.zeno_layer_norm(x2, w, b, want_checkpoint=True, y=far(x, (1 << 29) + 7))
    assert torch.equal(y, y2) and torch.equal(mean, mean2) and torch.equal(rstd, rstd2)
    assert torch.equal(ck.values, ck2.values) and torch.equal(ck.scales, ck2.scales)
    alone = B.zeno_checkpoint(x2)
    assert torch.equal(ck.values, alone.values) and torch.equal(ck.scales, alone.scales)
    assert torch.equal(B.zeno_checkpoint_values(ck, x.dtype), B.zeno_checkpoint_values(ck, x.dtype, out=y2))
    off = torch.tensor([0, 2, 7], dtype=torch.int32, device="cuda")
    one, two = (B.zeno_layer_norm_backward(d, q, mean, rstd, w, groups=off, dx=o)
                for d, q, o in ((dy, x, None), (dy2, x2, dy2)))
    for p, q in zip(one, two):
        assert torch.equal(p, q)


@pytest.mark.parametrize("ty", list(TYPES))
@pytest.mark.parametrize("out,width", [(10, 100), (130, 300)])
def test_gradients_far_apart(B, out, width, ty):
    g = torch.Generator().manual_seed(out)
    rows = 40
    dy, a = whole((rows, out), g).to(TYPES[ty]).cuda(), whole((rows, width), g).cuda()
    ck = B.zeno_checkpoint(a)
    off = torch.tensor([1, 33, 40], dtype=torch.int32, device="cuda")
    dw, db = B.zeno_weight_gradient(far(dy, (1 << 27) + 1), ck, groups=off)
    for i, (p, q) in enumerate(((1, 33), (33, 40))):
        assert torch.equal(dw[i].double().cpu(), (dy[p:q].double().cpu().T @ a[p:q].double().cpu()).reshape(-1))
        assert torch.equal(db[i].double().cpu(), dy[p:q].double().cpu().sum(0))


def test_a_checkpoint_past_32_bits(B):
    rows, width, last = 70001, 32768, 90
    g = torch.Generator().manual_seed(1)
    ck = B.alloc_checkpoint(rows, width)
    x = whole((last, width), g).bfloat16().cuda()
    end = B.zeno_checkpoint(x, out=B.Checkpoint(ck.values[-last:], ck.scales[-last:], width))
    everything = torch.empty(rows, width, dtype=torch.bfloat16, device="cuda")
    assert torch.equal(B.zeno_checkpoint_values(ck, torch.bfloat16, out=everything)[-last:], x)
    dy = torch.zeros(rows, 40, dtype=torch.bfloat16, device="cuda")
    dy[-last:] = whole((last, 40), g).bfloat16().cuda()
    off = torch.tensor([rows - last, rows], dtype=torch.int32, device="cuda")
    want = dy[-last:].double().cpu().T @ x.double().cpu()
    for out in (3, 40):
        dw, _ = B.zeno_weight_gradient(dy[:, :out], ck, groups=off)
        assert torch.equal(dw[0].double().cpu().reshape(out, width), want[:out])
    ck.values[-last:] = 0
    ck.scales[-last:] = 0
    again = B.zeno_checkpoint(everything, out=ck)
    assert torch.equal(again.values[-last:], B.zeno_checkpoint(x).values) and torch.equal(again.scales[-last:], B.zeno_checkpoint(x).scales)
    w = torch.ones(width, device="cuda")
    _, mean, rstd, _ = B.zeno_layer_norm(x, w)
    allmean, allrstd = torch.zeros(rows, device="cuda"), torch.zeros(rows, device="cuda")
    allmean[-last:], allrstd[-last:] = mean, rstd
    d = torch.zeros(rows, width, dtype=torch.bfloat16, device="cuda")
    d[-last:] = x.flip(1)
    got, gw, gb = B.zeno_layer_norm_backward(d, ck, allmean, allrstd, w, groups=off, dx=everything)
    one, ow, ob = B.zeno_layer_norm_backward(x.flip(1).contiguous(), end, mean, rstd, w)
    assert torch.equal(got[-last:], one) and torch.equal(gb, ob)
    # (the rows are cut into other chunks: as many additions of the same products, in another order)
    assert ((gw - ow).abs() <= 2 * last * 2.0 ** -24 * 4 * last * 10).all()


def test_more_rows_than_workgroups(B):
    """A launch has 2^20 workgroups at most and goes over the rows in steps."""
    rows = (1 << 22) + 5000
    g = torch.Generator().manual_seed(2)
    for vocab in (3, 260):
        z = torch.zeros(rows, vocab, dtype=torch.bfloat16, device="cuda")
        lab = torch.full((rows,), -1, dtype=torch.int32, device="cuda")
        tail = torch.randn(4999, vocab, generator=g).bfloat16().cuda()
        z[-4999:] = tail
        lab[-4999:] = 2
        got = B.zeno_logprobs(z, lab, top=2, want_entropy=True, want_stats=True)
        want = B.zeno_logprobs(tail, lab[-4999:], top=2, want_entropy=True, want_stats=True)
        for p, q in zip(got, want):
            assert torch.equal(p[-4999:], q)
        assert not got[0][:-4999].any() and (got[3][:-4999, 1] == 1).all()
        h = torch.ones(rows, device="cuda")
        d = B.zeno_logprobs_backward(z, got[2], labels=lab, grad_logp=h, out=z)
        assert torch.equal(d[-4999:], B.zeno_logprobs_backward(tail, want[2], labels=lab[-4999:], grad_logp=h[-4999:]))
        assert not d[:-4999].any()


@pytest.mark.parametrize("out,width", [(10, 64), (70, 96)])
def test_the_most_groups(B, out, width):
    g = torch.Generator().manual_seed(3)
    rows, m = 700, 1024
    dy, a = whole((rows, out), g).cuda(), whole((rows, width), g).cuda()
    cuts = torch.sort(torch.randint(0, rows + 1, (m + 1,), generator=g)).values
    G = torch.full((m, out * width + out), 7.0, device="cuda")
    B.zeno_weight_gradient(dy, B.zeno_checkpoint(a), groups=cuts.int().cuda(), dweight=G[:, :out * width], dbias=G[:, out * width:])
    for i in range(m):
        p, q = int(cuts[i]), int(cuts[i + 1])
        assert torch.equal(G[i, :out * width].reshape(out, width), dy[p:q].T @ a[p:q] if q > p else torch.zeros(out, width, device="cuda"))
        assert torch.equal(G[i, out * width:], dy[p:q].sum(0))


def off_line(shape, dtype):
    """A matrix whose rows do not start on memory lines."""
    return torch.empty(shape[0] * (shape[1] + 1) + 1, dtype=dtype, device="cuda").as_strided(shape, (shape[1] + 1, 1), 1)


@pytest.mark.parametrize("ty", list(TYPES))
def test_gradients_on_memory_lines_and_off_them(B, ty):
    """Rows on memory lines are written another way: the same bits."""
    g = torch.Generator().manual_seed(4)
    dt = TYPES[ty]
    for vocab in (128, 300 * 64, 40):
        z = torch.randn(9, vocab, generator=g).to(dt).cuda()
        lab = torch.randint(0, vocab, (9,), generator=g, dtype=torch.int32).cuda()
        _, _, stats, index, _ = B.zeno_logprobs(z, lab, want_stats=True, top=2)
        h, q = torch.randn(9, generator=g).cuda(), torch.randn(9, 2, generator=g).cuda()
        for kw in (dict(), dict(top_index=index, grad_top=q)):
            on, off = (B.zeno_logprobs_backward(z, stats, labels=lab, grad_logp=h, out=o, **kw) for o in (torch.empty_like(z), off_line(z.shape, dt)))
            assert torch.equal(on, off) and not torch.isnan(on).any()
    for width in (1024, 4096, 8192, 12032):
        x, dy = (torch.randn(40, width, generator=g).to(dt).cuda() for _ in range(2))
        w = torch.randn(width, generator=g).cuda()
        _, mean, rstd, _ = B.zeno_layer_norm(x, w)
        on, off = (B.zeno_layer_norm_backward(dy, x, mean, rstd, w, dx=o)[0] for o in (torch.empty_like(x), off_line(x.shape, dt)))
        assert torch.equal(on, off) and not torch.isnan(on).any()


@pytest.mark.parametrize("ty", list(TYPES))
@pytest.mark.parametrize("m,out,width,rows", [(256, 256, 256, 16700), (70, 300, 544, 4600), (40, 128, 128, 900), (256, 264, 288, 17000)])
def test_weight_gradients_on_memory_lines_and_off_them(B, m, out, width, rows, ty):
    """All shapes of tiles, inside the output and across its end; sums of small whole numbers."""
    g = torch.Generator().manual_seed(5)
    dy, a = whole((rows, out), g).to(TYPES[ty]).cuda(), whole((rows, width), g).cuda()
    cuts = torch.tensor([rows * i // m for i in range(m)] + [rows - 3])
    ck = B.zeno_checkpoint(a)
    off = cuts.int().cuda()
    one, one_b = B.zeno_weight_gradient(dy, ck, groups=off)
    G = off_line((m, out * width), torch.float32)
    two, two_b = B.zeno_weight_gradient(dy, ck, groups=off, dweight=G)
    assert torch.equal(one, two) and torch.equal(one_b, two_b)
    d32 = dy.float()
    for i in list(range(0, m, 37)) + [m - 1]:
        p, q = int(cuts[i]), int(cuts[i + 1])
        assert torch.equal(one[i].reshape(out, width), d32[p:q].T @ a[p:q]) and torch.equal(one_b[i], d32[p:q].sum(0))


def test_the_largest_vocabulary(B):
    """2^30 logits a row, shared by workgroups, and 2^23 in one workgroup each: s = sum exp(z - M) is known in closed form."""
    for rows, vocab, ty in ((1, 1 << 30, torch.bfloat16), (1, (1 << 30) - 3, torch.float32), (200, 1 << 23, torch.bfloat16)):
        z = torch.zeros(rows, vocab, dtype=ty, device="cuda")
        z[:, vocab - 1], z[:, vocab // 2 + 1] = 20.0, 10.0
        lab = torch.full((rows,), vocab // 2 + 1, dtype=torch.int32, device="cuda")
        logp, entropy, stats, index, top = B.zeno_logprobs(z, lab, top=4, want_entropy=True, want_stats=True)
        s = 1 + math.exp(-10) + (vocab - 2) * math.exp(-20)
        t = -10 * math.exp(-10) - 20 * (vocab - 2) * math.exp(-20)
        # at most 16384 values a thread and 22 joins; an exponential off by 4 EPS and its argument by EPS |20|
        tol = (16384 + 64) * 2.0 ** -24
        assert (logp.double() - (-10 - math.log(s))).abs().max() <= tol + 16 * 2.0 ** -24
        assert (entropy.double() - (math.log(s) - t / s)).abs().max() <= 40 * tol
        assert (index == torch.tensor([vocab - 1, vocab // 2 + 1, 0, 1], dtype=torch.int32, device="cuda")).all()
        g = torch.ones(rows, device="cuda")
        dz = B.zeno_logprobs_backward(z, stats, labels=lab, grad_logp=g, out=z)
        half = torch.finfo(ty).eps
        for at, want in ((vocab - 1, -1 / s), (vocab // 2 + 1, 1 - math.exp(-10) / s), (vocab - 2, -math.exp(-20) / s), (0, -math.exp(-20) / s)):
            assert (dz[:, at].double() - want).abs().max() <= (half + 2 * tol + 64 * 2.0 ** -24) * abs(want)
        del z, dz


def test_the_widest_rows(B):
    """2^24 columns of layer norm and of a checkpoint, and more weights than 32 bits count."""
    rows, width = 3, 1 << 24
    g = torch.Generator(device="cuda").manual_seed(6)
    x, dy = (torch.randn(rows, width, device="cuda", generator=g) for _ in range(2))
    w = torch.ones(width, device="cuda")
    y, mean, rstd, ck = B.zeno_layer_norm(x, w, want_checkpoint=True)
    alone = B.zeno_checkpoint(x)
    assert torch.equal(ck.values, alone.values) and torch.equal(ck.scales, alone.scales)
    x64 = x.double()
    m64, v64 = x64.mean(1), x64.var(1, unbiased=False)
    k = (16384 + 64) * 2.0 ** -24                    # additions of a thread and its joins, times half a step
    assert ((mean.double() - m64).abs() <= k * x64.abs().mean(1)).all()
    assert ((rstd.double() * (v64 + 1e-5).sqrt() - 1).abs() <= k).all()
    dx, dw, db = B.zeno_layer_norm_backward(dy, x, mean, rstd, w)
    xh = (x64 - mean.double()[:, None]) * rstd.double()[:, None]
    a = dy.double()
    c1, c2 = a.mean(1, keepdim=True), (a * xh).mean(1, keepdim=True)
    tol = rstd.double()[:, None] * (k * (a.abs().mean(1, keepdim=True) + xh.abs() * (a * xh).abs().mean(1, keepdim=True)) + 6 * 2.0 ** -24 * (a.abs() + (xh * c2).abs() + c1.abs()))
    assert ((dx.double() - rstd.double()[:, None] * (a - c1 - xh * c2)).abs() <= tol).all()
    assert ((dw[0].double() - (a * xh).sum(0)).abs() <= 8 * 2.0 ** -24 * (a * xh).abs().sum(0)).all()
    assert ((db[0].double() - a.sum(0)).abs() <= 4 * 2.0 ** -24 * a.abs().sum(0)).all()
    del x64, xh, a, tol, x, dy, y, dx, dw, db
    for rows, out in ((40, 130), (70, 130), (70, 3)):
        gen = torch.Generator().manual_seed(rows)
        a = whole((rows, 1 << 12), gen).cuda().repeat(1, 1 << 12)
        a[:, -5000:] = whole((rows, 5000), gen).cuda()
        dy = whole((rows, out), gen).bfloat16().cuda()
        dw, db = B.zeno_weight_gradient(dy, B.zeno_checkpoint(a))
        dw = dw.view(out, width)
        assert torch.equal(db[0], dy.float().sum(0))
        for o in (0, 1, out // 2, out - 1):
            assert torch.equal(dw[o], dy[:, o].float() @ a)
        del a, dw


@pytest.mark.parametrize("ty", list(TYPES))
def test_a_layer_into_a_large_vocabulary(B, ty):
    """The last layer of a token model: 50257 outputs, whole and in groups."""
    g = torch.Generator().manual_seed(7)
    rows, out, width = 300, 50257, 96
    dy, a = whole((rows, out), g).to(TYPES[ty]).cuda(), whole((rows, width), g).cuda()
    ck = B.zeno_checkpoint(a)
    for cuts in ([0, rows], [3, 100, 100, 101, 290]):
        dw, db = B.zeno_weight_gradient(dy, ck, groups=torch.tensor(cuts, dtype=torch.int32, device="cuda"))
        for i, (p, q) in enumerate(zip(cuts, cuts[1:])):
            d = dy[p:q].float()
            assert torch.equal(dw[i].view(out, width), d.t().contiguous() @ a[p:q]) and torch.equal(db[i], d.sum(0))


@pytest.mark.parametrize("ty", list(TYPES))
def test_large_gradients_on_memory_lines_and_off_them(B, ty):
    """From 128 MiB on, gradients of logits and of activations are written past the caches where their rows start on memory lines."""
    g = torch.Generator(device="cuda").manual_seed(8)
    dt = TYPES[ty]
    size = torch.finfo(dt).bits // 8

    def both(shape, call):
        one, two = call(torch.full(shape, 7.0, dtype=dt, device="cuda")), call(off_line(shape, dt).fill_(7.0))
        assert torch.equal(one, two) and not torch.isnan(one).any()

    for vocab in (128, 192, 4096, 33000 // 64 * 64):
        rows = (1 << 27) // (size * vocab) + 3
        z = torch.randn(rows, vocab, generator=g, device="cuda").to(dt)
        lab = torch.randint(0, vocab, (rows,), generator=g, device="cuda", dtype=torch.int32)
        _, entropy, stats, index, _ = B.zeno_logprobs(z, lab, want_stats=True, want_entropy=True, top=2)
        h, q = torch.randn(rows, generator=g, device="cuda"), torch.randn(rows, 2, generator=g, device="cuda")
        for kw in (dict(), dict(top_index=index, grad_top=q), dict(entropy=entropy, grad_entropy=h)):
            both(z.shape, lambda out: B.zeno_logprobs_backward(z, stats, labels=lab, grad_logp=h, out=out, **kw))
    for width in (512, 1024, 2048, 4096, 8192, 12032, 16384):
        rows = (1 << 27) // (size * width) + 3
        x, dy = (torch.randn(rows, width, generator=g, device="cuda").to(dt) for _ in range(2))
        w = torch.randn(width, generator=g, device="cuda")
        _, mean, rstd, ck = B.zeno_layer_norm(x, w, want_checkpoint=True)
        for src in (x, ck):
            both(x.shape, lambda out: B.zeno_layer_norm_backward(dy, src, mean, rstd, w, dx=out)[0])
