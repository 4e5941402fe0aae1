"""Log probabilities of given tokens, entropy, alternatives and their gradient against their definitions in float64."""
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


def make(rows, vocab, ty, seed, scale=3.0, pitch=None, offset=0):
    g = torch.Generator().manual_seed(seed)
    z = torch.randn(rows, vocab, generator=g) * scale
    labels = torch.randint(0, vocab, (rows,), generator=g, dtype=torch.int32)
    view, buf = T.strided(z, T.TYPES[ty], pitch, offset)
    return view, buf, labels, g


def bounds(ref, vocab, per_load):
    """Absolute bounds of logp-like values and of the entropy.  A part of a row is summed by 64 threads (rows of up to 2048 values)
    or 256, at most 64 parts are joined; an exponential is off by 2 units of the last place (4 EPS) and its argument by EPS |d|,
    which costs at most EPS e^-1 of the sum."""
    k = T.chain(vocab, 64 if vocab <= 2048 else 256, per_load) + 64 + 8
    with np.errstate(invalid="ignore"):
        sums = k * T.EPS
        log_s = np.abs(ref["log_s"])
        stat = sums + 2 * T.EPS * (log_s + 1)
        entropy = 2 * sums * (np.abs(ref["entropy"]) + 2) + 4 * T.EPS * (log_s + np.abs(ref["entropy"]) + 1)
    return stat, entropy


def close(got, want, tol, what):
    got, want = np.asarray(got, dtype=np.float64), np.asarray(want, dtype=np.float64)
    same = (got == want) | (np.isnan(got) & np.isnan(want))
    with np.errstate(invalid="ignore"):
        bad = ~same & ~(np.abs(got - want) <= tol)
    assert not bad.any(), (what, np.argwhere(bad)[:5].tolist(), got[bad][:5], want[bad][:5], np.broadcast_to(tol, got.shape)[bad][:5])


def check_forward(B, z, labels, top, ref=None):
    rows, vocab = z.shape
    per_load = 16 // z.element_size()
    lab = None if labels is None else labels.cuda()
    out = B.zeno_logprobs(z, lab, top=top, want_entropy=True, want_stats=True)
    torch.cuda.synchronize()
    logp, entropy, stats, index, top_logp = [None if o is None else o.cpu().numpy() for o in out]
    ref = ref or T.logprobs(z.double().cpu().numpy(), None if labels is None else labels.numpy(), top)
    stat, ent = bounds(ref, vocab, per_load)
    if labels is not None:
        with np.errstate(invalid="ignore"):
            close(logp, ref["logp"], stat + 3 * T.EPS * (np.abs(ref["logp"]) + np.abs(ref["log_s"])), "logp")
    close(entropy, ref["entropy"], ent, "entropy")
    close(stats[:, 0], ref["M"], 0.0, "max")
    close(stats[:, 1], ref["log_s"], stat, "log_s")
    if top:
        assert np.array_equal(index, ref["index"]), np.argwhere(index != ref["index"])[:5]
        with np.errstate(invalid="ignore"):
            close(top_logp, ref["top_logp"], stat[:, None] + 3 * T.EPS * (np.abs(ref["top_logp"]) + np.abs(ref["log_s"])[:, None]), "top")
    return out, ref


SHAPES = [  # rows, vocab, type, top, extra pitch, offset
    (1, 1, "fp32", 1, 0, 0), (3, 2, "bf16", 2, 0, 1), (5, 10, "fp32", 10, 0, 0), (7, 33, "fp16", 32, 1, 3),
    (130, 257, "bf16", 5, 0, 0), (9, 2048, "fp32", 8, 0, 1), (9, 2049, "fp32", 8, 0, 0), (600, 2500, "bf16", 3, 0, 0),
    (1, 32000, "bf16", 8, 0, 0), (4, 50257, "fp32", 32, 0, 0), (3, 50257, "bf16", 20, 0, 0), (2, 200003, "fp16", 1, 5, 7),
    (520, 8191, "fp16", 0, 1, 0), (513, 4099, "fp32", 32, 0, 2), (65, 20000, "bf16", 4, 0, 0),
]


@pytest.mark.parametrize("rows,vocab,ty,top,extra,offset", SHAPES)
def test_forward(B, rows, vocab, ty, top, extra, offset):
    z, _, labels, _ = make(rows, vocab, ty, rows * 7 + vocab, pitch=vocab + extra, offset=offset)
    if rows > 2:
        labels[1] = -1
    check_forward(B, z, labels, top)


@pytest.mark.parametrize("rows,vocab,ty", [(5, 10, "fp32"), (5, 70, "bf16"), (4, 2049, "fp16"), (520, 2100, "fp32"), (3, 33000, "bf16")])
def test_outputs_alone(B, rows, vocab, ty):
    """Every output may be asked for by itself and is the same as with the others."""
    z, _, labels, _ = make(rows, vocab, ty, 5)
    lab = labels.cuda()
    logp, entropy, stats, index, top_logp = B.zeno_logprobs(z, lab, top=4, want_entropy=True, want_stats=True)
    assert torch.equal(B.zeno_logprobs(z, lab)[0], logp)
    only = B.zeno_logprobs(z, want_entropy=True)
    assert only[0] is None and torch.equal(only[1], entropy)
    assert torch.equal(B.zeno_logprobs(z, want_stats=True)[2], stats)
    only = B.zeno_logprobs(z, top=4)
    assert torch.equal(only[3], index) and torch.equal(only[4], top_logp)


@pytest.mark.parametrize("ty", ["fp32", "bf16", "fp16"])
@pytest.mark.parametrize("rows,vocab", [(6, 40), (6, 2600), (6, 9000), (520, 2600)])
def test_masks(B, rows, vocab, ty):
    """Rows with few tokens left, with one, with none; masks of the type's lowest value; labels that are masked, left out, out of
    range.  More alternatives are asked for than tokens are left."""
    z, _, labels, _ = make(rows, vocab, ty, 11)
    low = torch.finfo(z.dtype).min
    z[0, 3:] = float("-inf")
    z[1, :] = float("-inf")
    z[2, :] = low
    z[3, 1:] = low
    z[4, :-1] = float("-inf")
    z[5, :] = 1.25
    labels[:6] = torch.tensor([1, 0, vocab - 1, 0, 2, -1], dtype=torch.int32)
    (logp, entropy, *_), ref = check_forward(B, z, labels, 7)
    assert float(logp[1]) == -np.inf and float(entropy[1]) == 0.0 and float(logp[4]) == -np.inf
    assert abs(float(entropy[2]) - np.log(vocab)) < 1e-4
    labels[0], labels[1] = vocab, -2
    check_forward(B, z, labels, 7)


@pytest.mark.parametrize("ty", ["fp32", "bf16", "fp16"])
@pytest.mark.parametrize("vocab", [40, 2600, 40000])
def test_values_that_are_not_finite(B, vocab, ty):
    z, _, labels, _ = make(6, vocab, ty, 12)
    z[0, 5] = float("nan")
    z[1, 7] = float("inf")
    z[2, :] = float("nan")
    z[3, 1] = float("inf")
    z[3, 2:] = float("-inf")
    z[4, :] = float("inf")
    check_forward(B, z, labels, 5)


@pytest.mark.parametrize("ty", ["fp32", "bf16"])
@pytest.mark.parametrize("vocab", [40, 2600, 20000])
def test_logits_at_the_ends_of_the_range(B, vocab, ty):
    """Large logits: log2(e) times them is out of float32's range; and an offset that cancels."""
    z, _, labels, _ = make(5, vocab, ty, 13)
    z[0, :] = -3.2e38
    z[0, 5] = -3.0e38
    z[1, :] = 1.0
    z[1, 9] = 3.3e38
    z[2, :] = 3.3e38
    z[3, :] += 30000.0
    z[4, :] = -1.5e38
    check_forward(B, z, labels, 5)


@pytest.mark.parametrize("rows,vocab,ty", [(3, 700, "bf16"), (3, 5000, "fp32"), (2, 70000, "bf16"), (600, 3000, "fp16")])
@pytest.mark.parametrize("kind", ["equal", "few", "rising", "crowded", "ties", "signed zeros"])
def test_alternatives_of_rows_that_are_hard_to_choose_from(B, rows, vocab, ty, kind):
    """Ties go to the lower index, in rows of one value, of few values, sorted rows, rows whose largest values crowd in the shares
    of few threads, rows with many copies of the k-th value."""
    g = torch.Generator().manual_seed(14)
    if kind == "equal":
        z = torch.zeros(rows, vocab)
    elif kind == "few":
        z = torch.randint(0, 3, (rows, vocab), generator=g).float()
    elif kind == "rising":
        z = torch.arange(vocab).float().expand(rows, vocab) / 64
    elif kind == "crowded":
        # every thread of a workgroup owns 16 bytes in each of its steps: one thread's columns hold the large values
        n = 16 // torch.tensor([], dtype=T.TYPES[ty]).element_size()
        z = torch.rand(rows, vocab, generator=g)
        for threads in (64, 256):
            for j in range(n):
                z[:, 5 * n + j::threads * n] += 10
    elif kind == "ties":
        z = torch.rand(rows, vocab, generator=g)
        z[:, vocab // 3:] = 2.0
        z[:, vocab // 2] = 3.0
    else:
        z = -torch.zeros(rows, vocab)
        z[:, ::3] = 0.0
    view, _ = T.strided(z, T.TYPES[ty])
    for top in (1, 7, 32):
        check_forward(B, view, None, top)


def grad_reference(ref, labels, g, h, q, index, vocab):
    rows = len(ref["M"])
    p, lp = np.nan_to_num(ref["p"], nan=np.nan), np.where(ref["p"] > 0, ref["lp"], 0.0)
    add = np.zeros((rows, vocab))
    total = np.zeros(rows)
    mag = np.zeros((rows, vocab))
    for r in range(rows):
        if g is not None and labels[r] != -1:
            if 0 <= labels[r] < vocab:
                add[r, labels[r]] += g[r]
                mag[r, labels[r]] += abs(g[r])
                total[r] += g[r]
            else:
                total[r] = np.nan
        if q is not None:
            for k in range(q.shape[1]):
                add[r, index[r, k]] += q[r, k]
                mag[r, index[r, k]] += abs(q[r, k])
                total[r] += q[r, k]
    h = np.zeros(rows) if h is None else h
    inner = total[:, None] + h[:, None] * (lp + ref["entropy"][:, None])
    with np.errstate(invalid="ignore"):
        dz = add - p * inner
    dz[ref["empty"]] = 0.0
    return dz, mag, np.abs(h)[:, None] * (np.abs(lp) + np.abs(ref["entropy"])[:, None])


def check_backward(B, z, labels, use_g=True, use_h=True, top=0, in_place=False, out=None, seed=3):
    rows, vocab = z.shape
    gen = torch.Generator().manual_seed(seed)
    lab = labels.cuda()
    ref = T.logprobs(z.double().cpu().numpy(), labels.numpy(), top)
    _, entropy, stats, index, _ = B.zeno_logprobs(z, lab, top=top, want_entropy=True, want_stats=True)
    g = torch.randn(rows, generator=gen) if use_g else None
    h = torch.randn(rows, generator=gen) * 0.3 if use_h else None
    q = torch.randn(rows, top, generator=gen) if top else None
    dev = lambda t: None if t is None else t.cuda()
    if in_place:
        out = z
    got = B.zeno_logprobs_backward(z, stats, labels=lab if use_g else None, grad_logp=dev(g), entropy=entropy if use_h else None,
                                   grad_entropy=dev(h), top_index=index if top else None, grad_top=dev(q), out=out)
    torch.cuda.synchronize()
    npd = lambda t: None if t is None else t.double().numpy()
    want, mag, ent_part = grad_reference(ref, labels.numpy(), npd(g), npd(h), npd(q), ref["index"], vocab)
    per_load = 16 // z.element_size()
    stat, ent = bounds(ref, vocab, per_load)
    with np.errstate(invalid="ignore"):
        lp_err = stat + 6 * T.EPS * (np.abs(np.where(ref["p"] > 0, ref["lp"], 0.0)).max(1) + np.abs(ref["log_s"]) + 1)
        gsum = (np.abs(npd(g)) if g is not None else 0) + (np.abs(npd(q)).sum(1) if q is not None else 0) + np.zeros(rows)
        hh = np.abs(npd(h)) if h is not None else np.zeros(rows)
        tol = ref["p"] * (gsum[:, None] + ent_part) * (lp_err[:, None] + (top + 8) * T.EPS) \
            + ref["p"] * (hh * (lp_err + ent))[:, None] + (top + 3) * T.EPS * mag
        tol = tol * 2 + np.abs(want) * T.half_step(z.dtype) * (1 + 2 ** -6) + T.smallest_half(z.dtype)
    close(got.double().cpu().numpy(), want, tol, "dlogits")
    return got


@pytest.mark.parametrize("rows,vocab,ty,top,extra,offset", SHAPES)
def test_backward(B, rows, vocab, ty, top, extra, offset):
    z, _, labels, _ = make(rows, vocab, ty, rows * 5 + vocab, pitch=vocab + extra, offset=offset)
    if rows > 2:
        labels[1] = -1
    check_backward(B, z, labels)
    if top:
        check_backward(B, z, labels, top=top)
        check_backward(B, z, labels, use_g=False, use_h=False, top=min(top, 3))
    check_backward(B, z, labels, use_h=False)
    check_backward(B, z, labels, use_g=False)


@pytest.mark.parametrize("ty", ["fp32", "bf16", "fp16"])
@pytest.mark.parametrize("vocab", [40, 2600, 20000])
def test_backward_of_masked_rows_and_labels(B, vocab, ty):
    z, _, labels, _ = make(7, vocab, ty, 17)
    z[0, 3:] = float("-inf")
    z[1, :] = float("-inf")
    z[2, :] = torch.finfo(z.dtype).min
    z[4, 6] = float("nan")
    labels[:7] = torch.tensor([1, 0, 5, vocab, 2, -1, -7], dtype=torch.int32)
    got = check_backward(B, z, labels, top=4)
    assert not got[1].any() and torch.isnan(got[3]).all() and torch.isnan(got[4]).all()


@pytest.mark.parametrize("vocab,ty,top", [(10, "fp32", 3), (500, "bf16", 0), (9000, "fp16", 32), (33000, "bf16", 5)])
def test_backward_in_place_and_what_lies_around(B, vocab, ty, top):
    z, buf, labels, _ = make(5, vocab, ty, 19, pitch=vocab + 3, offset=5)
    before = T.around(z, buf)
    keep = z.clone()
    got = check_backward(B, keep.clone(), labels, top=top)
    again = check_backward(B, z, labels, top=top, in_place=True)
    assert torch.equal(got, again)
    after = T.around(z, buf)
    assert torch.isnan(before).all() and torch.isnan(after).all()


def test_the_same_alternative_twice(B):
    """An index that stands twice counts twice, also where it is the label."""
    z, _, labels, _ = make(3, 300, "fp32", 23)
    labels[:] = 7
    _, _, stats, _, _ = B.zeno_logprobs(z, labels.cuda(), want_stats=True)
    index = torch.tensor([[7, 7], [9, 9], [0, 299]], dtype=torch.int32)
    q = torch.tensor([[1.0, 2.0], [0.5, -0.5], [1.0, 1.0]])
    g = torch.tensor([3.0, 1.0, 1.0])
    got = B.zeno_logprobs_backward(z, stats, labels=labels.cuda(), grad_logp=g.cuda(), top_index=index.cuda(), grad_top=q.cuda())
    ref = T.logprobs(z.double().cpu().numpy(), labels.numpy(), 2)
    want, _, _ = grad_reference(ref, labels.numpy(), g.double().numpy(), None, q.double().numpy(), index.numpy(), 300)
    # |dz| <= 12: six roundings of float32 and those of the statistics
    assert np.abs(got.double().cpu().numpy() - want).max() <= 12 * (40 * T.EPS)
    index[1, 1] = 300
    got = B.zeno_logprobs_backward(z, stats, top_index=index.cuda(), grad_top=q.cuda())
    assert torch.isnan(got[1]).all() and not torch.isnan(got[0]).any()


def test_gradient_against_differences(B):
    """Central differences of sum(g logp + h H + q top) in float64 of the definition, at the kernel's gradient in float32."""
    z, _, labels, _ = make(2, 12, "fp32", 29, scale=1.0)
    top = 3
    base = T.logprobs(z.double().cpu().numpy(), labels.numpy(), top)
    gen = torch.Generator().manual_seed(31)
    g, h, q = torch.randn(2, generator=gen), torch.randn(2, generator=gen), torch.randn(2, top, generator=gen)
    _, entropy, stats, index, _ = B.zeno_logprobs(z, labels.cuda(), top=top, want_entropy=True, want_stats=True)
    got = B.zeno_logprobs_backward(z, stats, labels=labels.cuda(), grad_logp=g.cuda(), entropy=entropy, grad_entropy=h.cuda(),
                                   top_index=index, grad_top=q.cuda()).double().cpu().numpy()

    def value(zz):
        r = T.logprobs(zz, labels.numpy(), top)
        return (g.double().numpy() * r["logp"]).sum() + (h.double().numpy() * r["entropy"]).sum() + \
            (q.double().numpy() * np.take_along_axis(r["lp"], base["index"], 1)).sum()

    z64, step = z.double().cpu().numpy(), 1e-5
    for r in range(2):
        for j in range(12):
            up, down = z64.copy(), z64.copy()
            up[r, j] += step
            down[r, j] -= step
            # truncation step^2 / 6 times a third derivative of at most about 50, rounding 2^-52 |value| / step
            assert abs((value(up) - value(down)) / (2 * step) - got[r, j]) <= 50 * step ** 2 + 1e-9 + 64 * T.EPS * 4


def test_long_rows_of_many(B):
    """Offsets past 2^31 elements: the last rows of a matrix of 4.4 GB of logits."""
    vocab, rows = 65536, 33000
    z = torch.zeros(rows, vocab, dtype=torch.bfloat16, device="cuda")
    tail, _, labels, _ = make(3, vocab, "bf16", 37)
    z[-3:] = tail
    lab = torch.full((rows,), -1, dtype=torch.int32, device="cuda")
    lab[-3:] = labels.cuda()
    logp, entropy, stats, index, top_logp = B.zeno_logprobs(z, lab, top=2, want_entropy=True, want_stats=True)
    ref = T.logprobs(tail.double().cpu().numpy(), labels.numpy(), 2)
    stat, ent = bounds(ref, vocab, 8)
    close(logp[-3:].cpu().numpy(), ref["logp"], stat + 3 * T.EPS * (np.abs(ref["logp"]) + np.abs(ref["log_s"])), "logp")
    assert np.array_equal(index[-3:].cpu().numpy(), ref["index"]) and not logp[:-3].any()
    g = torch.ones(rows, device="cuda")
    d = B.zeno_logprobs_backward(z, stats, labels=lab, grad_logp=g, out=z)
    assert not d[:100].any()
    dz = d[-3:].double().cpu().numpy()
    want = -ref["p"]
    want[np.arange(3), labels.numpy()] += 1
    close(dz, want, np.abs(want) * 2.0 ** -8 * 1.01 + ref["p"] * 200 * T.EPS + 2 * T.EPS, "dlogits")


def test_no_rows(B):
    z = torch.empty(0, 50, device="cuda")
    logp, entropy, stats, index, top = B.zeno_logprobs(z, torch.empty(0, dtype=torch.int32, device="cuda"), top=3, want_entropy=True,
                                                       want_stats=True)
    assert logp.shape == (0,) and index.shape == (0, 3)
    assert B.zeno_logprobs_backward(z, stats, labels=torch.empty(0, dtype=torch.int32, device="cuda"), grad_logp=logp).shape == (0, 50)


@pytest.mark.parametrize("vocab,ty", [(15, "fp32"), (64, "fp32"), (65, "fp32"), (127, "bf16"), (128, "fp16"), (129, "bf16"), (255, "fp16"),
                                      (256, "fp32"), (256, "bf16")])
def test_few_values(B, vocab, ty):
    """Rows that sixteen lanes hold, in one piece a lane and in several: masked, tied and broken rows, all the alternatives there are."""
    z, _, labels, _ = make(70, vocab, ty, 40 + vocab, pitch=vocab + 1, offset=1)
    z[0, 2:] = float("-inf")
    z[1, :] = float("-inf")
    z[2, :] = torch.finfo(z.dtype).min
    z[3, :] = 0.5
    z[4, vocab // 2] = float("nan")
    z[5, vocab - 1] = float("inf")
    z[6, vocab - 1] = z[6, 0]
    check_forward(B, z, labels, min(vocab, 32))
    check_forward(B, z, labels, 1)


def far_rows(vocab, fill, seed):
    """Rows with masks and logits of the size of `fill`, whole and in part: log2(e) times them has no fraction left in float32."""
    g = torch.Generator().manual_seed(seed)
    z = torch.randn(10, vocab, generator=g) * 3
    z[0, :] = fill
    z[1, :vocab // 2] = fill                                  # every thread's first pieces, none of its last
    z[2, torch.rand(vocab, generator=g) < 0.5] = fill
    z[3, 1:] = fill
    z[4, :] = fill
    z[4, 3 * vocab // 4:] = fill / 2                          # two sizes, both large
    z[5, vocab // 3] = -fill
    z[6, :] = -fill
    z[7, :] = torch.linspace(1, 0, vocab) * fill              # rises step by step
    z[8, vocab // 2:] = fill
    z[9, :] = fill + torch.linspace(0, 1, vocab) * 4000       # (the same value again where fill is that much larger)
    return z


@pytest.mark.parametrize("rows,vocab", [(10, 40), (10, 250), (10, 700), (10, 2600), (10, 20000), (520, 2600), (10, 70000)])
@pytest.mark.parametrize("ty", ["fp32", "bf16"])
@pytest.mark.parametrize("fill", [-3e4, -1.7e7, -1e8, -6e8, -1e9, -2e9, -1e10, -1e12, -1e20, -1e30, -1e38, 1e10, 1e30])
def test_large_finite_logits(B, rows, vocab, ty, fill):
    """Masks and logits of any finite size, in rows of one wave, of four, of sixteen and in rows shared by workgroups."""
    z = far_rows(vocab, fill, 51)
    g = torch.Generator().manual_seed(53)
    if rows > 10:
        z = torch.cat([torch.randn(rows - 10, vocab, generator=g), z])
    view, _ = T.strided(z, T.TYPES[ty])
    labels = torch.randint(0, vocab, (rows,), generator=g, dtype=torch.int32)
    labels[-3] = 0
    _, ref = check_forward(B, view, labels, 6)
    assert np.isfinite(ref["log_s"]).all()
    if fill in (-1e10, -1e30, 1e10):
        check_backward(B, view, labels, top=6)


SIGNALLING = {"fp32": (torch.int32, 0x7f800001), "bf16": (torch.int16, 0x7f81), "fp16": (torch.int16, 0x7c01)}


@pytest.mark.parametrize("ty", list(SIGNALLING))
@pytest.mark.parametrize("rows,vocab", [(16, 40), (16, 300), (16, 2600), (16, 20000), (530, 2600), (16, 70000)])
def test_signalling_nan_beside_the_largest(B, rows, vocab, ty):
    """A NaN that has not been quieted takes nothing with it: the others keep their ranks and the maximum is theirs."""
    z, _, labels, _ = make(rows, vocab, ty, 57)
    bits, code = SIGNALLING[ty]
    for r in range(16):
        z[rows - 16 + r, 16 + r] = 60.0
        z.view(bits)[rows - 16 + r, 16 + (r ^ 1)] = code
    check_forward(B, z, labels, 5)


@pytest.mark.parametrize("rows,vocab,ty,lanes", [(3, 60000, "fp32", 1), (3, 60000, "bf16", 31), (514, 40000, "fp32", 1), (514, 9000, "bf16", 31),
                                                 (5, 2048, "fp32", 31), (5, 2047, "fp16", 31), (1, 1 << 20, "bf16", 31), (2, 300000, "fp32", 20)])
def test_more_of_the_largest_in_few_lanes_than_the_list_holds(B, rows, vocab, ty, lanes):
    """The bound of the k-th value comes from 64 lanes' maxima: with the largest values in fewer than k of them it lies below more values
    than are kept, which may be all different, in a few groups of equal ones, or equal with one of them infinite."""
    n = 16 // torch.tensor([], dtype=T.TYPES[ty]).element_size()
    g = torch.Generator().manual_seed(61)
    lane = torch.arange(vocab) // n % 64
    held = lane < lanes
    assert int(held.sum()) > 512
    z = torch.rand(rows, vocab, generator=g)
    z[:, held] = 10 + torch.randint(0, 3000, (rows, int(held.sum())), generator=g).float() / 8
    z[rows - 1, held] = 20.0
    if rows > 1:
        z[0, held] = 10 + torch.randint(0, 3, (int(held.sum()),), generator=g).float()
    view, _ = T.strided(z, T.TYPES[ty])
    for top in (lanes + 1, 32):
        check_forward(B, view, None, top)
    if ty == "fp32":
        z[0, 4 * 64 + 1] = float("-inf")
        z[rows - 1, 4 * 64 + 2] = float("inf")
        view, _ = T.strided(z, T.TYPES[ty])
        check_forward(B, view, None, 32)
