"""Embedding and its gradient per worker against float64, with bounds that count roundings: a looked-up value is one product in float32
and one rounding to the output's type; a gradient is a sum of n terms in float32, whose longest chain of additions is no longer than n, and one product."""
import numpy as np
import pytest
import torch

from _tokens import EPS, TYPES, around, half_step, smallest_half, strided

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def B():
    from paper_1805_10032_amd import binding
    binding.load_library()
    return binding


def ids_of(rng, rows, vocab, kind="zipf"):
    if kind == "one":
        return np.full(rows, vocab - 1, dtype=np.int32)
    if kind == "distinct":
        return rng.permutation(max(rows, vocab))[:rows].astype(np.int32) % vocab
    ids = (np.exp(rng.random(rows) * np.log(vocab + 1)).astype(np.int64) - 1).clip(0, vocab - 1).astype(np.int32)
    ids[rng.random(rows) < 0.05] = -1
    return ids


def reference(dy, ids, vocab, scale, offsets):
    """(gradients, sums of magnitudes, counts) in float64, [m x vocab x width]."""
    m, width = len(offsets) - 1, dy.shape[1]
    grad, size, count = np.zeros((m, vocab, width)), np.zeros((m, vocab, width)), np.zeros((m, vocab, 1))
    for g in range(m):
        mine = np.arange(offsets[g], offsets[g + 1])
        mine = mine[(ids[mine] >= 0) & (ids[mine] < vocab)]
        np.add.at(grad[g], ids[mine], dy[mine])
        np.add.at(size[g], ids[mine], np.abs(dy[mine]))
        np.add.at(count[g], ids[mine], 1)
    return grad * scale, size * abs(scale), count


def check(got, ref, size, count, before=0.0):
    got = got.double().cpu().numpy().reshape(ref.shape)
    # n additions, the product with the scale, and the addition to what was there
    bound = (count + 1) * EPS * size * 1.001 + EPS * (np.abs(ref) + 2 * np.abs(before)) + 2.0 ** -126
    bound = np.where((count == 0) & (np.abs(before) == 0), 0.0, bound)
    err = np.abs(got - (ref + before))
    assert (err <= bound).all(), (float(err.max()), np.argwhere(err > bound)[:5].tolist())


@pytest.mark.parametrize("table_type", TYPES)
@pytest.mark.parametrize("out_type", TYPES)
@pytest.mark.parametrize("rows,vocab,width,pitch,offset", [(1, 1, 1, 1, 0), (3, 5, 7, 9, 1), (1, 32000, 64, 64, 0), (130, 11, 8, 8, 3),
                                                           (77, 1000, 515, 517, 1), (9000, 300, 40, 40, 0), (8193, 17, 9, 12, 5), (64, 50, 1030, 1032, 0)])
def test_lookup(B, table_type, out_type, rows, vocab, width, pitch, offset):
    rng = np.random.default_rng(rows * 7 + width)
    tt, ot = TYPES[table_type], TYPES[out_type]
    table, _ = strided(torch.from_numpy(rng.standard_normal((vocab, width))), tt, pitch, offset)
    ids = ids_of(rng, rows, vocab)
    ids[0] = vocab - 1
    if rows > 2:
        ids[1], ids[2] = vocab, -2
    out, buf = strided(torch.zeros(rows, width), ot, pitch, offset)
    before = around(out, buf)
    scale = 1.7
    B.zeno_embedding(torch.from_numpy(ids).cuda(), table, scale=scale, out=out)
    got = out.double().cpu().numpy()
    bad = (ids < -1) | (ids >= vocab)
    ref = table.double().cpu().numpy()[np.where(bad | (ids < 0), 0, ids)] * np.float64(np.float32(scale))
    ref[ids == -1] = 0
    assert np.isnan(got[bad]).all()
    err = np.abs(got - ref)[~bad]
    assert (err <= np.abs(ref[~bad]) * (EPS + half_step(ot)) * 1.001 + smallest_half(ot)).all()
    assert torch.equal(before.isnan(), around(out, buf).isnan())


def test_lookup_far_rows(B):
    """Offsets past 2^31 elements."""
    vocab, width = 70000, 32768
    table = torch.zeros(vocab, width, dtype=torch.bfloat16, device="cuda")
    table[-1] = torch.arange(width, device="cuda") % 251
    table[65537] = 3.0
    out = B.zeno_embedding(torch.tensor([vocab - 1, 0, 65537], dtype=torch.int32, device="cuda"), table)
    assert torch.equal(out[0].float().cpu(), (torch.arange(width) % 251).float())
    assert (out[1] == 0).all() and (out[2] == 3).all()


def test_lookup_keeps_specials(B):
    table = torch.tensor([[float("inf")], [float("nan")], [-0.0], [3e38]], device="cuda")
    out = B.zeno_embedding(torch.tensor([0, 1, 2, 3, -1], dtype=torch.int32, device="cuda"), table, scale=2.0).flatten()
    assert out[0] == float("inf") and out[1].isnan() and out[2] == 0 and torch.signbit(out[2]) and out[3] == float("inf") and out[4] == 0


CASES = [
    # rows, vocab, width, offsets, ids
    (1, 1, 1, None, "zipf"),
    (5, 3, 2, [0, 2, 2, 5], "zipf"),
    (31, 7, 9, [1, 20, 20, 29], "zipf"),
    (32, 4, 8, None, "one"),
    (33, 4, 8, None, "one"),
    (64, 1, 17, None, "one"),
    (65, 100, 16, None, "distinct"),
    (700, 13, 515, [0, 300, 301, 690], "zipf"),
    (2000, 500, 64, [0, 2000], "one"),
    (8192, 300, 24, [100, 3000, 3000, 8000], "zipf"),
    (16384, 300, 24, [100, 3000, 3000, 16000], "zipf"),
    (16385, 300, 24, [100, 3000, 3000, 16000], "zipf"),
    (16384, 70000, 2, [0, 9000, 16384], "zipf"),
    (8193, 300, 24, [100, 3000, 3000, 8000], "zipf"),
    (8200, 3, 5, None, "one"),
    (9000, 10000, 12, None, "distinct"),
    (20011, 2000, 33, [0] + [700 * i for i in range(1, 28)] + [20011], "zipf"),
    (70000, 50, 4, [0, 10, 69990], "zipf"),
    (70001, 2100, 3, [0, 65000, 70001], "one"),
]


@pytest.mark.parametrize("ty", TYPES)
@pytest.mark.parametrize("case", range(len(CASES)))
def test_gradient(B, case, ty):
    rows, vocab, width, offsets, kind = CASES[case]
    rng = np.random.default_rng(case)
    dtype = TYPES[ty]
    dy, _ = strided(torch.from_numpy(rng.standard_normal((rows, width))), dtype, width + case % 3, case % 4)
    ids = ids_of(rng, rows, vocab, kind)
    if rows > 40:
        ids[[3, 17]] = [vocab, -7]
    off = offsets or [0, rows]
    m = len(off) - 1
    G, buf = strided(torch.full((m, vocab * width), 7.0), torch.float32, vocab * width + case % 5, case % 7)
    before = around(G, buf)
    groups = None if offsets is None else torch.tensor(offsets, dtype=torch.int32, device="cuda")
    dev_ids = torch.from_numpy(ids).cuda()
    B.zeno_embedding_backward(dy, dev_ids, vocab, scale=0.75, groups=groups, dtable=G)
    ref, size, count = reference(dy.double().cpu().numpy(), ids, vocab, 0.75, off)
    check(G, ref, size, count)
    assert torch.equal(before.isnan(), around(G, buf).isnan())
    again = B.zeno_embedding_backward(dy, dev_ids, vocab, scale=0.75, groups=groups)
    assert torch.equal(again, G)
    # added to what is there
    start = torch.from_numpy(rng.standard_normal((m, vocab * width))).float().cuda()
    more = start.clone()
    B.zeno_embedding_backward(dy, dev_ids, vocab, scale=0.75, groups=groups, dtable=more, accumulate=True)
    before_sum = start.double().cpu().numpy().reshape(ref.shape)
    check(more, ref, size, count, before_sum)
    untouched = np.broadcast_to(count == 0, ref.shape)
    assert (more.cpu().numpy().reshape(ref.shape)[untouched] == start.cpu().numpy().reshape(ref.shape)[untouched]).all()


def test_gradient_against_differences(B):
    """sum(out * c) moves by scale * sum_t c_t h when a table row moves by h: the lookup is linear, so differences in float64 are exact."""
    rng = np.random.default_rng(5)
    vocab, width, rows = 6, 5, 40
    table = torch.from_numpy(rng.integers(-8, 9, (vocab, width))).float().cuda()
    c = torch.from_numpy(rng.integers(-4, 5, (rows, width))).float().cuda()
    ids = torch.from_numpy(ids_of(rng, rows, vocab)).cuda()
    grad = B.zeno_embedding_backward(c, ids, vocab, scale=0.5).view(vocab, width)
    base = (B.zeno_embedding(ids, table, scale=0.5) * c).double().sum()
    for v in range(vocab):
        for k in range(width):
            moved = table.clone()
            moved[v, k] += 1.0
            assert ((B.zeno_embedding(ids, moved, scale=0.5) * c).double().sum() - base).item() == grad[v, k].item()


def test_gradient_without_rows(B):
    G = torch.full((2, 50 * 9 + 3), 5.0, device="cuda")
    out = G[:, 1:1 + 450]
    B.zeno_embedding_backward(torch.empty(0, 9, device="cuda"), torch.empty(0, dtype=torch.int32, device="cuda"), 50,
                              groups=torch.zeros(3, dtype=torch.int32, device="cuda"), dtable=out)
    assert (out == 0).all() and (G[:, 0] == 5).all() and (G[:, 451:] == 5).all()
    B.zeno_embedding_backward(torch.empty(0, 9, device="cuda"), torch.empty(0, dtype=torch.int32, device="cuda"), 50,
                              groups=torch.zeros(3, dtype=torch.int32, device="cuda"), dtable=G[:, 1:451], accumulate=True)
    assert (out == 0).all()
    assert B.zeno_embedding(torch.empty(0, dtype=torch.int32, device="cuda"), torch.ones(4, 4, device="cuda")).shape == (0, 4)


@pytest.mark.parametrize("rows", [100, 9000])
def test_broken_offsets_stay_inside(B, rows):
    """Offsets that do not ascend or leave the batch: nothing outside the arguments is touched."""
    vocab, width = 20, 8
    G, buf = strided(torch.zeros(3, vocab * width), torch.float32, vocab * width + 40, 20)
    before = around(G, buf)
    dy = torch.ones(rows, width, device="cuda")
    ids = torch.arange(rows, dtype=torch.int32, device="cuda") % 25
    for bad in ([5, 3, 2, 90], [-4, 10, 1 << 30, 20], [1 << 30, 1 << 30, -1, 7]):
        B.zeno_embedding_backward(dy, ids, vocab, groups=torch.tensor(bad, dtype=torch.int32, device="cuda"), dtable=G)
    torch.cuda.synchronize()
    assert torch.equal(before.isnan(), around(G, buf).isnan())


def test_columns_past_32_bits(B):
    """A table of more than 2^31 values per worker."""
    vocab, width = 70000, 32768
    dy = torch.ones(3, width, dtype=torch.bfloat16, device="cuda")
    G = torch.full((1, vocab * width), 9.0, device="cuda")
    B.zeno_embedding_backward(dy, torch.tensor([69999, 69999, 0], dtype=torch.int32, device="cuda"), vocab, dtable=G)
    table = G.view(vocab, width)
    assert (table[-1] == 2).all() and (table[0] == 1).all() and table.sum(dtype=torch.float64).item() == 3 * width
    assert (table[1:-1] == 0).all()


@pytest.mark.parametrize("rows", [300, 20000])
def test_captured(B, rows):
    """A captured pass, replayed with other inputs and eager work between the replays."""
    rng = np.random.default_rng(1)
    vocab, width = 90, 40
    ids = torch.from_numpy(ids_of(rng, rows, vocab)).cuda()
    table = torch.randn(vocab, width, device="cuda")
    dy = torch.randn(rows, width, device="cuda")
    groups = torch.tensor([0, rows // 3, rows], dtype=torch.int32, device="cuda")
    ws = B.alloc_embedding_workspace(rows, vocab, width, 2)
    out, G = torch.empty(rows, width, device="cuda"), torch.empty(2, vocab * width, device="cuda")

    def call():
        B.zeno_embedding(ids, table, scale=2.0, out=out)
        B.zeno_embedding_backward(dy, ids, vocab, scale=2.0, groups=groups, dtable=G, workspace=ws)

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        call()
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call()
    for i in range(4):
        ids.copy_(torch.from_numpy(ids_of(rng, rows, vocab)).cuda())
        dy.normal_()
        G.fill_(float("nan"))
        out.fill_(float("nan"))
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, B.zeno_embedding(ids, table, scale=2.0))
        assert torch.equal(G, B.zeno_embedding_backward(dy, ids, vocab, scale=2.0, groups=groups))


def test_lookup_of_a_large_output(B):
    """160 MB on memory lines, which go past the caches."""
    table = torch.randn(300, 4096, device="cuda")
    ids = torch.randint(-1, 300, (20000,), device="cuda", dtype=torch.int32)
    out = B.zeno_embedding(ids, table, torch.bfloat16, scale=4.0)
    want = (table[ids.long().clamp(min=0)] * 4.0).bfloat16()
    want[ids < 0] = 0
    assert torch.equal(out, want)
