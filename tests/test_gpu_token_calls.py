"""How the token operators are called: captured into a graph and replayed, on another stream, two at once, with workspaces that held
something else, with wrong arguments."""
import pytest
import torch

from tests import _tokens as T

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def B():
    from paper_1805_10032_amd import binding
    binding.load_library()
    return binding


class Step:
    """One pass through all operators on buffers of its own; run() only enqueues and allocates nothing."""

    def __init__(self, B, dtype, rows=300, width=260, vocab=2500, m=3, split=False):
        self.B, self.dtype = B, dtype
        dev = "cuda"
        if split:
            rows, vocab = 3, 70000                      # a row shared by several workgroups
        self.rows = rows
        f32 = torch.float32
        self.x = torch.empty(rows, width, device=dev, dtype=dtype)
        self.weight, self.bias = torch.empty(width, device=dev), torch.empty(width, device=dev)
        self.logits = torch.empty(rows, vocab, device=dev, dtype=dtype)
        self.labels = torch.empty(rows, device=dev, dtype=torch.int32)
        self.g, self.h, self.q = (torch.empty(s, device=dev) for s in ((rows,), (rows,), (rows, 4)))
        self.groups = torch.tensor([0, rows // 3, rows // 3, rows], device=dev, dtype=torch.int32)
        self.dy = torch.empty(rows, width, device=dev, dtype=dtype)
        self.y, self.dx = torch.empty_like(self.x), torch.empty_like(self.x)
        self.mean, self.rstd = torch.empty(rows, device=dev), torch.empty(rows, device=dev)
        self.ckpt = B.alloc_checkpoint(rows, width)
        self.values = torch.empty(rows, width, device=dev, dtype=dtype)
        self.G = torch.empty(m, width * width + 3 * width, device=dev)
        self.logp, self.entropy, self.stats = torch.empty(rows, device=dev), torch.empty(rows, device=dev), torch.empty(rows, 2, device=dev)
        self.index, self.top = torch.empty(rows, 4, device=dev, dtype=torch.int32), torch.empty(rows, 4, device=dev)
        self.dlogits = torch.empty_like(self.logits)
        self.lp = torch.empty(m, rows, device=dev)
        self.scores = torch.empty(m, device=dev)
        self.ws = [B.alloc_logprobs_workspace(rows, vocab, 4), B.alloc_layer_norm_workspace(rows, width, m),
                   B.alloc_weight_gradient_workspace(rows, width, width, m), B.alloc_score_logprobs_workspace(m, self.G.shape[1])]

    def fill(self, seed):
        g = torch.Generator(device="cuda")
        g.manual_seed(seed)
        for t in (self.x, self.weight, self.bias, self.logits, self.g, self.h, self.q, self.dy, self.lp):
            t.copy_(torch.randn(t.shape, generator=g, device="cuda"))
        self.labels.copy_(torch.randint(-1, self.logits.shape[1], self.labels.shape, generator=g, device="cuda"))
        for w in self.ws:
            w.fill_(255)                                # NaN, whatever type it is read as
        return self

    def run(self):
        B, n = self.B, self.x.shape[1]
        B.zeno_layer_norm(self.x, self.weight, self.bias, y=self.y, mean=self.mean, rstd=self.rstd, checkpoint=self.ckpt)
        B.zeno_checkpoint_values(self.ckpt, out=self.values)
        B.zeno_logprobs(self.logits, self.labels, top=4, logp=self.logp, entropy=self.entropy, stats=self.stats, top_index=self.index,
                        top_logp=self.top, workspace=self.ws[0])
        B.zeno_logprobs_backward(self.logits, self.stats, labels=self.labels, grad_logp=self.g, entropy=self.entropy,
                                 grad_entropy=self.h, top_index=self.index, grad_top=self.q, out=self.dlogits)
        B.zeno_layer_norm_backward(self.dy, self.ckpt, self.mean, self.rstd, self.weight, groups=self.groups, dx=self.dx,
                                   dweight=self.G[:, :n], dbias=self.G[:, n:2 * n], workspace=self.ws[1])
        B.zeno_weight_gradient(self.dy, self.ckpt, groups=self.groups, dweight=self.G[:, 2 * n:2 * n + n * n],
                               dbias=self.G[:, 2 * n + n * n:], workspace=self.ws[2])
        B.zeno_score_logprobs(self.G, self.logp, self.lp, 1e-3, labels=self.labels, scores=self.scores, workspace=self.ws[3])

    def outputs(self):
        return [t.clone() for t in (self.y, self.mean, self.rstd, self.ckpt.values, self.ckpt.scales, self.values, self.dx, self.G, self.logp,
                                    self.entropy, self.stats, self.index, self.top, self.dlogits, self.scores)]


def same(a, b):
    return all(torch.equal(x, y) for x, y in zip(a, b))


@pytest.mark.parametrize("split", [False, True])
@pytest.mark.parametrize("dtype", list(T.TYPES.values()))
def test_captured_and_replayed(B, dtype, split):
    step = Step(B, dtype, split=split).fill(0)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step.run()
    torch.cuda.current_stream().wait_stream(side)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step.run()
    other = Step(B, dtype, split=split)
    for seed in (1, 2, 3, 4):
        other.fill(seed).run()                          # eager work between the replays
        torch.cuda.synchronize()
        want = other.outputs()
        step.fill(seed)
        graph.replay()
        torch.cuda.synchronize()
        got = step.outputs()
        assert same(got, want), seed
        assert all(torch.isfinite(t.float()).all() for t in (got[0], got[6], got[7], got[9], got[13], got[14]))


@pytest.mark.parametrize("dtype", list(T.TYPES.values()))
def test_two_streams_at_once(B, dtype):
    steps = [Step(B, dtype).fill(s) for s in (10, 11)]
    want = []
    for s in steps:
        s.run()
        torch.cuda.synchronize()
        want.append(s.outputs())
    streams = [torch.cuda.Stream() for _ in steps]
    for s, seed in zip(steps, (10, 11)):
        s.fill(seed)
    torch.cuda.synchronize()
    for _ in range(5):
        for s, stream in zip(steps, streams):
            with torch.cuda.stream(stream):
                s.run()
    torch.cuda.synchronize()
    for s, w in zip(steps, want):
        assert same(s.outputs(), w)


def test_two_graphs_replayed_at_once(B):
    """Graphs that have workspaces of their own do not disturb each other."""
    steps = [Step(B, torch.bfloat16).fill(s) for s in (20, 21)]
    graphs, want = [], []
    for s in steps:
        s.run()
        torch.cuda.synchronize()
        want.append(s.outputs())
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            s.run()
        graphs.append(graph)
    streams = [torch.cuda.Stream() for _ in steps]
    for _ in range(4):
        for graph, stream in zip(graphs, streams):
            with torch.cuda.stream(stream):
                graph.replay()
    torch.cuda.synchronize()
    for s, w in zip(steps, want):
        assert same(s.outputs(), w)


def test_records(B):
    step = Step(B, torch.bfloat16).fill(1)
    B.profile_enable(True)
    step.run()
    B.profile_enable(False)
    names = [r[0] for r in B.profile_collect()]
    assert names == ["layer_norm", "checkpoint", "logprobs", "logprobs_grad", "layer_norm_grad", "weight_grad", "score_logprobs"]


def test_the_binding_refuses(B):
    z = torch.randn(6, 40, device="cuda")
    lab = torch.zeros(6, dtype=torch.int32, device="cuda")
    w = torch.ones(40, device="cuda")
    stats = B.zeno_logprobs(z, lab, want_stats=True)[2]
    ck = B.zeno_checkpoint(z)
    y, mean, rstd, _ = B.zeno_layer_norm(z, w)
    groups = torch.tensor([0, 6], dtype=torch.int32, device="cuda")
    G, ws = torch.zeros(1, 50, device="cuda"), torch.empty(1 << 16, dtype=torch.uint8, device="cuda")
    bad = [
        lambda: B.zeno_logprobs(z.double(), lab), lambda: B.zeno_logprobs(z.t(), lab), lambda: B.zeno_logprobs(z[0], lab),
        lambda: B.zeno_logprobs(z, lab.long()), lambda: B.zeno_logprobs(z, lab[:5]), lambda: B.zeno_logprobs(z, lab.cpu()),
        lambda: B.zeno_logprobs(z, lab, logp=torch.zeros(7, device="cuda")), lambda: B.zeno_logprobs(z[:1].expand(6, 40), lab),
        lambda: B.zeno_logprobs(z, lab, workspace=torch.empty(256, device="cuda")),
        lambda: B.zeno_logprobs_backward(z, stats[:, :1], labels=lab, grad_logp=mean),
        lambda: B.zeno_logprobs_backward(z, stats, labels=lab, grad_logp=mean, out=z.bfloat16()),
        lambda: B.zeno_logprobs_backward(z, stats, grad_top=mean, top_index=lab),
        lambda: B.zeno_checkpoint(z.int()), lambda: B.zeno_checkpoint(z, out=B.alloc_checkpoint(6, 41)),
        lambda: B.zeno_checkpoint(z, out=B.alloc_checkpoint(5, 40)), lambda: B.zeno_checkpoint_values(z),
        lambda: B.zeno_layer_norm(z, w[:39]), lambda: B.zeno_layer_norm(z, w.double()), lambda: B.zeno_layer_norm(z, w, y=z.bfloat16()),
        lambda: B.zeno_layer_norm_backward(z, z.bfloat16(), mean, rstd, w), lambda: B.zeno_layer_norm_backward(z, z, mean[:3], rstd, w),
        lambda: B.zeno_layer_norm_backward(z, z, mean, rstd, w, groups=groups.long()),
        lambda: B.zeno_layer_norm_backward(z, z, mean, rstd, w, groups=groups[:1]),
        lambda: B.zeno_layer_norm_backward(z, z, mean, rstd, w, dweight=G),
        lambda: B.zeno_layer_norm_backward(z, B.alloc_checkpoint(6, 39), mean, rstd, w),
        lambda: B.zeno_weight_gradient(z, z), lambda: B.zeno_weight_gradient(z[:5], ck), lambda: B.zeno_weight_gradient(z, ck, dweight=G),
        lambda: B.zeno_score_logprobs(z, mean, z, 0.1), lambda: B.zeno_score_logprobs(z, z, z, 0.1),
    ]
    for i, call in enumerate(bad):
        with pytest.raises(ValueError):
            call()
            pytest.fail(f"call {i} was taken")
    refused = [
        (1, lambda: B.zeno_logprobs(z, lab, top=41)), (2, lambda: B.zeno_logprobs(z, lab, top=33, workspace=ws)), (1, lambda: B.zeno_logprobs(z)),
        (1, lambda: B.zeno_logprobs_backward(z, stats)), (1, lambda: B.zeno_logprobs_backward(z, stats, grad_logp=mean)),
        (1, lambda: B.zeno_layer_norm(z, w, eps=0.0)), (1, lambda: B.zeno_score_logprobs(z, mean, torch.zeros(6, 6, device="cuda"), -1.0)),
        (3, lambda: B.zeno_layer_norm_backward(z, z, mean, rstd, w, workspace=torch.empty(256, dtype=torch.uint8, device="cuda"))),
        (1, lambda: B.zeno_layer_norm_backward(z, z, mean, rstd, w, want_dx=False, want_weight=False, want_bias=False)),
    ]
    for status, call in refused:
        with pytest.raises(B.ZenoError) as e:
            call()
        assert e.value.status == status


def test_offsets_that_break_the_rules_stay_inside_the_arguments(B):
    """Wrong offsets give wrong gradients; everything around the outputs is as it was, and the next call is right."""
    rows, width, out = 200, 70, 40
    x = torch.randn(rows, width, device="cuda")
    dy = torch.randn(rows, out, device="cuda")
    w = torch.ones(width, device="cuda")
    _, mean, rstd, ck = B.zeno_layer_norm(x, w, want_checkpoint=True)
    for off in ([0, 500, 200], [-7, 90, 1 << 30], [150, 20, 190], [200, 100, 0], [-5, -3, -1]):
        groups = torch.tensor(off, dtype=torch.int32, device="cuda")
        G = torch.full((2, 4 + 2 * width), 7.0, device="cuda")
        H = torch.full((2, 4 + out * width + out), 7.0, device="cuda")
        dx, buf = T.strided(torch.zeros(rows, width), torch.float32, width + 3, 2)
        B.zeno_layer_norm_backward(x, ck, mean, rstd, w, groups=groups, dx=dx, dweight=G[:, 2:2 + width], dbias=G[:, 2 + width:2 + 2 * width])
        B.zeno_weight_gradient(dy, ck, groups=groups, dweight=H[:, 2:2 + out * width], dbias=H[:, 2 + out * width:2 + out * width + out])
        torch.cuda.synchronize()
        assert (G[:, :2] == 7).all() and (G[:, -2:] == 7).all() and (H[:, :2] == 7).all() and (H[:, -2:] == 7).all()
        assert torch.isnan(T.around(dx, buf)).all()
    _, dw, _ = B.zeno_layer_norm_backward(x, ck, mean, rstd, w)
    assert torch.isfinite(dw).all()
