"""Argument checks of the embedding and of the log probabilities of a linear layer: all of them on the host, before anything is enqueued, so they
run without a GPU.  The pointers are never dereferenced."""
import pytest
import torch

P = 1 << 20            # a well aligned address
INVALID, UNSUPPORTED, WORKSPACE = 1, 2, 3
ROOM = 1 << 40


@pytest.fixture(scope="module")
def B():
    import os
    from paper_1805_10032_amd import binding, build
    if not os.path.exists(binding.LIB_PATH):
        build.build(verbose=False)
    binding.load_library()
    return binding


CALLS = {
    "zeno_embedding": dict(table=P, ldt=40, table_dtype=0, vocab=100, width=40, ids=P, rows=3, scale=1.0, out=P, ldo=40, dtype=1, stream=None),
    "zeno_embedding_backward": dict(dy=P, lddy=40, dtype=1, rows=3, width=40, ids=P, vocab=100, scale=1.0, m=2, offsets=P, accumulate=0, dtable=P,
                                    ldg=4000, workspace=P, workspace_bytes=0, stream=None),
    "zeno_linear_logprobs": dict(hidden=P, ldh=40, weight=P, ldw=40, dtype=1, bias=P, rows=4, vocab=100, width=40, labels=P, logp=P, entropy=P,
                                 stats=P, workspace=P, workspace_bytes=0, stream=None),
    "zeno_linear_logprobs_backward": dict(hidden=P, ldh=40, weight=P, ldw=40, dtype=1, bias=P, rows=4, vocab=100, width=40, stats=P, labels=P,
                                          grad_logp=P, entropy=P, grad_entropy=P, m=2, offsets=P, dhidden=2 * P, lddh=40, dweight=P, ldg=4000,
                                          dbias=P, ldb=100, workspace=P, workspace_bytes=0, stream=None),
}
NAN, INF = float("nan"), float("inf")
REFUSED = [
    ("zeno_embedding", INVALID, dict(table=None), dict(ids=None), dict(out=None), dict(ldt=39), dict(ldo=39), dict(vocab=0), dict(vocab=-1),
     dict(width=0), dict(rows=-1), dict(table_dtype=3), dict(dtype=-1), dict(scale=NAN), dict(scale=INF), dict(ids=P + 2), dict(table=P + 2),
     dict(out=P + 1)),
    ("zeno_embedding", UNSUPPORTED, dict(width=(1 << 24) + 1, ldt=1 << 25, ldo=1 << 25), dict(vocab=(1 << 30) + 1), dict(rows=(1 << 30) + 1)),
    ("zeno_embedding_backward", INVALID, dict(dy=None), dict(ids=None), dict(dtable=None), dict(lddy=39), dict(ldg=3999), dict(vocab=0), dict(m=0),
     dict(m=1025), dict(offsets=None), dict(offsets=P + 2), dict(accumulate=2), dict(accumulate=-1), dict(scale=NAN), dict(dtype=3), dict(rows=-1),
     dict(dy=P + 1), dict(dtable=P + 2), dict(width=0), dict(ids=P + 1)),
    ("zeno_embedding_backward", UNSUPPORTED, dict(rows=(1 << 30) + 1), dict(vocab=1 << 30, ldg=1 << 40), dict(vocab=(1 << 30) + 1, ldg=1 << 40)),
    ("zeno_embedding_backward", WORKSPACE, dict(), dict(workspace=None, workspace_bytes=ROOM), dict(workspace=P + 128, workspace_bytes=ROOM)),
    ("zeno_linear_logprobs", INVALID, dict(hidden=None), dict(weight=None), dict(ldh=39), dict(ldw=39), dict(dtype=3), dict(rows=-1), dict(vocab=0),
     dict(width=0), dict(labels=None), dict(logp=None, entropy=None, stats=None), dict(hidden=P + 1), dict(weight=P + 1), dict(bias=P + 2),
     dict(labels=P + 2), dict(logp=P + 1), dict(entropy=P + 2), dict(stats=P + 2)),
    ("zeno_linear_logprobs", UNSUPPORTED, dict(width=(1 << 16) + 1, ldh=1 << 20, ldw=1 << 20), dict(vocab=(1 << 24) + 1), dict(rows=(1 << 22) + 1),
     dict(rows=(1 << 31) - 1), dict(vocab=1 << 24, width=1 << 13, ldh=1 << 13, ldw=1 << 13)),
    ("zeno_linear_logprobs", WORKSPACE, dict(), dict(workspace=None, workspace_bytes=ROOM), dict(workspace=P + 64, workspace_bytes=ROOM)),
    ("zeno_linear_logprobs_backward", INVALID, dict(hidden=None), dict(weight=None), dict(stats=None), dict(labels=None), dict(entropy=None),
     dict(grad_logp=None, grad_entropy=None), dict(dhidden=None, dweight=None, dbias=None), dict(lddh=39), dict(dhidden=P, lddh=41), dict(ldg=3999),
     dict(ldb=99), dict(m=0), dict(m=1025), dict(offsets=None), dict(offsets=P + 1), dict(dtype=4), dict(dweight=P + 1), dict(dbias=P + 2),
     dict(dhidden=P + 1), dict(stats=P + 2), dict(grad_logp=P + 2), dict(grad_entropy=P + 2), dict(entropy=P + 2), dict(bias=P + 1), dict(rows=-1),
     dict(vocab=0), dict(width=0)),
    ("zeno_linear_logprobs_backward", UNSUPPORTED, dict(rows=(1 << 22) + 1), dict(vocab=(1 << 24) + 1, ldg=1 << 40, ldb=1 << 30),
     dict(width=(1 << 16) + 1, ldh=1 << 20, ldw=1 << 20, lddh=1 << 20, ldg=1 << 40)),
    ("zeno_linear_logprobs_backward", WORKSPACE, dict(), dict(workspace=None, workspace_bytes=ROOM), dict(workspace=P + 8, workspace_bytes=ROOM)),
]


@pytest.mark.parametrize("name,status,changes", [(r[0], r[1], c) for r in REFUSED for c in r[2:]],
                         ids=lambda v: str(v) if not isinstance(v, dict) else "-".join(v) or "plain")
def test_refused(B, name, status, changes):
    args = dict(CALLS[name], **changes)
    assert set(args) == set(CALLS[name])
    assert getattr(B.load_library(), name)(*args.values()) == status


def test_calls_without_rows_need_no_memory(B):
    lib = B.load_library()
    assert lib.zeno_embedding(*dict(CALLS["zeno_embedding"], rows=0, ids=None, out=None).values()) == 0
    call = dict(CALLS["zeno_linear_logprobs"], rows=0, hidden=None, labels=None, logp=None, entropy=None, stats=None, workspace_bytes=ROOM)
    assert lib.zeno_linear_logprobs(*call.values()) == 0
    call = dict(CALLS["zeno_linear_logprobs_backward"], rows=0, hidden=None, stats=None, labels=None, grad_logp=None, entropy=None, grad_entropy=None,
                dhidden=None, dweight=None, dbias=None, workspace_bytes=ROOM)
    assert lib.zeno_linear_logprobs_backward(*call.values()) == 0


def test_workspace_queries(B):
    lib = B.load_library()
    for args in ((-1, 4, 4, 1), (1, 0, 4, 1), (1, 4, 0, 1), (1, 4, 4, 0), (1, 4, 4, 1025), (1, 1 << 30, 4, 2), (1, 4, (1 << 24) + 1, 1), ((1 << 30) + 1, 4, 4, 1)):
        assert lib.zeno_embedding_workspace_bytes(*args) == 0
    for args in ((-1, 4, 4, 1), (1, 0, 4, 1), (1, 4, 0, 1), (1, 4, 4, 3), (1, 4, 4, -1), ((1 << 22) + 1, 4, 4, 0), (1, (1 << 24) + 1, 4, 0),
                 (1, 4, (1 << 16) + 1, 0), (1, 1 << 24, 1 << 13, 0)):
        assert lib.zeno_linear_logprobs_workspace_bytes(*args) == 0
        assert lib.zeno_linear_logprobs_backward_workspace_bytes(*args, 1) == 0
    assert lib.zeno_linear_logprobs_backward_workspace_bytes(1, 4, 4, 0, 0) == 0 and lib.zeno_linear_logprobs_backward_workspace_bytes(1, 4, 4, 0, 1025) == 0
    sizes = [lib.zeno_embedding_workspace_bytes(*a) for a in ((0, 1, 1, 1), (1, 1, 1, 1), (70000, 200000, 64, 1024), (1 << 30, 4, 4, 1), (5, (1 << 30), 1, 1))]
    for dtype in range(3):
        for a in ((0, 1, 1), (1, 1, 1), (65, 32000, 4096), (1 << 22, 1, 1), (5, 1 << 24, 4096), (300, 1000, 1 << 16)):
            sizes += [lib.zeno_linear_logprobs_workspace_bytes(*a, dtype), lib.zeno_linear_logprobs_backward_workspace_bytes(*a, dtype, 1024)]
    assert all(n > 0 and n % 256 == 0 for n in sizes)


def test_the_binding_refuses_tensors_elsewhere_and_other_shapes(B):
    h, w, ids = torch.zeros(3, 5), torch.zeros(7, 5), torch.zeros(3, dtype=torch.int32)
    for call in (lambda: B.zeno_embedding(ids, w), lambda: B.zeno_embedding_backward(h, ids, 7), lambda: B.zeno_linear_logprobs(h, w, None, ids),
                 lambda: B.zeno_linear_logprobs_backward(h, w, None, h, labels=ids, grad_logp=h[:, 0]),
                 lambda: B.alloc_linear_logprobs_workspace(1, 1, 1, torch.float64)):
        with pytest.raises(ValueError):
            call()
    long = (1 << 32) + 5
    for call in (lambda: B.alloc_embedding_workspace(long, 10, 10), lambda: B.alloc_embedding_workspace(10, long, 10),
                 lambda: B.alloc_embedding_workspace(10, 10, long), lambda: B.alloc_embedding_workspace(10, 10, 10, long),
                 lambda: B.alloc_linear_logprobs_workspace(long, 10, 10), lambda: B.alloc_linear_logprobs_workspace(10, long, 10),
                 lambda: B.alloc_linear_logprobs_backward_workspace(10, 10, long), lambda: B.alloc_linear_logprobs_backward_workspace(10, 10, 10, torch.float32, long)):
        with pytest.raises(B.ZenoError):
            call()


def test_a_model_of_other_shapes_is_refused():
    from paper_1805_10032_amd.token_model import TokenModel
    for kw in (dict(inputs=0), dict(tied=True), dict(inputs=9, tied=True), dict(inputs=11, tied=True)):
        with pytest.raises(ValueError):
            TokenModel([24, 16, 11], **kw)
    plain, fed, tied = TokenModel([24, 24, 11]), TokenModel([24, 24, 11], inputs=11), TokenModel([24, 24, 11], inputs=11, tied=True)
    assert fed.num_params == plain.num_params + 11 * 24 and tied.num_params == plain.num_params
    assert tied.offsets[-1][2] == tied.table and plain.table is None
