"""Argument checks of the operators for models that answer with tokens: all of them on the host, before anything is enqueued, so
they run without a GPU.  The pointers are never dereferenced."""
import ctypes

import pytest
import torch

P = 1 << 20            # a well aligned address
INVALID, UNSUPPORTED, WORKSPACE = 1, 2, 3


@pytest.fixture(scope="module")
def B():
    from paper_1805_10032_amd import binding, build
    import os
    if not os.path.exists(binding.LIB_PATH):
        build.build(verbose=False)
    binding.load_library()
    return binding


CALLS = {
    "zeno_logprobs": dict(logits=P, ldz=100, dtype=1, rows=4, vocab=100, labels=P, logp=P, entropy=P, stats=P, top=2, top_index=P,
                          top_logp=P, workspace=P, workspace_bytes=0, stream=None),
    "zeno_logprobs_backward": dict(logits=P, ldz=100, dtype=0, rows=4, vocab=100, stats=P, labels=P, grad_logp=P, entropy=P,
                                   grad_entropy=P, top=2, top_index=P, grad_top=P, dlogits=2 * P, ldd=100, stream=None),
    "zeno_checkpoint": dict(x=P, ldx=40, dtype=2, rows=3, width=40, values=P, scales=P, stream=None),
    "zeno_checkpoint_values": dict(values=P, scales=P, rows=3, width=40, dtype=0, out=P, ldo=40, stream=None),
    "zeno_layer_norm": dict(x=P, ldx=40, dtype=1, rows=3, width=40, weight=P, bias=P, eps=1e-5, y=P, ldy=40, mean=P, rstd=P, values=P,
                            scales=P, stream=None),
    "zeno_layer_norm_backward": dict(dy=P, lddy=40, dtype=1, rows=3, width=40, x=P, ldx=40, values=None, scales=None, mean=P, rstd=P,
                                     weight=P, m=2, offsets=P, dx=2 * P, lddx=40, dweight=P, ldw=40, dbias=P, ldb=40, workspace=P,
                                     workspace_bytes=0, stream=None),
    "zeno_weight_gradient": dict(dy=P, lddy=10, dtype=1, rows=3, out=10, values=P, scales=P, width=40, m=2, offsets=P, dweight=P,
                                 ldw=400, dbias=P, ldb=10, workspace=P, workspace_bytes=0, stream=None),
    "zeno_score_logprobs": dict(G=P, ldg=50, m=3, d=50, logp_x=P, logp=P, ldp=7, n=7, labels=P, rho=0.1, scores=P, workspace=P,
                                workspace_bytes=0, stream=None),
}

REFUSED = [
    ("zeno_logprobs", INVALID, dict(logits=None), dict(ldz=99), dict(dtype=3), dict(dtype=-1), dict(rows=-1), dict(vocab=0, ldz=0),
     dict(labels=None), dict(top=-1), dict(top=3, vocab=2), dict(top_index=None), dict(top_logp=None), dict(logits=P + 1),
     dict(logp=P + 2), dict(labels=P + 2), dict(stats=P + 1), dict(entropy=P + 1),
     dict(logp=None, entropy=None, stats=None, top=0), dict(dtype=0, logits=P + 2)),
    ("zeno_logprobs", UNSUPPORTED, dict(top=33), dict(vocab=(1 << 30) + 1, ldz=1 << 31)),
    ("zeno_logprobs", WORKSPACE, dict(), dict(workspace=None, workspace_bytes=1 << 20), dict(workspace=P + 128, workspace_bytes=1 << 20),
     dict(workspace_bytes=255)),
    ("zeno_logprobs_backward", INVALID, dict(logits=None), dict(dlogits=None), dict(ldz=99), dict(ldd=99), dict(dtype=7), dict(stats=None),
     dict(labels=None), dict(entropy=None), dict(top_index=None), dict(grad_top=None), dict(top=0), dict(top=-1),
     dict(grad_logp=None, grad_entropy=None, grad_top=None, top=0), dict(dlogits=P, ldd=101), dict(grad_logp=P + 2), dict(dlogits=P + 2)),
    ("zeno_logprobs_backward", UNSUPPORTED, dict(top=40)),
    ("zeno_checkpoint", INVALID, dict(x=None), dict(values=None), dict(scales=None), dict(values=P + 8), dict(ldx=39), dict(width=0),
     dict(rows=-1), dict(dtype=5), dict(x=P + 1)),
    ("zeno_checkpoint", UNSUPPORTED, dict(width=(1 << 24) + 1, ldx=1 << 25)),
    ("zeno_checkpoint_values", INVALID, dict(out=None), dict(values=None), dict(scales=None), dict(values=P + 4), dict(ldo=39), dict(dtype=3),
     dict(out=P + 2)),
    ("zeno_layer_norm", INVALID, dict(x=None), dict(y=None), dict(weight=None), dict(eps=0.0), dict(eps=-1.0), dict(eps=float("nan")),
     dict(eps=float("inf")), dict(values=None), dict(scales=None), dict(ldx=39), dict(ldy=39), dict(weight=P + 2), dict(values=P + 8)),
    ("zeno_layer_norm", UNSUPPORTED, dict(width=(1 << 24) + 1, ldx=1 << 25, ldy=1 << 25)),
    ("zeno_layer_norm_backward", INVALID, dict(dy=None), dict(x=None), dict(values=P), dict(x=None, values=P), dict(values=P, scales=P),
     dict(mean=None), dict(rstd=None), dict(weight=None), dict(m=0), dict(m=1025), dict(offsets=None), dict(offsets=P + 2),
     dict(dx=None, dweight=None, dbias=None), dict(ldw=39), dict(ldb=39), dict(lddx=39), dict(dx=P, lddx=41), dict(dweight=P + 1)),
    ("zeno_layer_norm_backward", WORKSPACE, dict(), dict(workspace=None, workspace_bytes=1 << 20), dict(workspace=P + 4, workspace_bytes=1 << 20)),
    ("zeno_weight_gradient", INVALID, dict(dy=None), dict(values=None), dict(scales=None), dict(dweight=None), dict(ldw=399), dict(ldb=9),
     dict(width=0), dict(out=0), dict(m=0), dict(m=2000), dict(offsets=None), dict(values=P + 8), dict(lddy=9), dict(dtype=4)),
    ("zeno_weight_gradient", UNSUPPORTED, dict(out=1 << 19, lddy=1 << 19, width=1 << 19, ldw=1 << 40, ldb=1 << 19)),
    ("zeno_weight_gradient", WORKSPACE, dict(), dict(workspace=None, workspace_bytes=1 << 20), dict(workspace=P + 64, workspace_bytes=1 << 20)),
    ("zeno_score_logprobs", INVALID, dict(G=None), dict(logp=None), dict(logp_x=None), dict(scores=None), dict(m=0), dict(m=1025), dict(d=0),
     dict(ldg=49), dict(n=0), dict(ldp=6), dict(rho=-1.0), dict(rho=float("nan")), dict(G=P + 2), dict(labels=P + 1)),
    ("zeno_score_logprobs", WORKSPACE, dict(), dict(workspace=None, workspace_bytes=1 << 20), dict(workspace=P + 8, workspace_bytes=1 << 20)),
]


@pytest.mark.parametrize("name,status,changes", [(r[0], r[1], c) for r in REFUSED for c in r[2:]],
                         ids=lambda v: str(v) if not isinstance(v, dict) else "-".join(v) or "plain")
def test_refused(B, name, status, changes):
    args = dict(CALLS[name], **changes)
    assert set(args) == set(CALLS[name])
    assert getattr(B.load_library(), name)(*args.values()) == status


@pytest.mark.parametrize("name", [n for n in CALLS if "rows" in CALLS[n]])
def test_rows_beyond_the_most(B, name):
    """Row numbers keep room for a kernel's step in 32 bits."""
    for rows in ((1 << 30) + 1, (1 << 31) - 1):
        assert getattr(B.load_library(), name)(*dict(CALLS[name], rows=rows).values()) == UNSUPPORTED
    lib = B.load_library()
    rows = (1 << 30) + 1
    assert lib.zeno_logprobs_workspace_bytes(rows, 10, 0) == 0 and lib.zeno_layer_norm_workspace_bytes(rows, 4, 1) == 0
    assert lib.zeno_weight_gradient_workspace_bytes(rows, 4, 4, 1) == 0
    assert lib.zeno_logprobs_workspace_bytes(rows - 1, 10, 0) > 0 and lib.zeno_layer_norm_workspace_bytes(rows - 1, 4, 1) > 0


def test_calls_without_rows_need_no_memory(B):
    lib = B.load_library()
    none = {"zeno_logprobs": dict(rows=0, logits=None, labels=None, logp=None, top_index=None, top_logp=None, workspace_bytes=1 << 20),
            "zeno_logprobs_backward": dict(rows=0, logits=None, dlogits=None, stats=None),
            "zeno_checkpoint": dict(rows=0, x=None, values=None, scales=None),
            "zeno_checkpoint_values": dict(rows=0, out=None, values=None, scales=None),
            "zeno_layer_norm": dict(rows=0, x=None, y=None, values=None, scales=None)}
    for name, change in none.items():
        assert getattr(lib, name)(*dict(CALLS[name], **change).values()) == 0, name


def test_workspace_queries(B):
    lib = B.load_library()
    for args in ((-1, 10, 0), (1, 0, 0), (1, 10, 33), (1, 10, 11), (1, (1 << 30) + 1, 0), (1, 10, -1)):
        assert lib.zeno_logprobs_workspace_bytes(*args) == 0
    for args in ((-1, 4, 1), (4, 0, 1), (4, 4, 0), (4, 4, 1025), (4, (1 << 24) + 1, 1)):
        assert lib.zeno_layer_norm_workspace_bytes(*args) == 0
    for args in ((-1, 4, 4, 1), (4, 0, 4, 1), (4, 4, 0, 1), (4, 4, 4, 0), (4, 4, 4, 1025)):
        assert lib.zeno_weight_gradient_workspace_bytes(*args) == 0
    for args in ((0, 5), (1025, 5), (4, 0)):
        assert lib.zeno_score_logprobs_workspace_bytes(*args) == 0
    for n in (lib.zeno_logprobs_workspace_bytes(0, 1, 0), lib.zeno_logprobs_workspace_bytes(0, 200000, 8),
              lib.zeno_logprobs_workspace_bytes(3, 100000, 32),
              lib.zeno_layer_norm_workspace_bytes(0, 1, 1), lib.zeno_layer_norm_workspace_bytes(100, 77, 1024),
              lib.zeno_weight_gradient_workspace_bytes(0, 1, 1, 1), lib.zeno_weight_gradient_workspace_bytes(100000, 10, 10, 3),
              lib.zeno_score_logprobs_workspace_bytes(1, 1), lib.zeno_score_logprobs_workspace_bytes(1024, 1 << 33)):
        assert n > 0 and n % 256 == 0


def test_the_binding_refuses_tensors_elsewhere(B):
    z, lab = torch.zeros(3, 5), torch.zeros(3, dtype=torch.int32)
    ck = B.Checkpoint(torch.zeros(3, 32, dtype=torch.uint8), torch.zeros(3, 1, dtype=torch.uint8), 5)
    for call in (lambda: B.zeno_logprobs(z, lab), lambda: B.zeno_logprobs_backward(z, z), lambda: B.zeno_checkpoint(z),
                 lambda: B.zeno_layer_norm(z, z[0]), lambda: B.zeno_layer_norm_backward(z, z, z[:, 0], z[:, 0], z[0]),
                 lambda: B.zeno_weight_gradient(z, ck), lambda: B.zeno_score_logprobs(z, z[0], z, 0.1),
                 lambda: B.zeno_checkpoint_values(ck)):
        with pytest.raises(ValueError):
            call()


def test_the_binding_refuses_sizes_beyond_32_bits(B):
    """A size that the C call takes in 32 bits would otherwise arrive as another one.  The memory is never touched."""
    long = (1 << 32) + 5
    column = torch.empty(long, 1, dtype=torch.float16)
    for t in (column, column.t()):
        with pytest.raises(B.ZenoError) as e:
            B._matrix(t, "x", t.get_device())
        assert e.value.status == UNSUPPORTED
    offsets = torch.empty(long, dtype=torch.int32)
    with pytest.raises(B.ZenoError) as e:
        B._groups(offsets, offsets.get_device())
    assert e.value.status == UNSUPPORTED
    for call in (lambda: B.alloc_logprobs_workspace(long, 10, 0), lambda: B.alloc_logprobs_workspace(4, long, 0),
                 lambda: B.alloc_logprobs_workspace(4, 10, (1 << 32) + 1), lambda: B.alloc_layer_norm_workspace(long, 10, 1),
                 lambda: B.alloc_layer_norm_workspace(10, long, 1), lambda: B.alloc_layer_norm_workspace(10, 10, long),
                 lambda: B.alloc_weight_gradient_workspace(long, 10, 10, 1), lambda: B.alloc_weight_gradient_workspace(10, long, 10, 1),
                 lambda: B.alloc_weight_gradient_workspace(10, 10, long, 1), lambda: B.alloc_weight_gradient_workspace(10, 10, 10, long),
                 lambda: B.alloc_score_logprobs_workspace(long, 10)):
        with pytest.raises(B.ZenoError):
            call()
    weights = torch.empty(1, (1 << 31) + 5)        # (one layer's weights; the rows of such gradients are counted in 64 bits)
    assert B._grad_rows(weights, "dweight", 1, weights.shape[1], weights.get_device()) == (weights.data_ptr(), weights.shape[1])


def test_outputs_without_rows_have_no_address(B):
    """An empty tensor's pointer is NULL, whatever was asked for: no rows is no error."""
    lib = B.load_library()
    call = dict(CALLS["zeno_logprobs"], rows=0, logits=None, labels=None, logp=None, entropy=None, stats=None, top=0, top_index=None, top_logp=None,
                workspace_bytes=1 << 20)
    assert lib.zeno_logprobs(*call.values()) == 0
    assert lib.zeno_logprobs(*dict(call, rows=1, logits=P).values()) == INVALID
    call = dict(CALLS["zeno_layer_norm_backward"], rows=0, dy=None, x=None, mean=None, rstd=None, m=1, offsets=None, dx=None, dweight=None, dbias=None,
                workspace_bytes=1 << 20)
    assert lib.zeno_layer_norm_backward(*call.values()) == 0
    assert lib.zeno_layer_norm_backward(*dict(call, rows=1, dy=P, x=P, mean=P, rstd=P).values()) == INVALID
