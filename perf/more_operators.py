"""The measured cases of the operators at both ends of a model that answers with tokens.

A case is one pass through an operator, as a worker or the server of Algorithm 1 calls it:

  kind "embed"  rows of a table by token, times a scale; in training also the table's gradients of m workers, written into
                rows of G (every row of every worker's table, most of them zero)
  kind "loss"   log probabilities of given tokens straight from hidden states and the weights of the last layer, without keeping
                the logits; in training also the gradients of the hidden states and, of m workers, of the weights and the bias,
                written into rows of G

run() computes them in elementary torch operations where `own` is false, and through
paper_1805_10032_amd.binding where it is true.
"""
from __future__ import annotations

import math
import random

import torch

own = False

_TYPES = {"fp32": torch.float32, "bf16": torch.bfloat16, "fp16": torch.float16}


def listed():
    return [
        # serving: the state of one new token; launches and host time count
        {"name": "embed_token", "kind": "embed", "rows": 1, "vocab": 32000, "width": 4096, "table": "bf16", "type": "bf16", "m": 1,
         "train": False},
        # a long batch of prompts from the parameter vector itself: the lookup alone
        {"name": "embed_prompt", "kind": "embed", "rows": 65536, "vocab": 50257, "width": 2048, "table": "fp32", "type": "bf16", "m": 1,
         "train": False},
        # the paper's twenty workers: 2.6 GB of gradients, nearly all of them zero, and a few tokens that everybody uses
        {"name": "embed_workers", "kind": "embed", "rows": 16384, "vocab": 32000, "width": 1024, "table": "fp32", "type": "bf16", "m": 20,
         "train": True},
        # few values, many tokens: the sum over tokens is the long axis; odd width, odd number of tokens
        {"name": "embed_bytes", "kind": "embed", "rows": 50001, "vocab": 257, "width": 777, "table": "fp32", "type": "fp32", "m": 3,
         "train": True},
        # one token's log probability: the weights are read for a single row
        {"name": "loss_token", "kind": "loss", "rows": 1, "vocab": 32000, "width": 4096, "type": "bf16", "m": 1, "train": False,
         "entropy": True, "masked": 0.3},
        # a handful of tokens; odd width and vocabulary, so rows start anywhere
        {"name": "loss_few", "kind": "loss", "rows": 24, "vocab": 50257, "width": 1001, "type": "fp16", "m": 1, "train": False,
         "entropy": False, "masked": 0.0},
        # the server's batch at one of the m + 1 parameter vectors
        {"name": "loss_score", "kind": "loss", "rows": 4096, "vocab": 50257, "width": 2048, "type": "bf16", "m": 1, "train": False,
         "entropy": False, "masked": 0.0},
        # the same where differences of log probabilities are wanted finer
        {"name": "loss_score_fp32", "kind": "loss", "rows": 1000, "vocab": 32000, "width": 1024, "type": "fp32", "m": 1, "train": False,
         "entropy": False, "masked": 0.0},
        # training: thousands of tokens for each of four workers, the largest products
        {"name": "loss_train", "kind": "loss", "rows": 8192, "vocab": 64000, "width": 4096, "type": "bf16", "m": 4, "train": True,
         "entropy": False, "masked": 0.0},
        # twenty workers with a hundred tokens each: writing the rows of G counts
        {"name": "loss_workers", "kind": "loss", "rows": 2000, "vocab": 32000, "width": 1024, "type": "fp16", "m": 20, "train": True,
         "entropy": False, "masked": 0.0},
        # one short sequence, the entropy's gradient among the loss's, tokens ruled out
        {"name": "loss_sequence", "kind": "loss", "rows": 250, "vocab": 50257, "width": 1600, "type": "bf16", "m": 1, "train": True,
         "entropy": True, "masked": 0.3},
        # float32, odd sizes, ragged workers
        {"name": "loss_ragged", "kind": "loss", "rows": 777, "vocab": 10007, "width": 513, "type": "fp32", "m": 3, "train": True,
         "entropy": True, "masked": 0.0},
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    """Another case of the ranges that the listed ones stand for."""
    ty = rng.choice(["fp32", "bf16", "bf16", "fp16"])
    train = rng.random() < 0.6
    if rng.random() < 0.35:
        width = _log(rng, 8, 8192)
        if rng.random() < 0.5:
            width = max(64, width // 64 * 64)
        vocab = _log(rng, 10, 200000)
        m = _log(rng, 1, 64) if train else 1
        while m * vocab * width > 1 << 30:
            m, vocab = max(1, m // 2), max(10, vocab // 2)
        rows = _log(rng, 1, min(65536, (1 << 27) // width))
        return {"kind": "embed", "rows": rows, "vocab": vocab, "width": width, "table": rng.choice(["fp32", ty]), "type": ty, "m": m,
                "train": train}
    width = _log(rng, 8, 4096)
    if rng.random() < 0.6:
        width = max(64, width // 64 * 64)
    vocab = _log(rng, 10, 130000)
    rows = _log(rng, 1, 16384)
    m = _log(rng, 1, 32) if train else 1
    most = 1 << (37 if ty == "fp32" else 40)
    while rows * vocab > 1 << 29 or rows * vocab * width > most:
        rows = max(1, rows // 2)
    while m * vocab * width > 1 << 30:
        m = max(1, m // 2)
    return {"kind": "loss", "rows": rows, "vocab": vocab, "width": width, "type": ty, "m": m, "train": train,
            "entropy": rng.random() < 0.4, "masked": rng.choice([0.0, 0.0, 0.3])}


def _sizes(total, m, seed):
    """Rows of every worker: ragged, some may be empty; together all rows but the last few, which belong to nobody."""
    rng = random.Random(seed * 7919 + total * 31 + m)
    left = total - total // 64
    cuts = sorted(rng.randint(0, left) for _ in range(m - 1))
    if total >= 16 * m:   # ordinary batches: every worker within half and one and a half of the mean
        cuts = [int((i + 1 + rng.uniform(-0.25, 0.25)) * left / m) for i in range(m - 1)]
    return [0, *cuts, left]


def prepare(case, seed):
    dev = torch.device("cuda", torch.cuda.current_device())
    gen = torch.Generator(device=dev)
    gen.manual_seed(seed * 1000003 + 29)

    def randn(*shape, std=1.0):
        return torch.randn(shape, generator=gen, device=dev) * std

    def rand(*shape):
        return torch.rand(shape, generator=gen, device=dev)

    def filled(rows, width, ty, std):
        out = torch.empty(rows, width, device=dev, dtype=ty)
        for r in range(0, rows, 8192):
            out[r:r + 8192] = randn(min(8192, rows - r), width, std=std).to(ty)
        return out

    def tokens(rows, vocab):   # the j-th token is drawn about as often as 1 / (j + 1)
        return (torch.exp(rand(rows).double() * math.log(vocab + 1)).long() - 1).clamp(0, vocab - 1)

    st = {"case": dict(case)}
    rows, vocab, width, m, ty = case["rows"], case["vocab"], case["width"], case["m"], _TYPES[case["type"]]
    if case["train"]:
        st["offsets"] = _sizes(rows, m, seed)
        st["groups"] = torch.tensor(st["offsets"], dtype=torch.int32, device=dev)
    if case["kind"] == "embed":
        st["table"] = filled(vocab, width, _TYPES[case["table"]], width ** -0.5)
        st["scale"] = float(torch.tensor(math.sqrt(width), dtype=torch.float32))
        ids = tokens(rows, vocab)
        if case["train"]:
            ids[rand(rows) < 0.03] = -1                       # padding
            st["dy"] = filled(rows, width, ty, 0.01)
            st["G"] = torch.zeros(m, vocab * width, device=dev)
            if own:
                from paper_1805_10032_amd import binding as B
                st["workspace"] = B.alloc_embedding_workspace(rows, vocab, width, m)
        st["ids"] = ids.to(torch.int32)
        return st
    labels = tokens(rows, vocab)
    weight = filled(vocab, width, ty, 2.0 * width ** -0.5)
    # what a trained layer sees: states that lean towards the weights of the token that comes next, some of them strongly
    hidden = torch.empty(rows, width, device=dev, dtype=ty)
    lean = 1.5 * torch.abs(randn(rows, 1))
    for r in range(0, rows, 8192):
        part = randn(min(8192, rows - r), width)
        hidden[r:r + 8192] = (part + lean[r:r + 8192] * weight[labels[r:r + 8192]].float()).to(ty)
    st["hidden"], st["weight"] = hidden, weight
    st["bias"] = -0.5 * torch.log1p(torch.arange(vocab, device=dev, dtype=torch.float32))   # frequent tokens come first
    if case["masked"] > 0:                                    # tokens that a grammar or a filter rules out
        ban = rand(vocab) < case["masked"]
        ban[0] = False
        labels = torch.where(ban[labels], torch.zeros_like(labels), labels)
        st["bias"][ban] = float("-inf")
    if case["train"]:
        labels[rand(rows) < 0.06] = -1                        # padding
        st["grad_logp"] = -(1.0 + 0.1 * randn(rows)) / rows
        if case["entropy"]:
            st["grad_entropy"] = -(0.01 + 0.001 * randn(rows)) / rows
        st["dh"] = torch.zeros(rows, width, device=dev, dtype=ty)
        st["G"] = torch.zeros(m, vocab * width + vocab, device=dev)
    st["labels"] = labels.to(torch.int32)
    if own:
        from paper_1805_10032_amd import binding as B
        st["workspace"] = B.alloc_linear_logprobs_workspace(rows, vocab, width, ty)
        if case["train"]:
            st["workspace_back"] = B.alloc_linear_logprobs_backward_workspace(rows, vocab, width, ty, m)
    return st


# ---- the plain forms

def _plain_embed(st):
    case, table, ids = st["case"], st["table"], st["ids"].long()
    inside = ids >= 0
    picked = table[ids.clamp(min=0)].float() * st["scale"]
    out = {"out": torch.where(inside[:, None], picked, torch.zeros_like(picked)).to(_TYPES[case["type"]])}
    if case["train"]:
        vocab, width = table.shape
        G = st["G"].zero_().view(case["m"] * vocab, width)
        row = torch.arange(len(ids), device=ids.device)
        worker = torch.searchsorted(st["groups"][1:-1].contiguous(), row.int(), right=True)
        counts = inside & (row < st["offsets"][-1])
        part = torch.where(counts[:, None], st["dy"].float() * st["scale"], torch.zeros_like(picked))
        G.index_add_(0, worker * vocab + ids.clamp(min=0), part)
        out["G"] = st["G"]
    return out


def _plain_loss(st):
    case = st["case"]
    hidden, weight = st["hidden"].float(), st["weight"].float()
    z = torch.matmul(hidden, weight.t()) + st["bias"]
    labels = st["labels"].long()
    counted = labels >= 0
    y = labels.clamp(min=0)
    d = z - z.amax(1, keepdim=True)
    del z
    e = torch.exp(d)
    s = e.sum(1)
    log_s = torch.log(s)
    logp = d.gather(1, y[:, None])[:, 0] - log_s
    out = {"logp": torch.where(counted, logp, torch.zeros_like(logp))}
    entropy = None
    if case["entropy"]:
        entropy = log_s - torch.where(e > 0, e * d, torch.zeros_like(d)).sum(1) / s
        out["entropy"] = entropy
    if not case["train"]:
        return out
    g = torch.where(counted, st["grad_logp"], torch.zeros_like(st["grad_logp"]))
    p = e / s[:, None]
    if entropy is not None:
        lp = torch.where(p > 0, d - log_s[:, None], torch.zeros_like(d))
        dz = -p * (g[:, None] + st["grad_entropy"][:, None] * (lp + entropy[:, None]))
    else:
        dz = -p * g[:, None]
    dz.scatter_add_(1, y[:, None], g[:, None])
    last, n = st["offsets"][-1], weight.numel()
    st["dh"][:last] = torch.matmul(dz[:last], weight).to(st["dh"].dtype)
    for i, (a, b) in enumerate(zip(st["offsets"], st["offsets"][1:])):
        st["G"][i, :n] = torch.matmul(dz[a:b].t(), hidden[a:b]).view(-1)
        st["G"][i, n:] = dz[a:b].sum(0)
    out["dh"], out["G"] = st["dh"], st["G"]
    return out


# ---- the framework's calls

def _own_run(st):
    from paper_1805_10032_amd import binding as B
    case = st["case"]
    if case["kind"] == "embed":
        out = {"out": B.zeno_embedding(st["ids"], st["table"], _TYPES[case["type"]], scale=st["scale"])}
        if case["train"]:
            B.zeno_embedding_backward(st["dy"], st["ids"], case["vocab"], scale=st["scale"], groups=st["groups"], dtable=st["G"],
                                      workspace=st["workspace"])
            out["G"] = st["G"]
        return out
    train, want = case["train"], case["entropy"]
    logp, entropy, stats = B.zeno_linear_logprobs(st["hidden"], st["weight"], st["bias"], st["labels"], want_entropy=want, want_stats=train,
                                                  workspace=st["workspace"])
    out = {"logp": logp}
    if want:
        out["entropy"] = entropy
    if train:
        n = case["vocab"] * case["width"]
        B.zeno_linear_logprobs_backward(st["hidden"], st["weight"], st["bias"], stats, labels=st["labels"], grad_logp=st["grad_logp"],
                                        entropy=entropy, grad_entropy=st["grad_entropy"] if want else None, groups=st["groups"],
                                        dhidden=st["dh"], dweight=st["G"][:, :n], dbias=st["G"][:, n:], workspace=st["workspace_back"])
        out["dh"], out["G"] = st["dh"], st["G"]
    return out


def run(state):
    if own:
        return _own_run(state)
    return _plain_embed(state) if state["case"]["kind"] == "embed" else _plain_loss(state)


def work(case):
    """Bytes: what every call of the pass takes and returns, once; flops: the operations of the formulas."""
    rows, vocab, width, m = case["rows"], case["vocab"], case["width"], case["m"]
    e = 4 if case["type"] == "fp32" else 2
    if case["kind"] == "embed":
        t = 4 if case["table"] == "fp32" else 2
        total = rows * 4 + min(rows, vocab) * width * t + rows * width * e
        if not case["train"]:
            return {"bytes": total, "flops": rows * width}
        return {"bytes": total + rows * 4 + rows * width * e + 4 * m * vocab * width, "flops": 3 * rows * width}
    product = 2 * rows * vocab * width
    total = e * (rows * width + vocab * width) + 4 * vocab + 8 * rows + (4 * rows if case["entropy"] else 0)
    if not case["train"]:
        return {"bytes": total, "flops": product + 5 * rows * vocab}
    back = e * (2 * rows * width + vocab * width) + 4 * vocab + 24 * rows + 4 * m * (vocab * width + vocab)
    return {"bytes": total + back, "flops": 3 * product + 12 * rows * vocab}


# ---- the definitions in 64 bits

def _exact_embed(st):
    case = st["case"]
    table, ids = st["table"].double(), st["ids"].long()
    padded = torch.cat([table, torch.zeros_like(table[:1])])  # -1 takes the last row
    out = {"out": padded[ids] * st["scale"]}
    if case["train"]:
        vocab, width = case["vocab"], case["width"]
        G = torch.zeros(case["m"], vocab + 1, width, dtype=torch.float64, device=table.device)
        for i in range(case["m"]):
            mine = slice(st["offsets"][i], st["offsets"][i + 1])
            key = torch.where(ids[mine] < 0, vocab, ids[mine])
            G[i].index_put_((key,), st["dy"][mine].double(), accumulate=True)
        out["G"] = (G[:, :vocab] * st["scale"]).reshape(case["m"], -1)
    return out


def _exact_loss(st):
    case = st["case"]
    rows, vocab, n = case["rows"], case["vocab"], case["vocab"] * case["width"]
    weight, bias = st["weight"].double(), st["bias"].double()
    out = {"logp": []}
    if case["entropy"]:
        out["entropy"] = []
    if case["train"]:
        out["dh"] = torch.zeros(rows, case["width"], dtype=torch.float64, device=weight.device)
        out["G"] = torch.zeros(case["m"], n + vocab, dtype=torch.float64, device=weight.device)
        spans = list(enumerate(zip(st["offsets"], st["offsets"][1:]))) + [(None, (st["offsets"][-1], rows))]
    else:
        spans = [(None, (0, rows))]
    step = max(1, (1 << 28) // vocab)
    for who, (lo, hi) in spans:
        for a in range(lo, hi, step):
            part = slice(a, min(hi, a + step))
            h = st["hidden"][part].double()
            lab = st["labels"][part].long()
            z = torch.addmm(bias, h, weight.t())
            lp = torch.log_softmax(z, 1)
            at = torch.arange(len(lab), device=z.device)
            out["logp"].append(torch.where(lab >= 0, lp[at, lab.clamp(min=0)], 0.0))
            p = torch.exp(lp)
            plogp = torch.special.entr(p)                     # -p log p, 0 at 0
            ent = plogp.sum(1)
            if case["entropy"]:
                out["entropy"].append(ent)
            if who is None:
                continue
            g = st["grad_logp"][part].double() * (lab >= 0)
            dz = -p * g[:, None]
            if case["entropy"]:
                q = st["grad_entropy"][part].double()[:, None]
                dz += q * (plogp - p * ent[:, None])
            dz[at, lab.clamp(min=0)] += g
            out["dh"][part] = dz @ weight
            out["G"][who, :n] += (dz.t() @ h).reshape(-1)
            out["G"][who, n:] += dz.sum(0)
    return {name: torch.cat(v) if isinstance(v, list) else v for name, v in out.items()}


def exact(case, seed):
    global own
    was, own = own, False                                     # (the inputs alone: nothing that a call needs beside them)
    try:
        st = prepare(case, seed)
    finally:
        own = was
    return _exact_embed(st) if case["kind"] == "embed" else _exact_loss(st)
