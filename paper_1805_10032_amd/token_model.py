"""A model that answers with tokens, evaluated by the library's operators: layer norm and a linear layer, any number of times, the last
one into the vocabulary; f is the mean of -log p(label) over the tokens that count.

It stands on both sides of Algorithm 1.  A worker's gradient goes straight into its row of G (TokenModel.gradients: all workers'
tokens in one pass, activations kept in 8 bits for the backward pass), and the server scores the candidates from the log
probabilities of the m + 1 models (TokenModel.scores, Definition 2); zeno_aggregate_update takes them from there.

A parameter vector holds, layer by layer: the norm's weight and bias [width], the linear layer's weights [out x width] row-major
and its bias [out], all float32.  A model with `inputs` takes tokens instead of hidden states: a table [inputs x width] stands in front of the
layers, and its rows times sqrt(width) are the hidden states.  With `tied` the table is the last layer's weights too, which then have no
block of their own.

With keep_logits=False the logits are not formed: zeno_linear_logprobs takes the last layer's log probabilities and gradients straight from its input, whose
weights' gradients then come from that input itself instead of its 8 bits.

The operators' inputs and outputs are of the model's dtype, and so is what they cost in precision: activations are kept in 8 bits whatever the dtype
(a term of a weight's gradient is off by up to 2^-4 of itself), and scores are differences of log probabilities whose logits are half a step off.  A
server that needs them finer scores with a float32 model: the parameter vector is the same.
"""
from __future__ import annotations

import torch

from . import binding as B
from .workloads import ATTACKS


class TokenModel:
    """widths = [hidden width, ..., vocabulary]; activations are kept in `dtype`.  inputs: the vocabulary of the tokens that the model takes (None: it
    takes hidden states)."""

    def __init__(self, widths, dtype=torch.bfloat16, eps=1e-5, *, inputs=None, tied=False, keep_logits=True):
        if len(widths) < 2 or min(widths) < 1:
            raise ValueError("widths must name the hidden width and the vocabulary at least")
        if dtype not in B.DTYPE:
            raise ValueError(f"dtype must be one of {list(B.DTYPE)}")
        if inputs is not None and inputs < 1:
            raise ValueError("inputs must be the number of tokens that there are")
        if tied and (inputs is None or inputs != widths[-1] or widths[-2] != widths[0]):
            raise ValueError("a tied table has the last layer's shape: inputs = widths[-1] and widths[0] = widths[-2]")
        self.widths, self.dtype, self.eps = [int(w) for w in widths], dtype, float(eps)
        self.inputs, self.tied, self.keep_logits = None if inputs is None else int(inputs), bool(tied), bool(keep_logits)
        # What fp16's backward pass multiplies a token's gradient by.  Its steps end at 2^-24: the mean's 1/n would push the probabilities of a
        # large vocabulary below them (32000 values, 2500 tokens a worker: nine tenths of dlogits are 0), while 64 keeps 2^-30 of a token's
        # loss, and 65504 / 64 = 1023 times it before a gradient is infinite.  The other types have float32's range and need none.
        self.loss_scale = 64.0 if dtype == torch.float16 else 1.0
        self.scale = float(self.widths[0]) ** 0.5
        self.offsets, at = [], 0
        self.table = None if inputs is None else (0, self.inputs * self.widths[0])
        if self.table is not None:
            at = self.table[1]
        for i, (width, out) in enumerate(zip(self.widths, self.widths[1:])):
            parts = []
            for j, n in enumerate((width, width, out * width, out)):
                if j == 2 and self.tied and i == len(self.widths) - 2:
                    parts.append(self.table)
                    continue
                parts.append((at, n))
                at += n
            self.offsets.append(parts)
        self.num_params = at

    def init(self, seed=0, device="cuda"):
        """Norm weights 1, N(0, 1/width) weights and table, zero biases."""
        gen = torch.Generator(device=device)
        gen.manual_seed(int(seed))
        x = torch.zeros(self.num_params, dtype=torch.float32, device=device)
        if self.table is not None:
            x[:self.table[1]] = torch.randn(self.table[1], generator=gen, device=device) * self.widths[0] ** -0.5
        for i, ((nw, _, w, _), width) in enumerate(zip(self.offsets, self.widths)):
            x[nw[0]:nw[0] + nw[1]] = 1.0
            if not (self.tied and i == len(self.offsets) - 1):
                x[w[0]:w[0] + w[1]] = torch.randn(w[1], generator=gen, device=device) * width ** -0.5
        return x

    def _views(self, x):
        return [[x[at:at + n] for at, n in parts] for parts in self.offsets]

    def _states(self, x, hidden, keep):
        """The last layer's input, its weights in `dtype` and its bias, and what the backward pass needs of the layers."""
        h, kept = hidden, []
        if self.table is not None:
            h = B.zeno_embedding(hidden, x[:self.table[1]].view(self.inputs, self.widths[0]), self.dtype, scale=self.scale)
        last = len(self.offsets) - 1
        for i, ((norm_w, norm_b, w, b), width, out) in enumerate(zip(self._views(x), self.widths, self.widths[1:])):
            y, mean, rstd, ckpt = B.zeno_layer_norm(h, norm_w, norm_b, self.eps, want_checkpoint=keep)
            w = w.view(out, width).to(self.dtype)
            if keep:
                kept.append((ckpt, mean, rstd, B.zeno_checkpoint(y) if i < last or self.keep_logits else None, w))
            if i < last:
                h = torch.addmm(b.to(self.dtype), y, w.t())
        return y, w, b, kept

    def forward(self, x, hidden, *, keep=False):
        """Logits [tokens x vocabulary] for hidden states [tokens x width] (or int32 tokens); with keep=True also what the backward pass needs."""
        y, w, b, kept = self._states(x, hidden, keep)
        h = torch.addmm(b.to(self.dtype), y, w.t())
        return (h, kept) if keep else h

    def logprobs(self, x, hidden, labels):
        """log p(label) of every token (label -1: 0)."""
        if self.keep_logits:
            return B.zeno_logprobs(self.forward(x, hidden), labels)[0]
        y, w, b, _ = self._states(x, hidden, False)
        return B.zeno_linear_logprobs(y, w, b, labels)[0]

    def gradients(self, x, hidden, labels, groups, G):
        """G[i] = gradient at x of the mean loss over worker i's tokens, rows groups[i] .. groups[i + 1] - 1 (int32 offsets on
        the device); a worker without tokens that count sends zeros.  Returns the log probabilities."""
        m, tokens = G.shape[0], hidden.shape[0]
        if G.shape[1] != self.num_params or groups.numel() != m + 1:
            raise ValueError("G needs a row of num_params for every worker")
        if self.keep_logits:
            logits, kept = self.forward(x, hidden, keep=True)
            logp, _, stats, _, _ = B.zeno_logprobs(logits, labels, want_stats=True)
        else:
            y, w, b, kept = self._states(x, hidden, True)
            logp, _, stats = B.zeno_linear_logprobs(y, w, b, labels, want_stats=True)
        # -1 over the number of the worker's tokens that count
        counted = torch.zeros(tokens + 1, dtype=torch.int64, device=hidden.device)
        torch.cumsum(labels >= 0, 0, out=counted[1:])
        bounds = groups.long()
        per_worker = (counted[bounds[1:]] - counted[bounds[:-1]]).clamp(min=1)
        worker = torch.bucketize(torch.arange(tokens, device=hidden.device), bounds[1:], right=True).clamp(max=m - 1)
        unit = self.dtype == torch.float16    # the tokens' gradients are those of loss_scale times their own loss, not of the mean
        grad = torch.full((tokens,), -self.loss_scale, dtype=torch.float32, device=hidden.device) if unit else (-1.0 / per_worker[worker]).float()
        if self.keep_logits:
            dz = B.zeno_logprobs_backward(logits, stats, labels=labels, grad_logp=grad, out=logits)
        for layer in reversed(range(len(kept))):
            norm_w, norm_b, dw, db = [G[:, at:at + n] for at, n in self.offsets[layer]]
            ckpt_h, mean, rstd, ckpt_y, weights = kept[layer]
            if ckpt_y is None:
                dy, _, _ = B.zeno_linear_logprobs_backward(y, w, b, stats, labels=labels, grad_logp=grad, groups=groups, dweight=dw, dbias=db)
            else:
                B.zeno_weight_gradient(dz, ckpt_y, groups=groups, dweight=dw, dbias=db)
                dy = torch.mm(dz, weights)
            scale = x[self.offsets[layer][0][0]:self.offsets[layer][0][0] + self.offsets[layer][0][1]]
            down = layer > 0 or self.table is not None
            dz, _, _ = B.zeno_layer_norm_backward(dy, ckpt_h, mean, rstd, scale, groups=groups, want_dx=down,
                                                  dx=dy if down else None, dweight=norm_w, dbias=norm_b)
        if self.table is not None:
            B.zeno_embedding_backward(dz, hidden, self.inputs, scale=self.scale, groups=groups, dtable=G[:, :self.table[1]], accumulate=self.tied)
        if unit:
            G *= (1.0 / (self.loss_scale * per_worker)).float()[:, None]
        return logp

    def scores(self, x, G, hidden, labels, gamma, rho):
        """Definition 2 for every row of G on the server's tokens."""
        if G.shape[1] != self.num_params:
            raise ValueError("G needs rows of num_params")
        logp_x = self.logprobs(x, hidden, labels)
        logp = torch.empty((G.shape[0], hidden.shape[0]), dtype=torch.float32, device=hidden.device)
        for i in range(G.shape[0]):
            logp[i] = self.logprobs(torch.add(x, G[i], alpha=-gamma), hidden, labels)
        return B.zeno_score_logprobs(G, logp_x, logp, rho, labels=labels)


def token_worker_gradients(model, G, x, hidden, labels, groups, faulty, attack, *, scale=4.0):
    """Fill G with one iteration's candidates of the workers, those listed in `faulty` failing as worker_gradients describes it:
    label_flip (V-1-label before the gradient), bit_flip (negated, the first faulty row over the others), sign_flip, none."""
    if attack not in ATTACKS:
        raise ValueError(f"attack must be one of {ATTACKS}")
    faulty = list(faulty)
    if attack == "label_flip" and faulty:
        row = torch.arange(labels.numel(), device=labels.device)
        bad = torch.zeros_like(labels, dtype=torch.bool)
        for i in faulty:
            bad |= (row >= groups[i]) & (row < groups[i + 1])
        labels = torch.where(bad & (labels >= 0), model.widths[-1] - 1 - labels, labels).to(torch.int32)
    logp = model.gradients(x, hidden, labels, groups, G)
    if attack == "sign_flip":
        for i in faulty:
            G[i] *= -scale
    elif attack == "bit_flip" and faulty:
        G[faulty[0]] *= -1.0
        for i in faulty[1:]:
            G[i] = G[faulty[0]]
    return logp
