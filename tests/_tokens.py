"""Definitions in float64 of the operators for models that answer with tokens, and the error bounds that their tests use.

EPS is half a step of float32 relative to the value; half_step(dtype) that of an output type.  Bounds count roundings: a sum of n
terms whose longest chain of additions is k long is off by at most k EPS sum |term| (to first order)."""
import numpy as np
import torch

EPS = 2.0 ** -24
TYPES = {"fp32": torch.float32, "bf16": torch.bfloat16, "fp16": torch.float16}


def half_step(dtype):
    return torch.finfo(dtype).eps / 2


def smallest_half(dtype):
    """Half a step of the type's subnormals (float32 and bf16 results may be flushed: a whole smallest normal)."""
    return 2.0 ** -25 if dtype == torch.float16 else 2.0 ** -126


def strided(values, dtype, pitch=None, offset=0, device="cuda"):
    """`values` on the device as rows `pitch` elements apart, the first `offset` elements past the start of an allocation;
    everything around them is NaN."""
    rows, cols = values.shape
    pitch = pitch or cols
    buf = torch.full((offset + max(rows, 1) * pitch + 64,), float("nan"), dtype=dtype, device=device)
    view = buf[offset:offset + rows * pitch].view(rows, pitch)[:, :cols]
    view.copy_(values.to(dtype))
    return view, buf


def around(view, buf):
    """A copy of buf with the view's elements taken out: what a call must leave as it was."""
    mask = torch.ones_like(buf, dtype=torch.bool)
    rows, cols = view.shape
    if view.numel():
        off = view.storage_offset() - buf.storage_offset()
        idx = off + torch.arange(rows, device=buf.device)[:, None] * view.stride(0) + torch.arange(cols, device=buf.device)
        mask[idx.reshape(-1)] = False
    return buf[mask].clone()


def logprobs(z, labels, top):
    """z float64 [rows x vocab] (numpy).  logp, entropy, top_index, top_logp, stats, p."""
    z = np.asarray(z, dtype=np.float64)
    rows, vocab = z.shape
    with np.errstate(invalid="ignore", divide="ignore", over="ignore"):
        nan_row = np.isnan(z).any(1) | (z == np.inf).any(1)
        clean = np.where(np.isnan(z), -np.inf, z)
        M = clean.max(1)
        empty = (M == -np.inf) & ~nan_row
        safe = np.where(np.isfinite(M), M, 0.0)
        e = np.exp(z - safe[:, None])
        s = e.sum(1)
        log_s = np.where(empty, 0.0, np.log(np.where(empty, 1.0, s)))
        lp = (z - safe[:, None]) - log_s[:, None]
        p = e / np.where(empty, 1.0, s)[:, None]
        entropy = -np.where(p > 0, p * np.where(p > 0, lp, 0.0), 0.0).sum(1)
        lp[nan_row] = np.nan
        p[nan_row] = np.nan
        entropy[nan_row] = np.nan
        log_s[nan_row] = np.nan
        lp[empty] = -np.inf
        logp = np.zeros(rows)
        if labels is not None:
            for r, y in enumerate(labels):
                logp[r] = 0.0 if y == -1 else (lp[r, y] if 0 <= y < vocab else np.nan)
    order = np.argsort(-clean, axis=1, kind="stable")[:, :top]
    return dict(logp=logp, entropy=entropy, index=order, top_logp=np.take_along_axis(lp, order, 1), M=M, log_s=log_s, p=p, lp=lp,
                empty=empty)


def chain(n, threads, per_load):
    """Additions of the longest chain when `threads` threads each sum their share of n values and the threads' sums are joined."""
    return int(np.ceil(n / (threads * per_load))) * per_load + 16


def e4m3_grid():
    codes = np.arange(127)
    e, f = codes // 8, codes % 8
    return np.where(e == 0, f * 2.0 ** -9, (1 + f / 8) * 2.0 ** (e - 7.0))


def checkpoint(x):
    """(codes uint8 [rows x 32 blocks], scale bytes [rows x blocks]) of x, any float array, from the definition."""
    x = np.asarray(x, dtype=np.float64)
    rows, width = x.shape
    blocks = (width + 31) // 32
    pad = np.zeros((rows, blocks * 32))
    pad[:, :width] = x
    v = pad.reshape(rows, blocks, 32)
    big = np.where(np.isfinite(v), np.abs(v), 0.0).max(2)
    k = np.full(big.shape, -127)
    for i in np.ndindex(*big.shape):
        while big[i] > 448 * 2.0 ** k[i]:
            k[i] += 1
    q = v / (2.0 ** k.astype(float))[:, :, None]
    grid = e4m3_grid()
    t = np.abs(np.where(np.isfinite(q), q, 0.0))
    t = np.where((k == 120)[:, :, None], np.minimum(t, 240.0), t)
    hi = np.clip(np.searchsorted(grid, t), 0, 126)
    lo = np.maximum(hi - 1, 0)
    up, down = grid[hi] - t, t - grid[lo]
    code = np.where((up < down) | ((up == down) & (hi % 2 == 0)), hi, lo)
    code = np.where(np.isfinite(q), code, 127)
    code = code | np.where(np.signbit(q), 128, 0)
    return code.astype(np.uint8).reshape(rows, -1), (k + 127).astype(np.uint8)


def checkpoint_values(codes, scales, width):
    table = np.concatenate([e4m3_grid(), [np.nan]])
    table = np.concatenate([table, -table])
    v = table[codes.astype(int)].reshape(codes.shape[0], -1, 32) * (2.0 ** (scales.astype(float) - 127))[:, :, None]
    return v.reshape(codes.shape[0], -1)[:, :width]


def layer_norm(x, weight, bias, eps):
    x = np.asarray(x, dtype=np.float64)
    mean = x.mean(1)
    var = ((x - mean[:, None]) ** 2).mean(1)
    rstd = 1 / np.sqrt(var + eps)
    xh = (x - mean[:, None]) * rstd[:, None]
    return xh * weight + (0 if bias is None else bias), mean, rstd, xh


def layer_norm_grad(dy, xh, rstd, weight, offsets):
    a = dy * weight
    c1, c2 = a.mean(1, keepdims=True), (a * xh).mean(1, keepdims=True)
    dx = rstd[:, None] * (a - c1 - xh * c2)
    dw = np.stack([(dy[p:q] * xh[p:q]).sum(0) for p, q in zip(offsets, offsets[1:])])
    db = np.stack([dy[p:q].sum(0) for p, q in zip(offsets, offsets[1:])])
    return dx, dw, db, c1, c2
