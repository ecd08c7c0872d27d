"""Plain statements of the score-row operators in 64 bits, for the tests (no code of the package)."""
import math

import numpy as np

UNIT = {"f32": 2.0 ** -24, "f16": 2.0 ** -11, "bf16": 2.0 ** -8}   # half a step, relative
TINY = {"f32": 2.0 ** -126, "f16": 2.0 ** -24, "bf16": 2.0 ** -126}  # f16: half a step below the normal range is 2^-25


def act64(name, y):
    import torch
    if name == "relu":
        return torch.clamp(y, min=0.0)
    if name == "sigmoid":
        return torch.special.expit(y)
    if name == "tanh":
        return torch.tanh(y)
    if name == "gelu":
        return 0.5 * y * torch.special.erfc(-y / math.sqrt(2.0))
    if name == "silu":
        return y * torch.special.expit(y)
    return y


# largest slope of each activation
SLOPE = {"none": 1.0, "relu": 1.0, "sigmoid": 0.25, "tanh": 1.0, "gelu": 1.13, "silu": 1.10}


def layer64(x, weight, bias, act, scale, residual, residual_scale, out):
    """x [..., K], weight [N, K], residual [..., N] -> (result in 64 bits, bound on what fp32 sums and one rounding to
    `out` may add).  A sum of K products and the bias in fp32, in any order, is off by at most (K + 1) steps of 2^-23 of
    the sum of the magnitudes (2^-24 where every addition rounds to nearest; twice that is granted).  The activations'
    fp32 functions are off by at most 8 half steps of a value of at most max(1, |y|)."""
    import torch
    x, weight = x.double(), weight.double()
    K = x.shape[-1]
    y = x @ weight.t()
    mag = x.abs() @ weight.abs().t()
    if bias is not None:
        y = y + bias.double()
        mag = mag + bias.double().abs()
    z = act64(act, y)
    err = SLOPE[act] * (K + 1) * 2.0 ** -23 * mag
    if act not in ("none", "relu"):
        err = err + 8 * 2.0 ** -24 * y.abs().clamp(min=1.0)
    r = scale * z
    err = abs(scale) * (err + 2.0 ** -24 * z.abs())
    if residual is not None:
        r = r + residual_scale * residual.double()
        err = err + 2.0 ** -24 * (r.abs() + (residual_scale * residual.double()).abs())
    err = err + UNIT[out] * (r.abs() + err) + TINY[out]
    return r, err


def sample_row(x, random, temperature=1.0, top_k=0, top_p=1.0, min_p=0.0, listed=None, offset=0.0):
    """One row of fp32 scores (numpy) -> (label, log-probability, kept)."""
    x = np.asarray(x, np.float32).copy()
    if listed is not None and len(listed):
        at = np.unique(np.asarray(listed))
        x[at] = x[at] + np.float32(offset)
    with np.errstate(invalid="ignore"):
        keep = np.flatnonzero(x > -np.inf)
    if keep.size == 0:
        return -1, -math.inf, 0
    best = x[keep].max()
    if best == np.inf:
        keep = keep[x[keep] == np.inf]
    keep = keep[np.argsort(-x[keep].astype(np.float64), kind="stable")]
    if not temperature > 0:
        return int(keep[0]), 0.0, 1
    d = np.zeros(keep.size) if best == np.inf else (x[keep].astype(np.float64) - float(best)) / float(temperature)
    if 0 < top_k < keep.size:
        keep, d = keep[:top_k], d[:top_k]
    w = np.exp(d)
    n = keep.size
    if top_p < 1.0:
        before = np.concatenate([[0.0], np.cumsum(w)[:-1]])
        n = max(1, int(np.sum(before < float(top_p) * w.sum())))
    if min_p > 0.0:
        n = min(n, int(np.sum(w >= min(float(min_p), 1.0))))
    keep, d, w = keep[:n], d[:n], w[:n]
    back = np.argsort(keep)
    upto = np.cumsum(w[back])
    u = min(max(float(random), 0.0), 1.0) if random == random else 0.0
    passed = np.flatnonzero(upto > u * upto[-1])
    at = back[passed[0]] if passed.size else back[np.flatnonzero(w[back] > 0)[-1]]
    return int(keep[at]), float(d[at] - math.log(upto[-1])), int(n)
