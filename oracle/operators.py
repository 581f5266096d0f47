"""CPU reference of the operators for the last layers of a language model or
classifier (log probabilities and their gradient, orthogonalised updates, linear
layers in 8-bit integers), in fp64 numpy from their definitions.

TEST INFRASTRUCTURE ONLY, like ``oracle.mlp``: it shares no code with the GPU
library.  Where the definition itself rounds to fp32 (scaled logits, quantised
rows) the same fp32 operation is made here; everything else is fp64.
"""

from __future__ import annotations

import numpy as np

QUINTIC = (3.4445, -4.7750, 2.0315)
STEPS = 5


# -- log probabilities --------------------------------------------------------
def scaled(x: np.ndarray, scale: float) -> np.ndarray:
    """z = scale x in fp32, as fp64 values."""
    with np.errstate(over="ignore", invalid="ignore"):
        return (x.astype(np.float32) * np.float32(scale)).astype(np.float64)


def _rows(z):
    """(m, log s, p, log p, H) of each row; a row of minus infinities has log p of
    minus infinity and H = 0."""
    with np.errstate(all="ignore"):
        m = z.max(axis=1)
        empty = np.isneginf(m)
        d = z - np.where(empty, 0.0, m)[:, None]
        e = np.exp(d)
        s = e.sum(axis=1)
        ln = np.where(empty, -np.inf, np.log(s))
        p = e / np.where(empty, 1.0, s)[:, None]
        lp = np.where(empty[:, None], -np.inf, d - ln[:, None])
        terms = np.where(p == 0.0, 0.0, p * lp)
        return m, ln, p, lp, -terms.sum(axis=1)


def logprobs(x, scale=1.0, targets=None, n_top=0):
    """(log p of the targets, H, stat, ids, their log p)."""
    z = scaled(x, scale)
    n, v = z.shape
    m, ln, p, lp, entropy = _rows(z)
    logp = np.zeros(n)
    for i in range(n):
        t = -1 if targets is None else int(targets[i])
        logp[i] = 0.0 if t < 0 else np.nan if t >= v else lp[i, t]
    # NaN above all, then falling values, equal ones by index
    key = np.where(np.isnan(z), np.inf, z)
    order = np.lexsort((np.broadcast_to(np.arange(v), z.shape), -key, ~np.isnan(z)), axis=1)[:, :n_top]
    return logp, entropy, np.stack((m, ln), 1), order.astype(np.int32), np.take_along_axis(lp, order, 1)


def logprobs_grad(x, scale, targets, g, h):
    """d(sum of g log p_t + h H)/dx."""
    z = scaled(x, scale)
    n, v = z.shape
    m, ln, p, lp, entropy = _rows(z)
    dx = np.zeros_like(z)
    for i in range(n):
        t = -1 if targets is None else int(targets[i])
        if np.isneginf(m[i]) and t < v:
            continue
        gi = 0.0 if t < 0 or g is None else np.nan if t >= v else float(g[i])
        hi = 0.0 if h is None else float(h[i])
        dx[i] = -gi * p[i] - hi * np.where(p[i] == 0.0, 0.0, p[i] * (lp[i] + entropy[i]))
        if 0 <= t < v:
            dx[i, t] += gi
    return np.float64(np.float32(scale)) * dx


# -- orthogonalised updates -----------------------------------------------------
def orthogonalize(u: np.ndarray) -> np.ndarray:
    u = np.asarray(u, np.float64)
    norm = np.sqrt((u * u).sum())
    x = u / norm if norm != 0.0 else u
    turned = x.shape[0] > x.shape[1]
    if turned:
        x = x.T
    a, b, c = QUINTIC
    for _ in range(STEPS):
        gram = x @ x.T
        x = a * x + (b * gram + c * gram @ gram) @ x
    return x.T if turned else x


def muon_step(w, m, g, eta, momentum, nesterov, decay):
    w, m, g = (np.asarray(v, np.float64) for v in (w, m, g))
    m2 = momentum * m + g
    o = orthogonalize(g + momentum * m2 if nesterov else m2)
    return w * (1.0 - eta * decay) - eta * np.sqrt(max(1.0, w.shape[0] / w.shape[1])) * o, m2


# -- linear layers in 8-bit integers ----------------------------------------------
def quantize_rows(x: np.ndarray):
    """(q int8, scale fp32) of rows, in fp32 as the definition has it."""
    x = x.astype(np.float32)
    most = np.abs(x).max(axis=1)
    ok = np.isfinite(most) & (most > 0)
    with np.errstate(all="ignore"):
        factor = np.float32(127.0) / np.where(ok, most, np.float32(1.0))
        q = np.where(ok[:, None], np.rint(x * factor[:, None]), 0.0)
        scale = np.where(np.isfinite(most), most / np.float32(127.0), np.nan).astype(np.float32)
    return np.nan_to_num(np.clip(q, -127, 127)).astype(np.int8), scale


def linear_i8(xq, x_scale, wq, w_scale, bias=None, act=None):
    z = (xq.astype(np.int64) @ wq.astype(np.int64).T).astype(np.float64)
    z = z * x_scale.astype(np.float64)[:, None] * w_scale.astype(np.float64)[None, :]
    if bias is not None:
        z = z + bias.astype(np.float64)[None, :]
    with np.errstate(all="ignore"):
        if act is None:
            return z
        f = {"relu": lambda v: np.maximum(v, 0.0), "sigmoid": lambda v: 1.0 / (1.0 + np.exp(-v)),
             "tanh": np.tanh, "gaussian": lambda v: np.exp(-v * v),
             "step": lambda v: (v > 0).astype(np.float64)}[act](z)
        return np.where(np.isnan(z), np.nan, f)
