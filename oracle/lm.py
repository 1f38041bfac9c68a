"""64-bit oracle of the layer norm and of the calls on rows of logits (test infrastructure, not product code).

Plain numpy in float64, written from the definitions and sharing nothing with the CUDA path.  Matrices are float64
arrays of the rows' columns that count; the caller has rounded them to the type the kernels read.
"""
from __future__ import annotations

from typing import NamedTuple, Optional

import numpy as np


class NormFwd(NamedTuple):
    y: np.ndarray
    mean: np.ndarray
    rstd: np.ndarray


class NormBwd(NamedTuple):
    dx: np.ndarray
    dweight: np.ndarray
    dbias: np.ndarray


def layer_norm_fwd(x, weight, bias, eps) -> NormFwd:
    mean = x.mean(axis=1)
    rstd = 1.0 / np.sqrt(((x - mean[:, None]) ** 2).mean(axis=1) + eps)
    h = (x - mean[:, None]) * rstd[:, None]
    return NormFwd(h * (1.0 if weight is None else weight) + (0.0 if bias is None else bias), mean, rstd)


def layer_norm_bwd(dy, x, weight, mean, rstd) -> NormBwd:
    h = (x - mean[:, None]) * rstd[:, None]
    g = dy * (1.0 if weight is None else weight)
    dx = rstd[:, None] * (g - g.mean(axis=1, keepdims=True) - h * (g * h).mean(axis=1, keepdims=True))
    return NormBwd(dx, (dy * h).sum(axis=0), dy.sum(axis=0))


class LogProbs(NamedTuple):
    logp: np.ndarray          # [rows, vocab]
    entropy: np.ndarray
    max: np.ndarray
    logsum: np.ndarray


def log_probs(x, inv_t) -> LogProbs:
    rows, vocab = x.shape
    out = LogProbs(np.empty((rows, vocab)), np.empty(rows), np.empty(rows), np.empty(rows))
    for i in range(rows):
        z = x[i] * inv_t
        if np.isnan(z).any() or (z == np.inf).any():
            out.logp[i], out.entropy[i], out.logsum[i] = np.nan, np.nan, np.nan
            out.max[i] = np.max(z[~np.isnan(z)]) if (~np.isnan(z)).any() else -np.inf
            continue
        m = z.max()
        out.max[i] = m
        if m == -np.inf:
            out.logp[i], out.entropy[i], out.logsum[i] = -np.inf, 0.0, 0.0
            continue
        s = np.log(np.exp(z - m).sum())
        lp = z - m - s
        live = lp > -np.inf
        out.logp[i], out.logsum[i] = lp, s
        out.entropy[i] = -(np.exp(lp[live]) * lp[live]).sum()
    return out


def top_columns(row, k) -> np.ndarray:
    """The k best columns of one row: by value, NaN last, equal values by the lower column."""
    value = np.where(np.isnan(row), -np.inf, row)
    return np.lexsort((np.arange(len(row)), -value, np.isnan(row)))[:k].astype(np.int32)


def log_probs_bwd(x, inv_t, tokens, maximum, logsum, entropy, grad_logprob, grad_entropy) -> np.ndarray:
    rows, vocab = x.shape
    out = np.zeros((rows, vocab))
    for i in range(rows):
        if maximum[i] == -np.inf:
            continue
        lp = x[i] * inv_t - maximum[i] - logsum[i]
        p = np.exp(lp)
        if grad_logprob is not None and 0 <= tokens[i] < vocab:
            out[i] -= grad_logprob[i] * p
            out[i, tokens[i]] += grad_logprob[i]
        if grad_entropy is not None:
            live = p > 0
            out[i, live] -= grad_entropy[i] * p[live] * (lp[live] + entropy[i])
            out[i, np.isnan(p)] = np.nan
    return out * inv_t


class Distill(NamedTuple):
    loss: np.ndarray
    grad: np.ndarray


def distill(x, inv_t, ids, t, tail: bool, grad_loss: Optional[np.ndarray]) -> Distill:
    rows, vocab = x.shape
    loss, grad = np.zeros(rows), np.zeros((rows, vocab))
    for i in range(rows):
        z = x[i] * inv_t
        slots = [(int(c), float(v)) for c, v in zip(ids[i], t[i]) if 0 <= c < vocab]
        nan_teacher = any(np.isnan(v) for _, v in slots)
        weight = [v for _, v in slots if v > -np.inf]
        if not tail and not weight and not nan_teacher:
            continue
        if not np.isnan(z).any() and z.max() == -np.inf:
            continue
        if nan_teacher or np.isnan(z).any() or z.max() == np.inf:
            loss[i], grad[i] = np.nan, np.nan
            continue
        top = 0.0 if tail else max(weight)
        norm = 0.0 if tail else top + np.log(sum(np.exp(v - top) for v in weight))
        m = z.max()
        e = np.exp(z - m)
        log_total = np.log(e.sum())
        p = e / e.sum()
        mass = np.zeros(vocab)
        named = np.zeros(vocab, dtype=bool)
        q_sum = 0.0
        for c, v in slots:
            named[c] = True
            if v == -np.inf:
                continue
            q = np.exp(v - norm)
            mass[c] += q
            q_sum += q
            loss[i] += np.inf if z[c] == -np.inf else q * ((v - norm) - (z[c] - m - log_total))
        grad[i] = p - mass
        if tail:
            q_r = max(0.0, 1.0 - q_sum)
            rest = z[~named]
            if rest.size and rest.max() > -np.inf:
                r = rest.max()
                share = np.exp(rest - r)
                log_p_r = r + np.log(share.sum()) - m - log_total
                if q_r > 0:
                    loss[i] += q_r * (np.log(q_r) - log_p_r)
                grad[i, ~named] = share / share.sum() * (np.exp(log_p_r) - q_r)
            else:
                grad[i, ~named] = 0.0
    scale = np.ones(rows) if grad_loss is None else grad_loss
    return Distill(loss, grad * (scale * inv_t)[:, None])
