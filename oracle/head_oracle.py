"""Dropout, log probabilities and softmax cross entropy on fixed-point codes, written from their definitions.

Integers are Python / numpy int64 (dropout), everything else is in extended precision (numpy longdouble).
"""
from __future__ import annotations

import math

import numpy as np

from . import fxp_oracle as orc

SR, RN_HALF_UP = orc.SR, orc.RN_HALF_UP


def drop_threshold(p: float) -> int:
    """T: the 16-bit draws below it drop their element."""
    return math.floor(p * 65536 + 0.5)


def dropout_with_bits(x, fl_x, p, wl_o, fl_o, bits, mode=SR, res=None, fl_res=0):
    """The rule for given draws: floor((X + u)/K) where the draw is at least T."""
    x = np.asarray(x, dtype=np.int64)
    drop = drop_threshold(p)
    keep = 65536 - drop
    up = 16 + fl_o - fl_x
    big = x * (1 << up) if up >= 0 else x >> -up
    u = bits - drop if mode == SR else np.int64(keep // 2)
    y = np.where(bits >= drop, (big + u) // keep, 0)
    if res is not None:
        y = y + np.asarray(res, dtype=np.int64) * (1 << (fl_o - fl_res))
    return np.clip(y, -(1 << (wl_o - 1)), (1 << (wl_o - 1)) - 1)


def dropout(x, fl_x, p, wl_o, fl_o, mode=SR, seed=0, stream=0, res=None, fl_res=0):
    x = np.asarray(x)
    bits = orc.rounding_bits(x.size, SR, seed, stream).reshape(x.shape)
    return dropout_with_bits(x, fl_x, p, wl_o, fl_o, bits, mode, res, fl_res)


def values(logits, fl):
    """Codes (fl = None: fp32 values) as extended-precision numbers."""
    x = np.asarray(logits).astype(np.longdouble)
    return x if fl is None else x / np.longdouble(2) ** fl


def _row(x):
    """(kind, largest value, sum of exp(x - largest)) of a row: kind 'nan', 'empty' or 'ok'."""
    if np.any(np.isnan(x)) or np.any(np.isposinf(x)):
        return "nan", None, None
    m = x.max()
    if np.isneginf(m):
        return "empty", None, None
    return "ok", m, np.exp(x - m).sum()


def log_probs(logits, fl, labels, topk):
    """Returns dict(logp, lse, entropy, top_idx, top_logp, scale): longdouble; scale = sum p |x - m| + |m|, what the
    entropy's rounding errors are relative to."""
    x = values(logits, fl)
    rows, classes = x.shape
    out = {k: np.zeros(rows, dtype=np.longdouble) for k in ("logp", "lse", "entropy", "scale")}
    out["top_idx"] = np.zeros((rows, topk), dtype=np.int32)
    out["top_logp"] = np.zeros((rows, topk), dtype=np.longdouble)
    for i in range(rows):
        kind, m, s = _row(x[i])
        rank = np.where(np.isnan(x[i]), -np.inf, x[i])
        top = np.argsort(-rank, kind="stable")[:topk]
        out["top_idx"][i] = top
        if kind == "ok":
            lse = m + np.log(s)
            lp = x[i] - lse
            p = np.exp(lp)
            out["entropy"][i] = -np.sum(np.where(p > 0, p * np.where(p > 0, lp, 0), 0))
            out["scale"][i] = np.sum(np.where(p > 0, p * np.abs(np.where(p > 0, x[i] - m, 0)), 0)) + abs(m)
        else:
            lse = np.longdouble(np.nan if kind == "nan" else -np.inf)
            lp = np.full(classes, lse)
            out["entropy"][i] = np.nan if kind == "nan" else 0.0
        out["lse"][i] = lse
        out["top_logp"][i] = lp[top]
        if labels is not None:
            out["logp"][i] = 0.0 if labels[i] < 0 else lp[labels[i]] if labels[i] < classes else np.nan
    return out


def gradient(logits, fl, labels, weights=None):
    """weights (softmax - onehot), longdouble; zero rows where there is no label or no distribution."""
    x = values(logits, fl)
    g = np.zeros(x.shape, dtype=np.longdouble)
    for i in range(x.shape[0]):
        kind, m, s = _row(x[i])
        if kind != "ok" or not 0 <= labels[i] < x.shape[1]:
            continue
        e = np.exp(x[i] - m)
        hit = -np.delete(e, labels[i]).sum()
        e[labels[i]] = hit
        g[i] = e / s * (np.longdouble(1) if weights is None else np.longdouble(weights[i]))
    return g


def loss(logits, fl, labels, weights=None):
    """-sum_i weights_i logp_i in extended precision."""
    lp = log_probs(logits, fl, labels, 0)["logp"]
    return -np.sum(lp * (1 if weights is None else np.asarray(weights, dtype=np.longdouble)))


def quantize_real(g, wl, fl, mode=SR, seed=0, stream=0):
    """Quantize's rule for real values: element i of the flattened tensor takes draw i."""
    lim = np.longdouble(2) ** (wl - 1)
    t = np.floor(np.clip(g * np.longdouble(2) ** fl, -lim, lim - 1) * 65536).astype(np.int64)
    q = (t + orc.rounding_bits(g.size, mode, seed, stream).reshape(g.shape)) >> 16
    return np.minimum(q, (1 << (wl - 1)) - 1)
