"""The operators of include/igemm_rows.h from their definitions, in float64 and
exact integers on the CPU (numpy and torch), for tests/test_gpu_rows.py."""
from __future__ import annotations

import numpy as np
import torch

FLT_MAX = 3.402823466385288598e38


def route(logits, top_k, bias=None, groups=1, top_groups=1, group_best=1, score="softmax",
          renormalise=True, scale=1.0):
    """logits: a CPU tensor; returns (ids, weights float64, offsets, order)."""
    x = logits.double().numpy()
    T, E = x.shape
    x = np.where(np.isnan(x), -np.inf, np.minimum(x, FLT_MAX))
    used = x > -np.inf
    s = np.zeros((T, E))
    for t in range(T):
        u = used[t]
        if not u.any():
            continue
        if score == "softmax":
            e = np.exp(x[t, u] - x[t, u].max())
            s[t, u] = e / e.sum()
        else:
            with np.errstate(over="ignore"):
                s[t, u] = 1.0 / (1.0 + np.exp(-x[t, u]))
    if bias is None and (groups == 1 or group_best == 1):
        key = np.where(used, x, -np.inf)
    else:
        b = 0.0 if bias is None else bias.double().numpy()
        key = np.where(used, s + b, -np.inf)
    key = np.where(np.isnan(key), -np.inf, key)
    if groups > 1:
        g = -np.sort(-key.reshape(T, groups, -1), axis=2)
        total = g[:, :, 0].copy()
        if group_best == 2 and g.shape[2] > 1:
            total = total + np.where(g[:, :, 1] > -np.inf, g[:, :, 1], 0.0)
        best = np.argsort(-total, axis=1, kind="stable")[:, :top_groups]
        keep = np.zeros((T, groups), bool)
        np.put_along_axis(keep, best, True, axis=1)
        key = np.where(np.repeat(keep, E // groups, axis=1), key, -np.inf)
    best = np.argsort(-key, axis=1, kind="stable")[:, :top_k]
    ok = np.take_along_axis(key, best, axis=1) > -np.inf
    ids = np.where(ok, best, -1).astype(np.int32)
    w = np.where(ok, np.take_along_axis(s, best, axis=1), 0.0)
    if renormalise:
        total = w.sum(1, keepdims=True)
        w = np.divide(w, total, out=np.zeros_like(w), where=total > 0)
    flat = ids.ravel()
    order = np.full(T * top_k, -1, np.int32)
    slots = np.argsort(np.where(flat < 0, E, flat), kind="stable")[: int((flat >= 0).sum())]
    order[: len(slots)] = slots
    counts = np.bincount(flat[flat >= 0], minlength=E)
    offsets = np.concatenate([[0], np.cumsum(counts)]).astype(np.int32)
    return ids, w * scale, offsets, order


def grouped(A, B, offsets, order, scale_a, scale_b, slots, scatter, rows, out):
    """out: a float64 array to update; returns (out, the rows that were written)."""
    written = np.zeros(out.shape[0], bool)
    for g in range(B.shape[0]):
        lo, hi = (min(max(int(v), 0), rows) for v in offsets[g:g + 2])
        for i in range(lo, hi):
            s = i if order is None else int(order[i])
            a = i if slots == 0 else s // slots
            o = s if scatter else i
            if s < 0 or not 0 <= a < A.shape[0] or not 0 <= o < out.shape[0]:
                continue
            y = (A[a].astype(np.int64) @ B[g].astype(np.int64)).astype(np.float64)
            if scale_a is not None:
                y = y * float(scale_a[a])
            if scale_b is not None:
                y = y * scale_b[g].astype(np.float64)
            out[o] = y
            written[o] = True
    return out, written


def adapters(A, B, scale_a, scale_b, ids, down, up, ranks, scaling):
    """(out, base, reach, spread): the result, its shared part, the sum of the
    magnitudes that the adapter's sums run over, and the row's largest |u| times the
    sum of |up| (what a part of u relative to its row's largest value can move)."""
    a = A.astype(np.int64)
    y = (a @ B.astype(np.int64)).astype(np.float64)
    sa = np.ones(len(a)) if scale_a is None else scale_a.astype(np.float64)
    if scale_b is not None:
        y = y * scale_b.astype(np.float64)
    base = y * sa[:, None]
    out, reach, spread = base.copy(), np.zeros_like(base), np.zeros_like(base)
    if ids is None:
        return out, base, reach, spread
    for i, w in enumerate(ids):
        if not 0 <= w < down.shape[0]:
            continue
        r = down.shape[1] if ranks is None else min(max(int(ranks[w]), 0), down.shape[1])
        f = (1.0 if scaling is None else float(scaling[w])) * sa[i]
        d, v = down[w, :r].astype(np.float64), up[w, :, :r].astype(np.float64)
        u = d @ a[i] * f
        out[i] += v @ u
        reach[i] = np.abs(v) @ (np.abs(d) @ np.abs(a[i]) * abs(f))
        spread[i] = np.abs(v).sum(1) * (np.abs(u).max() if r else 0.0)
    return out, base, reach, spread
