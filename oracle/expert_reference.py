"""Routing to experts and low-rank adapters in numpy and 64 bits, from their definitions (include/regione.h): loops and
sorts over Python values, none of the library's code."""
from __future__ import annotations

import math

import numpy as np

FLOAT32_MAX = 3.4028234663852886e38


def _exp(x):
    return math.exp(x) if x < 709.0 else math.inf


def route(logits, bias, mask, score, n_groups, top_groups, group_best, top_k, renormalise, scale):
    """(expert [n, k] int32, weight [n, k] float64); score: "softmax" or "sigmoid"."""
    n, e = logits.shape
    per = e // n_groups
    expert, weight = np.full((n, top_k), -1, np.int32), np.zeros((n, top_k))
    for t in range(n):
        if mask is not None and not mask[t]:
            continue
        l = [float(v) for v in logits[t]]
        l = [-math.inf if math.isnan(v) else min(v, FLOAT32_MAX) for v in l]
        top = max(l)
        if top == -math.inf:
            continue
        if score == "softmax":
            p = [math.exp(v - top) if v > -math.inf else 0.0 for v in l]
            total = math.fsum(p)
            s = [v / total for v in p]
        else:
            s = [1.0 / (1.0 + _exp(-v)) if v > -math.inf else 0.0 for v in l]
        c = [s[i] + float(bias[i]) if bias is not None else s[i] for i in range(e)]
        out = [l[i] == -math.inf or math.isnan(c[i]) or c[i] == -math.inf for i in range(e)]
        order = list(range(e))
        if n_groups > 1:
            value = []
            for g in range(n_groups):
                best = sorted((c[i] for i in range(g * per, (g + 1) * per) if not out[i]), reverse=True)[:group_best]
                value.append(sum(best[1:], best[0]) if best else -math.inf)
            kept = sorted(range(n_groups), key=lambda g: (-value[g], g))[:top_groups]
            order = [i for i in order if i // per in kept]
        by = c if bias is not None else l
        chosen = sorted((i for i in order if not out[i]), key=lambda i: (-by[i], i))[:top_k]
        if score == "softmax" and renormalise and chosen:            # free of the other experts' size
            ref = max(l[i] for i in chosen)
            w = [math.exp(l[i] - ref) for i in chosen]
        else:
            w = [s[i] for i in chosen]
        if renormalise:
            total = math.fsum(w)
            w = [v / total if total > 0.0 else 0.0 for v in w]
        expert[t, :len(chosen)] = chosen
        weight[t, :len(chosen)] = [scale * v for v in w]
    return expert, weight


def slots(expert, n_experts, row_token_before):
    """(group_offsets, row_token, slot); entries of row_token past the end are those of `row_token_before`."""
    n, k = expert.shape
    pairs = [[] for _ in range(n_experts)]
    for t in range(n):
        for j in range(k):
            if 0 <= expert[t, j] < n_experts:
                pairs[expert[t, j]].append((t, j))
    offsets, row_token, slot, at = [0], np.array(row_token_before, np.int32), np.full((n, k), -1, np.int32), 0
    for mine in pairs:
        for t, j in mine:
            row_token[at], slot[t, j] = t, at
            at += 1
        offsets.append(at)
    return np.array(offsets, np.int32), row_token, slot


def combine(rows, slot, weight, base):
    """The sums, and the sums of the absolute values of their terms."""
    n, k = slot.shape
    out = np.zeros((n, rows.shape[1])) if base is None else base.astype(np.float64)
    size = np.abs(out)
    for t in range(n):
        for j in range(k):
            if 0 <= slot[t, j] < rows.shape[0]:
                term = (1.0 if weight is None else float(weight[t, j])) * rows[slot[t, j]].astype(np.float64)
                out[t] = out[t] + term
                size[t] = size[t] + np.abs(term)
    return out, size


def adapters(x, w, bias, a, b, which, weight):
    """x W^T + bias + the adapters' shares, each row's own; and the same with absolute values of everything."""
    y = x @ w.T + (0.0 if bias is None else bias)
    size = np.abs(x) @ np.abs(w).T + (0.0 if bias is None else np.abs(bias))
    for r in range(x.shape[0]):
        for s in range(which.shape[1]):
            i = which[r, s]
            if 0 <= i < a.shape[0]:
                f = 1.0 if weight is None else float(weight[r, s])
                y[r] += b[i] @ (f * (a[i] @ x[r]))
                size[r] += np.abs(b[i]) @ (abs(f) * (np.abs(a[i]) @ np.abs(x[r])))
    return y, size


def gelu_tanh(y):
    return 0.5 * y * (1.0 + np.tanh(math.sqrt(2.0 / math.pi) * (y + 0.044715 * y ** 3)))
