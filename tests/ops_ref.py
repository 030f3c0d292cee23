"""Plain 64-bit forms of the dense product and of routing by scores, for the
tests: numpy, one token at a time."""

import math

import numpy as np


def linear_fn(fn, v):
    v = np.asarray(v, np.float64)
    with np.errstate(over="ignore"):
        if fn == "relu":
            return np.where(np.isnan(v), v, np.maximum(v, 0.0))
        if fn == "silu":
            return v / (1.0 + np.exp(-v))
        if fn == "gelu":
            return 0.5 * v * np.vectorize(math.erfc)(-v / math.sqrt(2.0)) if v.size else v
        if fn == "gelu_tanh":
            return 0.5 * v * (1.0 + np.tanh(math.sqrt(2.0 / math.pi) * (v + 0.044715 * v ** 3)))
    return v


def linear(x, w, scale=None, bias=None, fn="none", residual=None):
    """(y, sum of |products| per output) of float64 arrays."""
    w = w if scale is None else w * scale[:, None]
    v = x @ w.T
    size = np.abs(x) @ np.abs(w).T
    if bias is not None:
        v = v + bias
        size = size + np.abs(bias)
    y = linear_fn(fn, v)
    return (y if residual is None else y + residual), size


def route(logits, k, bias=None, score="softmax", n_groups=1, top_groups=1, group_top=1, renorm=True, scale=1.0):
    """Expert ids and float64 weights by the rule's text."""
    T, E = logits.shape
    per = E // n_groups
    idx, wts = np.zeros((T, k), np.int32), np.zeros((T, k))
    for t in range(T):
        l = [float(v) for v in logits[t]]
        live = [math.isfinite(v) for v in l]
        top = max((v for v, ok in zip(l, live) if ok), default=0.0)

        def sigmoid(v):
            return 1.0 / (1.0 + math.exp(-v)) if v > -700 else 0.0

        if score == "sigmoid":
            s = [sigmoid(v) if ok else 0.0 for v, ok in zip(l, live)]
        else:
            s = [math.exp(v - top) if ok else 0.0 for v, ok in zip(l, live)]
            z = sum(s)
            s = [v / z if z else 0.0 for v in s]
        if bias is None:
            choice, pick = s, l
        else:
            choice = [a + float(b) for a, b in zip(s, bias)]
            live = [ok and math.isfinite(c) for ok, c in zip(live, choice)]
            s = [v if ok else 0.0 for v, ok in zip(s, live)]
            pick = choice
        kept = list(range(E))
        if n_groups > 1:
            def worth(g):
                ids = [e for e in range(g * per, g * per + per) if live[e]]
                if not ids:
                    return -math.inf
                if group_top == 1 and bias is None:
                    return max(l[e] for e in ids)
                return sum(sorted((choice[e] for e in ids), reverse=True)[:group_top])

            order = sorted(range(n_groups), key=lambda g: (-worth(g), g))[:top_groups]
            kept = [e for g in sorted(order) for e in range(g * per, g * per + per)]
        ids = sorted(kept, key=lambda e: (not live[e], -pick[e] if live[e] else 0.0, e))[:k]
        w = [s[e] for e in ids]
        if renorm:
            z = sum(w)
            w = [v / z if z else 0.0 for v in w]
        idx[t], wts[t] = ids, [scale * v for v in w]
    return idx, wts
