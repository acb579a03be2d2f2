"""Routing of rows to experts, in float64.  TEST INFRASTRUCTURE: the plain
statement of what the library's router computes, one row after the other.

s = softmax(l) or the logistic function of l; t = s + bias.  An expert whose
logit or bias is -inf cannot be chosen.  The experts form groups of consecutive
ids; a group's value is the sum of its group_best largest t; the top_groups
groups of the largest value stay, of their experts the k largest t are chosen
(ties: the lower group or id).  Weights are s of the chosen, divided by their
sum (renorm) and multiplied by a factor.  Places left over: id -1, weight 0.  A
row with a NaN or +inf logit or bias: ids -1, weights NaN.

Pins (tests/test_oracle_routing.py): PyTorch's softmax, sigmoid and topk, hand
examples (groups, ties, masks), and the invariances of the definition.
"""
import math

import numpy as np


def route_row(l, k, score="softmax", bias=None, n_groups=1, top_groups=1, group_best=1, renorm=True, factor=1.0):
    l = [float(v) for v in l]
    E = len(l)
    b = [0.0] * E if bias is None else [float(v) for v in bias]
    if any(math.isnan(v) or v == math.inf for v in l + b):
        return [-1] * k, [math.nan] * k
    if score == "softmax":
        top = max(l)
        e = [math.exp(v - top) if v > -math.inf else 0.0 for v in l]
        total = math.fsum(e)
        s = [v / total if total > 0 else 0.0 for v in e]
    else:
        s = [0.0 if v < -700 else 1.0 / (1.0 + math.exp(-v)) for v in l]
    t = {i: s[i] + b[i] for i in range(E) if l[i] > -math.inf and b[i] > -math.inf}
    per = E // n_groups
    values = {}
    for g in range(n_groups):
        best = sorted((t[i] for i in range(g * per, (g + 1) * per) if i in t), reverse=True)[:group_best]
        if best:
            values[g] = sum(best)
    stay = set(sorted(values, key=lambda g: (-values[g], g))[:top_groups])
    ids = sorted((i for i in t if i // per in stay), key=lambda i: (-t[i], i))[:k]
    w = [s[i] for i in ids]
    if renorm:
        total = math.fsum(w)
        w = [v / total if total > 0 else 0.0 for v in w]
    w = [v * factor for v in w]
    return ids + [-1] * (k - len(ids)), w + [0.0] * (k - len(w))


def route(logits, k, **kw):
    """logits [rows][experts] -> ids int32, weights float64 [rows][k]."""
    out = [route_row(l, k, **kw) for l in logits]
    return (np.array([o[0] for o in out], dtype=np.int32).reshape(len(out), k),
            np.array([o[1] for o in out], dtype=np.float64).reshape(len(out), k))
