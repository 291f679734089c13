"""Drawing tokens under temperature, top-k, top-p and min-p (oracle; test
infrastructure), in float64 with sums of high precision."""

import math

import numpy as np

__all__ = ["sample_row_ref"]


def sample_row_ref(x, u, temperature=1.0, top_k=0, top_p=1.0, min_p=0.0):
    """(token, prob, slack) of one row of logits: slack is how far, relative to the sum, the nearest border that the
    answer depends on is from another answer (of top-p, of min-p, of the drawn token)."""
    x = np.asarray(x, np.float64)
    live = np.flatnonzero(x > -np.inf)
    if len(live) == 0:
        return -1, 0.0, 1.0
    order = live[np.lexsort((live, -x[live]))]
    if not temperature > 0:
        return int(order[0]), 1.0, 1.0
    order = order[:top_k] if top_k > 0 else order
    w = np.exp((x[order] - x[order[0]]) / float(temperature))
    sums = np.concatenate([[0.0], np.cumsum(w)])
    slack, n = 1.0, len(w)
    if top_p < 1:
        target = float(top_p) * math.fsum(w)
        n = max(1, int((sums[:-1] < target).sum()))
        if 0 < target < sums[-1]:
            slack = min(slack, np.abs(sums[1:] - target).min() / sums[-1])
    if min_p > 0:
        n = min(n, max(1, int((w >= float(min_p)).sum())))
        slack = min(slack, np.abs(w[w != 1] / float(min_p) - 1).min(initial=1.0))
    total = sums[n]
    i = min(int((sums[1:n + 1] <= float(u) * total).sum()), n - 1)
    if n > 1:
        slack = min(slack, np.abs(sums[1:n] / total - float(u)).min())
    return int(order[i]), w[i] / total, slack
