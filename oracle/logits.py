"""TEST INFRASTRUCTURE ONLY -- the bending of logits by definition, in 64 bits with numpy."""

from __future__ import annotations

import numpy as np

PROMPT = 1 << 30


def path(tree, j):
    """Rows of the tree's contiguous cache on query j's path."""
    rows, u = [], int(tree.query_node[j])
    while u >= 0:
        rows.append(np.arange(tree.node_tok_begin[u], tree.node_tok_begin[u] + tree.node_tok_len[u]))
        u = int(tree.node_parent[u])
    return np.concatenate(rows)


def adjust(tree, x, tokens, repetition=None, frequency=None, presence=None, bias=None, bias_row=None, mask=None, mask_row=None):
    """(logits, mag) of float64 x [nq, vocab]; tokens: of the rows of the tree's contiguous cache.  mag: the sum of the magnitudes of
    the terms that a logit is made of."""
    x = np.array(x, dtype=np.float64)
    nq, vocab = x.shape
    mag = np.abs(x)
    with np.errstate(invalid="ignore", over="ignore"):
        for j in range(nq):
            if repetition is not None or frequency is not None or presence is not None:
                t = np.asarray(tokens)[path(tree, j)].astype(np.int64)
                t = t[(t >= 0) & (t % PROMPT < vocab)]
                every, c = np.bincount(t % PROMPT, minlength=vocab), np.bincount(t[t < PROMPT], minlength=vocab)
                if repetition is not None:
                    r = float(repetition[j])
                    x[j] = np.where(every > 0, np.where(x[j] > 0, x[j] / r, x[j] * r), x[j])
                f = 0.0 if frequency is None else float(frequency[j])
                p = 0.0 if presence is None else float(presence[j])
                mag[j] = np.abs(x[j]) + np.where(c > 0, abs(f) * c + abs(p), 0)
                x[j] = np.where(c > 0, x[j] - (f * c + p), x[j])
            b = 0 if bias_row is None else int(bias_row[j])
            if bias is not None and 0 <= b < len(bias):
                mag[j] += np.abs(bias[b])
                x[j] += bias[b]
            m = 0 if mask_row is None else int(mask_row[j])
            if mask is not None and 0 <= m < len(mask):
                for v in range(vocab):
                    if not (int(mask[m][v // 32]) >> (v % 32)) & 1:
                        x[j, v] = -np.inf
    return x, mag
