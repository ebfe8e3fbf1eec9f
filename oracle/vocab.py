"""fp64 oracle of the embedding and of low-rank adapters: row by row from the
definitions. Inputs are the values the device arrays hold, as float64.

TEST INFRASTRUCTURE ONLY (see the package docstring).

    out[t] = scale * table[token t]                  (zeros for a token outside the table)
    out[t] = base[t] + s_k (x[t] a_k^T) b_k^T        k = rows[t] (base[t] for k outside the adapters)

and their gradients. The sums of magnitudes beside the results are what rounding
errors are measured against.

Pins (tests/test_vocab_oracle.py): hand-made rows; float64 autograd.
"""

from __future__ import annotations

import numpy as np


def embedding(table, tokens, scale):
    """scale * table[token] per token, zeros for a token outside the table."""
    out = np.zeros((len(tokens), table.shape[1]))
    for t, v in enumerate(tokens):
        if 0 <= v < table.shape[0]:
            out[t] = scale * table[v]
    return out


def embedding_backward(grad, tokens, V, scale):
    """(gradient [V, d] of the table, the sum of the magnitudes behind each element, rows behind each token)."""
    total, size, n = np.zeros((V, grad.shape[1])), np.zeros((V, grad.shape[1])), np.zeros(V, dtype=np.int64)
    for t, v in enumerate(tokens):
        if 0 <= v < V:
            total[v] += grad[t]
            size[v] += np.abs(grad[t])
            n[v] += 1
    return scale * total, abs(scale) * size, n


def adapters_add(base, x, rows, a, b, scales):
    """(base + the rows' adapters [T, N], the magnitude of what is summed for each element)."""
    T = x.shape[0]
    out = np.zeros((T, b.shape[1])) if base is None else base.copy()
    size = np.abs(out)
    for t in range(T):
        k = rows[t]
        if 0 <= k < a.shape[0]:
            s = 1.0 if scales is None else scales[k]
            out[t] += s * (b[k] @ (a[k] @ x[t]))
            size[t] += abs(s) * (np.abs(b[k]) @ (np.abs(a[k]) @ np.abs(x[t])))
    return out, size


def adapters_backward(grad, x, rows, a, b, scales):
    """((grad_x, grad_a, grad_b), the magnitudes of what is summed for each of their elements)."""
    out = np.zeros(x.shape), np.zeros(a.shape), np.zeros(b.shape)
    size = np.zeros(x.shape), np.zeros(a.shape), np.zeros(b.shape)
    for t in range(x.shape[0]):
        k = rows[t]
        if not 0 <= k < a.shape[0]:
            continue
        s = 1.0 if scales is None else scales[k]
        for (gx, ga, gb), f in ((out, lambda z: z), (size, np.abs)):
            g, xt, A, B, c = f(grad[t]), f(x[t]), f(a[k]), f(b[k]), f(s)
            v, u = c * (g @ B), c * (A @ xt)
            gx[t] = v @ A
            ga[k] += np.outer(v, xt)
            gb[k] += np.outer(g, u)
    return out, size
