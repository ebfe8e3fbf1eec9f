"""fp64 oracle: logits changed by penalties, biases and grammar masks, their
log-probabilities, and the gradient through both.

TEST INFRASTRUCTURE ONLY (see the package docstring).

A row's rule is a dict; every key may be missing:

    prompt, output   token lists of its history
    repetition, frequency, presence   penalties
    bias             list of (id, value)
    allowed          bool [V]

    x = z
    x = x / repetition (x > 0) or x * repetition       for tokens of prompt and output
    x = x - frequency * c - presence [c > 0]           c = count in the output
    x = x + bias                                       of an id's last entry
    x = x / temperature
    x = -inf                                           where not allowed

    logp = x_token - lse, entropy = -sum p log p, lse = log sum e^x
    grad = slope (g ([v = token] - p) - e p (log p + H)),  slope = dx / dz

Pins (tests/test_policy_oracle.py): hand-made rows; float64 autograd and finite
differences through the textbook formulas; agreement with ``logprobs`` without
rules.
"""

from __future__ import annotations

from collections import Counter

import numpy as np


def change_logits(z, rules, temperature: float = 1.0) -> tuple[np.ndarray, np.ndarray]:
    """(x, slope) fp64 [T, V] of logits z [T, V] under one rule per row."""
    z = np.asarray(z, dtype=np.float64)
    T, V = z.shape
    x, slope = z.copy(), np.ones_like(z)
    for i, rule in enumerate(rules):
        prompt = [t for t in rule.get("prompt", ()) if 0 <= t < V]
        output = Counter(t for t in rule.get("output", ()) if 0 <= t < V)
        rho = float(rule.get("repetition", 1.0))
        for t in set(prompt) | set(output):
            k = 1.0 / rho if z[i, t] > 0 else rho
            x[i, t] = z[i, t] / rho if z[i, t] > 0 else z[i, t] * rho
            slope[i, t] = k
        for t, c in output.items():
            x[i, t] -= float(rule.get("frequency", 0.0)) * c + float(rule.get("presence", 0.0))
        for t, b in dict(rule.get("bias", ())).items():
            if 0 <= t < V:
                x[i, t] += b
        x[i] /= float(temperature)
        slope[i] /= float(temperature)
        if "allowed" in rule:
            x[i][~rule["allowed"]] = -np.inf
            slope[i][~rule["allowed"]] = 0.0
    return x, slope


def _softmax(x):
    """(p, log p, lse) of each row; a row of -inf has p = 0 and lse = -inf. log p is taken from the row's maximum, as an
    lse of a magnitude near the largest numbers holds no log sum."""
    m = x.max(axis=1, keepdims=True)
    none = np.isneginf(m[:, 0])
    with np.errstate(invalid="ignore"):
        e = np.exp(x - np.where(none, 0.0, m[:, 0])[:, None])
        s = e.sum(axis=1, keepdims=True)
        lse = np.where(none, -np.inf, m[:, 0] + np.log(np.where(none, 1.0, s[:, 0])))
        p = e / np.where(none[:, None], 1.0, s)
        logp = np.where(none[:, None], -np.inf, x - m - np.log(np.where(none[:, None], 1.0, s)))
    return p, logp, lse


def _at_positive(p, a):
    """a where p > 0 (or NaN), else 0: the factor of a product p a."""
    return np.where(p == 0, 0.0, a)


def changed_logprobs(z, tokens, rules, temperature: float = 1.0):
    """(logp, entropy, lse) fp64 [T]; logp NaN for tokens outside [0, V)."""
    x, _ = change_logits(z, rules, temperature)
    T, V = x.shape
    p, logp_all, lse = _softmax(x)
    tok = np.asarray(tokens)
    ok = (tok >= 0) & (tok < V)
    logp = np.full(T, np.nan)
    for i in np.nonzero(ok)[0]:
        logp[i] = logp_all[i, tok[i]]
    return logp, -(p * _at_positive(p, logp_all)).sum(axis=1), lse


def changed_logprobs_grad(z, tokens, rules, grad_logp, grad_entropy=None, temperature: float = 1.0) -> np.ndarray:
    """Gradient fp64 [T, V] of sum grad_logp logp + grad_entropy entropy with respect to z."""
    x, slope = change_logits(z, rules, temperature)
    T, V = x.shape
    p, logp_all, _ = _softmax(x)
    logp_all = _at_positive(p, logp_all)
    H = -(p * logp_all).sum(axis=1)
    tok = np.asarray(tokens)
    ok = (tok >= 0) & (tok < V)
    g = np.where(ok, np.asarray(grad_logp, dtype=np.float64), 0.0)
    e = np.zeros(T) if grad_entropy is None else np.asarray(grad_entropy, dtype=np.float64)
    onehot = np.zeros((T, V))
    onehot[np.nonzero(ok)[0], tok[ok]] = 1.0
    grad = slope * (g[:, None] * (onehot - p) - e[:, None] * p * (logp_all + H[:, None]))
    return np.where(np.isneginf(x).all(axis=1)[:, None], 0.0, grad)
