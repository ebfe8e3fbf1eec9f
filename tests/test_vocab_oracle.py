"""Pins of oracle/vocab.py: hand-made rows, float64 autograd, magnitudes by hand."""

import numpy as np
import torch

import oracle


def test_embedding_by_hand():
    table = np.array([[1.0, -2.0], [3.0, 4.0], [5.0, 0.5]])
    out = oracle.embedding(table, [2, -1, 0, 3, 2], 2.0)
    assert (out == [[10, 1], [0, 0], [2, -4], [0, 0], [10, 1]]).all()
    g = np.array([[1.0, 2], [9, 9], [3, -1], [9, 9], [-4, 7]])
    grad, size, n = oracle.embedding_backward(g, [2, -1, 0, 3, 2], 3, -2.0)
    assert (grad == [[-6, 2], [0, 0], [6, -18]]).all()
    assert (size == [[6, 2], [0, 0], [10, 18]]).all() and (n == [1, 0, 2]).all()


def test_embedding_against_autograd():
    rng = np.random.default_rng(0)
    table, g, tok = rng.standard_normal((20, 7)), rng.standard_normal((50, 7)), rng.integers(0, 20, 50)
    w = torch.tensor(table, requires_grad=True)
    out = 0.3 * torch.nn.functional.embedding(torch.as_tensor(tok), w)
    out.backward(torch.as_tensor(g))
    assert np.allclose(out.detach().numpy(), oracle.embedding(table, tok, 0.3), rtol=1e-14)
    assert np.allclose(w.grad.numpy(), oracle.embedding_backward(g, tok, 20, 0.3)[0], rtol=1e-12)


def test_adapters_by_hand():
    a, b = np.array([[[1.0, 2.0]], [[3.0, -1.0]]]), np.array([[[1.0], [0.0], [2.0]], [[-1.0], [1.0], [0.5]]])
    x, base = np.array([[1.0, 1.0], [2.0, 0.0], [5.0, 5.0]]), np.ones((3, 3))
    out, size = oracle.adapters_add(base, x, [0, 1, -1], a, b, [2.0, 10.0])
    assert (out == [[7, 1, 13], [-59, 61, 31], [1, 1, 1]]).all()
    assert (size == [[7, 1, 13], [61, 61, 31], [1, 1, 1]]).all()
    assert (oracle.adapters_add(None, x, [0, 1, 2], a, b, None)[0] == [[3, 0, 6], [-6, 6, 3], [0, 0, 0]]).all()


def test_adapters_against_autograd():
    rng = np.random.default_rng(1)
    T, d, N, n, r = 12, 5, 7, 3, 2
    rows = np.array([0, 1, 2, -1, 3, 1, 1, 0, 2, 2, 2, 7])
    x, a, b = rng.standard_normal((T, d)), rng.standard_normal((n, r, d)), rng.standard_normal((n, N, r))
    base, g, s = rng.standard_normal((T, N)), rng.standard_normal((T, N)), rng.random(n)
    X, A, B = (torch.tensor(t, requires_grad=True) for t in (x, a, b))
    y = torch.as_tensor(base)
    for k in range(n):  # the textbook form, masked
        y = y + torch.as_tensor((rows == k)[:, None] * s[k]) * (X @ A[k].T @ B[k].T)
    y.backward(torch.as_tensor(g))
    assert np.allclose(y.detach().numpy(), oracle.adapters_add(base, x, rows, a, b, s)[0], rtol=1e-12)
    (gx, ga, gb), (sx, sa, sb) = oracle.adapters_backward(g, x, rows, a, b, s)
    for got, want, size in ((gx, X.grad, sx), (ga, A.grad, sa), (gb, B.grad, sb)):
        assert np.allclose(got, want.numpy(), rtol=1e-10, atol=1e-13)
        assert (size >= np.abs(got) - 1e-12).all()


def test_sizes_are_sums_of_magnitudes():
    rng = np.random.default_rng(2)
    T, d, N = 6, 4, 5
    pos = [np.abs(rng.standard_normal(s)) for s in ((T, N), (T, d), (2, 3, d), (2, N, 3), (2,))]
    g, x, a, b, s = pos
    rows = [0, 1, 0, 1, -1, 0]
    out, size = oracle.adapters_backward(g, x, rows, a, b, s)
    for o, m in zip(out, size):
        assert np.allclose(o, m)
    flipped = oracle.adapters_backward(-g, x, rows, -a, b, -s)[1]
    for m, f in zip(size, flipped):
        assert np.allclose(m, f)
