"""The oracle of the calls on parameters, against other ways to the same values."""

import numpy as np
import pytest

from oracle import parameters as op


def test_embed():
    r = np.random.default_rng(0)
    w = r.normal(size=(7, 3))
    got = op.embed(w, [0, 6, -1, 3, 7, -2], 2.0)
    assert np.array_equal(got[[0, 1, 3]], 2.0 * w[[0, 6, 3]]) and np.array_equal(got[2], np.zeros(3))
    assert np.isnan(got[4:]).all()


def test_embed_grad_is_the_gradient_of_embed():
    """embed is linear in the table: its gradient is the sum that a difference of any size gives."""
    r = np.random.default_rng(1)
    V, H, tokens = 5, 4, np.array([0, 3, 3, -1, 4, 3, 0])
    w, d = r.normal(size=(V, H)), r.normal(size=(len(tokens), H))
    got, count, size = op.embed_grad(d, tokens, V, 1.5)
    for v in range(V):
        for h in range(H):
            up, down = w.copy(), w.copy()
            up[v, h] += 0.5
            down[v, h] -= 0.5
            diff = np.sum(d * (op.embed(up, tokens, 1.5) - op.embed(down, tokens, 1.5)))
            assert abs(diff - got[v, h]) < 1e-12
    assert count.tolist() == [2, 0, 0, 3, 1]
    assert (np.abs(got) <= size + 1e-15).all()


@pytest.mark.parametrize("m,n", [(1, 1), (1, 9), (9, 1), (16, 16), (12, 40), (40, 12)])
def test_orthogonalize_goes_by_singular_values(m, n):
    g = np.random.default_rng(m * n).normal(size=(m, n))
    a, b = op.orthogonalize(g, scale=0.5), op.orthogonalize_singular(g, scale=0.5)
    assert np.abs(a - b).max() < 1e-10 * np.abs(b).max()
    s = np.linalg.svd(op.orthogonalize(g), compute_uv=False)
    start = np.linalg.svd(g / np.linalg.norm(g), compute_uv=False)
    assert (s[start > 0.01] > 0.67).all() and (s < 1.21).all()


@pytest.mark.parametrize("m,n", [(40, 40), (24, 100), (100, 24)])
@pytest.mark.parametrize("together", [1, 2])
@pytest.mark.parametrize("steps", [1, 2, 5])
def test_rounded_products_are_near(m, n, together, steps):
    g = np.random.default_rng(3).normal(size=(m, n))
    ref = op.orthogonalize(g, (op.QUINTIC,) * steps)
    off = [np.linalg.norm(op.orthogonalize_rounded(g, (op.QUINTIC,) * steps, parts=p, together=together) - ref) / np.linalg.norm(ref)
           for p in (1, 2)]
    assert 1e-5 < off[0] < 2e-3 and off[1] < 3e-6


def test_zeros_and_epsilon():
    assert np.array_equal(op.orthogonalize(np.zeros((3, 4))), np.zeros((3, 4)))
    g = np.full((1, 1), 1e-9)
    assert abs(op.orthogonalize(g, epsilon=1e-7)[0, 0] - op.orthogonalize(np.ones((1, 1)) * 1e-2, epsilon=1.0)[0, 0]) < 1e-12
