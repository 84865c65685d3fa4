"""fp64 oracle of the calls on a token policy's parameters: rows of the vocabulary's table, their
gradient, and Newton-Schulz products.  NumPy, from the definitions."""

from __future__ import annotations

import numpy as np

from .tokens import NO_TOKEN, _f64

QUINTIC = (3.4445, -4.7750, 2.0315)


def embed(weight, tokens, scale=1.0):
    """[N,H] of tokens [N]: zeros for NO_TOKEN, NaN for what is not in the vocabulary."""
    tokens = np.asarray(tokens, dtype=np.int64)
    w = _f64(weight)
    valid = (tokens >= 0) & (tokens < len(w))
    rows = scale * w[np.where(valid, tokens, 0)]
    return np.where((tokens == NO_TOKEN)[:, None], 0.0, np.where(valid[:, None], rows, np.nan))


def embed_grad(d_embedded, tokens, V, scale=1.0):
    """d_weight [V,H], each token's steps [N], and the sum of the sizes of what is summed [V,H]."""
    tokens = np.asarray(tokens, dtype=np.int64)
    use = (tokens >= 0) & (tokens < V)
    x = _f64(d_embedded)[use]
    total, size = np.zeros((V, x.shape[1])), np.zeros((V, x.shape[1]))
    np.add.at(total, tokens[use], x)
    np.add.at(size, tokens[use], np.abs(x))
    return scale * total, np.bincount(tokens[use], minlength=V), abs(scale) * size


def _start(g, epsilon):
    g = _f64(g)
    return g / max(np.sqrt(np.sum(g * g)), epsilon)


def orthogonalize(g, coefficients=(QUINTIC,) * 5, epsilon=1e-7, scale=1.0):
    x = _start(g, epsilon)
    tall = x.shape[0] > x.shape[1]
    x = x.T if tall else x
    for a, b, c in coefficients:
        gram = x @ x.T
        x = a * x + (b * gram + c * (gram @ gram)) @ x
    return scale * (x.T if tall else x)


def orthogonalize_singular(g, coefficients=(QUINTIC,) * 5, epsilon=1e-7, scale=1.0):
    """The same by way of the singular values."""
    u, s, v = np.linalg.svd(_start(g, epsilon), full_matrices=False)
    for a, b, c in coefficients:
        s = a * s + b * s ** 3 + c * s ** 5
    return scale * (u * s) @ v


def _operand(x, scale, parts):
    """x as operands of a scale: float16, and (2 parts) what that leaves of x."""
    y = (x * scale).astype(np.float32)
    high = y.astype(np.float16).astype(np.float32)
    low = (y - high).astype(np.float16).astype(np.float32)
    return [_f64(high) / scale] + ([_f64(low) / scale] if parts == 2 else [])


def _product(a, b):
    """Of operands in parts, low parts first and low times low left out, as the matrix cores sum
    them: 32 products at a time are added to a float32 sum."""
    pairs = [(a[0], b[0])] if len(a) == 1 else [(a[1], b[0]), (a[0], b[1]), (a[0], b[0])]
    total = np.zeros((a[0].shape[0], b[0].shape[1]))
    for p, q in pairs:
        for k in range(0, p.shape[1], 32):
            total = _f64((total + p[:, k:k + 32] @ q[k:k + 32]).astype(np.float32))
    return total


class _Symmetric:
    """A symmetric matrix as it is kept: its diagonal in float32, the rest as an operand."""

    def __init__(self, off, diagonal, parts):
        self.diagonal = diagonal.astype(np.float32).astype(np.float64)
        off = off.astype(np.float32).astype(np.float64)
        self.operand = _operand(off - np.diag(np.diagonal(off)), 8192.0, parts)
        self.off = sum(self.operand)


def _combine(m, n, of_m, of_n, of_mn, parts):
    """of_m M + of_n N + of_mn M N."""
    oo = _product(m.operand, n.operand)
    dm, dn = m.diagonal[:, None], n.diagonal[None, :]
    off = of_m * m.off + of_n * n.off + of_mn * (dm * n.off + m.off * dn + oo)
    return _Symmetric(off, of_m * m.diagonal + of_n * n.diagonal + of_mn * (m.diagonal * n.diagonal + np.diagonal(oo)), parts)


def orthogonalize_rounded(g, coefficients=(QUINTIC,) * 5, epsilon=1e-7, scale=1.0, parts=1, together=1):
    """orthogonalize() with the roundings of the operands, of the sums of products and of what is
    kept between the products: X float32, operands float16 in one part or two, diagonals apart.
    together 2: the first two steps at once, the second's matrices from the first's."""
    single = lambda y: _f64(np.asarray(y).astype(np.float32))  # noqa: E731
    x = single(_start(g, epsilon))
    tall = x.shape[0] > x.shape[1]
    x = x.T if tall else x
    k = 0
    while k < len(coefficients):
        a, b, c = coefficients[k]
        xs = _operand(x, 4096.0, parts)
        gram = _product(xs, [y.T for y in xs])
        m = _Symmetric(gram, np.diagonal(gram).copy(), parts)
        p = _combine(m, m, b, 0.0, c, parts)
        k += 1
        if together == 2 and k == 1 and k < len(coefficients):
            a2, b2, c2 = coefficients[k]
            t = _combine(m, p, a, 0.0, 1.0, parts)
            m = _combine(t, p, a, 0.0, 1.0, parts)
            q = _combine(m, m, b2, 0.0, c2, parts)
            p = _combine(q, p, a, a2, 1.0, parts)
            a = float(np.float32(a * a2))
            k += 1
        x = single(single(a + p.diagonal)[:, None] * x + _product(p.operand, xs))
    return scale * (x.T if tall else x)
