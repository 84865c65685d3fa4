"""How exact Newton-Schulz products are at the sizes of layers, where the kernels' own choices are those
that a program gets, against products in float64 on the GPU.

Tolerance: a result's rounding to its type, measured on the float64 result, and twice what a model of the
operands' roundings is off (steps one by one, and the first two at once, whichever is more).  The two
are independent of each other, so that their squares add: a value's place between two bfloat16
ones says nothing about the error that it has.  Errors of a million elements and more spread
over the norms of several hundred directions, so that the kernel's and the model's are within a few
percent of each other if they have the same roundings; twice is for what differs (the order of sums
that are rounded to operands), and 1% for the first."""

import functools
import math

import pytest
import torch

import paper_1802_01561_amd as vt
from oracle import parameters as op
from test_gpu_orthogonalize import check

pytestmark = pytest.mark.gpu

F32, BF16 = torch.float32, torch.bfloat16


def matrix(seed, m, n, dtype, kind="strong"):
    """A few strong directions above noise, or noise."""
    g = torch.Generator(device="cuda").manual_seed(seed)
    x = torch.randn((m, n), generator=g, device="cuda")
    if kind == "strong":
        r = max(1, min(m, n) // 16)
        x = torch.randn((m, r), generator=g, device="cuda") @ torch.randn((r, n), generator=g, device="cuda") / math.sqrt(r) + 0.3 * x
    return (1e-3 * x).to(dtype)


def _turned(x):
    return x.t().contiguous() if x.shape[0] > x.shape[1] else x


def _start(g):
    x = _turned(g.double())
    return x / torch.linalg.vector_norm(x)


def _steps(steps):
    return [[float(torch.tensor(v)) for v in s] for s in steps]


def exact(g, steps):
    x = _start(g)
    for a, b, c in _steps(steps):
        s = x @ x.t().contiguous()
        x = a * x + (b * s + c * (s @ s)) @ x
    return x.t() if g.shape[0] > g.shape[1] else x


def _operand(x, scale):
    return (x * scale).half().double() / scale


class _Symmetric:
    """The diagonal in float32, the rest as an operand."""

    def __init__(self, off, diagonal):
        self.diagonal = diagonal.float().double()
        self.off = _operand(off - torch.diag(torch.diagonal(off)), 8192.0)


def _combine(m, n, of_m, of_n, of_mn):
    oo = m.off @ n.off
    dm, dn = m.diagonal[:, None], n.diagonal[None, :]
    off = of_m * m.off + of_n * n.off + of_mn * (dm * n.off + m.off * dn + oo)
    return _Symmetric(off, of_m * m.diagonal + of_n * n.diagonal + of_mn * (m.diagonal * n.diagonal + torch.diagonal(oo)))


def rounded(g, steps, together):
    """bfloat16 matrices: float16 operands, and sums without rounding, which is far less."""
    x, k, steps = _start(g), 0, _steps(steps)
    while k < len(steps):
        a, b, c = steps[k]
        xs = _operand(x, 4096.0)
        gram = xs @ xs.t().contiguous()
        m = _Symmetric(gram, torch.diagonal(gram))
        p = _combine(m, m, b, 0.0, c)
        k += 1
        if together == 2 and k == 1 and k < len(steps):
            a2, b2, c2 = steps[k]
            t = _combine(m, p, a, 0.0, 1.0)
            m = _combine(t, p, a, 0.0, 1.0)
            p = _combine(_combine(m, m, b2, 0.0, c2), p, a, a2, 1.0)
            a *= a2
            k += 1
        x = (a + p.diagonal)[:, None] * x + p.off @ xs
    return x.t() if g.shape[0] > g.shape[1] else x


def _norm(x):
    return torch.linalg.vector_norm(x).item()


@functools.lru_cache(maxsize=None)
def _model(seed, m, n, kind, steps):
    g = matrix(seed, m, n, BF16, kind)
    ref = exact(g, steps)
    return g, ref, max(_norm(rounded(g, steps, k) - ref) for k in (1, 2)), _norm(ref.to(BF16).double() - ref)


STEPS = (op.QUINTIC,) * 5


@pytest.mark.parametrize("m,n,kind", [(2048, 2048, "strong"), (2048, 2048, "normal"), (4096, 1024, "strong"), (4096, 4096, "strong")])
@pytest.mark.parametrize("kernel", [None, "ortho_128x2", "ortho_256x1", "ortho_256x2"])
def test_bfloat16_layers(m, n, kind, kernel, monkeypatch):
    monkeypatch.delenv("VTRACE_KERNEL", raising=False)
    if kernel:
        monkeypatch.setenv("VTRACE_KERNEL", kernel)
    g, ref, off, rounding = _model(m + n, m, n, kind, STEPS)
    got, = vt.vtrace_orthogonalize([g])
    err = _norm(got.double() - ref)
    print(f"[case] {m} x {n} {kind} {kernel}: {err / _norm(ref):.3e}, rounding {rounding / _norm(ref):.3e}, model {off / _norm(ref):.3e}", flush=True)
    assert err <= math.hypot(1.01 * rounding, 2.0 * off)


@pytest.mark.parametrize("m,n", [(90, 100), (400, 300), (1100, 1030)])
@pytest.mark.parametrize("steps", [1, 2, 3, 5])
@pytest.mark.parametrize("kernel", [None] + [f"ortho_{size}x{together}" for size in (64, 128, 256) for together in (1, 2)])
def test_bfloat16_matrices_keep_22_bits_from_step_to_step(m, n, steps, kernel, monkeypatch):
    """Steps that change nothing give G / |G| rounded once.  X is float32 behind each step and then two
    float16 parts, the second at most half a step of the first, 2^-11, and so off by 2^-22 at most; where
    the first leaves float16's range the second's step is 2^-24 2^-11 of X 2^12.  Twice for the float32 operations'
    2^-24, a step more for the start.  A single part, 2^-11, is an eighth of bfloat16's half step."""
    monkeypatch.delenv("VTRACE_KERNEL", raising=False)
    if kernel:
        monkeypatch.setenv("VTRACE_KERNEL", kernel)
    g = matrix(m + steps, m, n, BF16)
    got, = vt.vtrace_orthogonalize([g], steps=steps, coefficients=(1.0, 0.0, 0.0))
    ref = g.double() / torch.linalg.vector_norm(g.double())
    half_step = torch.exp2(torch.floor(torch.log2(ref.abs().clamp(min=1e-30))) - 8)
    tol = half_step + 2.0 * (steps + 1) * (2.0 ** -22 * ref.abs() + 2.0 ** -47)
    assert ((got.double() - ref).abs() <= tol).all()


def _half_steps(ref, dtype):
    """Half the distance between the values of `dtype` around each element."""
    return torch.exp2(torch.floor(torch.log2(ref.abs().clamp(min=1e-30))) - (8 if dtype is BF16 else 24))


@pytest.mark.parametrize("m,n", [(1, 1), (2, 2), (4, 4), (3, 5), (1, 257), (300, 1), (16, 192), (31, 33), (32, 32), (256, 32), (32, 4096),
                                 (20, 65536)])
@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("kind", ["strong", "normal"])
@pytest.mark.parametrize("coefficients", [STEPS, ((1.5, -0.5, 0.0),) * 12])
def test_few_rows_are_float64_up_to_one_rounding(m, n, dtype, kind, coefficients, monkeypatch):
    """All steps of up to 32 rows in float64.  An entry of a 32 x 32 product has a rounding error of 32 2^-53
    of the sizes that are summed, 12 at most: 2^-44.4.  Those of A beside small eigenvalues grow by a^2 with
    each step that follows, 3.4445^8 = 2^14.3 until the last of five (the cubic's 1.5^22 = 2^12.9), and P
    has |b| + 2 |c| t, at most 9, of them: 2^-27 of the result's norm, twice for what the earlier steps' add.
    Then comes the result's own rounding, to one bit more where that carries it over a power of two."""
    monkeypatch.delenv("VTRACE_KERNEL", raising=False)
    g = matrix(m + n, m, n, dtype, kind)
    got, = vt.vtrace_orthogonalize([g], steps=len(coefficients), coefficients=coefficients)
    ref = exact(g, coefficients)
    more, half_steps = 2.0 ** -26 * _norm(ref), _half_steps(ref, dtype)
    near = _half_steps(ref.abs() + more, dtype)
    err = (got.double() - ref).abs()
    assert (err <= torch.maximum(half_steps, near) + more).all()
    assert _norm(err) <= 1.01 * _norm(torch.maximum(half_steps, near)) + more


@pytest.mark.parametrize("m,n", [(65536, 32768), (65536, 5000), (4000, 65536)])
def test_both_parts_of_the_largest_float32_matrices(m, n, monkeypatch):
    """A small matrix's rows and columns among zeros, from the first to the last: the same result there and zeros
    elsewhere.  With either part of an operand lost or from elsewhere it would be off by 2^-12 and more;
    the bound is that of the small matrix, whose sums' terms are the same (each of them is added by itself,
    no more than 200 roundings of 2^-24, for which the bound has 15)."""
    monkeypatch.delenv("VTRACE_KERNEL", raising=False)
    steps = STEPS[:3]
    small = matrix(m + n, 200, 150, F32, "strong")
    g = torch.Generator(device="cuda").manual_seed(n)

    def places(size, count):
        p = torch.randperm(size - 2, generator=g, device="cuda")[:count - 2] + 1
        return torch.cat([torch.tensor([0, size - 1], device="cuda"), p]).sort().values

    rows, columns = places(m, 200), places(n, 150)
    large = torch.zeros((m, n), device="cuda")
    large[rows[:, None], columns[None, :]] = small
    ws = vt.OrthogonalWorkspace([large])
    vt.vtrace_orthogonalize([large], steps=3, out=[large], workspace=ws)
    got = large[rows[:, None], columns[None, :]]
    check(small, got, steps=steps)
    large[rows[:, None], columns[None, :]] = 0.0
    assert all(int(torch.count_nonzero(large[at:at + 8192])) == 0 for at in range(0, m, 8192))
