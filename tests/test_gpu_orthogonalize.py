"""Newton-Schulz products against the oracle, in float64.

Tolerance: the result's rounding, and twice what the oracle's models (steps one by one, and two
at once) of the operands' roundings and of the float32 sums' roundings is off: the kernel's are as many and of the same sizes, but
not the same ones, since a sum in another order may round an operand the other way, and
the matrix cores' sums are within one step of float32 where the model's are within half.  Where
one singular value has it all (a single row), the model's error is one sample and may be near
zero, so that a bound of its own is added: a + b t + c t^2, with sizes 3.4 + 4.8 + 2.0 against
a sum of down to 0.7, weighs a float32 rounding up to 15 times, in each of the steps.

A single element may take more than its share of that.  Errors along the smallest singular
values grow most (3.44 a step), so that an error can be nearly x y^T with x and y about normally
distributed: of m of those the largest is above sqrt(2 ln(2 m / p)) root mean squares with a
probability below p (2 exp(-t^2 / 2) each), and never above sqrt(m); the element's share
is the product of both.  p is 1e-6."""

import functools

import numpy as np
import pytest
import torch

import paper_1802_01561_amd as vt
from oracle import parameters as op

pytestmark = pytest.mark.gpu

F32, BF16 = torch.float32, torch.bfloat16
HALF_STEP = {F32: 2.0 ** -24, BF16: 2.0 ** -8}
STEPS = (op.QUINTIC,) * 5


def matrix(seed, m, n, dtype, kind="normal"):
    g = torch.Generator().manual_seed(seed)
    x = torch.randn((m, n), generator=g)
    if kind == "strong":  # a few strong directions above noise
        r = max(1, min(m, n) // 16)
        x = torch.randn((m, r), generator=g) @ torch.randn((r, n), generator=g) + 0.3 * x
    return (1e-3 * x).to(dtype)


def largest(m):
    return min(np.sqrt(m), np.sqrt(2.0 * np.log(2e6 * m)))


@functools.lru_cache(maxsize=None)
def _reference(data, shape, f32, steps, scale, epsilon):
    """The oracle's result, and how far its models of the roundings are off."""
    x = np.frombuffer(data).reshape(shape)
    ref = op.orthogonalize(x, steps, epsilon, scale)
    off = max(np.linalg.norm(op.orthogonalize_rounded(x, steps, epsilon, scale, parts=2 if f32 else 1, together=k) - ref) for k in (1, 2))
    return ref, off


def check(g, got, steps=STEPS, scale=1.0, epsilon=1e-7):
    steps = tuple(tuple(float(np.float32(v)) for v in s) for s in steps)
    ref, off = _reference(g.cpu().double().numpy().tobytes(), tuple(g.shape), g.dtype == F32, steps, float(np.float32(scale)),
                          float(np.float32(epsilon)))
    assert got.dtype == g.dtype and got.shape == g.shape
    err = np.abs(got.cpu().double().numpy() - ref)
    off = off + 15.0 * np.sqrt(len(steps)) * 2.0 ** -24 * np.linalg.norm(ref)
    u = HALF_STEP[g.dtype]
    assert np.linalg.norm(err) <= 2.0 * off + u * np.linalg.norm(ref), (np.linalg.norm(err), off, np.linalg.norm(ref))
    tol = 2.0 * off / np.sqrt(err.size) * largest(err.shape[0]) * largest(err.shape[1]) + u * np.abs(ref)
    assert (err <= tol).all(), (np.argwhere(~(err <= tol))[:5], err.max())


SIZES = [(1, 1), (1, 2), (2, 1), (1, 300), (300, 1), (2, 2), (3, 5), (16, 16), (15, 17), (63, 64), (64, 65), (65, 130), (127, 128),
         (128, 129), (129, 127), (200, 72), (256, 256), (257, 255), (83, 1001), (1000, 83), (513, 300), (640, 640)]


@pytest.fixture(params=[None] + [f"{size}x{together}" for size in (32, 64, 128, 256) for together in (1, 2)])
def tile(request, monkeypatch):
    """The kernels that the sizes choose, and each of them for all sizes, steps one by one and two at once."""
    if request.param is None:
        monkeypatch.delenv("VTRACE_KERNEL", raising=False)
    else:
        monkeypatch.setenv("VTRACE_KERNEL", f"ortho_{request.param}")


@pytest.mark.parametrize("m,n", SIZES)
@pytest.mark.parametrize("dtype", [F32, BF16])
def test_one_matrix(m, n, dtype, tile):
    for kind in ("normal", "strong"):
        g = matrix(m + 7 * n, m, n, dtype, kind)
        got, = vt.vtrace_orthogonalize([g.cuda()])
        check(g, got)


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_many_matrices_of_all_sizes(dtype, tile):
    """More than one launch's table, wide and tall, in both types."""
    shapes = (SIZES[:16] * 4)[:60]
    gs = [matrix(i, m, n, dtype if i % 5 else (F32 if dtype is BF16 else BF16)) for i, (m, n) in enumerate(shapes)]
    scales = [1.0 + 0.25 * (i % 3) for i in range(len(gs))]
    ws = vt.OrthogonalWorkspace([g.cuda() for g in gs])
    ws.tensor[4352:].fill_(0xFF)
    out = vt.vtrace_orthogonalize([g.cuda() for g in gs], scales, workspace=ws)
    for g, o, s in zip(gs, out, scales):
        check(g, o, scale=s)


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("shapes", [[(1100, 1030)], [(700, 2100), (2100, 700)], [(520, 512)] * 9])
def test_larger_matrices(dtype, shapes, tile):
    gs = [matrix(i, m, n, dtype, "strong") for i, (m, n) in enumerate(shapes)]
    for g, o in zip(gs, vt.vtrace_orthogonalize([g.cuda() for g in gs])):
        check(g, o)
