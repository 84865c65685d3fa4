"""The C ABI of the token-policy operators on the host: exported symbols and argument
validation.  Every call carries an invalid argument, so nothing is launched and the fake
pointers are never dereferenced."""

import ctypes
import math
import os
import re

import pytest
import torch

import paper_1802_01561_amd as vt
from paper_1802_01561_amd import _lib, tokens

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
HEADER = os.path.join(ROOT, "include", "vtrace_tokens.h")
OK, NULL, SHAPE, DTYPE, PARAM, ALIGN, WS = 0, 1, 2, 3, 4, 5, 6
P = 0x10000


@pytest.fixture(scope="module")
def L():
    return _lib.lib()


def test_library_exports_every_declared_symbol(L):
    text = re.sub(r"/\*.*?\*/", "", open(HEADER).read(), flags=re.S)
    names = set(re.findall(r"\b(vtrace_[a-z_]+)\s*\(", text))
    assert names == set(_lib.TOKEN_SIGNATURES) and len(names) == 7
    assert all(hasattr(L, n) for n in names)
    assert int(re.search(r"VTRACE_CLIP_WORKSPACE_BYTES (\d+)", text).group(1)) == _lib.CLIP_WORKSPACE_BYTES
    assert int(re.search(r"VTRACE_NO_TOKEN \((-?\d+)\)", text).group(1)) == vt.NO_TOKEN
    assert set(tokens.__all__) <= set(dir(vt))


def test_workspace_bytes(L):
    n = L.vtrace_vocab_workspace_bytes
    assert 256 < n(1, 1, 1000, 64) < n(100, 32, 1000, 64)
    g = L.vtrace_vocab_grad_workspace_bytes
    assert g(100, 32, 1000, 64, 1) < g(100, 32, 1000, 64, 0)
    bad = [(0, 4, 9, 64), (4, 0, 9, 64), (4, 4, 0, 64), (4, 4, 9, 0), (4, 4, 9, 4), (4, 4, 9, 65), (4, 4, 9, 32776),
           (4, 4, (1 << 24) + 1, 64), (1 << 13, 1 << 13, 9, 8), (1 << 10, 1 << 10, 9, 1024), (1 << 24, 2, 1 << 14, 8),
           (-1, -1, 9, 64), (1 << 62, 1 << 62, 9, 64)]
    for s in bad:
        assert n(*s) == 0 and g(*s, 0) == 0, s
    assert g(4, 4, 9, 64, 2) == 0
    m = L.vtrace_log_prob_workspace_bytes
    assert m(1, 1) >= 256 + 24 and m(1 << 20, 1) > m(1, 1)
    for s in [(0, 1), (1, 0), (1, (1 << 27) + 1), (1 << 30, 1 << 20)]:
        assert m(*s) == 0, s


def _log_probs(L, **kw):
    a = dict(T=5, B=4, V=100, H=64, h=P, w=P, b=None, t=P, lp=P, ls=P, ent=None, ws=P, n=1 << 24)
    a.update(kw)
    return L.vtrace_vocab_log_probs(*(a[k] for k in ("T", "B", "V", "H", "h", "w", "b", "t", "lp", "ls", "ent", "ws", "n")), None)


SHAPES = [(dict(T=0), SHAPE), (dict(B=-1), SHAPE), (dict(V=0), SHAPE), (dict(V=(1 << 24) + 1), SHAPE), (dict(H=0), SHAPE),
          (dict(H=12), SHAPE), (dict(H=40000), SHAPE), (dict(T=1 << 20, B=1 << 6), SHAPE),
          (dict(T=1 << 16, B=1 << 8, H=64), SHAPE), (dict(T=1 << 24, B=1, H=8, V=1 << 15), SHAPE)]


@pytest.mark.parametrize("kw,status", SHAPES + [
    (dict(h=None), NULL), (dict(w=None), NULL), (dict(t=None), NULL), (dict(lp=None), NULL), (dict(ls=None), NULL),
    (dict(h=P + 8), ALIGN), (dict(w=P + 2), ALIGN), (dict(b=P + 2), ALIGN), (dict(t=P + 1), ALIGN), (dict(lp=P + 2), ALIGN),
    (dict(ls=P + 2), ALIGN), (dict(ent=P + 3), ALIGN), (dict(ws=P + 8), ALIGN), (dict(ws=None), WS), (dict(n=256), WS)])
def test_log_probs_rejects(L, kw, status):
    assert _log_probs(L, **kw) == status


def test_log_probs_workspace_is_exact(L):
    for T, B, V, H in [(1, 1, 100, 64), (5, 40, 1000, 8)]:
        n = L.vtrace_vocab_workspace_bytes(T, B, V, H)
        assert _log_probs(L, T=T, B=B, V=V, H=H, n=n - 1) == WS


def _grad(L, **kw):
    a = dict(T=5, B=4, V=100, H=64, dt=0, h=P, w=P, b=None, t=P, ls=P, ent=None, dl=P, de=None, dh=P, dw=P, db=None, ws=P,
             n=1 << 30)
    a.update(kw)
    keys = ("T", "B", "V", "H", "dt", "h", "w", "b", "t", "ls", "ent", "dl", "de", "dh", "dw", "db", "ws", "n")
    return L.vtrace_vocab_grad(*(a[k] for k in keys), None)


@pytest.mark.parametrize("kw,status", SHAPES + [
    (dict(h=None), NULL), (dict(w=None), NULL), (dict(t=None), NULL), (dict(ls=None), NULL), (dict(dl=None), NULL),
    (dict(dh=None), NULL), (dict(dw=None), NULL), (dict(de=P), NULL), (dict(dt=2), DTYPE), (dict(dt=-1), DTYPE),
    (dict(h=P + 8), ALIGN), (dict(w=P + 2), ALIGN), (dict(dh=P + 8), ALIGN), (dict(dw=P + 8), ALIGN), (dict(b=P + 2), ALIGN),
    (dict(t=P + 1), ALIGN), (dict(ls=P + 2), ALIGN), (dict(ent=P + 2), ALIGN), (dict(dl=P + 2), ALIGN),
    (dict(ent=P, de=P + 2), ALIGN), (dict(db=P + 2), ALIGN), (dict(ws=P + 8), ALIGN), (dict(ws=None), WS), (dict(n=256), WS)])
def test_grad_rejects(L, kw, status):
    assert _grad(L, **kw) == status


def _loss(L, **kw):
    a = dict(T=5, B=4, lp=P, lm=P, ent=P, r=P, d=P, v=P, boot=P, n=None, rho=1.0, c=1.0, lam=1.0, bc=0.5, ec=0.01, var=None,
             losses=P, dl=P, de=P, dv=P, vs=None, pg=None, ws=P, nb=1 << 20)
    a.update(kw)
    keys = ("T", "B", "lp", "lm", "ent", "r", "d", "v", "boot", "n", "rho", "c", "lam", "bc", "ec", "var", "losses", "dl",
            "de", "dv", "vs", "pg", "ws", "nb")
    return L.vtrace_log_prob_loss_grad(*(a[k] for k in keys), None)


V = _lib.Variant


@pytest.mark.parametrize("kw,status", [(dict(**{k: None}), NULL) for k in ("lp", "lm", "r", "d", "v", "boot", "losses", "dl", "dv")] + [
    (dict(**{k: P + 2}), ALIGN) for k in ("lp", "lm", "ent", "r", "d", "v", "boot", "n", "losses", "dl", "de", "dv", "vs", "pg")] + [
    (dict(T=0), SHAPE), (dict(B=0), SHAPE), (dict(B=(1 << 27) + 1), SHAPE), (dict(T=1 << 30, B=1 << 20), SHAPE),
    (dict(rho=math.nan), PARAM), (dict(rho=-1.0), PARAM), (dict(c=math.nan), PARAM), (dict(lam=1.5), PARAM),
    (dict(lam=math.nan), PARAM), (dict(bc=math.inf), PARAM), (dict(ec=math.nan), PARAM),
    (dict(var=ctypes.byref(V(9, 0, 0.0))), PARAM), (dict(var=ctypes.byref(V(2, 0, 0.0))), PARAM),
    (dict(var=ctypes.byref(V(0, 0, 0.0, 5, 0, 0))), PARAM), (dict(var=ctypes.byref(V(0, 0, 0.0, 1, 0, 7))), DTYPE),
    (dict(ws=None), WS), (dict(ws=P + 8), ALIGN), (dict(nb=256), WS)])
def test_log_prob_loss_rejects(L, kw, status):
    assert _loss(L, **kw) == status


def _clip(L, ins, outs, sizes, dtypes, max_norm=1.0, norm=P, ws=2 * P, n=_lib.CLIP_WORKSPACE_BYTES, count=None):
    k = len(sizes)
    arr = lambda t, x: (t * max(1, k))(*x) if x is not None else None  # noqa: E731
    return L.vtrace_clip_grad_norm(k if count is None else count, arr(ctypes.c_void_p, ins), arr(ctypes.c_void_p, outs),
                                   arr(ctypes.c_int64, sizes), arr(ctypes.c_int32, dtypes), max_norm, norm, ws, n, None)


def test_clip_rejects(L):
    A, B, C = 0x100000, 0x200000, 0x300000
    assert _clip(L, [A], [B], [4], [0], norm=None) == NULL
    assert _clip(L, None, [B], [4], [0]) == NULL
    assert _clip(L, [A], [B], [4], None) == NULL
    assert _clip(L, [None], [B], [4], [0]) == NULL
    assert _clip(L, [A], [None], [4], [0]) == NULL
    assert _clip(L, [A], [B], [4], [0], count=-1) == SHAPE
    assert _clip(L, [A], [B], [4], [0], count=(1 << 16) + 1) == SHAPE
    assert _clip(L, [A], [B], [-1], [0]) == SHAPE
    assert _clip(L, [A], [B], [1 << 41], [0]) == SHAPE
    assert _clip(L, [A], [B], [4], [2]) == DTYPE
    assert _clip(L, [A], [B], [4], [0], max_norm=math.nan) == PARAM
    assert _clip(L, [A], [B], [4], [0], max_norm=-1.0) == PARAM
    assert _clip(L, [A + 2], [B], [4], [0]) == ALIGN
    assert _clip(L, [A], [B + 1], [4], [1]) == ALIGN
    assert _clip(L, [A], [B], [4], [0], norm=P + 2) == ALIGN
    assert _clip(L, [A], [B], [4], [0], ws=None) == WS
    assert _clip(L, [A], [B], [4], [0], ws=P + 8) == ALIGN
    assert _clip(L, [A], [B], [4], [0], n=_lib.CLIP_WORKSPACE_BYTES - 1) == WS
    # outputs that overlap something: another output, another gradient, their own gradient in part, the norm
    assert _clip(L, [A, C], [B, B + 12], [4, 4], [0, 0]) == PARAM
    assert _clip(L, [A, A], [A, A], [4, 4], [0, 0]) == PARAM
    assert _clip(L, [A, B], [C, A + 8], [4, 4], [0, 0]) == PARAM
    assert _clip(L, [A], [A + 8], [4], [0]) == PARAM
    assert _clip(L, [A + 8], [A], [4], [0]) == PARAM
    assert _clip(L, [A, A + 64], [A, B], [4, 1 << 20], [0, 0], norm=A) == PARAM
    assert _clip(L, [A, B], [A, C], [1 << 12, 4], [0, 0], norm=A + 64) == PARAM
    assert _clip(L, [A], [2 * P], [4], [0]) == PARAM
    # a long gradient that is only read hides nothing behind a short one
    assert _clip(L, [A, A + 8, C], [B, B + 64, A + 4096], [4096, 1, 4], [0, 0, 0]) == PARAM


def test_python_binding_validates_before_calling():
    h, w = torch.zeros(2, 3, 64, dtype=torch.bfloat16), torch.zeros(10, 64, dtype=torch.bfloat16)
    t, f = torch.zeros(2, 3, dtype=torch.int32), torch.zeros(2, 3)
    for call in (lambda: vt.vtrace_vocab_log_probs(h, w, None, t), lambda: vt.vtrace_vocab_log_probs(h[0], w, None, t),
                 lambda: vt.vtrace_vocab_grad(h, w, None, t, f, None, f),
                 lambda: vt.vtrace_vocab_grad(h, w, None, t, f, None, f, grad_dtype=torch.float16),
                 lambda: vt.vtrace_log_prob_loss_grad(f, f, None, f, f, f, torch.zeros(3)),
                 lambda: vt.vtrace_log_prob_loss_grad(f, f, None, f, f, f, torch.zeros(3), correction="retrace"),
                 lambda: vt.vtrace_clip_grad_norm([f], 1.0), lambda: vt.vtrace_clip_grad_norm([], 1.0),
                 lambda: vt.vtrace_clip_grad_norm([f], None, out=[f]), lambda: vt.vtrace_clip_grad_norm([f], 1.0, out=[]),
                 lambda: vt.VocabWorkspace(0, 1, 10, 64, device="cpu"), lambda: vt.VocabWorkspace(1, 1, 10, 64, device="cpu"),
                 lambda: vt.LogProbWorkspace(1, 0, device="cpu")):
        with pytest.raises(ValueError):
            call()
    with pytest.raises(TypeError):
        vt.vtrace_vocab_log_probs(None, w, None, t)
    with pytest.raises(TypeError):
        vt.vtrace_clip_grad_norm([1.0], 1.0)
