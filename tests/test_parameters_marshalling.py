"""The calls on parameters: two ways into the library, on the host."""

import ctypes

import numpy as np
import pytest
import torch

import paper_1802_01561_amd as vt
from paper_1802_01561_amd import parameters


def _workspace(kind):
    w = object.__new__(kind)
    w.tensor, w.nbytes = torch.empty(32768, dtype=torch.uint8), 32768
    return w


def _declines(seen):
    """Stands in for native code that takes no call."""
    def record(*args):
        seen.append(args)
    names = dict(vocab_embed=0, vocab_embed_grad=0, orthogonalize=0, device=staticmethod(lambda: 0),
                 stream=staticmethod(lambda device: 0), call_vocab_embed=staticmethod(record),
                 call_vocab_embed_grad=staticmethod(record), call_orthogonalize=staticmethod(record))
    return type("Declines", (), names)


def test_matrices_and_outputs_are_taken_from_iterators_once(monkeypatch):
    """Where native code declines, the Python path has the same matrices and outputs."""
    seen = []
    monkeypatch.setattr(parameters, "_fast_call", lambda first: _declines(seen))
    g = [torch.ones(3, 4), torch.ones(4, 2)]
    with pytest.raises(ValueError, match="GPU"):  # past the counts
        vt.vtrace_orthogonalize(iter(g), out=(t.clone() for t in g), workspace=_workspace(vt.OrthogonalWorkspace))
    assert [len(part) for part in seen[0][1:3]] == [2, 2]


def test_coefficients_reach_native_code_as_one_table(monkeypatch):
    seen = []
    monkeypatch.setattr(parameters, "_fast_call", lambda first: _declines(seen))
    each = [(1.5, -0.5, 0.0), (2.0, -1.0, 0.25)]
    for steps, given, expect in ((2, each, [x for r in each for x in r]), (3, (1.5, -0.5, 0.0), [1.5, -0.5, 0.0] * 3)):
        tables = []
        Declines = _declines(seen)
        Declines.call_orthogonalize = staticmethod(
            lambda fn, ms, outs, scale, n, table, *rest: tables.append(list((ctypes.c_float * (3 * n)).from_address(table))))
        monkeypatch.setattr(parameters, "_fast_call", lambda first: Declines)
        with pytest.raises(ValueError, match="GPU"):
            vt.vtrace_orthogonalize([torch.ones(2, 2)], steps=steps, coefficients=given, workspace=_workspace(vt.OrthogonalWorkspace))
        assert tables == [expect]
    with pytest.raises(ValueError, match="coefficients"):
        vt.vtrace_orthogonalize([torch.ones(2, 2)], steps=3, coefficients=each)


@pytest.mark.parametrize("scale", [2, True, torch.tensor(2.0), "2"])
def test_scales_that_are_no_float_go_through_python(monkeypatch, scale):
    seen = []
    monkeypatch.setattr(parameters, "_fast_call", lambda first: _declines(seen))
    t, w, d = torch.zeros((2, 3), dtype=torch.int32), torch.zeros(5, 8), torch.zeros(2, 3, 8)
    with pytest.raises(ValueError, match="GPU"):
        vt.vtrace_vocab_embed(w, t, scale)
    with pytest.raises(ValueError, match="GPU"):
        vt.vtrace_vocab_embed_grad(d, t, 5, scale, workspace=_workspace(vt.EmbedWorkspace))
    assert not seen


def test_workspaces_of_other_calls_and_types_are_not_native(monkeypatch):
    """A workspace of another kind is refused in Python; embed takes any, for its flag."""
    seen = []
    monkeypatch.setattr(parameters, "_fast_call", lambda first: _declines(seen))
    t, w, d = torch.zeros((2, 3), dtype=torch.int32), torch.zeros(5, 8), torch.zeros(2, 3, 8)
    with pytest.raises(ValueError, match="GPU"):
        vt.vtrace_vocab_embed(w, t, workspace=_workspace(vt.ClipWorkspace))
    assert len(seen) == 1
    with pytest.raises((TypeError, ValueError)):
        vt.vtrace_vocab_embed_grad(d, t, 5, workspace=_workspace(vt.ClipWorkspace))
    with pytest.raises((TypeError, ValueError)):
        vt.vtrace_orthogonalize([w], workspace=_workspace(vt.ClipWorkspace))
    with pytest.raises(ValueError, match="one or the other"):
        vt.vtrace_vocab_embed_grad(d, t, 5, accumulate_into=w, out=w)
    assert len(seen) == 1


@pytest.mark.parametrize("scale", [torch.tensor(0.5), np.array(0.5), np.float32(0.5), 1, [0.5, 2.0], torch.tensor([0.5, 2.0])])
def test_scales_of_updates_as_numbers_tensors_and_arrays(monkeypatch, scale):
    """One, of no dimension, or one for each matrix: past the checks, to where the library is called."""
    g = [torch.ones(3, 4), torch.ones(4, 2)]
    with pytest.raises(ValueError, match="GPU"):
        vt.vtrace_orthogonalize(g, scale)
    with pytest.raises(ValueError, match="3 scales for 2"):
        vt.vtrace_orthogonalize(g, [1.0, 2.0, 3.0])


@pytest.mark.parametrize("given", [torch.tensor([1.5, -0.5, 0.25]), np.array([1.5, -0.5, 0.25]), torch.tensor([[1.5, -0.5, 0.25]] * 3)])
def test_coefficients_as_tensors_and_arrays(given):
    assert list(parameters._coefficients(given, 3)) == [1.5, -0.5, 0.25] * 3
    if given.ndim == 1:
        assert list(parameters._coefficients(given, 2)) == [1.5, -0.5, 0.25] * 2
        for short in (given[:2], [given[0], given[1]], [1.5, given], given[0:1]):
            with pytest.raises(ValueError, match="coefficients"):
                parameters._coefficients(short, len(short))


def test_the_type_asked_for_reaches_native_code(monkeypatch):
    """Which declines an output of another."""
    seen = []
    monkeypatch.setattr(parameters, "_fast_call", lambda first: _declines(seen))
    t, w = torch.zeros((2, 3), dtype=torch.int32), torch.zeros(5, 8)
    out = torch.zeros(2, 3, 8)
    with pytest.raises(TypeError, match="out has dtype"):
        vt.vtrace_vocab_embed(w, t, out_dtype=torch.bfloat16, out=out)
    with pytest.raises(ValueError, match="GPU"):
        vt.vtrace_vocab_embed(w, t, out=out.bfloat16())
    assert [args[4] for args in seen] == [True, True]
