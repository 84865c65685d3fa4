"""Torch-tensor front end of the calls on a token policy's parameters
(include/vtrace_parameters.h): argument marshalling only, as in binding.py.

vtrace_vocab_embed and vtrace_vocab_embed_grad are the input end of the network whose
output end is in tokens.py; vtrace_orthogonalize follows vtrace_clip_grad_norm.  Calls run
on ``stream``, or on the current stream of the tensors' device, which need not be the
current device.
"""

from __future__ import annotations

import ctypes
from typing import Optional, Sequence, Union

import torch

from ._lib import check, lib
from .binding import _fast_call, _p, _require
from .tokens import _DTYPES, _CallWorkspace, _grad_dtype_code, _On, _outputs, _workspace

__all__ = [
    "QUINTIC",
    "EmbedWorkspace",
    "OrthogonalWorkspace",
    "vtrace_orthogonalize",
    "vtrace_orthogonalize_workspace_bytes",
    "vtrace_vocab_embed",
    "vtrace_vocab_embed_grad",
    "vtrace_vocab_embed_grad_workspace_bytes",
]

# Coefficients of the Newton-Schulz steps (Jordan et al., "Muon", 2024): s -> a s + b s^3 + c s^5 with the steepest slope at
# 0 for which singular values near 1 stay there.
QUINTIC = (3.4445, -4.7750, 2.0315)


class EmbedWorkspace(_CallWorkspace):
    """Workspace of vtrace_vocab_embed_grad (and of vtrace_vocab_embed, for its flag), for calls
    of so many steps, tokens and elements of a row, or fewer."""

    def __init__(self, T: int, B: int, V: int, H: int, device=None, stream=None):
        n = vtrace_vocab_embed_grad_workspace_bytes(T, B, V, H)
        if n == 0:
            raise ValueError(f"invalid shape T={T} B={B} V={V} H={H}")
        super().__init__(n, device, stream)


class OrthogonalWorkspace(_CallWorkspace):
    """Workspace of vtrace_orthogonalize, for matrices of these shapes and types, or some of them."""

    def __init__(self, matrices: Sequence[torch.Tensor], device=None, stream=None):
        matrices = list(matrices)
        n = vtrace_orthogonalize_workspace_bytes(matrices)
        if n == 0:
            raise ValueError("invalid shapes of matrices")
        super().__init__(n, matrices[0].device if device is None and matrices else device, stream)


def vtrace_vocab_embed_grad_workspace_bytes(T: int, B: int, V: int, H: int) -> int:
    return lib().vtrace_vocab_embed_grad_workspace_bytes(T, B, V, H)


def _shapes(matrices: Sequence[torch.Tensor]):
    n = len(matrices)
    rows, columns, dtypes = (ctypes.c_int64 * n)(), (ctypes.c_int64 * n)(), (ctypes.c_int32 * n)()
    for i, m in enumerate(matrices):
        if not isinstance(m, torch.Tensor):
            raise TypeError("matrices must be torch.Tensors")
        if m.dim() != 2:
            raise ValueError(f"matrices[{i}] must have two dimensions, got {m.dim()}")
        if m.dtype not in _DTYPES:
            raise TypeError(f"matrices[{i}] must be float32 or bfloat16, got {m.dtype}")
        rows[i], columns[i] = m.shape
        dtypes[i] = _DTYPES[m.dtype]
    return rows, columns, dtypes


def vtrace_orthogonalize_workspace_bytes(matrices: Sequence[torch.Tensor]) -> int:
    matrices = list(matrices)
    return lib().vtrace_orthogonalize_workspace_bytes(len(matrices), *_shapes(matrices))


def _dtype_code(dtype, name: str) -> int:
    try:
        return _DTYPES[dtype]
    except (KeyError, TypeError):
        raise ValueError(f"{name} must be torch.float32 or torch.bfloat16, got {dtype}") from None


def _tokens_shape(tokens, device):
    if not isinstance(tokens, torch.Tensor):
        raise TypeError("tokens must be a torch.Tensor")
    if tokens.dim() != 2:
        raise ValueError("tokens must be [T, B]")
    _require(tokens, "tokens", tuple(tokens.shape), torch.int32, device)
    return tuple(tokens.shape)


def vtrace_vocab_embed(vocab_weight, tokens, scale: float = 1.0, *, out_dtype=None, workspace=None,
                       out: Optional[torch.Tensor] = None, stream=None) -> torch.Tensor:
    """scale * vocab_weight[tokens]: [T,B,H] of ``out_dtype`` (float32 or bfloat16; None: that
    of ``out`` or of the table) from a table [V,H] of either type; zeros for NO_TOKEN, NaN
    for a token that is not in the vocabulary.

    ``workspace`` (any of this library's) is there for its error flag alone."""
    # As in tokens.py, native code takes the ordinary call, or declines.
    if stream is None and type(scale) is float and (workspace is None or isinstance(workspace, _CallWorkspace)):
        fast = _fast_call(vocab_weight)
        if fast:
            given = out if type(out) is torch.Tensor else vocab_weight
            wanted = given.dtype if out_dtype is None else out_dtype
            if wanted in _DTYPES:
                device = fast.device()
                r = fast.call_vocab_embed(fast.vocab_embed, vocab_weight, tokens, scale, wanted is torch.bfloat16, out,
                                          None if workspace is None else workspace.tensor,
                                          0 if workspace is None else workspace.nbytes, device, fast.stream(device))
                if r is not None:
                    return _outputs(r)[0]
    if not isinstance(vocab_weight, torch.Tensor):
        raise TypeError("vocab_weight must be a torch.Tensor")
    if vocab_weight.dim() != 2:
        raise ValueError("vocab_weight must be [V, H]")
    if out is not None and not isinstance(out, torch.Tensor):
        raise TypeError("out must be a torch.Tensor")
    V, H = vocab_weight.shape
    dev = vocab_weight.device
    if out_dtype is None:
        out_dtype = (vocab_weight if out is None else out).dtype
    elif out is not None and out.dtype != out_dtype:
        raise TypeError(f"out has dtype {out.dtype}, expected {out_dtype}")
    codes = _dtype_code(vocab_weight.dtype, "vocab_weight.dtype"), _dtype_code(out_dtype, "out_dtype")
    if dev.type != "cuda":
        raise ValueError("inputs must be on a GPU device")
    _require(vocab_weight, "vocab_weight", (V, H), None, dev)
    T, B = _tokens_shape(tokens, dev)
    if workspace is not None and workspace.tensor.device != dev:
        raise ValueError(f"workspace is on {workspace.tensor.device}, expected {dev}")
    with _On(dev, stream) as s:
        if out is None:
            out = torch.empty((T, B, H), dtype=out_dtype, device=dev)
        _require(out, "out", (T, B, H), out_dtype, dev)
        check(lib().vtrace_vocab_embed(T, B, V, H, *codes, _p(vocab_weight), _p(tokens), scale, _p(out),
                                       None if workspace is None else _p(workspace.tensor),
                                       0 if workspace is None else workspace.nbytes, s))
    return out


def vtrace_vocab_embed_grad(d_embedded, tokens, vocab_size: int, scale: float = 1.0, *, grad_dtype=torch.float32,
                            accumulate_into: Optional[torch.Tensor] = None, out: Optional[torch.Tensor] = None,
                            workspace: Optional[EmbedWorkspace] = None, stream=None) -> torch.Tensor:
    """The table's gradient [V,H] from those of vtrace_vocab_embed's rows, [T,B,H] (float32 or
    bfloat16): the sum over each token's steps, times ``scale``.

    ``accumulate_into`` [V,H] is added to in place (rows of tokens that steps have; the others
    are not touched) and returned; otherwise all of ``out`` or a new tensor is written, rows
    that no step has with zeros.  ``grad_dtype`` is a new tensor's: that of ``accumulate_into``
    or ``out`` decides otherwise."""
    if accumulate_into is not None and out is not None:
        raise ValueError("out and accumulate_into are one or the other")
    given = accumulate_into if out is None else out
    if stream is None and type(scale) is float and type(workspace) is EmbedWorkspace:
        fast = _fast_call(d_embedded)
        wanted = given.dtype if type(given) is torch.Tensor else grad_dtype
        if fast and wanted in _DTYPES:
            device = fast.device()
            r = fast.call_vocab_embed_grad(fast.vocab_embed_grad, d_embedded, tokens, vocab_size, scale,
                                           wanted is torch.bfloat16, accumulate_into is not None, given,
                                           workspace.tensor, workspace.nbytes, device, fast.stream(device))
            if r is not None:
                return _outputs(r)[0]
    if not isinstance(d_embedded, torch.Tensor):
        raise TypeError("d_embedded must be a torch.Tensor")
    if d_embedded.dim() != 3:
        raise ValueError("d_embedded must be [T, B, H]")
    T, B, H = d_embedded.shape
    dev = d_embedded.device
    if given is not None:
        if not isinstance(given, torch.Tensor):
            raise TypeError("out and accumulate_into must be torch.Tensors")
        grad_dtype = given.dtype
    codes = _dtype_code(d_embedded.dtype, "d_embedded.dtype"), _grad_dtype_code(grad_dtype)
    if dev.type != "cuda":
        raise ValueError("inputs must be on a GPU device")
    _require(d_embedded, "d_embedded", (T, B, H), None, dev)
    _require(tokens, "tokens", (T, B), torch.int32, dev)
    with _On(dev, stream) as s:
        workspace = _workspace(workspace, EmbedWorkspace, dev, T, B, vocab_size, H, stream=stream)
        if given is None:
            given = torch.empty((vocab_size, H), dtype=grad_dtype, device=dev)
        _require(given, "accumulate_into" if accumulate_into is not None else "out", (vocab_size, H), grad_dtype, dev)
        check(lib().vtrace_vocab_embed_grad(T, B, vocab_size, H, *codes, _p(d_embedded), _p(tokens), scale,
                                            accumulate_into is not None, _p(given), _p(workspace.tensor),
                                            workspace.nbytes, s))
    return given


def _is_number(x) -> bool:
    """One value and no sequence: tensors and arrays of no dimension have a length that raises."""
    return not hasattr(x, "__len__") or getattr(x, "ndim", 1) == 0


_quintic = {}  # steps -> the table of QUINTIC for so many


def _coefficients(coefficients, steps: int):
    """3 floats for each step, from one triple for all or a triple for each."""
    if coefficients is QUINTIC and steps in _quintic:
        return _quintic[steps]
    rows = list(coefficients)
    if len(rows) == 3 and all(_is_number(r) for r in rows):
        rows = [rows] * steps
    if len(rows) != steps or any(_is_number(r) or len(r) != 3 for r in rows):
        raise ValueError(f"coefficients must be a triple, or {steps} of them")
    table = (ctypes.c_float * (3 * steps))(*(float(x) for r in rows for x in r))
    if coefficients is QUINTIC:
        _quintic[steps] = table
    return table


def vtrace_orthogonalize(matrices: Sequence[torch.Tensor], scale: Union[float, Sequence[float]] = 1.0, *, steps: int = 5,
                         coefficients=QUINTIC, epsilon: float = 1e-7, out: Optional[Sequence[torch.Tensor]] = None,
                         workspace: Optional[OrthogonalWorkspace] = None, stream=None) -> list:
    """Nearly orthogonal matrices with the singular vectors of the given ones (float32 or
    bfloat16, two dimensions, contiguous), by ``steps`` Newton-Schulz products of
    X = G / max(|G|, epsilon), times ``scale`` (one factor, or one for each).

    ``coefficients``: (a, b, c) of s -> a s + b s^3 + c s^5, for all steps or for each.
    Results go to ``out`` (tensors of the same shapes and types, each of which may be its own
    matrix) or new tensors, which are returned as a list."""
    matrices = list(matrices)
    if not matrices:
        raise ValueError("no matrices")
    n = len(matrices)
    outs = None if out is None else list(out)
    if outs is not None and len(outs) != n:
        raise ValueError(f"{len(outs)} outputs for {n} matrices")
    if isinstance(steps, bool) or not isinstance(steps, int) or not 1 <= steps <= 64:
        raise ValueError(f"steps must be 1 to 64, got {steps}")
    table = _coefficients(coefficients, steps)
    if stream is None and type(scale) is float and type(epsilon) is float and type(workspace) is OrthogonalWorkspace:
        fast = _fast_call(matrices[0])
        if fast:
            device = fast.device()
            r = fast.call_orthogonalize(fast.orthogonalize, matrices, outs, scale, steps, ctypes.addressof(table), epsilon,
                                        workspace.tensor, workspace.nbytes, device, fast.stream(device))
            if r is not None:
                return list(_outputs(r))
    if _is_number(scale):
        scales = (ctypes.c_float * n)(*([float(scale)] * n))
    else:
        if len(scale) != n:
            raise ValueError(f"{len(scale)} scales for {n} matrices")
        scales = (ctypes.c_float * n)(*(float(x) for x in scale))
    rows, columns, dtypes = _shapes(matrices)
    dev = matrices[0].device
    if dev.type != "cuda":
        raise ValueError("inputs must be on a GPU device")
    with _On(dev, stream) as s:
        if outs is None:
            outs = [torch.empty_like(m) for m in matrices]
        ins_p, outs_p = (ctypes.c_void_p * n)(), (ctypes.c_void_p * n)()
        for i, (m, o) in enumerate(zip(matrices, outs)):
            _require(m, f"matrices[{i}]", m.shape, None, dev)
            if o is not m:
                _require(o, f"out[{i}]", m.shape, m.dtype, dev)
            ins_p[i], outs_p[i] = m.data_ptr(), o.data_ptr()
        if workspace is None:
            workspace = OrthogonalWorkspace(matrices, device=dev, stream=stream)
        workspace = _workspace(workspace, OrthogonalWorkspace, dev)
        check(lib().vtrace_orthogonalize(n, ins_p, outs_p, rows, columns, dtypes, scales, steps, table, epsilon,
                                         _p(workspace.tensor), workspace.nbytes, s))
    return outs
