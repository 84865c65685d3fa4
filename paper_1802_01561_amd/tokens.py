"""Torch-tensor front end of the token-policy operators (include/vtrace_tokens.h):
argument marshalling only, as in binding.py.

A learner step of a policy over a vocabulary is vtrace_vocab_log_probs,
vtrace_log_prob_loss_grad, vtrace_vocab_grad and vtrace_clip_grad_norm in turn.
Calls run on ``stream``, or on the current stream of the tensors' device, which need
not be the current device.
"""

from __future__ import annotations

import ctypes
from typing import NamedTuple, Optional, Sequence

import torch

from ._lib import CLIP_WORKSPACE_BYTES, VTRACE_BF16, VTRACE_F32, check, lib
from .binding import _allocating_on, _fast_call, _fast_variant, _p, _require, _variant

__all__ = [
    "NO_TOKEN",
    "ClipWorkspace",
    "LogProbLossGrad",
    "LogProbWorkspace",
    "VocabGrad",
    "VocabLogProbs",
    "VocabWorkspace",
    "vtrace_clip_grad_norm",
    "vtrace_log_prob_loss_grad",
    "vtrace_log_prob_workspace_bytes",
    "vtrace_vocab_grad",
    "vtrace_vocab_grad_workspace_bytes",
    "vtrace_vocab_log_probs",
    "vtrace_vocab_workspace_bytes",
]

# The ordinary call (plain tensors, a workspace, the current stream of the current device) is
# checked and marshalled, and its outputs allocated, in native code (csrc/fast_call.cpp),
# which declines whatever is not exactly that.

# The token of a step that takes no part (a prompt, the padding behind a sequence).
NO_TOKEN = -1

_DTYPES = {torch.float32: VTRACE_F32, torch.bfloat16: VTRACE_BF16}


class _On:
    """The device and the stream of a call, both current inside the block."""

    def __init__(self, device: torch.device, stream):
        if device.type != "cuda":
            raise ValueError("inputs must be on a GPU device")
        if stream is not None and stream.device != device:
            raise ValueError(f"stream is on {stream.device}, inputs are on {device}")
        self._device = torch.cuda.device(device)
        self._allocating = _allocating_on(stream)
        self._stream, self._on = stream, device

    def __enter__(self):
        self._device.__enter__()
        self._allocating.__enter__()
        s = torch.cuda.current_stream(self._on) if self._stream is None else self._stream
        return ctypes.c_void_p(s.cuda_stream)

    def __exit__(self, *e):
        self._allocating.__exit__(*e)
        self._device.__exit__(*e)


def _grad_dtype_code(dtype) -> int:
    try:
        return _DTYPES[dtype]
    except (KeyError, TypeError):
        raise ValueError(f"grad_dtype must be torch.float32 or torch.bfloat16, got {dtype}") from None


class _CallWorkspace:
    """Device memory for one kind of call, cleared on creation."""

    def __init__(self, nbytes: int, device, stream):
        device = torch.device("cuda" if device is None else device)
        if device.index is None and device.type == "cuda":
            device = torch.device("cuda", torch.cuda.current_device())
        self.nbytes = nbytes
        with _On(device, stream) as s:
            self.tensor = torch.empty(nbytes, dtype=torch.uint8, device=device)
            check(lib().vtrace_workspace_init(_p(self.tensor), nbytes, s))


class VocabWorkspace(_CallWorkspace):
    """Workspace of vtrace_vocab_log_probs, or with ``grad_dtype`` of vtrace_vocab_grad."""

    def __init__(self, T: int, B: int, V: int, H: int, device=None, stream=None, *, grad_dtype=None):
        n = (vtrace_vocab_workspace_bytes(T, B, V, H) if grad_dtype is None
             else vtrace_vocab_grad_workspace_bytes(T, B, V, H, grad_dtype))
        if n == 0:
            raise ValueError(f"invalid shape T={T} B={B} V={V} H={H}")
        super().__init__(n, device, stream)


class LogProbWorkspace(_CallWorkspace):
    """Workspace of vtrace_log_prob_loss_grad."""

    def __init__(self, T: int, B: int, device=None, stream=None):
        n = vtrace_log_prob_workspace_bytes(T, B)
        if n == 0:
            raise ValueError(f"invalid shape T={T} B={B}")
        super().__init__(n, device, stream)


class ClipWorkspace(_CallWorkspace):
    """Workspace of vtrace_clip_grad_norm, whatever the gradients."""

    def __init__(self, device=None, stream=None):
        super().__init__(CLIP_WORKSPACE_BYTES, device, stream)


def _workspace(given, kind, device, *args, **kw):
    if given is None:
        return kind(*args, device=device, **kw)
    if not isinstance(given, kind):
        raise TypeError(f"workspace must be a {kind.__name__}")
    if given.tensor.device != device:
        raise ValueError(f"workspace is on {given.tensor.device}, expected {device}")
    return given


def _native_out(out, kind, required: int) -> bool:
    """Whether native code takes these outputs: none, or all that are required."""
    return out is None or (type(out) is kind and all(t is not None for t in out[:required]))


def _outputs(result, out=None, kind=tuple):
    """The outputs of a call that native code took, or its error."""
    if type(result) is int:
        check(result)
    return out if out is not None else result if kind is tuple else kind._make(result)


def vtrace_vocab_workspace_bytes(T: int, B: int, V: int, H: int) -> int:
    return lib().vtrace_vocab_workspace_bytes(T, B, V, H)


def vtrace_vocab_grad_workspace_bytes(T: int, B: int, V: int, H: int, grad_dtype=torch.float32) -> int:
    return lib().vtrace_vocab_grad_workspace_bytes(T, B, V, H, _grad_dtype_code(grad_dtype))


def vtrace_log_prob_workspace_bytes(T: int, B: int) -> int:
    return lib().vtrace_log_prob_workspace_bytes(T, B)


def _vocab_inputs(hidden, vocab_weight, vocab_bias, tokens):
    if not isinstance(hidden, torch.Tensor) or not isinstance(vocab_weight, torch.Tensor):
        raise TypeError("hidden and vocab_weight must be torch.Tensors")
    if hidden.dim() != 3 or vocab_weight.dim() != 2:
        raise ValueError("hidden must be [T, B, H] and vocab_weight [V, H]")
    T, B, H = hidden.shape
    V = vocab_weight.shape[0]
    dev = hidden.device
    if dev.type != "cuda":
        raise ValueError("inputs must be on a GPU device")
    _require(hidden, "hidden", (T, B, H), torch.bfloat16, dev)
    _require(vocab_weight, "vocab_weight", (V, H), torch.bfloat16, dev)
    if vocab_bias is not None:
        _require(vocab_bias, "vocab_bias", (V,), torch.float32, dev)
    _require(tokens, "tokens", (T, B), torch.int32, dev)
    return T, B, V, H, dev


class VocabLogProbs(NamedTuple):
    log_probs: torch.Tensor  # [T,B] log pi(a_t|x_t)
    log_sums: torch.Tensor  # [T,B] log sum of the exponentials of all logits
    entropy: Optional[torch.Tensor]  # [T,B]


def vtrace_vocab_log_probs(hidden, vocab_weight, vocab_bias, tokens, *,
                           workspace: Optional[VocabWorkspace] = None, with_entropy=True,
                           out: Optional[VocabLogProbs] = None, stream=None) -> VocabLogProbs:
    """log pi(a_t|x_t) and the policy's entropy from hidden states [T,B,H] (bfloat16) and
    a vocabulary layer [V,H] (bfloat16, a row for each token) with an optional bias [V]
    (float32, -inf rules a token out), without keeping the logits.

    ``tokens`` [T,B] int32; NO_TOKEN marks steps that take no part (their outputs are 0).
    With ``out``, its entropy decides instead of ``with_entropy``."""
    if stream is None and type(workspace) is VocabWorkspace and _native_out(out, VocabLogProbs, 2):
        fast = _fast_call(hidden)
        if fast:
            device = fast.device()
            r = fast.call_vocab_log_probs(
                fast.vocab_log_probs, hidden, vocab_weight, vocab_bias, tokens, out is None and with_entropy,
                *(out or (None, None, None)), workspace.tensor, workspace.nbytes, device, fast.stream(device))
            if r is not None:
                return _outputs(r, out, VocabLogProbs)
    T, B, V, H, dev = _vocab_inputs(hidden, vocab_weight, vocab_bias, tokens)
    with _On(dev, stream) as s:
        workspace = _workspace(workspace, VocabWorkspace, dev, T, B, V, H, stream=stream)
        if out is None:
            f32 = dict(dtype=torch.float32, device=dev)
            out = VocabLogProbs(torch.empty((T, B), **f32), torch.empty((T, B), **f32),
                                torch.empty((T, B), **f32) if with_entropy else None)
        for name, t in zip(out._fields, out):
            if t is not None or name != "entropy":
                _require(t, name, (T, B), torch.float32, dev)
        check(lib().vtrace_vocab_log_probs(
            T, B, V, H, _p(hidden), _p(vocab_weight), _p(vocab_bias), _p(tokens), _p(out.log_probs),
            _p(out.log_sums), _p(out.entropy), _p(workspace.tensor), workspace.nbytes, s))
    return out


class VocabGrad(NamedTuple):
    d_hidden: torch.Tensor  # [T,B,H]
    d_weight: torch.Tensor  # [V,H]
    d_bias: Optional[torch.Tensor]  # [V], where the layer has a bias


def vtrace_vocab_grad(hidden, vocab_weight, vocab_bias, tokens, log_sums, entropy=None, d_log_probs=None,
                      d_entropy=None, *, grad_dtype=torch.float32, workspace: Optional[VocabWorkspace] = None,
                      out: Optional[VocabGrad] = None, stream=None) -> VocabGrad:
    """Gradients of the hidden states and of the vocabulary layer from those of the
    log-probabilities and (optional) of the entropies, both [T,B] float32.

    ``log_sums`` and (with d_entropy) ``entropy`` are vtrace_vocab_log_probs' outputs;
    ``grad_dtype`` (float32 or bfloat16) is the type of d_hidden and d_weight."""
    code = _grad_dtype_code(grad_dtype)
    if stream is None and type(workspace) is VocabWorkspace and _native_out(out, VocabGrad, 2):
        fast = _fast_call(hidden)
        if fast:
            device = fast.device()
            r = fast.call_vocab_grad(
                fast.vocab_grad, hidden, vocab_weight, vocab_bias, tokens, log_sums, entropy, d_log_probs, d_entropy,
                grad_dtype is torch.bfloat16, *(out or (None, None, None)), out is None and vocab_bias is not None,
                workspace.tensor, workspace.nbytes, device, fast.stream(device))
            if r is not None:
                return _outputs(r, out, VocabGrad)
    T, B, V, H, dev = _vocab_inputs(hidden, vocab_weight, vocab_bias, tokens)
    if d_entropy is not None and entropy is None:
        raise ValueError("d_entropy needs entropy")
    for name, t in (("log_sums", log_sums), ("d_log_probs", d_log_probs)):
        _require(t, name, (T, B), torch.float32, dev)
    for name, t in (("entropy", entropy), ("d_entropy", d_entropy)):
        if t is not None:
            _require(t, name, (T, B), torch.float32, dev)
    with _On(dev, stream) as s:
        workspace = _workspace(workspace, VocabWorkspace, dev, T, B, V, H, stream=stream, grad_dtype=grad_dtype)
        if out is None:
            kw = dict(dtype=grad_dtype, device=dev)
            out = VocabGrad(torch.empty((T, B, H), **kw), torch.empty((V, H), **kw),
                            None if vocab_bias is None else torch.empty(V, dtype=torch.float32, device=dev))
        _require(out.d_hidden, "d_hidden", (T, B, H), grad_dtype, dev)
        _require(out.d_weight, "d_weight", (V, H), grad_dtype, dev)
        if out.d_bias is not None:
            _require(out.d_bias, "d_bias", (V,), torch.float32, dev)
        check(lib().vtrace_vocab_grad(
            T, B, V, H, code, _p(hidden), _p(vocab_weight), _p(vocab_bias), _p(tokens), _p(log_sums), _p(entropy),
            _p(d_log_probs), _p(d_entropy), _p(out.d_hidden), _p(out.d_weight), _p(out.d_bias), _p(workspace.tensor),
            workspace.nbytes, s))
    return out


class LogProbLossGrad(NamedTuple):
    losses: torch.Tensor  # [4] total, policy gradient, baseline, entropy
    d_log_probs: torch.Tensor  # [T,B]
    d_values: torch.Tensor  # [T,B]
    d_entropy: Optional[torch.Tensor]  # [T,B]
    vs: Optional[torch.Tensor]
    pg_advantages: Optional[torch.Tensor]


def vtrace_log_prob_loss_grad(target_log_probs, behaviour_log_probs, entropy, rewards, discounts, values,
                              bootstrap_value, lengths=None, rho_bar=1.0, c_bar=1.0, lam=1.0, baseline_cost=0.5,
                              entropy_cost=0.01, *, workspace: Optional[LogProbWorkspace] = None, with_vs=False,
                              with_pg_advantages=False, out: Optional[LogProbLossGrad] = None, stream=None,
                              correction="vtrace", q_estimate="vtrace", epsilon=1e-6,
                              reward_transform=None) -> LogProbLossGrad:
    """V-trace targets, losses and gradients from log-probabilities [T,B] (float32), for
    lanes of different ``lengths`` ([B] int32 on the device, None = T).

    ``entropy`` [T,B] is the policy's (None: no entropy loss and no d_entropy); the
    variant arguments are as in vtrace_loss_grad."""
    if stream is None and type(workspace) is LogProbWorkspace and _native_out(out, LogProbLossGrad, 3):
        fast = _fast_call(target_log_probs)
        known = fast and _fast_variant(correction, q_estimate, epsilon, "log_probs", reward_transform, torch.float32)
        if known:
            device = fast.device()
            r = fast.call_log_prob_loss(
                fast.log_prob_loss, target_log_probs, behaviour_log_probs, entropy, rewards, discounts, values,
                bootstrap_value, lengths, rho_bar, c_bar, lam, baseline_cost, entropy_cost, known[1],
                *(out or (None,) * 6), out is None and entropy is not None, out is None and bool(with_vs),
                out is None and bool(with_pg_advantages), workspace.tensor, workspace.nbytes, device, fast.stream(device))
            if r is not None:
                return _outputs(r, out, LogProbLossGrad)
    variant = _variant(correction, q_estimate, epsilon, "log_probs", reward_transform)
    if not isinstance(target_log_probs, torch.Tensor):
        raise TypeError("target_log_probs must be a torch.Tensor")
    if target_log_probs.dim() != 2:
        raise ValueError("target_log_probs must be [T, B]")
    T, B = target_log_probs.shape
    dev = target_log_probs.device
    if dev.type != "cuda":
        raise ValueError("inputs must be on a GPU device")
    for name, t in (("target_log_probs", target_log_probs), ("behaviour_log_probs", behaviour_log_probs),
                    ("entropy", entropy), ("rewards", rewards), ("discounts", discounts), ("values", values)):
        if t is not None or name != "entropy":
            _require(t, name, (T, B), torch.float32, dev)
    _require(bootstrap_value, "bootstrap_value", (B,), torch.float32, dev)
    if lengths is not None:
        _require(lengths, "lengths", (B,), torch.int32, dev)
    with _On(dev, stream) as s:
        workspace = _workspace(workspace, LogProbWorkspace, dev, T, B, stream=stream)
        if out is None:
            new = lambda wanted=True: torch.empty((T, B), dtype=torch.float32, device=dev) if wanted else None  # noqa: E731
            out = LogProbLossGrad(torch.empty(4, dtype=torch.float32, device=dev), new(), new(), new(entropy is not None),
                                  new(with_vs), new(with_pg_advantages))
        _require(out.losses, "losses", (4,), torch.float32, dev)
        for name, t in zip(out._fields[1:], out[1:]):
            if t is not None or name in ("d_log_probs", "d_values"):
                _require(t, name, (T, B), torch.float32, dev)
        check(lib().vtrace_log_prob_loss_grad(
            T, B, _p(target_log_probs), _p(behaviour_log_probs), _p(entropy), _p(rewards), _p(discounts), _p(values),
            _p(bootstrap_value), _p(lengths), rho_bar, c_bar, lam, baseline_cost, entropy_cost, ctypes.byref(variant),
            _p(out.losses), _p(out.d_log_probs), _p(out.d_entropy), _p(out.d_values), _p(out.vs),
            _p(out.pg_advantages), _p(workspace.tensor), workspace.nbytes, s))
    return out


def vtrace_clip_grad_norm(gradients: Sequence[torch.Tensor], max_norm: Optional[float], *,
                          out: Optional[Sequence[torch.Tensor]] = None,
                          workspace: Optional[ClipWorkspace] = None, norm: Optional[torch.Tensor] = None,
                          stream=None) -> torch.Tensor:
    """Clips the gradients (float32 or bfloat16, contiguous) by their global norm, in place
    or into ``out`` (tensors of the same shapes and types); returns the norm before
    clipping, a float32 scalar on the device.  max_norm None: the norm alone."""
    gradients = list(gradients)
    if not gradients:
        raise ValueError("no gradients")
    if max_norm is None and out is not None:
        raise ValueError("out needs max_norm")
    first = gradients[0]
    outs = gradients if out is None else list(out)  # once: an iterator has nothing left for the second way in
    if stream is None and type(workspace) is ClipWorkspace:
        fast = _fast_call(first)
        if fast:
            device = fast.device()
            r = fast.call_clip(fast.clip, gradients, outs, max_norm is not None, max_norm, norm, workspace.tensor,
                               workspace.nbytes, device, fast.stream(device))
            if r is not None:
                return _outputs(r)[0]
    if not isinstance(first, torch.Tensor):
        raise TypeError("gradients must be torch.Tensors")
    dev = first.device
    if len(outs) != len(gradients):
        raise ValueError(f"{len(outs)} outputs for {len(gradients)} gradients")
    n = len(gradients)
    ins_p, outs_p = (ctypes.c_void_p * n)(), (ctypes.c_void_p * n)()
    sizes, dtypes = (ctypes.c_int64 * n)(), (ctypes.c_int32 * n)()
    for i, (g, o) in enumerate(zip(gradients, outs)):
        _require(g, f"gradients[{i}]", getattr(g, "shape", ()), None, dev)
        if g.dtype not in _DTYPES:
            raise TypeError(f"gradients[{i}] must be float32 or bfloat16, got {g.dtype}")
        if o is not g:
            _require(o, f"out[{i}]", g.shape, g.dtype, dev)
        ins_p[i], outs_p[i] = g.data_ptr(), o.data_ptr()
        sizes[i], dtypes[i] = g.numel(), _DTYPES[g.dtype]
    with _On(dev, stream) as s:
        workspace = _workspace(workspace, ClipWorkspace, dev, stream=stream)
        if norm is None:
            norm = torch.empty((), dtype=torch.float32, device=dev)
        _require(norm, "norm", (), torch.float32, dev)
        check(lib().vtrace_clip_grad_norm(n, ins_p, None if max_norm is None else outs_p, sizes, dtypes,
                                          0.0 if max_norm is None else max_norm, _p(norm), _p(workspace.tensor),
                                          workspace.nbytes, s))
    return norm
