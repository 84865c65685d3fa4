"""One workspace for calls of different kinds in turn: the completion counters of one kind
are no other kind's data, so every call finds them at zero."""

import pytest
import torch

import paper_1802_01561_amd as vt
from paper_1802_01561_amd._lib import check, lib

pytestmark = pytest.mark.gpu


def _kinds():
    """name -> (workspace, call): calls of several workgroups each, whose outputs do not depend
    on what the workspace held."""
    g = torch.Generator(device="cuda").manual_seed(1)
    kw = dict(generator=g, device="cuda")
    f = lambda *s: torch.randn(*s, **kw)  # noqa: E731
    kinds = {}

    T, B, A, H = 20, 1024, 9, 64
    act = torch.randint(0, A, (T, B), **kw).int()
    z, y, rest = f(T, B, A), f(T, B, A), (f(T, B), torch.full((T, B), 0.97, device="cuda"), f(T, B), f(B))
    kinds["loss"] = (vt.Workspace(T, B, A), lambda ws: vt.vtrace_loss_grad(z, y, act, *rest, workspace=ws)[:3])
    hidden, wt, bias = f(T, B, H).bfloat16(), (f(H, A + 1) * 0.1).bfloat16(), f(A + 1)
    kinds["head"] = (vt.Workspace(T, B, A, H=H),
                     lambda ws: vt.vtrace_head_loss_grad(hidden, wt, bias, y.bfloat16(), act, rest[0], rest[1], rest[3],
                                                         workspace=ws)[:4])
    for name, n in (("few", 40), ("tiles", 300)):
        V, h = 3001, f(n, 1, H).bfloat16()
        w, b, tok = f(V, H).bfloat16(), f(V), torch.randint(0, V, (n, 1), **kw).int()
        args = (h, w, b, tok)
        kinds["vocab_" + name] = (vt.VocabWorkspace(n, 1, V, H), lambda ws, args=args: vt.vtrace_vocab_log_probs(*args, workspace=ws))
        o, d = vt.vtrace_vocab_log_probs(*args), (f(n, 1), f(n, 1))
        kinds["vocab_grad_" + name] = (vt.VocabWorkspace(n, 1, V, H, grad_dtype=torch.float32),
                                       lambda ws, args=args, o=o, d=d: vt.vtrace_vocab_grad(*args, *o[1:], *d, workspace=ws))
    for name, (T1, B1) in (("wide", (10, 2000)), ("long", (5000, 3))):
        x = (-f(T1, B1).abs(), -f(T1, B1).abs(), f(T1, B1), f(T1, B1), torch.full((T1, B1), 0.97, device="cuda"), f(T1, B1), f(B1))
        kinds["losses_" + name] = (vt.LogProbWorkspace(T1, B1), lambda ws, x=x: vt.vtrace_log_prob_loss_grad(*x, workspace=ws)[:4])
    grads = [f(n) for n in (70000, 5, 4097)]

    def clip(ws):
        out = [torch.full_like(t, 7.0) for t in grads]
        return [vt.vtrace_clip_grad_norm(grads, 0.5, out=out, workspace=ws), *out]

    kinds["clip"] = (vt.ClipWorkspace(), clip)
    return kinds


def test_calls_of_every_kind_take_turns():
    kinds = _kinds()
    expect = {}
    for name, (ws, call) in kinds.items():
        expect[name] = [t.clone() for t in call(ws) if t is not None]
    size = max(ws.nbytes for ws, _ in kinds.values())
    shared = torch.full((size,), 0xA5, dtype=torch.uint8, device="cuda")
    check(lib().vtrace_workspace_init(shared.data_ptr(), size, torch.cuda.current_stream().cuda_stream))
    for ws, _ in kinds.values():
        ws.tensor, ws.nbytes = shared, size
    wrong = []
    for first in kinds:
        for then in kinds:
            for name in (first, then):
                ws, call = kinds[name]
                got = [t for t in call(ws) if t is not None]
                if not all(torch.equal(a, b) for a, b in zip(got, expect[name])):
                    wrong.append((first, then, name))
    assert not wrong, wrong
