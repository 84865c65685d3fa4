"""The token-policy operators as a program uses them: both ways into the library, calls at
the same time, graphs that share a workspace, sizes at which another kernel takes over."""

import ctypes
import math

import numpy as np
import pytest
import torch

import paper_1802_01561_amd as vt
from oracle import tokens as ot
from paper_1802_01561_amd._lib import lib
from test_gpu_log_prob_loss import _batch as _loss_batch
from test_gpu_log_prob_loss import PLAIN, _dev
from test_gpu_log_prob_loss import _check as _check_losses
from test_gpu_vocab import _batch, _check_grad, _check_log_probs, _gpu, _grad_inputs

pytestmark = pytest.mark.gpu


def _same(a, b):
    assert len(a) == len(b)
    for p, q in zip(a, b):
        assert (p is None) == (q is None)
        assert p is None or torch.equal(p, q)


@pytest.mark.parametrize("bias", [False, True])
@pytest.mark.parametrize("N", [1, 15, 16, 17, 32, 33, 48, 49, 63, 64, 65, 127, 128, 129, 255, 256, 257])
def test_steps_where_another_kernel_takes_over(N, bias):
    H, V = 192 + 8, 3001
    x, w, b, tokens, _, _ = _batch(N, N, 1, H, V, bias=bias, none=0.1)
    _check_log_probs(x, w, b, tokens, vt.vtrace_vocab_log_probs(*_gpu(x, w, b, tokens)))


@pytest.mark.parametrize("N,H,V", [(20, 512, 33000), (16, 8, 20001), (33, 520, 33003), (64, 1032, 16400), (100, 8, 70001),
                                   (128, 328, 66001), (1, 520, 33003), (16, 1400, 12301), (32, 1032, 16400), (31, 1376, 24575),
                                   (17, 768, 24576), (40, 72, 12288), (64, 72, 12287), (33, 72, 6144), (64, 8, 300), (2, 136, 140001)])
def test_layers_where_another_kernel_takes_over(N, H, V):
    """On both sides of 2^24 elements, of the bounds on V, of 16, 32 and 64 tokens a workgroup, and of one round."""
    x, w, b, tokens, _, _ = _batch(N + V, N, 1, H, V, bias=True, none=0.1)
    ws = vt.VocabWorkspace(N, 1, V, H)
    ws.tensor[256:].fill_(0xFF)
    _check_log_probs(x, w, b, tokens, vt.vtrace_vocab_log_probs(*_gpu(x, w, b, tokens), workspace=ws))


@pytest.mark.parametrize("N,H,V", [(129, 8, 1), (300, 64, 2), (1, 2048, 3), (2, 8, 40000), (63, 72, 129), (128, 128, 128),
                                   (257, 256, 257), (512, 264, 1)])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_smallest_and_flat_layers(N, H, V, dtype):
    x, w, b, tokens, d_lp, d_h = _batch(N + V, 1, N, H, V, bias=True, none=0.1)
    _check_log_probs(x, w, b, tokens, vt.vtrace_vocab_log_probs(*_gpu(x, w, b, tokens)))
    ls, ent = _grad_inputs(x, w, b, tokens)
    out = vt.vtrace_vocab_grad(*_gpu(x, w, b, tokens, ls, ent, d_lp, d_h), grad_dtype=dtype)
    _check_grad(x, w, b, tokens, d_lp, d_h, out, dtype)


@pytest.mark.parametrize("none", [0.0, 0.9, 1.0])
def test_parts_of_d_hidden_follow_the_steps_that_count(none):
    """A workspace for 2000 steps, of which few, most or none have a token; then the others'
    turn in the same workspace."""
    T, B, H, V = 250, 8, 72, 2500
    ws = vt.VocabWorkspace(T, B, V, H, grad_dtype=torch.float32)
    ws.tensor[256:].fill_(0xFF)
    for seed, share in ((1, none), (2, 0.5), (3, none)):
        x, w, b, tokens, d_lp, d_h = _batch(seed, T, B, H, V, none=share)
        ls, ent = _grad_inputs(x, w, b, tokens)
        out = vt.vtrace_vocab_grad(*_gpu(x, w, b, tokens, ls, ent, d_lp, d_h), workspace=ws)
        _check_grad(x, w, b, tokens, d_lp, d_h, out, torch.float32)


@pytest.mark.parametrize("N,H,V", [(8192, 64, 130), (8193, 72, 300), (20011, 64, 257), (200000, 8, 40)])
def test_many_steps(N, H, V):
    """On both sides of the number of steps up to which one launch lists and gathers them."""
    x, w, b, tokens, d_lp, d_h = _batch(N, N, 1, H, V, bias=True, none=0.3)
    tokens[:300] = vt.NO_TOKEN
    ws = vt.VocabWorkspace(N, 1, V, H)
    ws.tensor[256:].fill_(0xFF)
    _check_log_probs(x, w, b, tokens, vt.vtrace_vocab_log_probs(*_gpu(x, w, b, tokens), workspace=ws))
    ls, ent = _grad_inputs(x, w, b, tokens)
    d_lp, d_h = (torch.where(tokens >= 0, t, 0.0) for t in (d_lp, d_h))
    out = vt.vtrace_vocab_grad(*_gpu(x, w, b, tokens, ls, ent, d_lp, d_h))
    _check_grad(x, w, b, tokens, d_lp, d_h, out, torch.float32)


@pytest.mark.parametrize("T,B", [(200000, 1), (70000, 3)])
def test_losses_of_the_longest_lanes(T, B):
    y = _loss_batch(T, T, B, lengths=(lambda r: r.integers(0, T + 1, B)) if B > 1 else None)
    out = vt.vtrace_log_prob_loss_grad(**_dev(y), **PLAIN, with_vs=True, with_pg_advantages=True)
    _check_losses(y, out, PLAIN)


def test_losses_of_many_lanes():
    """The recursion of all lanes at once in float64 (the oracle walks them one by one)."""
    T, B = 3, 300001
    y = _loss_batch(T, T, B)
    out = vt.vtrace_log_prob_loss_grad(**_dev(y), **PLAIN, with_vs=True, with_pg_advantages=True)
    f = {k: v.astype(np.float64) for k, v in y.items() if v is not None}
    rho = np.minimum(1.0, np.exp(f["target_log_probs"] - f["behaviour_log_probs"]))
    r, g, v = f["rewards"], f["discounts"], f["values"]
    vs, adv = np.empty((T, B)), np.empty((T, B))
    after, v_after = f["bootstrap_value"], f["bootstrap_value"]
    for t in reversed(range(T)):
        adv[t] = rho[t] * (r[t] + g[t] * after - v[t])
        vs[t] = v[t] + rho[t] * (r[t] + g[t] * v_after - v[t]) + g[t] * rho[t] * (after - v_after)
        after, v_after = vs[t], v[t]
    for got, ref in ((out.vs, vs), (out.pg_advantages, adv), (out.d_log_probs, -adv), (out.d_values, 0.5 * (v - vs))):
        # as in _check of the losses' tests
        assert (np.abs(got.cpu().double().numpy() - ref) <= 2.0 ** -24 * np.abs(ref) + 1e-9 * (1.0 + np.abs(ref).max())).all()


def test_native_and_python_marshalling_agree():
    """A workspace and no stream goes through native code, a stream through Python."""
    T, B, H, V = 40, 3, 64, 700
    x, w, b, tokens, d_lp, d_h = _gpu(*_batch(5, T, B, H, V, bias=True, none=0.2))
    here = torch.cuda.current_stream()
    fw = vt.VocabWorkspace(T, B, V, H)
    native = vt.vtrace_vocab_log_probs(x, w, b, tokens, workspace=fw)
    _same(native, vt.vtrace_vocab_log_probs(x, w, b, tokens, workspace=fw, stream=here))
    plain = vt.vtrace_vocab_log_probs(x, w, b, tokens, workspace=fw, with_entropy=False)
    _same(plain[:2], native[:2])
    assert plain.entropy is None
    out = vt.VocabLogProbs(*(torch.empty_like(t) for t in native))
    assert vt.vtrace_vocab_log_probs(x, w, b, tokens, workspace=fw, out=out) is out
    _same(out, native)
    for dtype in (torch.float32, torch.bfloat16):
        gw = vt.VocabWorkspace(T, B, V, H, grad_dtype=dtype)
        args = (x, w, b, tokens, native.log_sums, native.entropy, d_lp, d_h)
        grads = vt.vtrace_vocab_grad(*args, grad_dtype=dtype, workspace=gw)
        _same(grads, vt.vtrace_vocab_grad(*args, grad_dtype=dtype, workspace=gw, stream=here))
        out = vt.VocabGrad(*(torch.empty_like(t) for t in grads))
        assert vt.vtrace_vocab_grad(*args, grad_dtype=dtype, workspace=gw, out=out) is out
        _same(out, grads)
        # the gradient of a bias that is not asked for, and one of a layer without a bias
        _same(vt.vtrace_vocab_grad(*args, grad_dtype=dtype, workspace=gw, out=vt.VocabGrad(*out[:2], None))[:2], grads[:2])
        free = (x, w, None, tokens, native.log_sums, native.entropy, d_lp, d_h)
        zero = (x, w, torch.zeros_like(b), tokens, native.log_sums, native.entropy, d_lp, d_h)
        _same(vt.vtrace_vocab_grad(*free, grad_dtype=dtype, workspace=gw, out=out),
              vt.vtrace_vocab_grad(*zero, grad_dtype=dtype, workspace=gw))
    y = _dev(_loss_batch(9, 300, 9))
    lw = vt.LogProbWorkspace(300, 9)
    native = vt.vtrace_log_prob_loss_grad(**y, workspace=lw, with_vs=True, with_pg_advantages=True)
    _same(native, vt.vtrace_log_prob_loss_grad(**y, workspace=lw, with_vs=True, with_pg_advantages=True, stream=here))
    cw = vt.ClipWorkspace()
    g = [torch.randn(n, device="cuda") for n in (5, 4000, 1)]
    outs = [[torch.empty_like(t) for t in g] for _ in range(2)]
    norms = [vt.vtrace_clip_grad_norm(g, 1, out=o, workspace=cw, stream=s) for o, s in zip(outs, (None, here))]
    assert torch.equal(*norms)
    _same(*outs)


def test_calls_at_the_same_time():
    """Two streams, a workspace each, several rounds: what each gets alone."""
    T, B, H, V = 60, 4, 128, 5000
    sets = []
    for seed in (1, 2):
        x, w, b, tokens, d_lp, d_h = _gpu(*_batch(seed, T, B, H, V, bias=True, none=0.1))
        y = _dev(_loss_batch(seed, 3000, 5))
        sets.append((x, w, b, tokens, d_lp, d_h, y, vt.VocabWorkspace(T, B, V, H),
                     vt.VocabWorkspace(T, B, V, H, grad_dtype=torch.bfloat16), vt.LogProbWorkspace(3000, 5), vt.ClipWorkspace()))

    def step(x, w, b, tokens, d_lp, d_h, y, fw, gw, lw, cw):
        o = vt.vtrace_vocab_log_probs(x, w, b, tokens, workspace=fw)
        g = vt.vtrace_vocab_grad(x, w, b, tokens, o.log_sums, o.entropy, d_lp, d_h, grad_dtype=torch.bfloat16, workspace=gw)
        loss = vt.vtrace_log_prob_loss_grad(**y, workspace=lw)
        return [*o, *g, loss.losses, loss.d_log_probs, vt.vtrace_clip_grad_norm(list(g), 0.1, workspace=cw)]

    alone = [step(*s) for s in sets]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in sets]
    for _ in range(4):
        got = []
        for s, stream in zip(sets, streams):
            with torch.cuda.stream(stream):
                got.append(step(*s))
        torch.cuda.synchronize()
        for a, b in zip(alone, got):
            _same(a, b)


def test_two_graphs_share_workspaces():
    """Captured apart, replayed one after the other in either order, with eager calls between."""
    T, B, H, V = 60, 3, 64, 900
    fw, gw = vt.VocabWorkspace(T, B, V, H), vt.VocabWorkspace(T, B, V, H, grad_dtype=torch.float32)
    lw, cw = vt.LogProbWorkspace(T, B), vt.ClipWorkspace()
    rest = _dev(_loss_batch(3, T, B))

    def step(x, w, b, tokens):
        o = vt.vtrace_vocab_log_probs(x, w, b, tokens, workspace=fw)
        y = dict(rest, target_log_probs=o.log_probs, entropy=o.entropy)
        loss = vt.vtrace_log_prob_loss_grad(**y, workspace=lw)
        g = vt.vtrace_vocab_grad(x, w, b, tokens, o.log_sums, o.entropy, loss.d_log_probs, loss.d_entropy, workspace=gw)
        return [*o, loss.losses, *g, vt.vtrace_clip_grad_norm(list(g), 0.3, workspace=cw)]

    inputs = [_gpu(*_batch(seed, T, B, H, V, bias=True, none=none)[:4]) for seed, none in ((41, 0.0), (42, 0.6))]
    expect = [[t.clone() for t in step(*i)] for i in inputs]
    graphs, held = [], []
    for i in inputs:
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            held.append(step(*i))
        graphs.append(graph)
    for order in ((0, 1), (1, 0), (0, 0, 1)):
        for k in order:
            graphs[k].replay()
        torch.cuda.synchronize()
        for k in (0, 1):
            _same(held[k], expect[k])
        _same(step(*inputs[1]), expect[1])


def test_log_probs_that_are_infinite():
    """A ruled-out token (log pi = -inf) has ratio 0: no gradient through it, and none before it."""
    T, B = 30, 2
    y = _loss_batch(11, T, B)
    y["target_log_probs"][12, 0] = -math.inf
    out = vt.vtrace_log_prob_loss_grad(**_dev(y), with_vs=True, with_pg_advantages=True)
    assert out.pg_advantages[12, 0] == 0 and out.d_log_probs[12, 0] == 0
    assert out.vs[12, 0] == out.vs[12, 0] and torch.isfinite(out.vs).all() and torch.isfinite(out.d_values).all()
    assert out.vs[12, 0].item() == np.float32(y["values"][12, 0])
    # the same with a behaviour that never takes its token: an infinite ratio is truncated
    y = _loss_batch(11, T, B)
    y["behaviour_log_probs"][12, 0] = -math.inf
    out = vt.vtrace_log_prob_loss_grad(**_dev(y), with_vs=True)
    assert all(torch.isfinite(t).all() for t in (out.losses, out.d_log_probs, out.vs))
    y["behaviour_log_probs"][12, 0] = -1e4
    _same(out[:5], vt.vtrace_log_prob_loss_grad(**_dev(y), with_vs=True)[:5])


def test_clip_of_nothing_and_of_many():
    """Empty tensors alone, more of them than a launch holds, and single elements among them."""
    empty = [torch.empty(0, device="cuda") for _ in range(300)]
    assert vt.vtrace_clip_grad_norm(empty, 1.0).item() == 0.0
    some = list(empty)
    for i in range(0, 300, 7):
        some[i] = torch.full((1,), 2.0, device="cuda", dtype=torch.bfloat16 if i % 2 else torch.float32)
    n = len(range(0, 300, 7))
    assert vt.vtrace_clip_grad_norm(some, None).item() == np.float32(math.sqrt(4.0 * n))
    vt.vtrace_clip_grad_norm(some, 1.0, workspace=vt.ClipWorkspace())
    for i in range(0, 300, 7):
        # factor and product round once each, bfloat16 2^-8
        assert abs(some[i].item() - 1.0 / math.sqrt(n)) <= (2.0 ** -8 + 2.0 ** -23 if i % 2 else 2.0 ** -23) / math.sqrt(n)
    twice = torch.ones(5, device="cuda")
    with pytest.raises(vt.VtraceError, match="PARAM"):
        vt.vtrace_clip_grad_norm([twice, twice], 1.0)
    assert (twice == 1).all()
    assert vt.vtrace_clip_grad_norm([twice, twice], None).item() == np.float32(math.sqrt(10.0))


def test_rows_behind_the_outputs_of_a_shorter_call():
    """A call on the first rows of larger tensors leaves the others as they were."""
    T, B, H, V = 20, 2, 64, 300
    x, w, b, tokens, d_lp, d_h = _gpu(*_batch(6, T, B, H, V, bias=True))
    keep = T - 7
    outs = vt.VocabLogProbs(*(torch.full((T, B), 5.0, device="cuda") for _ in range(3)))
    grads = vt.VocabGrad(torch.full((T, B, H), 5.0, device="cuda"), torch.empty((V, H), device="cuda"), torch.empty(V, device="cuda"))
    o = vt.vtrace_vocab_log_probs(x[:keep], w, b, tokens[:keep], out=vt.VocabLogProbs(*(t[:keep] for t in outs)))
    vt.vtrace_vocab_grad(x[:keep], w, b, tokens[:keep], o.log_sums, o.entropy, d_lp[:keep], d_h[:keep],
                         out=vt.VocabGrad(grads.d_hidden[:keep], *grads[1:]))
    assert all((t[keep:] == 5.0).all() for t in (*outs, grads.d_hidden))
    _same([t[:keep] for t in outs], vt.vtrace_vocab_log_probs(x[:keep], w, b, tokens[:keep]))


def test_errors_leave_the_library_usable():
    """A refused call, then the right one; the C entries return codes for what Python refuses."""
    T, B, H, V = 9, 2, 64, 100
    x, w, b, tokens, _, _ = _gpu(*_batch(7, T, B, H, V))
    ws = vt.VocabWorkspace(T, B, V, H)
    o = torch.empty((T, B), device="cuda")
    p = lambda t: ctypes.c_void_p(None if t is None else t.data_ptr())  # noqa: E731
    call = lambda n, h=x: lib().vtrace_vocab_log_probs(T, B, V, H, p(h), p(w), None, p(tokens), p(o), p(o), None,  # noqa: E731
                                                       p(ws.tensor), n, None)
    assert call(ws.nbytes - 1) != 0 and call(ws.nbytes, None) != 0
    with pytest.raises(TypeError):
        vt.vtrace_vocab_log_probs(x, w, b, tokens.long(), workspace=ws)
    _same(vt.vtrace_vocab_log_probs(x, w, b, tokens, workspace=ws), vt.vtrace_vocab_log_probs(x, w, b, tokens))
