"""The calls on a token policy's parameters as a program uses them: one learner step of all of
them, both ways into the library, calls at the same time, graphs that share a workspace, tensors
at any element, entries that are not finite, tensors of more than 2^31 elements."""

import math

import numpy as np
import pytest
import torch

import paper_1802_01561_amd as vt
from oracle import parameters as op
from paper_1802_01561_amd import binding
from test_gpu_embed import _check_embed, _normal, _tokens, check_grad
from test_gpu_log_prob_loss import _batch as _loss_batch
from test_gpu_log_prob_loss import _dev
from test_gpu_orthogonalize import check, matrix
from test_gpu_vocab import _check_grad, _check_log_probs

pytestmark = pytest.mark.gpu

F32, BF16 = torch.float32, torch.bfloat16
CUBIC = (1.5, -0.5, 0.0)


def _same(a, b):
    assert len(a) == len(b)
    for p, q in zip(a, b):
        assert p.dtype == q.dtype and torch.equal(p, q)


class Policy:
    """A tied table and one layer: hidden = tanh(embedded layer^T)."""

    def __init__(self, seed, T=24, B=5, H=72, V=901):
        g = torch.Generator().manual_seed(seed)
        self.T, self.B, self.H, self.V = T, B, H, V
        self.table = (torch.randn(V, H, generator=g) / H ** 0.5).bfloat16().cuda()
        self.layer = (torch.randn(H, H, generator=g) / H ** 0.5).cuda()
        t = _tokens(seed, T * B, V, "text", 0.1).reshape(T, B)
        self.inputs = torch.from_numpy(t).cuda()
        self.actions = torch.from_numpy(np.roll(t, -1, axis=0).copy()).cuda()
        self.rest = _dev(_loss_batch(seed, T, B))
        self.vocab, self.vocab_grad = vt.VocabWorkspace(T, B, V, H), vt.VocabWorkspace(T, B, V, H, grad_dtype=F32)
        self.embed, self.loss, self.clip = vt.EmbedWorkspace(T, B, V, H), vt.LogProbWorkspace(T, B), vt.ClipWorkspace()
        self.ortho = vt.OrthogonalWorkspace([self.layer])

    def step(self):
        scale = math.sqrt(self.H)
        x = vt.vtrace_vocab_embed(self.table, self.inputs, scale, out_dtype=F32, workspace=self.embed)
        flat = x.view(-1, self.H)
        hidden = torch.tanh(flat @ self.layer.t())
        states = hidden.bfloat16().view(self.T, self.B, self.H)
        o = vt.vtrace_vocab_log_probs(states, self.table, None, self.actions, workspace=self.vocab)
        y = dict(self.rest, target_log_probs=o.log_probs, entropy=o.entropy)
        loss = vt.vtrace_log_prob_loss_grad(**y, workspace=self.loss)
        g = vt.vtrace_vocab_grad(states, self.table, None, self.actions, o.log_sums, o.entropy, loss.d_log_probs, loss.d_entropy,
                                 grad_dtype=F32, workspace=self.vocab_grad)
        outer = g.d_weight.clone()
        d_pre = g.d_hidden.view(-1, self.H) * (1.0 - hidden * hidden)
        d_layer = d_pre.t().contiguous() @ flat
        d_x = (d_pre @ self.layer).view(self.T, self.B, self.H)
        d_table = vt.vtrace_vocab_embed_grad(d_x, self.inputs, self.V, scale, accumulate_into=g.d_weight, workspace=self.embed)
        assert d_table is g.d_weight
        both, d_layer_was = d_table.clone(), d_layer.clone()
        norm = vt.vtrace_clip_grad_norm([d_table, d_layer], 0.5, workspace=self.clip)
        clipped = d_layer.clone()
        update, = vt.vtrace_orthogonalize([d_layer], 0.2, out=[d_layer], workspace=self.ortho)
        assert update is d_layer
        return [x, states, *o, loss.losses, loss.d_log_probs, loss.d_entropy, g.d_hidden, outer, d_x, both, d_layer_was, d_table,
                norm, clipped, update]


def test_learner_step_of_all_calls():
    """Each against its oracle, with the inputs that it had."""
    p = Policy(3)
    x, states, lp, ls, ent, losses, d_lp, d_ent, d_hidden, outer, d_x, both, d_layer, d_table, norm, clipped, update = p.step()
    scale = math.sqrt(p.H)
    tokens, actions = p.inputs.cpu().numpy(), p.actions.cpu()
    _check_embed(p.table, tokens, scale, F32, x)
    c = lambda t: t.cpu()  # noqa: E731
    _check_log_probs(c(states), c(p.table), None, actions, vt.VocabLogProbs(lp, ls, ent))
    check_grad(d_x, tokens, p.V, scale, both, before=outer)
    _check_grad(c(states), c(p.table), None, actions, c(d_lp), c(d_ent), vt.VocabGrad(d_hidden, outer, None), F32)
    total = math.sqrt(sum((t.double() ** 2).sum().item() for t in (both, d_layer)))
    assert abs(norm.item() - total) <= 2.0 ** -23 * total and total > 0.5  # clipped
    for was, now in ((both, d_table), (d_layer, clipped)):
        # the norm, the factor and the product are rounded once each
        assert torch.allclose(now.double(), was.double() * (0.5 / total), rtol=2.0 ** -22, atol=2.0 ** -149)
    check(clipped, update, scale=0.2)
    for ws in (p.vocab, p.vocab_grad, p.embed, p.loss, p.clip, p.ortho):
        assert vt.vtrace_error_flag(ws) == 0


def test_learner_steps_in_graphs_that_share_workspaces():
    """Two captured apart, replayed in either order, with eager steps between."""
    ps = [Policy(7), Policy(8)]
    for name in ("vocab", "vocab_grad", "embed", "loss", "clip", "ortho"):
        setattr(ps[1], name, getattr(ps[0], name))
    expect = [[t.clone() for t in p.step()] for p in ps]
    torch.cuda.synchronize()
    graphs, held = [], []
    for p in ps:
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            held.append(p.step())
        graphs.append(graph)
    for order in ((0, 1), (1, 0), (0, 0, 1), (1, 1, 0)):
        for k in order:
            graphs[k].replay()
        torch.cuda.synchronize()
        for k in (0, 1):
            _same(held[k], expect[k])
        _same(ps[1].step(), expect[1])
        torch.cuda.synchronize()


MIXED = [(1, 1), (40, 70), (70, 40), (130, 257), (300, 300), (32, 500), (33, 20)]


def _mixed(seed, dtypes=(F32, BF16)):
    return [matrix(seed + i, m, n, dtypes[i % len(dtypes)], "strong").cuda() for i, (m, n) in enumerate(MIXED)]


def test_updates_in_graphs_replayed():
    """Matrices of all the kernels in one call, on data that changes between replays."""
    gs, other = _mixed(50), _mixed(90)
    ws = vt.OrthogonalWorkspace(gs)
    expect = [vt.vtrace_orthogonalize(x, workspace=ws) for x in (gs, other)]
    into, out = [g.clone() for g in gs], [torch.empty_like(g) for g in gs]
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        vt.vtrace_orthogonalize(into, out=out, workspace=ws)
    for k in (1, 0, 0, 1, 1):
        for a, b in zip(into, (gs, other)[k]):
            a.copy_(b)
        graph.replay()
        torch.cuda.synchronize()
        _same(out, expect[k])
        _same(vt.vtrace_orthogonalize(gs, workspace=ws), expect[0])


def test_calls_at_the_same_time():
    """Two streams, a workspace each, several rounds: what each gets alone."""
    T, B, H, V = 900, 40, 72, 5000  # past what one pass ranks
    sets = []
    for seed in (1, 2):
        gs = _mixed(100 * seed)
        sets.append((_normal(seed, (V, H), BF16).cuda(), torch.from_numpy(_tokens(seed, T * B, V, "text")).cuda().view(T, B),
                     _normal(seed + 9, (T, B, H), BF16).cuda(), gs, vt.EmbedWorkspace(T, B, V, H), vt.OrthogonalWorkspace(gs)))

    def calls(w, t, d, gs, ew, ow):
        return [vt.vtrace_vocab_embed(w, t, workspace=ew), vt.vtrace_vocab_embed_grad(d, t, V, workspace=ew),
                *vt.vtrace_orthogonalize(gs, workspace=ow), vt.vtrace_vocab_embed_grad(d[:20], t[:20], V, workspace=ew)]

    alone = [calls(*s) for s in sets]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in sets]
    for _ in range(4):
        got = []
        for s, stream in zip(sets, streams):
            with torch.cuda.stream(stream):
                got.append(calls(*s))
        torch.cuda.synchronize()
        for a, b in zip(alone, got):
            _same(a, b)


def test_native_and_python_marshalling_agree(monkeypatch):
    """A workspace and no stream goes through native code, a stream through Python."""
    fast = binding._fast_call(torch.empty(1, device="cuda"))
    ran = []
    for name in ("call_vocab_embed", "call_vocab_embed_grad", "call_orthogonalize"):
        def counted(*args, _f=getattr(fast, name)):
            r = _f(*args)
            ran.append(r is not None)
            return r
        monkeypatch.setattr(fast, name, counted)
    here = torch.cuda.current_stream()
    T, B, H, V = 31, 3, 24, 200
    t = torch.from_numpy(_tokens(1, T * B, V)).cuda().view(T, B)
    ew = vt.EmbedWorkspace(T, B, V, H)
    for table, wanted in ((F32, BF16), (BF16, F32), (BF16, None)):
        w, d = _normal(2, (V, H), table).cuda(), _normal(3, (T, B, H), table).cuda()
        a = vt.vtrace_vocab_embed(w, t, 2.5, out_dtype=wanted, workspace=ew)
        b = vt.vtrace_vocab_embed(w, t, 2.5, out_dtype=wanted, workspace=ew, stream=here)
        c = vt.vtrace_vocab_embed(w, t, 2.5, out=torch.empty_like(a))
        _same([a, a], [b, c])
        assert a.dtype == (wanted or table)
        wanted = wanted or F32
        a = vt.vtrace_vocab_embed_grad(d, t, V, 2.5, grad_dtype=wanted, workspace=ew)
        b = vt.vtrace_vocab_embed_grad(d, t, V, 2.5, grad_dtype=wanted, workspace=ew, stream=here)
        into = torch.zeros_like(a)
        c = vt.vtrace_vocab_embed_grad(d, t, V, 2.5, accumulate_into=into, workspace=ew)
        e = vt.vtrace_vocab_embed_grad(d, t, V, 2.5, out=torch.empty_like(a))
        _same([a, a, a], [b, c, e])
        assert c is into
    gs = _mixed(7)
    ow = vt.OrthogonalWorkspace(gs)
    a = vt.vtrace_orthogonalize(gs, 0.5, workspace=ow)
    b = vt.vtrace_orthogonalize(gs, 0.5, workspace=ow, stream=here)
    c = vt.vtrace_orthogonalize(iter(gs), [0.5] * len(gs), out=(torch.empty_like(g) for g in gs), workspace=ow)
    e = vt.vtrace_orthogonalize(iter(gs), 0.5, out=(torch.empty_like(g) for g in gs), workspace=ow)
    for other in (b, c, e):
        _same(a, other)
    # embed native: two of three calls each; gradients with a workspace and without a stream; two of the four updates
    assert sum(ran) == 6 + 6 + 2, ran


def test_scales_one_for_each_and_single_bits():
    gs = _mixed(20)
    scales = [0.25 * 2.0 ** i for i in range(len(gs))]
    a, b = vt.vtrace_orthogonalize(gs, scales), vt.vtrace_orthogonalize(gs)
    for x, y, s in zip(a, b, scales):
        assert torch.equal(x, y * s)  # powers of two
    for x in vt.vtrace_orthogonalize(gs, 0.0):
        assert (x == 0).all()


@pytest.mark.parametrize("first", [1, 2, 3])
def test_tensors_at_any_element(first):
    """Inputs and outputs that start, and rows that lie, at no multiple of 16 bytes; what is around them stays."""
    def moved(t):
        around = torch.full((t.numel() + 2 * first + 8,), 7.0, dtype=t.dtype, device="cuda")
        inside = around[first:first + t.numel()].view(t.shape)
        inside.copy_(t)
        return around, inside

    def untouched(around, n):
        assert (around[:first] == 7).all() and (around[first + n:] == 7).all()

    gs = _mixed(30)
    expect = vt.vtrace_orthogonalize(gs)
    for in_place in (False, True):
        ins = [moved(g) for g in gs]
        outs = ins if in_place else [moved(torch.zeros_like(g)) for g in gs]
        got = vt.vtrace_orthogonalize([i for _, i in ins], out=[o for _, o in outs])
        _same(got, expect)
        for (around, o) in outs:
            untouched(around, o.numel())
        if not in_place:
            _same([i for _, i in ins], gs)


@pytest.mark.parametrize("H", [8, 40, 72])
def test_embed_outputs_leave_what_is_around_them(H):
    """Rows and the gradient's table between others of the same tensor, at 16 bytes."""
    T, B, V = 50, 3, 90
    t = torch.from_numpy(_tokens(H, T * B, V)).cuda().view(T, B)
    w, d = _normal(1, (V, H), BF16).cuda(), _normal(2, (T, B, H), BF16).cuda()
    rows = torch.full((T + 2, B, H), 7.0, dtype=BF16, device="cuda")
    vt.vtrace_vocab_embed(w, t, out=rows[1:-1])
    assert torch.equal(rows[1:-1], vt.vtrace_vocab_embed(w, t)) and (rows[0] == 7).all() and (rows[-1] == 7).all()
    for dtype in (F32, BF16):
        table = torch.full((V + 2, H), 7.0, dtype=dtype, device="cuda")
        vt.vtrace_vocab_embed_grad(d, t, V, out=table[1:-1])
        assert torch.equal(table[1:-1], vt.vtrace_vocab_embed_grad(d, t, V, grad_dtype=dtype))
        assert (table[0] == 7).all() and (table[-1] == 7).all()


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("value", [math.nan, math.inf, -math.inf])
def test_what_is_not_finite_stays_in_its_matrix(dtype, value):
    gs = _mixed(40, (dtype,))
    expect = vt.vtrace_orthogonalize(gs)
    for which in range(len(gs)):
        bad = [g.clone() for g in gs]
        bad[which].view(-1)[-1] = value
        got = vt.vtrace_orthogonalize(bad)
        assert torch.isnan(got[which]).all()
        _same([o for i, o in enumerate(got) if i != which], [o for i, o in enumerate(expect) if i != which])


@pytest.mark.parametrize("m,n", [(1, 9), (20, 30), (64, 40), (200, 300)])
@pytest.mark.parametrize("dtype", [F32, BF16])
def test_zeros_and_norms_below_epsilon(m, n, dtype):
    g = matrix(m, m, n, dtype).cuda()
    zero, small, large = torch.zeros_like(g), (g.double() * 2.0 ** -40).to(dtype), (g.double() * 2.0 ** 100).to(dtype)
    got = vt.vtrace_orthogonalize([zero, small, large])
    assert (got[0] == 0).all()
    check(small, got[1])
    check(large, got[2])
    got, = vt.vtrace_orthogonalize([g], epsilon=1.0)
    check(g, got, epsilon=1.0)


@pytest.mark.parametrize("m,n", [(2, 2), (20, 33), (32, 500), (90, 100), (300, 140)])
@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("coefficients", [(op.QUINTIC,), (op.QUINTIC,) * 2, (op.QUINTIC,) * 3, (op.QUINTIC,) * 4, (op.QUINTIC,) * 6,
                                          (CUBIC,) * 3, (CUBIC,) * 12, (op.QUINTIC, (2.5, -2.0, 0.5), CUBIC)])
def test_other_steps(m, n, dtype, coefficients):
    g = matrix(m + n, m, n, dtype)
    got, = vt.vtrace_orthogonalize([g.cuda()], steps=len(coefficients), coefficients=coefficients)
    check(g, got, steps=coefficients)


@pytest.mark.parametrize("m,n", [(1, 3), (9, 20), (32, 32)])
@pytest.mark.parametrize("steps", [7, 8, 64])
def test_many_steps_of_few_rows(m, n, steps):
    """On both sides of what the small matrices' own steps take, of full rank and of less."""
    for rank in (m, max(1, m // 3)):
        g = torch.Generator().manual_seed(steps + rank)
        x = (torch.randn(m, rank, generator=g) @ torch.randn(rank, n, generator=g)).cuda()
        got, = vt.vtrace_orthogonalize([x], steps=steps)
        s = np.linalg.svd(got.double().cpu().numpy(), compute_uv=False)
        # of full rank in its float32 elements they have all come near 1; no direction ever leaves the range
        assert s[:rank].min() > 0.6 and s.max() < 1.3


def test_a_workspace_for_more_serves_less_and_other_calls():
    gs = _mixed(60)
    T, B, H, V = 40, 5, 24, 300
    t = torch.from_numpy(_tokens(4, T * B, V)).cuda().view(T, B)
    d = _normal(5, (T, B, H), F32).cuda()
    ws, big = vt.OrthogonalWorkspace(gs), vt.EmbedWorkspace(T, B, V, H)
    ws.tensor[4352:].fill_(0xFF)
    expect = [vt.vtrace_orthogonalize(gs[k:k + 2]) for k in range(5)]
    for k in range(5):
        _same(vt.vtrace_orthogonalize(gs[k:k + 2], workspace=ws), expect[k])
        vt.vtrace_orthogonalize(gs, workspace=ws)
    whole = vt.vtrace_vocab_embed_grad(d, t, V)
    part = vt.vtrace_vocab_embed_grad(d[:7], t[:7], V)
    for _ in range(3):
        _same([vt.vtrace_vocab_embed_grad(d, t, V, workspace=big), vt.vtrace_vocab_embed_grad(d[:7], t[:7], V, workspace=big)], [whole, part])


@pytest.mark.parametrize("N", [300, 20000])
def test_gradient_against_differences(N):
    """The lookup is linear: with small integers, (embed(w + e) - embed(w)) . d = gradient . e, exactly."""
    H, V, scale = 16, 70, 2.0
    r = np.random.default_rng(N)
    whole = lambda *shape: torch.from_numpy(r.integers(-3, 4, shape).astype(np.float32)).cuda()  # noqa: E731
    w, e, d = whole(V, H), whole(V, H), whole(N, 1, H)
    t = torch.from_numpy(_tokens(N, N, V, "text")).cuda().view(N, 1)
    change = (vt.vtrace_vocab_embed(w + e, t, scale) - vt.vtrace_vocab_embed(w, t, scale)).double()
    grad = vt.vtrace_vocab_embed_grad(d, t, V, scale).double()
    assert (change * d.double()).sum().item() == (grad * e.double()).sum().item()


def test_more_than_2_31_elements():
    """A table, outputs and a gradient past 32 bits: every token once, in another order."""
    H, V = 8192, 270001
    w = torch.empty((V, H), dtype=BF16, device="cuda").random_(-100, 100)
    order = torch.randperm(V, generator=torch.Generator().manual_seed(1)).int()
    t = order.cuda().view(V, 1)
    rows = vt.vtrace_vocab_embed(w, t)
    ws = vt.EmbedWorkspace(V, 1, V, H)
    grad = vt.vtrace_vocab_embed_grad(rows, t, V, grad_dtype=BF16, workspace=ws)
    assert torch.equal(grad, w)
    for at in (0, 1000, 262143, 262144, 262145, V - 1):
        assert torch.equal(rows[at, 0], w[order[at].item()])
    assert vt.vtrace_error_flag(ws) == 0


def test_most_steps_and_most_tokens():
    """2^25 steps of the shortest rows, 2^24 tokens: sums of small integers, exactly."""
    T, B, H, V = 4096, 8192, 8, 1 << 24
    g = torch.Generator(device="cuda").manual_seed(2)
    t = torch.randint(-1, V, (T, B), generator=g, device="cuda", dtype=torch.int32)
    t[::7] %= 1000  # frequent ones
    t[5] = vt.NO_TOKEN
    d = torch.randint(-3, 4, (T, B, H), generator=g, device="cuda").to(BF16)
    ws = vt.EmbedWorkspace(T, B, V, H)
    flat, rows = t.view(-1).long(), d.view(-1, H).float()
    expect = torch.zeros((V + 1, H), device="cuda").index_add_(0, torch.where(flat < 0, V, flat), rows)[:V]
    got = vt.vtrace_vocab_embed_grad(d, t, V, workspace=ws)
    assert torch.equal(got, expect)
    before = torch.randint(-3, 4, (V, H), generator=g, device="cuda").float()
    assert torch.equal(vt.vtrace_vocab_embed_grad(d, t, V, 2.0, accumulate_into=before.clone(), workspace=ws), before + 2.0 * expect)
    out = vt.vtrace_vocab_embed(expect, t, 0.5, out_dtype=F32, workspace=ws)
    assert torch.equal(out.view(-1, H), torch.where((flat < 0)[:, None], 0.0, 0.5 * expect[flat.clamp(min=0)]))
    assert vt.vtrace_error_flag(ws) == 0


def test_tokens_at_any_element():
    T, B, H, V = 30, 7, 16, 50
    w, d = _normal(1, (V, H), F32).cuda(), _normal(2, (T, B, H), F32).cuda()
    t = torch.from_numpy(_tokens(3, T * B, V)).cuda()
    around = torch.full((T * B + 9,), 2 ** 30, dtype=torch.int32, device="cuda")
    for first in (1, 2, 3):
        inside = around[first:first + T * B]
        inside.copy_(t)
        ws = vt.EmbedWorkspace(T, B, V, H)
        _same([vt.vtrace_vocab_embed(w, inside.view(T, B), workspace=ws), vt.vtrace_vocab_embed_grad(d, inside.view(T, B), V, workspace=ws)],
              [vt.vtrace_vocab_embed(w, t.view(T, B)), vt.vtrace_vocab_embed_grad(d, t.view(T, B), V)])
        assert vt.vtrace_error_flag(ws) == 0
        around.fill_(2 ** 30)


@pytest.mark.parametrize("dtype,m,n", [(BF16, 65536, 32768), (BF16, 32768, 65536), (F32, 65536, 32768), (BF16, 65536, 40),
                                       (F32, 24, 65536), (F32, 65536, 5000)])
def test_largest_matrices(dtype, m, n):
    """Three singular values with vectors of signs, whose products are small integers; anything out of
    place is off by its whole size.  bfloat16: an operand's rounding (2^-11) counts up to 5 times in B X in each of
    five steps, on singular values that steps take at most apart by 3.4 once and then by about 1: 2^-6.
    Float32: terms of few values, of whose sums the roundings do not cancel.  k terms are k / 32
    additions, each off by up to 2^-24 of what is reached, half of the sum on average: for k = 65536
    2^10 2^-24 = 2^-14 of A, as much of B and of B X; times B's sizes (4.8 + 2 * 2.0), in five steps, one of
    which takes them apart by 3.4: 2^-14 * 8.8 * 5 * 3.4 = 2^-6.8."""
    def signs(count, mask):
        i = torch.arange(count, device="cuda")
        p = i & mask
        for s in (8, 4, 2, 1):
            p = p ^ (p >> s)
        return 1.0 - 2.0 * (p & 1).float()

    u = torch.stack([signs(m, k) for k in (0x2D31, 0x0000, 0x7B06)])
    # orthogonal columns for the sizes that are no power of two as well: halves, quarters, eighths
    i = torch.arange(n, device="cuda")
    e = n // 8
    v = torch.stack([1.0 - 2.0 * ((i // (e * k)) % 2).float() for k in (4, 2, 1)])
    sizes = torch.tensor([4.0, 2.0, 1.0], device="cuda")
    g = ((u * sizes[:, None]).t().contiguous() @ v).to(dtype)
    ws = vt.OrthogonalWorkspace([g])
    got, = vt.vtrace_orthogonalize([g], workspace=ws)
    f = sizes.double().cpu().numpy() / math.sqrt(21.0)
    for _ in range(5):
        f = f * (3.4445 - 4.7750 * f ** 2 + 2.0315 * f ** 4)
    f = torch.tensor(f, device="cuda").float()[:, None]
    worst = size = 0.0
    for at in range(0, m, 4096):
        expect = (u[:, at:at + 4096] * f).t().contiguous() @ v / math.sqrt(m * n)
        worst = max(worst, (got[at:at + 4096].float() - expect).abs().max().item())
        size = max(size, expect.abs().max().item())
    print(f"[case] {dtype} {m} x {n}: {worst / size:.2e}", flush=True)
    assert worst <= 2.0 ** -6 * size


@pytest.mark.parametrize("kernel", [f"ortho_{size}x{together}k{pieces}" for size in (128, 256) for together in (1, 2) for pieces in (2, 3)])
@pytest.mark.parametrize("dtype", [F32, BF16])
def test_tiles_split_along_k(kernel, dtype, monkeypatch):
    """Pieces of even and uneven lengths, several matrices' tiles, twice in one workspace, in a graph."""
    monkeypatch.setenv("VTRACE_KERNEL", kernel)
    shapes = [(130, 700), (640, 640), (257, 255), (70, 64), (300, 1000), (1000, 300)]
    gs = [matrix(i, m, n, dtype, "strong") for i, (m, n) in enumerate(shapes)]
    on = [g.cuda() for g in gs]
    ws = vt.OrthogonalWorkspace(on)
    ws.tensor[4352:].fill_(0xFF)
    got = vt.vtrace_orthogonalize(on, workspace=ws)
    for g, o in zip(gs, got):
        check(g, o)
    out = [torch.empty_like(g) for g in on]
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        vt.vtrace_orthogonalize(on, out=out, workspace=ws)
    for _ in range(3):
        for o in out:
            o.zero_()
        graph.replay()
        torch.cuda.synchronize()
        _same(out, got)
        _same(vt.vtrace_orthogonalize(on, workspace=ws), got)
    assert int(ws.tensor[:4352].count_nonzero()) == 0  # flag and counters


def test_empty_matrices_and_very_many():
    """Nothing to do, nothing among something, and more than one launch's table many times over."""
    empty = [torch.empty((0, 5), device="cuda"), torch.empty((7, 0), dtype=BF16, device="cuda")]
    for got, g in zip(vt.vtrace_orthogonalize(empty), empty):
        assert got.shape == g.shape and got.dtype == g.dtype
    gs = [matrix(i, 1 + i % 9, 1 + i % 7, F32 if i % 3 else BF16) for i in range(2000)]
    gs[500], gs[777] = matrix(1, 100, 130, F32), matrix(2, 100, 130, BF16)
    on = [g.cuda() for g in gs]
    on.insert(3, empty[0])
    gs.insert(3, empty[0].cpu())
    got = vt.vtrace_orthogonalize(on)
    assert got[3].numel() == 0
    for i in (0, 1, 2, 4, 8, 38, 39, 501, 778, 1999, 2000):
        check(gs[i], got[i])
    again = vt.vtrace_orthogonalize(on, out=on)
    _same(again, got)


def test_same_matrix_twice_and_refused_overlaps():
    g = matrix(9, 40, 60, F32).cuda()
    a, b = vt.vtrace_orthogonalize([g, g])
    assert torch.equal(a, b) and torch.equal(a, vt.vtrace_orthogonalize([g])[0])
    both = torch.empty(2 * g.numel(), device="cuda")
    overlapping = [both[:g.numel()].view(g.shape), both[g.numel() - 1:-1].view(g.shape)]
    for outs in ([g, torch.empty_like(g)], [a, a], overlapping):
        with pytest.raises(vt.VtraceError, match="PARAM"):
            vt.vtrace_orthogonalize([g, g], out=outs)
    assert torch.equal(g, matrix(9, 40, 60, F32).cuda())


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("long", [False, True])
def test_few_rows_beside_others(dtype, long):
    """With the others' X, or their first A: whichever launch has them, what they get alone, in place too."""
    few = [matrix(i, m, n, dtype, "strong") for i, (m, n) in enumerate([(1, 3), (32, 500), (700, 20), (32, 32), (9, 65)])]
    gs = [few[0], matrix(7, 90, 2500 if long else 100, dtype), *few[1:3], matrix(8, 70, 66, dtype), *few[3:]]
    on = [g.cuda() for g in gs]
    ws = vt.OrthogonalWorkspace(on)
    ws.tensor[4352:].fill_(0xFF)
    got = vt.vtrace_orthogonalize(on, 0.5, workspace=ws)
    for g, o in zip(gs, got):
        check(g, o, scale=0.5)
    alone = vt.vtrace_orthogonalize([g.cuda() for g in few], 0.5)
    _same([o for i, o in enumerate(got) if i not in (1, 4)], alone)
    _same(vt.vtrace_orthogonalize(on, 0.5, out=on, workspace=ws), got)


@pytest.mark.parametrize("dtype,shapes,fewer", [
    (BF16, [(512, 2048)] * 9, (8, 5, 1)), (BF16, [(2048, 512)] * 11, (10,)), (F32, [(512, 512)] * 15, (14, 3)),
    (F32, [(700, 2100), (90, 100), (20, 500), (700, 2100), (33, 64), (640, 640)] * 7, (41, 39, 20)),
    (BF16, [(4096, 4096)] * 2 + [(4096, 16384)], (2, 1))])
def test_a_workspace_for_all_matrices_serves_some_of_them(dtype, shapes, fewer):
    """The last ones alone, whose tiles are others than those of all: what they get in a workspace of their own, and
    nothing behind the workspace's bytes is written."""
    gs = [(1e-3 * torch.randn(s, generator=torch.Generator(device="cuda").manual_seed(i), device="cuda")).to(dtype) for i, s in enumerate(shapes)]
    ws = vt.OrthogonalWorkspace(gs)
    ws.tensor = torch.full((ws.nbytes + 65536,), 0xFF, dtype=torch.uint8, device="cuda")
    ws.tensor[:4352] = 0
    whole = vt.vtrace_orthogonalize(gs, workspace=ws)
    for k in fewer:
        own = vt.OrthogonalWorkspace(gs[-k:])
        assert own.nbytes <= ws.nbytes
        own.tensor = torch.full((own.nbytes + 65536,), 0xFF, dtype=torch.uint8, device="cuda")
        own.tensor[:4352] = 0
        _same(vt.vtrace_orthogonalize(gs[-k:], workspace=ws), vt.vtrace_orthogonalize(gs[-k:], workspace=own))
        assert (own.tensor[own.nbytes:] == 0xFF).all()
    _same(vt.vtrace_orthogonalize(gs, workspace=ws), whole)
    assert (ws.tensor[ws.nbytes:] == 0xFF).all()


def test_scales_as_tensors():
    gs = _mixed(25)
    expect = vt.vtrace_orthogonalize(gs, 0.5)
    for scale in (torch.tensor(0.5), torch.tensor(0.5, device="cuda"), torch.full((len(gs),), 0.5), np.array(0.5)):
        _same(vt.vtrace_orthogonalize(gs, scale), expect)
