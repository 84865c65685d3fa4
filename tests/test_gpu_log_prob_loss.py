"""V-trace losses from log-probabilities, and clipping by the global norm, on the GPU
against the fp64 oracle.

Ratios, recursion and sums are float64 and outputs float32.  The ratio's exponential is
within 6e-11 of itself and a step's value is a sum over the steps behind it, so an output
is within a float32 rounding (2^-24) of its value plus 1e-9 of the largest value in the
batch (a hundred thousand steps' errors of 6e-11 that decay would not reach 1e-9 a step;
the weights of these batches are at most about 1)."""

import math

import numpy as np
import pytest
import torch

import paper_1802_01561_amd as vt
from oracle import tokens as ot

pytestmark = pytest.mark.gpu

U = 2.0 ** -24


def _batch(seed, T, B, *, entropy=True, lengths=None):
    r = np.random.default_rng(seed)
    f = lambda x: np.ascontiguousarray(x, dtype=np.float32)  # noqa: E731
    lp = f(-r.exponential(1.5, (T, B)))
    lm = f(np.minimum(lp + 0.3 * r.normal(size=(T, B)), 0.0))
    x = dict(target_log_probs=lp, behaviour_log_probs=lm, entropy=f(r.random((T, B)) * 3) if entropy else None,
             rewards=f(r.normal(size=(T, B)) * (r.random((T, B)) < 0.3)),
             discounts=f(np.where(r.random((T, B)) < 0.01, 0.0, 0.97)), values=f(r.normal(size=(T, B))),
             bootstrap_value=f(r.normal(size=B)))
    x["lengths"] = None if lengths is None else np.asarray(lengths(r), dtype=np.int32)
    return x


def _dev(x):
    return {k: None if v is None else torch.from_numpy(np.array(v)).cuda() for k, v in x.items()}


def _f32(v):
    return float(np.float32(v))


def _check(x, out, scalars, **kw):
    s = {k: _f32(v) for k, v in scalars.items()}
    if "epsilon" in kw:
        kw["epsilon"] = _f32(kw["epsilon"])
    o = ot.log_prob_loss_and_grads(**x, **s, **kw)
    for name in ("d_log_probs", "d_values", "d_entropy", "vs", "pg_advantages"):
        got, ref = getattr(out, name), getattr(o, name)
        if got is None:
            continue
        # tanhf of the asymmetric rewards: a few float32 roundings of rewards below 5
        slack = 1e-9 if kw.get("reward_transform") != "asymmetric" else 40 * U
        err = np.abs(got.cpu().double().numpy() - ref)
        assert (err <= U * np.abs(ref) + slack * (1.0 + np.abs(ref).max())).all(), (name, err.max())
    rss = np.sqrt((o.step_losses ** 2).sum(axis=(0, 1)))
    slack = 1e-8 if kw.get("reward_transform") != "asymmetric" else 1e-4
    tol = U * np.abs(o.losses) + slack * np.concatenate([[rss.sum()], rss]) * 10 + 1e-12
    assert (np.abs(out.losses.cpu().double().numpy() - o.losses) <= tol).all(), (out.losses, o.losses)
    return o


PLAIN = dict(rho_bar=1.0, c_bar=1.0, lam=1.0, baseline_cost=0.5, entropy_cost=0.01)
SHAPES = [(1, 1), (2, 3), (7, 1), (100, 32), (128, 16), (129, 17), (2049, 1), (5000, 2), (3000, 3), (4096, 5), (777, 100),
          (20, 5000)]


def _ragged(T, B):
    return lambda r: np.concatenate([[0, T, -3, T + 5, 1], r.integers(0, T + 1, B)])[:B]


@pytest.mark.parametrize("ragged", [False, True])
@pytest.mark.parametrize("T,B", SHAPES)
def test_losses_and_gradients(T, B, ragged):
    x = _batch(T + B, T, B, entropy=ragged or T % 2 == 0, lengths=_ragged(T, B) if ragged else None)
    d = _dev(x)
    if ragged:  # whatever lies behind a lane's last step
        behind = torch.arange(T, device="cuda").unsqueeze(1) >= d["lengths"].unsqueeze(0)
        for k in ("target_log_probs", "behaviour_log_probs", "entropy", "rewards", "discounts", "values"):
            d[k][behind] = float("nan")
    ws = vt.LogProbWorkspace(T, B)
    ws.tensor[256 + 4096:].fill_(0xFF)  # behind the counters, which every call leaves at zero
    for s in (PLAIN, dict(rho_bar=0.9, c_bar=0.5, lam=0.95, baseline_cost=0.3, entropy_cost=0.1)):
        out = vt.vtrace_log_prob_loss_grad(**d, **s, workspace=ws, with_vs=True, with_pg_advantages=True)
        assert (out.d_entropy is None) == (x["entropy"] is None)
        _check(x, out, s)
        again = vt.vtrace_log_prob_loss_grad(**d, **s, workspace=ws)
        assert torch.equal(again.losses, out.losses) and torch.equal(again.d_log_probs, out.d_log_probs)
        assert again.vs is None and again.pg_advantages is None
    if ragged:
        for t in (out.d_log_probs, out.d_values, out.d_entropy, out.vs, out.pg_advantages):
            assert not t[behind].any()


@pytest.mark.parametrize("kw", [dict(correction="none"), dict(correction="epsilon", epsilon=1e-2), dict(q_estimate="baseline"),
                                dict(correction="one_step_is", reward_transform="clip"), dict(reward_transform="asymmetric")])
def test_variants(kw):
    for T, B in ((50, 7), (3000, 2)):
        x = _batch(5, T, B, lengths=_ragged(T, B))
        out = vt.vtrace_log_prob_loss_grad(**_dev(x), **PLAIN, **kw, with_vs=True, with_pg_advantages=True)
        _check(x, out, PLAIN, **kw)


def test_against_the_calls_on_logits():
    """The same batch through vtrace_loss_grad: its V-trace outputs to its own tolerance."""
    T, B, A = 60, 40, 9
    g = torch.Generator(device="cuda").manual_seed(2)
    z, y = (torch.randn((T, B, A), generator=g, device="cuda") for _ in range(2))
    act = torch.randint(0, A, (T, B), generator=g, device="cuda").int()
    x = _dev(_batch(3, T, B))
    rest = [x[k] for k in ("rewards", "discounts", "values", "bootstrap_value")]
    full = vt.vtrace_loss_grad(z, y, act, *rest, with_vs=True, with_pg_advantages=True)
    pick = lambda q: torch.log_softmax(q.double(), -1).gather(-1, act.long().unsqueeze(-1)).squeeze(-1).float()  # noqa: E731
    lz = torch.log_softmax(z.double(), -1)
    ent = -(lz.exp() * lz).sum(-1).float()
    out = vt.vtrace_log_prob_loss_grad(pick(z), pick(y), ent, *rest, with_vs=True, with_pg_advantages=True)
    for a, b in ((out.vs, full.vs), (out.pg_advantages, full.pg_advantages), (out.d_values, full.d_values)):
        assert ((a - b).abs() <= 1e-5 + 1e-4 * b.abs()).all()
    assert ((out.losses - full.losses).abs() <= 1e-3 + 1e-4 * full.losses.abs()).all()


def test_nan_reaches_earlier_steps_of_its_lane_alone():
    x = _batch(6, 3000, 3)
    d = _dev(x)
    d["rewards"][1500, 1] = float("nan")
    out = vt.vtrace_log_prob_loss_grad(**d, **PLAIN, with_vs=True)
    bad = torch.isnan(out.vs).cpu()
    cut = int(np.nonzero(x["discounts"][:1501, 1] == 0)[0][-1]) if (x["discounts"][:1501, 1] == 0).any() else -1
    assert bad[max(cut, 0):1501, 1].all() and not bad[1501:].any() and not bad[:, [0, 2]].any()
    assert torch.isnan(out.losses[0])


def test_infinite_truncation_and_masked_behaviour():
    x = _batch(7, 40, 3)
    s = dict(PLAIN, rho_bar=math.inf, c_bar=math.inf)
    out = vt.vtrace_log_prob_loss_grad(**_dev(x), **s, with_vs=True)
    o = ot.log_prob_loss_and_grads(**x, **s)
    # products of up to 40 ratios, each within 6e-11 of itself
    assert (np.abs(out.vs.cpu().double().numpy() - o.vs) <= U * np.abs(o.vs) + 1e-8 * (1 + np.abs(o.vs).max())).all()


def test_streams_and_refusals():
    x = _dev(_batch(8, 300, 9))
    base = vt.vtrace_log_prob_loss_grad(**x)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    o = vt.vtrace_log_prob_loss_grad(**x, stream=s)
    s.synchronize()
    assert torch.equal(base.losses, o.losses) and torch.equal(base.d_log_probs, o.d_log_probs)
    with pytest.raises(TypeError):
        vt.vtrace_log_prob_loss_grad(**dict(x, rewards=x["rewards"].double()))
    with pytest.raises(TypeError):
        vt.vtrace_log_prob_loss_grad(**dict(x, lengths=torch.full((9,), 3, device="cuda")))
    with pytest.raises(ValueError, match="shape"):
        vt.vtrace_log_prob_loss_grad(**dict(x, bootstrap_value=x["bootstrap_value"][:8].contiguous()))
    with pytest.raises(ValueError, match="contiguous"):
        vt.vtrace_log_prob_loss_grad(**{k: v.t().contiguous().t() if v is not None and v.dim() == 2 else v for k, v in x.items()})
    with pytest.raises(vt.VtraceError, match="PARAM"):
        vt.vtrace_log_prob_loss_grad(**x, lam=2.0)
    with pytest.raises(vt.VtraceError, match="WORKSPACE"):
        vt.vtrace_log_prob_loss_grad(**x, workspace=vt.LogProbWorkspace(1, 1))


# Clipping: squares and sums float64, the norm one rounding; the factor one rounding, its
# product another, bfloat16 outputs 2^-8.
def _grads(seed, sizes, dtypes, shift=0, scale=1.0):
    g = torch.Generator(device="cuda").manual_seed(seed)
    out = []
    for i, (n, t) in enumerate(zip(sizes, dtypes)):
        whole = (torch.randn(n + 8, generator=g, device="cuda") * scale).to(t)
        k = (i * shift) % 8
        out.append(whole[k:k + n])
    return out


def _check_clip(grads, max_norm, norm, outs):
    ref_norm = math.sqrt(sum(float((g.double() ** 2).sum()) for g in grads))
    assert abs(float(norm) - ref_norm) <= U * ref_norm * 1.01
    factor = _f32(max_norm) / max(ref_norm, _f32(max_norm)) if ref_norm > 0 else 1.0
    for g, o in zip(grads, outs):
        ref = g.double() * factor
        tol = (2.1 * U + (2.0 ** -8 if g.dtype == torch.bfloat16 else 0.0)) * ref.abs() + 1e-38
        assert ((o.double() - ref).abs() <= tol).all()
        if factor == 1.0:
            assert torch.equal(o, g)


F, H = torch.float32, torch.bfloat16
CLIP = [([1], [F]), ([1], [H]), ([5, 0, 3], [F, H, H]), ([16384, 16385, 16383, 1], [F, H, F, H]), ([100003, 7, 65536], [H, F, H]),
        ([257 + i for i in range(250)], [(F, H)[i % 3 == 0] for i in range(250)]), ([3000001, 1000], [H, F])]


@pytest.mark.parametrize("shift", [0, 1, 3])
@pytest.mark.parametrize("sizes,dtypes", CLIP)
def test_clip(sizes, dtypes, shift):
    ws = vt.ClipWorkspace()
    ws.tensor[256 + 4096:].fill_(0xFF)
    grads = _grads(len(sizes), sizes, dtypes, shift)
    for max_norm in (0.25, 1e6):
        outs = _grads(9, sizes, dtypes, shift if max_norm < 1 else 0)  # alike and other alignments
        norm = vt.vtrace_clip_grad_norm(grads, max_norm, out=outs, workspace=ws)
        _check_clip(grads, max_norm, norm, outs)
        mine = [g.clone() for g in grads]
        mine = [torch.cat([m[:0], m]) for m in mine]
        same = vt.vtrace_clip_grad_norm(mine, max_norm, workspace=ws)
        assert torch.equal(same, norm)
        _check_clip(grads, max_norm, same, mine)
    alone = vt.vtrace_clip_grad_norm(grads, None, workspace=ws)
    assert torch.equal(alone, norm)


def test_clip_in_place_of_views():
    """Pieces of one buffer, side by side, at every alignment."""
    whole = torch.randn(20000, device="cuda")
    keep = whole.clone()
    cuts = [0, 1, 8, 9, 4000, 4003, 19990, 20000]
    views = [whole[a:b] for a, b in zip(cuts, cuts[1:])]
    norm = vt.vtrace_clip_grad_norm(views[:-1], 2.0)
    _check_clip([keep[:19990]], 2.0, norm, [whole[:19990]])
    assert torch.equal(whole[19990:], keep[19990:])


def test_clip_extremes():
    big, tiny = torch.full((1000,), 1e30, device="cuda"), torch.full((1000,), 1e-30, device="cuda")
    for g in (big, tiny, big.bfloat16(), tiny.bfloat16()):
        _check_clip([g], 1.0, vt.vtrace_clip_grad_norm([g], 1.0, out=[o := torch.empty_like(g)]), [o])
    zero = torch.zeros(10, device="cuda")
    assert float(vt.vtrace_clip_grad_norm([zero], 0.0)) == 0.0 and not zero.any()
    x = torch.ones(10, device="cuda")
    assert float(vt.vtrace_clip_grad_norm([x], 0.0)) == pytest.approx(10 ** 0.5) and not x.any()
    x = torch.ones(10, device="cuda")
    vt.vtrace_clip_grad_norm([x], math.inf)
    assert (x == 1).all()
    x = torch.tensor([1.0, math.inf, -2.0], device="cuda")
    assert math.isinf(float(vt.vtrace_clip_grad_norm([x], 1.0)))
    assert x[0] == 0 and torch.isnan(x[1]) and x[2] == 0
    x, y = torch.tensor([1.0, math.nan], device="cuda"), torch.ones(3, device="cuda").bfloat16()
    assert math.isnan(float(vt.vtrace_clip_grad_norm([x, y], 1.0))) and torch.isnan(x).all() and torch.isnan(y).all()
    assert float(vt.vtrace_clip_grad_norm([torch.empty(0, device="cuda")], 1.0)) == 0.0


def test_clip_refusals_and_streams():
    g = torch.ones(100, device="cuda")
    with pytest.raises(vt.VtraceError, match="PARAM"):
        vt.vtrace_clip_grad_norm([g, g], 1.0)
    with pytest.raises(vt.VtraceError, match="PARAM"):
        vt.vtrace_clip_grad_norm([g[:60], g[50:]], 1.0)
    with pytest.raises(vt.VtraceError, match="PARAM"):
        vt.vtrace_clip_grad_norm([g[:50]], 1.0, out=[g[10:60]])
    assert float(vt.vtrace_clip_grad_norm([g, g], None)) == pytest.approx(200 ** 0.5)
    with pytest.raises(vt.VtraceError, match="PARAM"):
        vt.vtrace_clip_grad_norm([g], -1.0)
    with pytest.raises(ValueError, match="contiguous"):
        vt.vtrace_clip_grad_norm([g[::2]], 1.0)
    with pytest.raises(TypeError):
        vt.vtrace_clip_grad_norm([g.half()], 1.0)
    with pytest.raises(TypeError):
        vt.vtrace_clip_grad_norm([g], 1.0, out=[g.bfloat16()])
    assert (g == 1).all()
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    vt.vtrace_clip_grad_norm([g], 1.0, stream=s)
    s.synchronize()
    assert ((g - 0.1).abs() <= 0.1 * 2.1 * U).all()


def test_a_learner_step_as_a_whole():
    """Hidden states to clipped gradients, against the oracles one after the other.

    The chain's only inexact hand-overs are float32 log-probabilities (about 1e-6), so each
    gradient is within 1e-4 of its largest element."""
    T, B, H, V = 40, 6, 64, 800
    r = np.random.default_rng(4)
    g = torch.Generator().manual_seed(4)
    hidden = torch.randn(T, B, H, generator=g).bfloat16()
    weight = (torch.randn(V, H, generator=g) * 0.25).bfloat16()
    lengths = torch.tensor([40, 3, 0, 39, 21, 40], dtype=torch.int32)
    tokens = torch.randint(0, V, (T, B), generator=g).int()
    tokens[torch.arange(T).unsqueeze(1) >= lengths] = vt.NO_TOKEN
    x = _batch(5, T, B)
    x["lengths"] = lengths.numpy()

    ref = ot.vocab_log_probs(hidden.double().numpy().reshape(-1, H), weight.double().numpy(), None, tokens.numpy().reshape(-1))
    x["target_log_probs"], x["entropy"] = ref.log_probs.reshape(T, B), ref.entropy.reshape(T, B)
    x["behaviour_log_probs"] = np.minimum(x["target_log_probs"] + 0.3 * r.normal(size=(T, B)), 0).astype(np.float32)
    lo = ot.log_prob_loss_and_grads(**x, **{k: _f32(v) for k, v in PLAIN.items()})
    go = ot.vocab_grad(hidden.double().numpy().reshape(-1, H), weight.double().numpy(), None, tokens.numpy().reshape(-1),
                       lo.d_log_probs.reshape(-1), lo.d_entropy.reshape(-1))
    norm, clipped = ot.clip_grad_norm([go.d_hidden, go.d_weight], 0.5)

    d = _dev({k: v for k, v in x.items() if k not in ("target_log_probs", "entropy")})
    hd, wd, td = hidden.cuda(), weight.cuda(), tokens.cuda()
    f = vt.vtrace_vocab_log_probs(hd, wd, None, td)
    loss = vt.vtrace_log_prob_loss_grad(f.log_probs, d.pop("behaviour_log_probs"), f.entropy, **d, **PLAIN)
    grad = vt.vtrace_vocab_grad(hd, wd, None, td, f.log_sums, f.entropy, loss.d_log_probs, loss.d_entropy)
    got = vt.vtrace_clip_grad_norm([grad.d_hidden, grad.d_weight], 0.5)
    assert np.abs(loss.losses.cpu().double().numpy() - lo.losses).max() <= 1e-4 * np.abs(lo.losses).max()
    assert abs(float(got) - norm) <= 1e-4 * norm
    for a, b in zip((grad.d_hidden, grad.d_weight), clipped):
        assert np.abs(a.cpu().double().numpy().reshape(b.shape) - b).max() <= 1e-4 * np.abs(b).max()
