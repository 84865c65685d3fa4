"""The token-policy oracle against definitions it does not share: differences of the
losses, the [T,B,A] oracle on small action sets, and exact sums."""

import math

import numpy as np
import pytest

import oracle
from oracle import tokens as ot


def _layer(seed, N=7, H=5, V=11, bias=True):
    r = np.random.default_rng(seed)
    x, w = r.normal(size=(N, H)), r.normal(size=(V, H))
    b = r.normal(size=V) if bias else None
    tokens = r.integers(0, V, N)
    tokens[2] = ot.NO_TOKEN
    return x, w, b, tokens, r.normal(size=N), r.normal(size=N)


def _objective(x, w, b, tokens, g, h):
    o = ot.vocab_log_probs(x, w, b, tokens)
    return np.sum(g * o.log_probs) + np.sum(h * o.entropy)


@pytest.mark.parametrize("bias", [False, True])
def test_vocab_grad_is_the_difference_quotient(bias):
    x, w, b, tokens, g, h = _layer(3, bias=bias)
    o = ot.vocab_grad(x, w, b, tokens, g, h)
    r = np.random.default_rng(4)
    eps = 1e-6
    for name, arr, grad in [("hidden", x, o.d_hidden), ("weight", w, o.d_weight)] + ([("bias", b, o.d_bias)] if bias else []):
        for _ in range(6):
            d = r.normal(size=arr.shape)
            args = dict(hidden=x, weight=w, bias=b)
            up, down = dict(args), dict(args)
            up[name], down[name] = arr + eps * d, arr - eps * d
            q = (_objective(up["hidden"], up["weight"], up["bias"], tokens, g, h)
                 - _objective(down["hidden"], down["weight"], down["bias"], tokens, g, h)) / (2 * eps)
            assert q == pytest.approx(np.sum(grad * d), rel=1e-6, abs=1e-7), name


def test_log_probs_are_the_small_action_sets():
    x, w, b, tokens, _, _ = _layer(5)
    o = ot.vocab_log_probs(x, w, b, tokens)
    log_pi = oracle.log_softmax((x @ w.T + b)[None])[0]
    use = tokens >= 0
    assert np.allclose(o.log_probs[use], log_pi[use, tokens[use]], rtol=1e-13, atol=1e-13)
    assert np.allclose(o.entropy[use], -(np.exp(log_pi) * log_pi).sum(-1)[use], rtol=1e-13)
    assert o.log_probs[2] == 0.0 and o.log_sums[2] == 0.0 and o.entropy[2] == 0.0


def test_ruled_out_tokens_are_as_if_absent():
    x, w, b, tokens, g, h = _layer(6)
    tokens = np.where(tokens >= 9, 0, tokens)
    masked = b.copy()
    masked[9:] = -np.inf
    a, c = ot.vocab_grad(x, w, masked, tokens, g, h), ot.vocab_grad(x, w[:9], b[:9], tokens, g, h)
    assert np.allclose(a.d_hidden, c.d_hidden, rtol=1e-12, atol=1e-12)
    assert np.allclose(a.d_weight[:9], c.d_weight, rtol=1e-12, atol=1e-12) and not a.d_weight[9:].any()


@pytest.mark.parametrize("kw", [{}, dict(correction="none"), dict(correction="epsilon", epsilon=1e-2),
                                dict(correction="one_step_is", q_estimate="baseline"), dict(reward_transform="asymmetric")])
def test_loss_from_log_probs_is_the_loss_from_logits(kw):
    r = np.random.default_rng(8)
    T, B, A = 6, 4, 5
    z, y = r.normal(size=(T, B, A)), r.normal(size=(T, B, A))
    act = r.integers(0, A, (T, B))
    rew, disc, val, boot = r.normal(size=(T, B)), 0.9 * (r.random((T, B)) > 0.2), r.normal(size=(T, B)), r.normal(size=B)
    scal = dict(rho_bar=1.5, c_bar=0.8, lam=0.9, baseline_cost=0.4, entropy_cost=0.03)
    full = oracle.loss_and_grads(z, y, act, rew, disc, val, boot, **scal, **kw)
    pick = lambda q: np.take_along_axis(oracle.log_softmax(q), act[..., None], -1)[..., 0]  # noqa: E731
    log_pi = oracle.log_softmax(z)
    ent = -(np.exp(log_pi) * log_pi).sum(-1)
    o = ot.log_prob_loss_and_grads(pick(z), pick(y), ent, rew, disc, val, boot, **scal, **kw)
    assert np.allclose(o.losses, full.losses, rtol=1e-12)
    assert np.allclose(o.vs, full.vs, rtol=1e-12) and np.allclose(o.pg_advantages, full.pg_advantages, rtol=1e-12)
    assert np.allclose(o.d_values, full.d_values, rtol=1e-12, atol=1e-14)
    # through the softmax: d_logits = d_log_probs (1[a] - pi) + d_entropy dH/dz
    onehot = np.eye(A)[act]
    pi = np.exp(log_pi)
    dz = o.d_log_probs[..., None] * (onehot - pi) - o.d_entropy[..., None] * pi * (log_pi + ent[..., None])
    assert np.allclose(dz, full.d_logits, rtol=1e-12, atol=1e-14)


def test_lengths_cut_the_lanes():
    r = np.random.default_rng(9)
    T, B = 5, 4
    a = [r.normal(size=(T, B)) for _ in range(6)]
    boot, n = r.normal(size=B), np.array([0, 2, 5, 9])
    o = ot.log_prob_loss_and_grads(*a, boot, n)
    for b in range(1, B):
        m = min(int(n[b]), T)
        one = ot.log_prob_loss_and_grads(*[x[:m, b:b + 1] for x in a], boot[b:b + 1])
        assert np.allclose(o.vs[:m, b], one.vs[:, 0], rtol=1e-13) and not o.vs[m:, b].any()
        assert np.allclose(o.d_log_probs[:m, b], one.d_log_probs[:, 0], rtol=1e-13) and not o.d_log_probs[m:, b].any()
    assert not o.d_values[:, 0].any()


def test_clip():
    g = [np.array([3.0, 0.0]), np.array([[4.0]])]
    norm, c = ot.clip_grad_norm(g, 1.0)
    assert norm == 5.0 and np.allclose(c[0], [0.6, 0.0]) and np.allclose(c[1], [[0.8]])
    assert all((x == y).all() for x, y in zip(ot.clip_grad_norm(g, 5.0)[1], g))
    assert ot.clip_grad_norm([np.zeros(3)], 0.0)[0] == 0.0
    norm, c = ot.clip_grad_norm([np.array([np.inf, 1.0])], 1.0)
    assert norm == math.inf and np.isnan(c[0][0]) and c[0][1] == 0.0
    assert np.isnan(ot.clip_grad_norm([np.array([np.nan, 1.0])], 1.0)[1][0]).all()
