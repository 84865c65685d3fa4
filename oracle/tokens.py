"""fp64 oracle of the token-policy operators: a vocabulary layer's log-probabilities and
their gradients, V-trace losses from log-probabilities of lanes of different lengths, and
clipping by the global norm.  NumPy, from the definitions, logits and all."""

from __future__ import annotations

from typing import NamedTuple, Optional

import numpy as np

from .definitions import pg_advantages, temporal_differences, transform_rewards, vtrace_targets_recursive

NO_TOKEN = -1


def _f64(x):
    return np.asarray(x, dtype=np.float64)


class VocabOut(NamedTuple):
    log_probs: np.ndarray  # [N]
    log_sums: np.ndarray
    entropy: np.ndarray
    log_pi: np.ndarray  # [N,V]


def vocab_log_probs(hidden, weight, bias, tokens) -> VocabOut:
    """Of steps [N,H] with tokens [N] (NO_TOKEN: zeros); a bias of -inf rules a token out."""
    tokens = np.asarray(tokens, dtype=np.int64)
    use = tokens != NO_TOKEN
    x = np.where(use[:, None], _f64(hidden), 0.0)
    z = x @ _f64(weight).T
    if bias is not None:
        z = z + _f64(bias)
    top = z.max(axis=1, keepdims=True)
    log_sums = top[:, 0] + np.log(np.exp(z - top).sum(axis=1))
    log_pi = z - log_sums[:, None]
    pi = np.exp(log_pi)
    entropy = -np.sum(np.where(pi > 0.0, pi * np.where(pi > 0.0, log_pi, 0.0), 0.0), axis=1)
    valid = (tokens >= 0) & (tokens < z.shape[1])
    lp = np.where(valid, log_pi[np.arange(len(tokens)), np.where(valid, tokens, 0)], np.nan)
    return VocabOut(np.where(use, lp, 0.0), np.where(use, log_sums, 0.0), np.where(use, entropy, 0.0), log_pi)


class VocabGradOut(NamedTuple):
    d_hidden: np.ndarray  # [N,H]
    d_weight: np.ndarray  # [V,H]
    d_bias: np.ndarray  # [V]
    g: np.ndarray  # [N,V]


def vocab_grad(hidden, weight, bias, tokens, d_log_probs, d_entropy=None) -> VocabGradOut:
    """Of sum_n d_log_probs log pi(a_n) + d_entropy H_n."""
    tokens = np.asarray(tokens, dtype=np.int64)
    use = tokens != NO_TOKEN
    x = np.where(use[:, None], _f64(hidden), 0.0)
    o = vocab_log_probs(hidden, weight, bias, tokens)
    pi = np.exp(o.log_pi)
    onehot = np.zeros_like(pi)
    onehot[np.arange(len(tokens)), np.where(use, tokens, 0)] = 1.0
    g = np.where(use, _f64(d_log_probs), 0.0)[:, None] * (onehot - pi)
    if d_entropy is not None:
        log_pi = np.where(pi > 0.0, o.log_pi, 0.0)
        g = g - np.where(use, _f64(d_entropy), 0.0)[:, None] * pi * (log_pi + o.entropy[:, None])
    g = np.where(use[:, None], g, 0.0)
    return VocabGradOut(g @ _f64(weight), g.T @ x, g.sum(axis=0), g)


class LogProbLossOut(NamedTuple):
    losses: np.ndarray  # [4]
    d_log_probs: np.ndarray  # [T,B]
    d_values: np.ndarray
    d_entropy: np.ndarray
    vs: np.ndarray
    pg_advantages: np.ndarray
    step_losses: np.ndarray  # [T,B,3]


def log_prob_loss_and_grads(target_log_probs, behaviour_log_probs, entropy, rewards, discounts, values, bootstrap_value,
                            lengths=None, rho_bar=1.0, c_bar=1.0, lam=1.0, baseline_cost=0.5, entropy_cost=0.01, *,
                            correction="vtrace", q_estimate="vtrace", epsilon=1e-6,
                            reward_transform: Optional[str] = None) -> LogProbLossOut:
    """Each lane on its own, its first ``lengths[b]`` steps alone; zeros behind them."""
    T, B = np.shape(target_log_probs)
    n = np.full(B, T) if lengths is None else np.clip(np.asarray(lengths, dtype=np.int64), 0, T)
    d_lp, d_v, d_h, vs, adv = (np.zeros((T, B)) for _ in range(5))
    step = np.zeros((T, B, 3))
    for b in range(B):
        m = int(n[b])
        if m == 0:
            continue
        lane = lambda x: _f64(x)[:m, b:b + 1]  # noqa: E731
        lp, r, g, v, boot = (lane(target_log_probs), transform_rewards(lane(rewards), reward_transform),
                             lane(discounts), lane(values), _f64(bootstrap_value)[b:b + 1])
        ratio = np.exp(lp - lane(behaviour_log_probs))
        rho, c = np.minimum(rho_bar, ratio), lam * np.minimum(c_bar, ratio)
        rho_v, c_v, rho_pg = rho, c, rho
        if correction != "vtrace":
            rho_v, c_v = np.ones_like(rho), lam * np.ones_like(rho)
            rho_pg = rho if correction == "one_step_is" else rho_v
        deltas = temporal_differences(rho_v, r, g, v, boot)
        target = vtrace_targets_recursive(v, boot, deltas, g, c_v)
        a = pg_advantages(rho_pg, r, g, v, target, boot, q_estimate)
        log_p, w = lp, np.ones_like(lp)
        if correction == "epsilon":
            log_p, w = np.log(np.exp(lp) + epsilon), np.exp(lp) / (np.exp(lp) + epsilon)
        vs[:m, b:b + 1], adv[:m, b:b + 1] = target, a
        d_lp[:m, b:b + 1] = -a * w
        d_v[:m, b:b + 1] = baseline_cost * (v - target)
        d_h[:m, b] = -entropy_cost
        step[:m, b, 0] = (-a * log_p)[:, 0]
        step[:m, b, 1] = (0.5 * baseline_cost * (target - v) ** 2)[:, 0]
        if entropy is not None:
            step[:m, b, 2] = -entropy_cost * lane(entropy)[:, 0]
    parts = step.sum(axis=(0, 1))
    return LogProbLossOut(np.concatenate([[parts.sum()], parts]), d_lp, d_v, d_h, vs, adv, step)


def clip_grad_norm(gradients, max_norm):
    """(norm, clipped gradients)."""
    norm = np.sqrt(sum(np.sum(_f64(g) ** 2) for g in gradients))
    with np.errstate(invalid="ignore"):
        return norm, [_f64(g) * (max_norm / np.maximum(norm, max_norm) if norm > 0.0 or np.isnan(norm) else 1.0)
                      for g in gradients]
