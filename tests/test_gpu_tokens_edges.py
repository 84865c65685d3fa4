"""The token-policy operators where the definition is finite and a careless form of it is not."""

import math

import numpy as np
import pytest
import torch

import paper_1802_01561_amd as vt
from oracle import tokens as ot
from test_gpu_log_prob_loss import PLAIN, _dev
from test_gpu_vocab import U, _batch, _check_grad, _check_log_probs, _gpu, _grad_inputs

pytestmark = pytest.mark.gpu


def _growing_lanes(T, B, log_ratio, ends):
    """Importance ratios above 1 throughout; rewards in the first two steps alone, so that every
    value behind them is 0 however large the product of the ratios is."""
    x = dict(target_log_probs=np.full((T, B), -0.5), behaviour_log_probs=np.full((T, B), -0.5 - log_ratio),
             entropy=np.ones((T, B)), rewards=np.zeros((T, B)), discounts=np.ones((T, B)), values=np.zeros((T, B)),
             bootstrap_value=np.zeros(B))
    x["rewards"][:2] = np.arange(1, 3)[:, None]
    if ends:
        x["discounts"][T // 2] = 0.0
    x = {k: np.ascontiguousarray(v, dtype=np.float32) for k, v in x.items()}
    return dict(x, lengths=np.arange(T, T - 7 * B, -7, dtype=np.int32))


@pytest.mark.parametrize("ends", [False, True])
@pytest.mark.parametrize("T,B", [(1000, 1), (1100, 3), (6000, 1), (12000, 5), (3000, 40)])
@pytest.mark.parametrize("c_bar,log_ratio", [(math.inf, 1.0), (2.0, 1.0), (math.inf, 30.0)])
def test_products_of_ratios_beyond_float64(T, B, c_bar, log_ratio, ends):
    """Thousands of steps' ratios multiply to more than the largest double; the recursion
    multiplies them with zeros one after the other."""
    x = _growing_lanes(T, B, log_ratio, ends)
    s = dict(PLAIN, c_bar=c_bar, rho_bar=1.0)
    out = vt.vtrace_log_prob_loss_grad(**_dev(x), **s, with_vs=True, with_pg_advantages=True)
    o = ot.log_prob_loss_and_grads(**x, **{k: float(np.float32(v)) for k, v in s.items()})
    for name in ("vs", "pg_advantages", "d_log_probs", "d_values", "losses"):
        got, ref = getattr(out, name).cpu().double().numpy(), getattr(o, name)
        # values of the first two steps: two ratios, each within 1e-9 of itself, and one rounding
        assert (np.abs(got - ref) <= (U + 1e-8) * np.abs(ref) + 1e-8 * (name == "losses") * T).all(), (name, got, ref)


@pytest.mark.parametrize("mask", [-1e9, -1e10, -1e15, -1e20, -1e30, -9e36])
@pytest.mark.parametrize("N,V", [(3, 3000), (20, 40000), (48, 30011), (100, 20000), (200, 3000), (700, 9000)])
def test_low_finite_biases_over_whole_pieces(N, V, mask):
    """A bias of -1e30 rules tokens out as well as -inf does, where a whole stretch of the
    vocabulary has it: beside allowed tokens its exponentials are 0."""
    H = 72
    x, w, b, tokens, d_lp, d_h = _batch(N + V, N, 1, H, V, bias=True, none=0.1)
    b[V // 3:] = mask
    b[:40] = mask
    ruled_out = b == b[0]
    tokens = torch.where(ruled_out[tokens.long().clamp(min=0)] & (tokens >= 0), 40 + tokens % (V // 3 - 40), tokens).int()
    b64 = torch.where(ruled_out, torch.tensor(-math.inf), b)
    args = _gpu(x, w, b, tokens)
    _check_log_probs(x, w, b64, tokens, vt.vtrace_vocab_log_probs(*args))
    plain = vt.vtrace_vocab_log_probs(*args, with_entropy=False)
    _check_log_probs(x, w, b64, tokens, plain)
    ls, ent = _grad_inputs(x, w, b64, tokens)
    out = vt.vtrace_vocab_grad(*args, *_gpu(ls, ent, d_lp, d_h))
    _check_grad(x, w, b64, tokens, d_lp, d_h, out, torch.float32)
    assert not out.d_weight[ruled_out.cuda()].any()


@pytest.mark.parametrize("offset", [-1e30, -1e10, 3e8, 1e30])
@pytest.mark.parametrize("N,V", [(3, 3000), (48, 30011), (100, 20000), (200, 3000)])
def test_a_large_bias_common_to_all_tokens(N, V, offset):
    """What is left of the logits beside it is float32's rounding of their sum: equal logits."""
    H = 72
    x, w, _, tokens, _, _ = _batch(N + V, N, 1, H, V)
    x[:] = 0
    out = vt.vtrace_vocab_log_probs(*_gpu(x, w, torch.full((V,), offset), tokens))
    # sums of equal terms: 64 roundings of the log-sum's argument, as in the other tests
    for got in (out.log_probs, -out.entropy):
        assert ((got.double() + math.log(V)).abs() <= U * (64.0 + 2.0 * math.log(V))).all()
    assert (out.log_sums.double() - np.float32(offset)).abs().max() <= 2.0 * U * abs(offset)


def test_clipped_into_an_iterator():
    """``out`` may be any iterable, by either way of marshalling."""
    g = [torch.ones(4, device="cuda"), torch.ones(12, device="cuda").bfloat16()]
    marked = torch.ones(0, device="cuda").as_subclass(type("Marked", (torch.Tensor,), {}))  # which native code declines
    for extra in ([], [marked]):
        for kw in (dict(workspace=vt.ClipWorkspace()), dict()):
            out = [torch.zeros_like(t) for t in g]
            norm = vt.vtrace_clip_grad_norm(iter([*g, *extra]), 1.0, out=(t for t in [*out, *extra]), **kw)
            assert float(norm) == 4.0 and all((t == 0.25).all() for t in out)


def test_wanted_outputs_by_truth():
    """with_vs = 1 asks for vs, whichever way the call is marshalled."""
    y = _dev(_growing_lanes(40, 3, 0.1, False))
    for kw in (dict(workspace=vt.LogProbWorkspace(40, 3)), dict()):
        out = vt.vtrace_log_prob_loss_grad(**y, with_vs=1, with_pg_advantages=np.bool_(True), **kw)
        assert out.vs is not None and out.pg_advantages is not None
        out = vt.vtrace_log_prob_loss_grad(**y, with_vs=0, with_pg_advantages=None, **kw)
        assert out.vs is None and out.pg_advantages is None
