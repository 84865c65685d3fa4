"""The token-policy operators where the definition is finite and a careless form of it is not."""

import math

import numpy as np
import pytest

import paper_1802_01561_amd as vt
from oracle import tokens as ot
from test_gpu_log_prob_loss import PLAIN, _dev
from test_gpu_vocab import U

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
