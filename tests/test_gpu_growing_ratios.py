"""Calls on logits whose importance ratios multiply to more than the largest double, while the
values they are multiplied with are 0: as the recursion, one step after the other."""

import math

import pytest
import torch

import paper_1802_01561_amd as vt

pytestmark = pytest.mark.gpu


def _batch(T, B, A, log_ratio):
    """A reward in the first step alone, so that every value behind them is 0; probability of
    the action 1 - (A - 1) e^-60 under pi, about e^-log_ratio under mu."""
    z = torch.zeros(T, B, A)
    z[..., 0] = 60.0
    y = torch.zeros(T, B, A)
    y[..., 0] = -log_ratio
    r = torch.zeros(T, B)
    r[0] = 1.0
    return [t.cuda() for t in (z, y, torch.zeros(T, B, dtype=torch.int32), r, torch.ones(T, B), torch.zeros(T, B), torch.zeros(B))]


@pytest.mark.parametrize("kernel", ["auto", "wide", "tiled", "tiled_short", "lane_serial"])
@pytest.mark.parametrize("log_ratio", [12.0, 50.0, 85.0])
@pytest.mark.parametrize("T,B,A", [(256, 2, 9), (200, 3, 18), (128, 2, 4), (64, 5, 9), (300, 40, 6), (256, 2, 48), (100, 4, 200)])
def test_loss_and_targets(T, B, A, log_ratio, kernel, monkeypatch):
    monkeypatch.delenv("VTRACE_KERNEL", raising=False)
    if kernel != "auto":
        monkeypatch.setenv("VTRACE_KERNEL", kernel)
    x = _batch(T, B, A, log_ratio)
    out = vt.vtrace_loss_grad(*x, 1.0, math.inf, with_vs=True, with_pg_advantages=True, with_lane_losses=True)
    vs, adv = vt.vtrace_targets(*x, 1.0, math.inf)
    # v_0 = V + rho (1 + 0), and 0 behind it
    for got in (out.vs, vs, out.pg_advantages, adv):
        assert (got[0] == 1.0).all() and not got[1:].any()
    for t in (*out[:6], adv):
        assert not torch.isnan(t).any()


@pytest.mark.parametrize("T,B,log_ratio", [(100, 4, 85.0), (16, 40, 85.0), (300, 3, 50.0), (64, 2000, 85.0)])
def test_output_layer(T, B, log_ratio):
    H, A = 64, 9
    hidden = torch.ones(T, B, H, device="cuda", dtype=torch.bfloat16)
    w = torch.zeros(H, A + 1, device="cuda", dtype=torch.bfloat16)
    w[0, 0] = 60.0
    x = _batch(T, B, A, log_ratio)
    out = vt.vtrace_head_loss_grad(hidden, w, torch.zeros(A + 1, device="cuda"), x[1], x[2], x[3], x[4], x[6], 1.0, math.inf,
                                   with_vs=True, with_pg_advantages=True)
    assert not any(torch.isnan(t).any() for t in out if t is not None)
    assert (out.vs[0] == 1.0).all() and not out.vs[1:].any()
