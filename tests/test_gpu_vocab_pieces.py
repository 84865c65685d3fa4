"""Gradients of a layer with a bias whose G takes several pieces of the vocabulary: what
starts, sums and ends a piece behind the first.  The reference is the same formulas in float64
on the GPU, the bounds those of the gradients' other tests."""

import math

import pytest
import torch

import paper_1802_01561_amd as vt
from test_gpu_vocab import HALF_BF16, U, _batch, _gpu

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("bias", [True, False])
@pytest.mark.parametrize("T,B,H,V", [(1030, 2, 64, 60007), (150, 1, 40, 600001)])
def test_several_pieces(T, B, H, V, bias, dtype):
    x, w, b, tokens, d_lp, d_h = _batch(V, T, B, H, V, bias=bias, none=0.1)
    ruled_out = torch.zeros(V, dtype=torch.bool)
    if bias:  # in the first piece, in the last, and across the vocabulary
        ruled_out[:100], ruled_out[-70:], ruled_out[::1001] = True, True, True
        b[ruled_out] = -math.inf
        tokens = torch.where(ruled_out[tokens.long().clamp(min=0)] & (tokens >= 0), 101, tokens).int()
        tokens[1, 0] = V - 71
    x, w, b, tokens, d_lp, d_h, ruled_out = _gpu(x, w, b, tokens, d_lp, d_h, ruled_out)
    row_bytes = -(-T * B // 256) * 256 * (4 if dtype == torch.float32 else 2)
    ws = vt.VocabWorkspace(T, B, V, H, grad_dtype=dtype)
    assert row_bytes * V > ws.nbytes  # a G of all tokens does not fit
    fwd = vt.vtrace_vocab_log_probs(x, w, b, tokens)
    out = vt.vtrace_vocab_grad(x, w, b, tokens, fwd.log_sums, fwd.entropy, d_lp, d_h, grad_dtype=dtype, workspace=ws)

    use = (tokens.view(-1) >= 0).unsqueeze(1)
    X, W = x.view(-1, H).double() * use, w.double()
    z, m = X @ W.t(), X.abs() @ W.abs().t()
    if bias:
        z, m = z + b.double(), m + torch.where(ruled_out, 0.0, b).double().abs()
    tau = ((H ** 0.5 + 8.0) * U * m).amax(1, keepdim=True)
    lse = torch.logsumexp(z, 1, keepdim=True)
    p = (z - lse).exp()
    lp = torch.where(p > 0, z - lse, 0.0)
    e = -(p * lp).sum(1, keepdim=True)
    del z, m
    g, h = (t.view(-1, 1).double() * use for t in (d_lp, d_h))
    G = (-g * p - h * p * (lp + e)).scatter_add_(1, tokens.view(-1, 1).clamp(min=0).long(), g)
    # the kernel's own log-sums and entropies: their errors enter as p's relative one
    rel = 2.0 * tau + U * 128.0 + U * (lp.abs() + 8.0)
    dG = p * (g.abs() + h.abs() * (lp.abs() + e + 1.0)) * rel * 2.0 + U * G.abs()
    mag = G.abs() + dG
    del rel, p, lp
    operand, stored = (HALF_BF16 ** 2, U) if dtype == torch.float32 else (HALF_BF16, HALF_BF16)

    def within(got, ref, sum_of, k):
        bound = (sum_of(dG) + (operand + (k ** 0.5 + 8.0) * U) * sum_of(mag)) * (1.0 + stored) + stored * ref.abs() + 1e-37
        assert ((got.double().view(ref.shape) - ref).abs() <= bound).all()

    within(out.d_hidden, G @ W, lambda t: t @ W.abs(), V)
    within(out.d_weight, G.t().contiguous() @ X, lambda t: t.t().contiguous() @ X.abs(), T * B)
    assert (out.d_bias is not None) == bias
    if bias:
        ref = G.sum(0)
        assert ((out.d_bias.double() - ref).abs() <= dG.sum(0) + 80.0 * U * mag.sum(0) + U * ref.abs() + 1e-37).all()
        assert not out.d_weight[ruled_out].any() and not out.d_bias[ruled_out].any()
    assert not out.d_hidden.view(-1, H)[~use.view(-1)].any()
