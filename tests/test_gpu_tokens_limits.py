"""The token-policy operators at the largest sizes that their header allows, and gradients of
policies that are nearly certain."""

import math

import numpy as np
import pytest
import torch

import paper_1802_01561_amd as vt
from oracle import tokens as ot
from test_gpu_vocab import HALF_BF16, U, _batch, _check_grad, _check_log_probs, _flat, _gpu, _grad_inputs

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("N,V", [(1, 300), (40, 77), (150, 300)])
def test_largest_hidden_size(N, V, dtype):
    x, w, b, tokens, d_lp, d_h = _batch(N, N, 1, 32768, V, bias=True, none=0.1)
    ls, ent = _grad_inputs(x, w, b, tokens)
    _check_log_probs(x, w, b, tokens, vt.vtrace_vocab_log_probs(*_gpu(x, w, b, tokens)))
    out = vt.vtrace_vocab_grad(*_gpu(x, w, b, tokens, ls, ent, d_lp, d_h), grad_dtype=dtype)
    _check_grad(x, w, b, tokens, d_lp, d_h, out, dtype)


@pytest.mark.parametrize("N", [2, 50, 130])
def test_largest_vocabulary(N):
    """2^24 tokens, the last ones taken."""
    H, V = 8, 1 << 24
    g = torch.Generator(device="cuda").manual_seed(N)
    w = torch.randn((V, H), generator=g, device="cuda").bfloat16()
    x = torch.randn((N, 1, H), generator=g, device="cuda").bfloat16()
    tokens = (V - 1 - torch.arange(N, device="cuda").view(N, 1) * 3).int()
    out = vt.vtrace_vocab_log_probs(x, w, None, tokens)
    X = x.view(N, H).double()
    parts = [X @ w[at:at + (1 << 20)].double().t() for at in range(0, V, 1 << 20)]
    lse = torch.logsumexp(torch.stack([torch.logsumexp(z, 1) for z in parts]), 0)
    entropy = lse - sum((torch.exp(z - lse.unsqueeze(1)) * z).sum(1) for z in parts)
    taken = torch.cat(parts[-1:], 1).gather(1, (tokens.long() - (V - (1 << 20))))
    del parts
    # as in _check_log_probs, the magnitudes of the products bounded by the largest
    tau = (H ** 0.5 + 8.0) * U * (X.abs().sum(1) * w.abs().max().double())
    bound = tau + U * (64.0 + lse.abs())
    assert ((out.log_sums.view(-1).double() - lse).abs() <= bound).all()
    assert ((out.log_probs.view(-1).double() - (taken.view(-1) - lse)).abs() <= 2 * bound + U * taken.view(-1).abs()).all()
    # spread: sum p |log p + H| is at most a few units for these logits (deviation sqrt 8)
    assert ((out.entropy.view(-1).double() - entropy).abs() <= (2 * tau + 64 * U) * 8.0 + U * (entropy + 64)).all()
    d = torch.ones((N, 1), device="cuda")
    grad = vt.vtrace_vocab_grad(x, w, None, tokens, out.log_sums, None, d, grad_dtype=torch.bfloat16)
    rows = torch.tensor([0, 1, 262143, 262144, V // 2, V - 2, V - 1, *tokens.view(-1)[:8].tolist()], device="cuda")
    z = X @ w[rows].double().t()
    G = (tokens.view(-1, 1) == rows).double() - torch.exp(z - lse.unsqueeze(1))
    ref = G.t() @ X
    bound = (HALF_BF16 + 1e-4) * (G.abs().t() @ X.abs()) + HALF_BF16 * ref.abs() + 1e-37
    assert ((grad.d_weight[rows].double() - ref).abs() <= bound * 1.01).all()


def test_most_hidden_elements():
    """N H just below 2^30: the last rows of the hidden states and of their gradients."""
    N, H, V = 131071, 8184, 70
    g = torch.Generator(device="cuda").manual_seed(7)
    x = torch.randn((N, 1, H), generator=g, device="cuda", dtype=torch.bfloat16)
    w = (torch.randn((V, H), generator=g, device="cuda") * (2.0 / H ** 0.5)).bfloat16()
    tokens = torch.randint(0, V, (N, 1), generator=g, device="cuda").int()
    d_lp = torch.randn((N, 1), generator=g, device="cuda")
    out = vt.vtrace_vocab_log_probs(x, w, None, tokens)
    grad = vt.vtrace_vocab_grad(x, w, None, tokens, out.log_sums, None, d_lp)
    W = w.double()
    tail = slice(N - 300, N)
    X = x.view(N, H)[tail].double()
    z = X @ W.t()
    lse = torch.logsumexp(z, 1)
    tau = ((H ** 0.5 + 8.0) * U * (X.abs() @ W.abs().t())).amax(1)
    assert ((out.log_sums.view(-1)[tail].double() - lse).abs() <= tau + U * (64.0 + lse.abs())).all()
    G = torch.zeros((N, V), dtype=torch.float64, device="cuda")
    for at in range(0, N, 1 << 14):  # of all steps, from the kernel's own log-sums
        part = slice(at, at + (1 << 14))
        p = torch.exp(x.view(N, H)[part].double() @ W.t() - out.log_sums.view(-1, 1)[part].double())
        G[part] = -p * d_lp[part].double()
    G.scatter_add_(1, tokens.long(), d_lp.double())
    # G's terms within p (2 tau + 128 u) and 2^-16; sums of V and N terms
    dG = G.abs() * U + d_lp.double().abs() * (2.0 * tau.max() + 128.0 * U)
    operand = HALF_BF16 ** 2
    ref = G[tail] @ W
    bound = dG[tail] @ W.abs() + (operand + (V ** 0.5 + 8) * U) * (G[tail].abs() @ W.abs()) + U * ref.abs() + 1e-37
    assert ((grad.d_hidden.view(N, H)[tail].double() - ref).abs() <= bound).all()
    ref, terms = torch.zeros((V, H), dtype=torch.float64, device="cuda"), torch.zeros((V, H), dtype=torch.float64, device="cuda")
    for at in range(0, N, 1 << 14):
        part = slice(at, at + (1 << 14))
        X = x.view(N, H)[part].double()
        ref += G[part].t().contiguous() @ X
        terms += (dG[part] + (operand + (N ** 0.5 + 8) * U) * G[part].abs()).t().contiguous() @ X.abs()
    assert ((grad.d_weight.double() - ref).abs() <= terms + U * ref.abs()).all()


def test_clip_beyond_32_bits():
    """A gradient of more than 2^32 elements, at an odd place of its buffer, clipped in place."""
    n = (1 << 32) + 12345
    whole = torch.full((n + 3,), 2.0 ** -7, device="cuda", dtype=torch.bfloat16)
    g = whole[1:n + 1]
    g[-1] = 3.0
    norm = vt.vtrace_clip_grad_norm([g, torch.zeros(5, device="cuda")], 256.0)
    ref = math.sqrt((n - 1) * 2.0 ** -14 + 9.0)
    assert abs(float(norm) - ref) <= 1.01 * U * ref
    factor = 256.0 / ref
    for part in (g[:1000], g[n // 2:n // 2 + 1000], g[(1 << 31) - 5:(1 << 31) + 5], g[-1001:-1]):
        assert ((part.double() - factor * 2.0 ** -7).abs() <= 1.01 * HALF_BF16 * factor * 2.0 ** -7).all()
    assert abs(float(g[-1]) - 3.0 * factor) <= 1.01 * HALF_BF16 * 3.0 * factor
    assert float(whole[0]) == float(whole[-1]) == float(whole[-2]) == 2.0 ** -7
    assert not (g[:: 1 << 20] == 2.0 ** -7).any()


def _flushed_back(x, w, b, tokens, d_lp, d_h, out):
    """The gradients with what subnormal numbers may have lost put back.  The matrix cores and the
    exponential take a number below 2^-126 as 0: each of G's two parts in a product is off by up to
    2^-126 beside its rounding, and so is a partial sum, so that a sum of products G y is off by
    up to 2^-126 sum (2 |y| + 1)."""
    f = _flat(x, w, b, tokens)
    use = (f[3] != vt.NO_TOKEN)[:, None]
    o = ot.vocab_grad(*f, *(t.double().numpy().reshape(-1) for t in (d_lp, d_h)))

    def back(got, ref, operand):
        lost = 2.0 ** -126 * (2.0 * np.abs(operand) + 1.0).sum(0)
        now = got.double().cpu().numpy().reshape(ref.shape)
        return torch.from_numpy(now + np.clip(ref - now, -lost, lost)).view(got.shape).cuda()

    return vt.VocabGrad(back(out.d_hidden, o.d_hidden, f[1]),
                        back(out.d_weight, o.d_weight, np.where(use, f[0], 0.0)), out.d_bias)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("scale", [10.0, 40.0])
@pytest.mark.parametrize("T,B", [(1, 3), (30, 2), (150, 2)])
def test_gradients_of_peaked_policies(T, B, scale, dtype):
    """Most probabilities near 0 or 1, the taken token among the likely ones and among the others."""
    x, w, b, tokens, d_lp, d_h = _batch(3, T, B, 64, 700, bias=True, none=0.1, scale=scale)
    top = (x.double() @ w.double().t() + b.double()).argmax(-1).int()
    tokens = ((torch.arange(T * B).view(T, B) % 3 > 0) & (tokens >= 0)).int() * (top - tokens) + tokens
    ls, ent = _grad_inputs(x, w, b, tokens)
    out = vt.vtrace_vocab_grad(*_gpu(x, w, b, tokens, ls, ent, d_lp, d_h), grad_dtype=dtype)
    assert out.d_hidden.dtype == out.d_weight.dtype == dtype
    _check_grad(x, w, b, tokens, d_lp, d_h, _flushed_back(x, w, b, tokens, d_lp, d_h, out), dtype)
