"""npd_ce_fwd_bwd of up to 8 tokens (and the first sizes beyond) at widths and vocabularies where a warp goes through
several batches of k-steps and a block through several groups of vocabulary rows.  Against 64 bits on the GPU; tolerances as
derived in test_gpu_ce.py."""

import pytest
import torch

from paper_2605_05940_b200 import binding as B

from _device_reference import u

pytestmark = pytest.mark.gpu
DEV, BF16, F32 = "cuda", torch.bfloat16, torch.float32


def _head(d, V, pad=0):
    g = torch.Generator(device=DEV).manual_seed(d + V)
    buf = (torch.randn((V, d + pad), device=DEV, generator=g) * (2.0 / d ** 0.5)).to(BF16)
    return g, buf[:, :d]


def _labels(T, V, first):
    """Classes in the first, a middle and the last group of 16 rows, and in groups that a block takes second and third."""
    places = [0, V - 1, V // 2, 16 * 444 + 3, 16 * 296 + 1, 15, V - 16, 16 * 600 + 5]
    return torch.tensor([places[(i + first) % 8] for i in range(T)], device=DEV, dtype=torch.int32)


def _tolerance(H, W, tau, lse):
    absz = (H.abs() @ W.abs().t()).amax(1) / tau
    return 4 * u(F32) * (H.shape[1] / 16 + 16) * absz + 64 * u(F32) * (1 + lse.abs() + absz)


def _check(hidden, weight, labels, tau, nll, lse):
    H, W = hidden.double(), weight.double()
    Z = H @ W.t() / tau
    want_lse = torch.logsumexp(Z, 1)
    want = want_lse - Z.gather(1, labels.long()[:, None])[:, 0]
    tol = _tolerance(H, W, tau, want_lse)
    assert bool(((nll.double() - want).abs() <= tol).all()) and bool(((lse.double() - want_lse).abs() <= tol).all())


@pytest.mark.parametrize("d", [64, 320, 640, 768, 1024, 1536, 2048, 2304, 4096, 4160])
@pytest.mark.parametrize("V", [12000, 20011])
def test_few_tokens_with_several_batches_and_groups(d, V):
    g, weight = _head(d, V, pad=8 if V % 2 else 0)
    for T in (1, 2, 5, 8, 9, 17):
        hidden = torch.randn((T, d), device=DEV, generator=g).to(BF16)
        for first in range(0, 8, 8 if T > 5 else 2):
            labels = _labels(T, V, first)
            for tau in (1.0, 0.5):
                nll, lse, _, _ = B.npd_cross_entropy(hidden, weight, labels, temperature=tau, grads=False)
                _check(hidden, weight, labels, tau, nll, lse)


@pytest.mark.parametrize("T,d", [(8, 1536), (3, 2048)])
def test_gradients_of_few_tokens_at_real_widths(T, d):
    V = 12000
    g, weight = _head(d, V)
    hidden = torch.randn((T, d), device=DEV, generator=g).to(BF16)
    labels = _labels(T, V, 1)
    labels[T // 2] = -100                          # does not count
    w = torch.rand(T, device=DEV, generator=g) + 0.5
    nll, lse, dH, dW = B.npd_cross_entropy(hidden, weight, labels, token_weight=w, grad_scale=0.25, dw_dtype=F32)
    on = labels >= 0
    _check(hidden[on], weight, labels[on], 1.0, nll[on], lse[on])
    assert not nll[~on].any() and not dH[~on].any()
    H, W = hidden.double(), weight.double()
    Z = H @ W.t()
    G = torch.softmax(Z, 1)
    k = (0.25 * w.double() * on)[:, None]
    eg = (_tolerance(H, W, 1.0, torch.logsumexp(Z, 1)) + 4 * u(F32))[:, None] * G * k       # G's error from the logits
    G.scatter_add_(1, labels.long().clamp(min=0)[:, None], -torch.ones((T, 1), dtype=torch.float64, device=DEV))
    G *= k
    rel = u(BF16) * 1.01 + 2 * u(F32) * (V / 16 + 64)      # G's rounding to bf16, the accumulation of the products
    sH, sW = (rel * G.abs() + eg) @ W.abs(), (rel * G.abs() + eg).t() @ H.abs()
    assert bool(((dH.double() - G @ W).abs() <= u(BF16) * 1.01 * (G @ W).abs() + sH + 1e-30).all())
    assert bool(((dW.double() - G.t() @ H).abs() <= u(F32) * (G.t() @ H).abs() + sW + 1e-30).all())
