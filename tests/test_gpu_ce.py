"""npd_ce_fwd_bwd against the fp64 oracle.

Tolerances.  Logits are sums of d exact products of bf16 numbers, accumulated in fp32 by the tensor core, which
aligns the addends of a step and cuts what falls below the accumulator's last place: at most one unit (not half)
per addend group of 16 and accumulation, so a logit is off by at most 2 u (d/16 + 16) of the sum of the
absolute products.  lse and nll inherit the largest error of the row's logits (their derivatives with respect to
the logits are probabilities), plus a few dozen fp32 roundings of the values themselves.
A gradient element sums products of G (bf16) with bf16 operands; each G is off by u(bf16) of itself (its
probability's own relative error is the logits' absolute error, far below) and the result by its own type's
rounding.  With s_abs the sum of the absolute products, |got - want| <= u(out)|want| + (u(bf16) + e) s_abs."""

import numpy as np
import pytest
import torch

from oracle import npd_oracle as orc
from paper_2605_05940_b200 import binding as B

from _tolerance import host, u

pytestmark = pytest.mark.gpu
DEV = "cuda"
F32, BF16 = torch.float32, torch.bfloat16


def _batch(T, d, V, seed=0, pad=0, masked=True, weighted=False, spread=1.0):
    g = torch.Generator(device=DEV).manual_seed(seed + 7 * T + 3 * d + V)
    r = lambda n, std: (torch.randn((n, d + pad), device=DEV, generator=g) * std).to(BF16)
    hidden, weight = r(T, 1.0)[:, :d], r(V, spread / np.sqrt(d))[:, :d]
    labels = torch.randint(0, V, (T,), device=DEV, generator=g, dtype=torch.int32)
    mask = None
    if masked:
        mask = (torch.rand(T, device=DEV, generator=g) < 0.7).to(torch.uint8)
        labels[::5] = -100
        labels[3::11] = V                    # beyond the vocabulary: does not count
    w = torch.rand(T, device=DEV, generator=g) * 2 if weighted else None
    return hidden, weight, labels, mask, w


def _check(hidden, weight, labels, mask, w, tau, gs, got, base_dw=None):
    H, W = host(hidden), host(weight)
    y = labels.cpu().numpy()
    m = None if mask is None else mask.cpu().numpy()
    ww = None if w is None else host(w)
    nll, lse, dH, dW = orc.cross_entropy_step(H, W, y, m, ww, tau, gs)
    T, V, d = H.shape[0], W.shape[0], H.shape[1]
    on = (y >= 0) & (y < V) & ((m != 0) if m is not None else True)
    absz = np.zeros(T)
    absz[on] = (np.abs(H[on]) @ np.abs(W).T).max(axis=1) / tau
    ez = 2 * u(F32) * (d / 16 + 16) * absz                     # error of a row's logits
    tol = 2 * ez + 64 * u(F32) * (1 + np.abs(lse) + absz)
    gn, gl = host(got[0]), host(got[1]) if got[1] is not None else None
    assert np.all(np.abs(gn - nll) <= tol), np.max(np.abs(gn - nll) - tol)
    assert np.all(gn[~on] == 0)
    if gl is not None:
        assert np.all(np.abs(gl - lse) <= tol) and np.all(gl[~on] == 0)
    if got[2] is None and got[3] is None:
        return
    Z = H @ W.T / tau
    G = np.exp(Z - Z.max(1, keepdims=True))
    G /= G.sum(1, keepdims=True)
    # where the label's probability is near 1 the difference p - 1 carries the fp32 rounding of p
    absG = G.copy()
    absG[np.arange(T)[on], y[on]] = np.abs(G[np.arange(T)[on], y[on]] - 1)
    k = gs / tau * (np.ones(T) if ww is None else ww) * on
    eg = (tol + 4 * u(F32))[:, None] * G * k[:, None]          # absolute error of G from the logits
    absG *= k[:, None]
    rel = u(BF16) * 1.01 + 2 * u(F32) * (max(T, V) / 16 + 64)  # rounding of G; accumulation of the products
    if got[2] is not None:
        t = u(BF16) * np.abs(dH) * 1.01 + rel * (absG @ np.abs(W)) + eg @ np.abs(W) + 1e-30
        err = np.abs(host(got[2]) - dH)
        assert np.all(err <= t), (np.max(err / np.maximum(t, 1e-300)))
        assert np.all(host(got[2])[~on] == 0)
    if got[3] is not None:
        base = 0.0 if base_dw is None else base_dw
        t = u(got[3].dtype) * np.abs(dW + base) * 1.01 + rel * (absG.T @ np.abs(H)) + eg.T @ np.abs(H) + 1e-30 \
            + 4 * u(F32) * np.abs(base)
        err = np.abs(host(got[3]) - (dW + base))
        assert np.all(err <= t), (np.max(err / np.maximum(t, 1e-300)))


SHAPES = [(1, 64, 1), (1, 64, 2), (1, 128, 1000), (2, 64, 255), (7, 192, 257), (129, 64, 513), (256, 64, 1000), (257, 128, 300),
          (300, 320, 2111), (1000, 256, 777), (33, 1536, 5000)]


@pytest.mark.parametrize("T,d,V", SHAPES)
@pytest.mark.parametrize("tau,weighted,masked", [(1.0, False, False), (2.0, True, True), (0.7, False, True)])
def test_losses_and_gradients(T, d, V, tau, weighted, masked):
    hidden, weight, labels, mask, w = _batch(T, d, V, pad=8 * (T % 3), masked=masked, weighted=weighted, spread=2.0)
    dw = F32 if (T + V) % 2 else BF16
    s = B.CEStep(hidden, weight, labels, loss_mask=mask, token_weight=w, temperature=tau, grad_scale=0.125, dw_dtype=dw)
    for t in (s.nll, s.lse, s.d_hidden, s.d_weight):
        t.fill_(float("nan"))
    s.run()
    assert s.status() == B.NPD_OK
    _check(hidden, weight, labels, mask, w, tau, 0.125, (s.nll, s.lse, s.d_hidden, s.d_weight))
    f = B.npd_cross_entropy(hidden, weight, labels, loss_mask=mask, token_weight=w, temperature=tau, grads=False)
    assert torch.equal(f[0], s.nll) and torch.equal(f[1], s.lse) and f[2] is None and f[3] is None


@pytest.mark.parametrize("cols", [1, 256, 600, 1 << 20])
def test_pieces_of_the_vocabulary(cols):
    hidden, weight, labels, mask, w = _batch(300, 128, 1500, weighted=True)
    got = B.npd_cross_entropy(hidden, weight, labels, loss_mask=mask, token_weight=w, grad_scale=0.01, grad_chunk_cols=cols)
    _check(hidden, weight, labels, mask, w, 1.0, 0.01, got)


def test_one_gradient_alone_and_accumulation():
    hidden, weight, labels, mask, w = _batch(400, 192, 900, weighted=True)
    both = B.npd_cross_entropy(hidden, weight, labels, loss_mask=mask, token_weight=w, grad_scale=0.02)
    only_w = B.npd_cross_entropy(hidden, weight, labels, loss_mask=mask, token_weight=w, grad_scale=0.02, d_hidden=None)
    assert only_w[2] is None and torch.equal(only_w[3], both[3])
    only_h = B.npd_cross_entropy(hidden, weight, labels, loss_mask=mask, token_weight=w, grad_scale=0.02, d_weight=None)
    assert only_h[3] is None
    _check(hidden, weight, labels, mask, w, 1.0, 0.02, only_h)
    g = torch.Generator(device=DEV).manual_seed(5)
    base = torch.randn((900, 192), device=DEV, generator=g) * 0.01
    acc = base.clone()
    got = B.npd_cross_entropy(hidden, weight, labels, loss_mask=mask, token_weight=w, grad_scale=0.02, d_weight=acc,
                              accumulate_dw=True)
    assert got[3] is acc
    _check(hidden, weight, labels, mask, w, 1.0, 0.02, got, base_dw=host(base))


@pytest.mark.parametrize("T", [1, 130, 600])
def test_no_token_counts(T):
    hidden, weight, labels, _, _ = _batch(T, 64, 300, masked=False)
    hidden.fill_(float("nan"))                       # never read
    for kw in (dict(loss_mask=torch.zeros(T, dtype=torch.uint8, device=DEV)), dict(labels=torch.full_like(labels, -1)),
               dict(labels=torch.full_like(labels, 300))):
        y = kw.pop("labels", labels)
        nll, lse, dH, dW = B.npd_cross_entropy(hidden, weight, y, **kw)
        assert not nll.any() and not lse.any() and not dH.any() and not dW.any()


def test_masked_rows_are_not_read_and_bad_rows_stay_alone():
    hidden, weight, labels, mask, _ = _batch(500, 128, 700)
    want = B.npd_cross_entropy(hidden, weight, labels, loss_mask=mask)
    on = (mask != 0) & (labels >= 0) & (labels < 700)
    h2 = hidden.clone()
    h2[~on] = float("nan")
    got = B.npd_cross_entropy(h2, weight, labels, loss_mask=mask)
    assert all(torch.equal(a, b) for a, b in zip(got[:2], want[:2])) and torch.equal(got[3], want[3])
    bad = int(torch.nonzero(on)[17])
    h2[bad, 3] = float("inf")
    got = B.npd_cross_entropy(h2, weight, labels, loss_mask=mask)
    keep = torch.arange(500, device=DEV) != bad
    assert torch.isnan(got[0][bad]) and torch.equal(got[0][keep], want[0][keep])
    assert torch.isnan(got[2][bad]).any() and torch.isfinite(got[2][keep].float()).all()


def test_far_logits():
    # a row decided by one class, and logits of hundreds: no overflow, exact zeros where they belong
    T, d, V = 4, 64, 600
    weight = torch.zeros((V, d), device=DEV, dtype=BF16)
    weight[:, 0] = torch.linspace(-8, 8, V, device=DEV).to(BF16)
    hidden = torch.zeros((T, d), device=DEV, dtype=BF16)
    hidden[:, 0] = torch.tensor([100.0, -100.0, 1.0, 0.0], device=DEV).to(BF16)
    labels = torch.tensor([V - 1, V - 1, 5, 9], device=DEV, dtype=torch.int32)
    got = B.npd_cross_entropy(hidden, weight, labels)
    _check(hidden, weight, labels, None, None, 1.0, 1.0, got)
    assert abs(float(got[0][3]) - np.log(V)) < 1e-5


def test_same_bits_other_stream_and_graph():
    hidden, weight, labels, mask, w = _batch(700, 256, 3000, weighted=True)
    kw = dict(loss_mask=mask, token_weight=w, grad_scale=0.01)
    want = B.npd_cross_entropy(hidden, weight, labels, **kw)
    again = B.npd_cross_entropy(hidden, weight, labels, flags=B.NPD_CE_SERIALIZE_LAUNCHES, **kw)
    for i in (0, 1, 3):
        assert torch.equal(want[i], again[i])
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    got = B.npd_cross_entropy(hidden, weight, labels, stream=side, **kw)
    side.synchronize()
    assert torch.equal(got[0], want[0]) and torch.equal(got[3], want[3])
    step = B.CEStep(hidden, weight, labels, **kw)
    step.run()
    graph = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        step.run()
    h0 = hidden.clone()
    hidden.copy_(h0.flip(0))
    graph.replay()
    other = B.npd_cross_entropy(hidden, weight, labels, **kw)
    assert torch.equal(step.nll, other[0]) and torch.equal(step.d_weight, other[3])
    hidden.copy_(h0)
    graph.replay()
    torch.cuda.synchronize()
    assert torch.equal(step.nll, want[0]) and torch.equal(step.d_weight, want[3]) and step.status() == B.NPD_OK


def test_agrees_with_the_composite_objective_of_the_distillation_step():
    from paper_2605_05940_b200 import synth_inputs as syn
    b = syn.scaled("c2", device=DEV, T=600, d=128, V=2504, min_len=20, max_len=200)
    kd = B.KDStep(b, kd_lambda=0.0, dw_dtype=F32)
    kd.run()
    ce = B.npd_cross_entropy(b.hidden, b.weight, b.labels, loss_mask=b.loss_mask, grad_scale=kd.grad_scale, dw_dtype=F32)
    torch.cuda.synchronize()
    assert torch.allclose(ce[0], kd.nll_student, rtol=1e-5, atol=1e-5)
    rel = lambda a, r: float((a.double() - r.double()).norm() / r.double().norm())
    # the two round the logit gradients to bf16 at different scales, and d_hidden once more
    assert rel(ce[3], kd.d_weight) < 2 * u(BF16) and rel(ce[2], kd.d_hidden) < 4 * u(BF16)


def test_scores_feed_the_segment_statistics():
    # the scoring pass: losses of a packed batch, per-segment sums, against the oracle
    from paper_2605_05940_b200 import synth_inputs as syn
    b = syn.scaled("c2", device=DEV, T=500, d=64, V=1200, min_len=10, max_len=90)
    nll = B.npd_cross_entropy(b.hidden, b.weight, b.labels, loss_mask=b.loss_mask, grads=False)[0]
    _, s_sum, _, count, _ = B.npd_segment_stats(b.cu_seqlens, b.loss_mask, b.labels, None, nll, None)
    y, m, cu = b.labels.cpu().numpy(), b.loss_mask.cpu().numpy(), b.cu_seqlens.cpu().numpy()
    want = orc.cross_entropy_step(host(b.hidden), host(b.weight), y, m)[0]
    ref = orc.segment_stats(cu, m, y, want, want, want)
    assert np.array_equal(count.cpu().numpy(), ref[3]) and np.allclose(host(s_sum), ref[1], rtol=1e-4)


def test_a_large_case_against_fp64_on_the_gpu():
    # full tiles, several pieces of the vocabulary, several pairs of row blocks
    hidden, weight, labels, mask, w = _batch(3000, 512, 30011, weighted=True, spread=3.0)
    nll, lse, dH, dW = B.npd_cross_entropy(hidden, weight, labels, loss_mask=mask, token_weight=w, grad_scale=1e-3,
                                           grad_chunk_cols=8192)
    on = (mask != 0) & (labels >= 0) & (labels < 30011)
    H, W = hidden.double(), weight.double()
    Z = H @ W.t()
    L = torch.logsumexp(Z, 1)
    at = labels.long().clamp(0, 30010)[:, None]
    ref = torch.where(on, L - Z.gather(1, at)[:, 0], torch.zeros_like(L))
    assert float((nll.double() - ref).abs().max()) < 1e-4
    P = torch.exp(Z - L[:, None])
    P.scatter_add_(1, at, -torch.ones_like(P[:, :1]))
    P *= (torch.where(on, w.double(), torch.zeros_like(L)) * 1e-3)[:, None]
    rel = lambda a, r: float((a.double() - r).norm() / r.norm())
    assert rel(dH, P @ W) < 3 * u(BF16) and rel(dW, P.t() @ H) < 3 * u(BF16)


def test_accumulation_into_a_new_d_weight_starts_at_zero():
    g = torch.Generator(device=DEV).manual_seed(33)
    T, d, V = 150, 128, 700
    H, W = (torch.randn(T, d, device=DEV, generator=g)).to(BF16), (torch.randn(V, d, device=DEV, generator=g) * 0.1).to(BF16)
    y = torch.randint(0, V, (T,), device=DEV, generator=g, dtype=torch.int32)
    junk = torch.full((V, d), float("nan"), device=DEV)   # its memory is what the next tensor of this size gets
    del junk
    step = B.CEStep(H, W, y, grad_scale=1.0 / T, dw_dtype=torch.float32, accumulate_dw=True)
    step.run()
    plain = B.npd_cross_entropy(H, W, y, grad_scale=1.0 / T, dw_dtype=torch.float32)[3]
    assert torch.equal(step.d_weight, plain)              # one add to zero per element
    step.run()
    assert torch.equal(step.d_weight, 2 * plain)          # x + x is exact
