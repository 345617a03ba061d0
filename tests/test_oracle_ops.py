"""Pins of the oracle's functions around the loss step: torch's own routines in fp64 and central finite
differences."""

import numpy as np
import pytest
import torch

from oracle import npd_oracle as orc


def _diff(f, a, step=1e-6):
    """Central differences of the scalar f at the array a."""
    g = np.zeros_like(a)
    for i in np.ndindex(a.shape):
        keep = a[i]
        a[i] = keep + step
        up = f()
        a[i] = keep - step
        g[i] = (up - f()) / (2 * step)
        a[i] = keep
    return g


@pytest.mark.parametrize("tau", [1.0, 0.7, 2.0])
def test_cross_entropy_matches_torch_and_differences(tau):
    rng = np.random.default_rng(3)
    T, d, V = 6, 4, 9
    H, W = rng.normal(size=(T, d)), rng.normal(size=(V, d))
    y = np.array([0, 8, -100, 3, 9, 5])              # none, and one beyond the vocabulary
    m = np.array([1, 1, 1, 0, 1, 1])
    w = rng.random(T) * 2
    nll, lse, dH, dW = orc.cross_entropy_step(H, W, y, m, w, tau, 0.3)
    on = [0, 1, 5]
    want = torch.nn.functional.cross_entropy(torch.from_numpy(H @ W.T / tau)[on], torch.from_numpy(y[on]), reduction="none")
    assert np.allclose(nll[on], want.numpy(), rtol=1e-12)
    assert np.all(nll[[2, 3, 4]] == 0) and np.all(lse[[2, 3, 4]] == 0) and np.all(dH[[2, 3, 4]] == 0)
    assert np.allclose(lse[on], torch.logsumexp(torch.from_numpy(H @ W.T / tau)[on], 1).numpy(), rtol=1e-12)
    loss = lambda: 0.3 * float(np.sum(w * orc.cross_entropy_step(H, W, y, m, w, tau, 0.3)[0]))
    assert np.allclose(dH, _diff(loss, H), atol=1e-8) and np.allclose(dW, _diff(loss, W), atol=1e-8)


def test_cross_entropy_is_the_composite_objective_without_its_distillation_term():
    rng = np.random.default_rng(4)
    H, W, Z = rng.normal(size=(5, 3)), rng.normal(size=(7, 3)), rng.normal(size=(5, 7))
    y, m = np.array([1, 6, -100, 0, 2]), np.array([1, 1, 1, 0, 1])
    dH, dW = orc.composite_backward(H, W, Z, y, m, 1.0, 0.25, 0.0)
    got = orc.cross_entropy_step(H, W, y, m, None, 1.0, 0.25)
    assert np.allclose(got[2], dH) and np.allclose(got[3], dW)


@pytest.mark.parametrize("post_norm", [False, True])
@pytest.mark.parametrize("gate", ["none", "shared", "token"])
@pytest.mark.parametrize("offset", [0.0, 1.0])
def test_norm_join_matches_torch_and_differences(post_norm, gate, offset):
    rng = np.random.default_rng(5)
    T, d, eps = 3, 5, 1e-3
    x, r = rng.normal(size=(T, d)), rng.normal(size=(T, d))
    wp, wq = rng.normal(size=d), rng.normal(size=d)
    g = {"none": None, "shared": rng.normal(size=d), "token": rng.normal(size=(T, d))}[gate]
    how = dict(gate=g, post_weight=wp, pre_weight=wq, post_norm=post_norm, eps=eps, weight_offset=offset,
               residual_scale=0.7, branch_scale=1.3)
    h, y = orc.norm_join(x, r, **how)
    want = torch.nn.functional.rms_norm(torch.from_numpy(h), (d,), torch.from_numpy(wq + offset), eps)
    assert np.allclose(y, want.numpy(), rtol=1e-12)
    if post_norm and gate == "none":
        n = torch.nn.functional.rms_norm(torch.from_numpy(x), (d,), torch.from_numpy(wp + offset), eps).numpy()
        assert np.allclose(h, 0.7 * r + 1.3 * n)
    cy, ch = rng.normal(size=(T, d)), rng.normal(size=(T, d))
    loss = lambda: float(sum(np.sum(c * v) for c, v in zip((ch, cy), orc.norm_join(x, r, **how))))
    got = orc.norm_join_backward(cy, h, x, dh=ch, **how)
    assert np.allclose(got["dx"], _diff(loss, x), atol=1e-7)
    assert np.allclose(got["dresidual"], _diff(loss, r), atol=1e-7)
    assert np.allclose(got["d_pre_weight"], _diff(loss, wq), atol=1e-7)
    if post_norm:
        assert np.allclose(got["d_post_weight"], _diff(loss, wp), atol=1e-7)
    if g is not None:
        dg = got["d_gate"] if gate == "token" else got["d_gate"].sum(0)
        assert np.allclose(dg, _diff(loss, g), atol=1e-7)


@pytest.mark.parametrize("act", ["none", "relu", "gelu", "gelu_tanh", "silu"])
def test_linear_matches_torch_and_differences(act):
    rng = np.random.default_rng(6)
    M, N, K = 4, 3, 5
    x, w, b, r = rng.normal(size=(M, K)), rng.normal(size=(N, K)), rng.normal(size=N), rng.normal(size=(M, N))
    f = torch.nn.functional
    fn = {"none": lambda v: v, "relu": torch.relu, "gelu": f.gelu, "gelu_tanh": lambda v: f.gelu(v, approximate="tanh"),
          "silu": f.silu}[act]
    y, z = orc.linear(x, w, b, r, act)
    want = fn(torch.from_numpy(x @ w.T + b)).numpy() + r
    assert np.allclose(y, want, rtol=1e-12, atol=1e-14)
    c = rng.normal(size=(M, N))
    loss = lambda: float(np.sum(c * orc.linear(x, w, b, r, act)[0]))
    dx, dw, db, _ = orc.linear_backward(c, x, w, z, act)
    assert np.allclose(dx, _diff(loss, x), atol=1e-7) and np.allclose(dw, _diff(loss, w), atol=1e-7)
    assert np.allclose(db, _diff(loss, b), atol=1e-7)
