"""The operators as a student uses them one after the other: the last block's down projection, its join with the
residual stream and the final norm, the LM head with its loss, and the way back through all of them.

Tolerance.  Against the oracle's chain in fp64 on the same bf16 inputs.  Every stage rounds its result to bf16 once
(relative error u = 2^-8 at most, a fraction of it on average): on the way forward x (1), h and the hidden states (2);
on the way back the logit gradients, d_hidden (2), dx, dresidual (1) and dz, the products of the projection (1).  The
errors add up to at most 8 u of a result's norm; logits of unit size turn a relative error of the hidden states into
one of the same size in the probabilities."""

import numpy as np
import pytest
import torch

from oracle import npd_oracle as orc
from paper_2605_05940_b200 import binding as B
from paper_2605_05940_b200 import synth_inputs as syn

from _tolerance import host, u

pytestmark = pytest.mark.gpu
DEV = "cuda"
BF16 = torch.bfloat16


def _rel(got, want):
    return float(np.linalg.norm(host(got) - want) / np.linalg.norm(want))


def _tail(T, d, seed):
    g = torch.Generator(device=DEV).manual_seed(seed)
    r = lambda n, m, std=1.0: (torch.randn((n, m), device=DEV, generator=g) * std).to(BF16)
    act = r(T, 4 * d)
    w_down, b_down = r(d, 4 * d, 0.5 / np.sqrt(d)), torch.randn(d, device=DEV, generator=g) * 0.1
    how = dict(gate=(0.5 + torch.rand(d, device=DEV, generator=g)).to(BF16), post_weight=1 + 0.2 * torch.randn(d, device=DEV, generator=g),
               pre_weight=1 + 0.2 * torch.randn(d, device=DEV, generator=g), post_norm=True, eps=1e-6, residual_scale=0.8,
               branch_scale=1.0)
    return act, w_down, b_down, r(T, d, 2.0), how


def _oracle_forward(act, w_down, b_down, residual, how):
    x = orc.linear(host(act), host(w_down), host(b_down))[0]
    hh = {k: host(v) if torch.is_tensor(v) else v for k, v in how.items()}
    h, y = orc.norm_join(x, host(residual), **hh)
    return x, hh, h, y


@pytest.mark.parametrize("loss", ["ce", "kd"])
def test_forward_and_backward_through_the_tail(loss):
    T, d, V = 300, 192, 1504
    act, w_down, b_down, residual, how = _tail(T, d, 3)
    b = syn.scaled("c2", device=DEV, T=T, d=d, V=V, min_len=20, max_len=90)
    hidden, weight = torch.empty((T, d), device=DEV, dtype=BF16), b.weight
    b.hidden = hidden                                     # the step's hidden states come from the join
    gs = 1.0 / b.n_loss
    x, _ = B.npd_linear_fwd(act, w_down, bias=b_down)
    norm = B.NormJoin(x, residual, **how)
    if loss == "ce":
        step = B.CEStep(hidden, weight, b.labels, loss_mask=b.loss_mask, grad_scale=gs, norm=norm)
    else:
        step = B.KDStep(b, grad_scale=gs, norm=norm)
    step.run()
    d_act, d_down, d_bias = B.npd_linear_bwd(norm.dx, act, w_down, want_dbias=True)
    torch.cuda.synchronize()
    assert step.status() == B.NPD_OK

    ox, hh, oh, oy = _oracle_forward(act, w_down, b_down, residual, how)
    y, m, W = b.labels.cpu().numpy(), b.loss_mask.cpu().numpy(), host(weight)
    if loss == "ce":
        nll, _, dH, dW = orc.cross_entropy_step(oy, W, y, m, None, 1.0, gs)
        # a loss is a difference of logits that the hidden states' rounding moves by u of their size
        assert np.all(np.abs(host(step.nll) - nll) <= 8 * u(BF16) * (np.abs(oy) @ np.abs(W).T).max(1))
    else:
        dH, dW = orc.kd_backward(oy, W, host(b.teacher), m, b.tau, gs)
    back = orc.norm_join_backward(dH, oh, ox, **hh)
    o_act, o_down, o_bias, _ = orc.linear_backward(back["dx"], host(act), host(w_down))
    tol = 8 * u(BF16)
    for name, got, want in (("hidden", hidden, oy), ("d_weight", step.d_weight, dW), ("dx", norm.dx, back["dx"]),
                            ("dresidual", norm.dresidual, back["dresidual"]), ("d_post", norm.d_post_weight, back["d_post_weight"]),
                            ("d_pre", norm.d_pre_weight, back["d_pre_weight"]), ("d_gate", norm.d_gate, back["d_gate"].sum(0)),
                            ("d_act", d_act, o_act), ("d_down", d_down, o_down), ("d_bias", d_bias, o_bias)):
        assert _rel(got, want) < tol, (name, _rel(got, want))


def test_a_captured_tail_replays_on_new_values():
    T, d, V = 260, 128, 900
    act, w_down, b_down, residual, how = _tail(T, d, 5)
    g = torch.Generator(device=DEV).manual_seed(6)
    weight = (torch.randn((V, d), device=DEV, generator=g) * 0.1).to(BF16)
    labels = torch.randint(0, V, (T,), device=DEV, generator=g, dtype=torch.int32)
    hidden, x = torch.empty((T, d), device=DEV, dtype=BF16), torch.empty((T, d), device=DEV, dtype=BF16)
    norm = B.NormJoin(x, residual, **how)
    step = B.CEStep(hidden, weight, labels, grad_scale=1.0 / T, norm=norm)

    def run():
        B.npd_linear_fwd(act, w_down, bias=b_down, y=x)
        step.run()
        return B.npd_linear_bwd(norm.dx, act, w_down, want_dbias=True)

    run()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = run()
    act.copy_((torch.randn(act.shape, device=DEV, generator=g)).to(BF16))
    graph.replay()
    torch.cuda.synchronize()
    got = [t.clone() for t in (step.nll, step.d_weight)]
    run()
    torch.cuda.synchronize()
    assert torch.equal(got[0], step.nll) and torch.equal(got[1], step.d_weight) and step.status() == B.NPD_OK


def test_one_decoded_token_through_the_tail():
    # serving: one row, forward only, and the token's log-probability
    d, V = 192, 5000
    act, w_down, b_down, residual, how = _tail(1, d, 9)
    g = torch.Generator(device=DEV).manual_seed(10)
    weight = (torch.randn((V, d), device=DEV, generator=g) * 0.1).to(BF16)
    label = torch.tensor([4321], device=DEV, dtype=torch.int32)
    x, _ = B.npd_linear_fwd(act, w_down, bias=b_down)
    h, y = B.npd_norm_fwd(x, residual, **how)
    nll, lse, _, _ = B.npd_cross_entropy(y, weight, label, grads=False)
    _, _, _, oy = _oracle_forward(act, w_down, b_down, residual, how)
    want = orc.cross_entropy_step(oy, host(weight), label.cpu().numpy())
    bound = 8 * u(BF16) * (np.abs(oy) @ np.abs(host(weight)).T).max()
    assert abs(float(nll) - want[0][0]) <= bound and abs(float(lse) - want[1][0]) <= bound


def test_a_timed_step_runs_the_join_too():
    T, d, V = 200, 128, 904
    act, w_down, b_down, residual, how = _tail(T, d, 13)
    b = syn.scaled("c2", device=DEV, T=T, d=d, V=V, min_len=20, max_len=90)
    b.hidden = torch.zeros((T, d), device=DEV, dtype=BF16)
    x, _ = B.npd_linear_fwd(act, w_down, bias=b_down)
    norm = B.NormJoin(x, residual, **how)
    step = B.KDStep(b, grad_scale=1.0 / b.n_loss, norm=norm)
    times = step.run_with_phase_times()
    got = [t.clone() for t in (b.hidden, step.nll_student, step.kl, norm.d_pre_weight)]
    assert len(times) == len(step.phase_names()) and float(got[0].abs().max()) > 0
    step.run()
    torch.cuda.synchronize()
    for a, c in zip(got[:3], (b.hidden, step.nll_student, step.kl)):
        assert torch.equal(a, c)
    # d_hidden's sums over pieces of the vocabulary have no fixed order
    assert _rel(got[3], host(norm.d_pre_weight)) < 2 * u(BF16)
