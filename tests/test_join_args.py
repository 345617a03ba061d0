"""What CEStep and KDStep check about the join that they are given (NormJoin).  No GPU needed: the library behind
the binding is replaced, tensors lie in host memory."""

import contextlib
import types

import pytest
import torch

from paper_2605_05940_b200 import binding as B

T, D, V = 6, 64, 24
BF16 = torch.bfloat16


@pytest.fixture
def calls(monkeypatch):
    """Names of the library's calls, in order."""
    log = []

    class Lib:
        def __getattr__(self, name):
            if name == "npd_strerror":
                return lambda code: b""
            return lambda *a: log.append(name) or B.NPD_OK

    monkeypatch.setattr(B, "lib", Lib)
    monkeypatch.setattr(B, "_device_of", lambda t, where: t.get_device())
    monkeypatch.setattr(B, "_scope", lambda dev, stream: contextlib.nullcontext())
    monkeypatch.setattr(B, "_current", lambda dev: 0)
    monkeypatch.setattr(B, "_stream", lambda stream: 0)
    return log


def _mat(rows=T, cols=D):
    return torch.zeros((rows, cols), dtype=BF16)


def _step(kind, hidden, grads, norm, **kw):
    if kind == "ce":
        if not grads:
            kw["d_hidden"] = None
        return B.CEStep(hidden, _mat(V), torch.zeros(T, dtype=torch.int32), norm=norm, **kw)
    batch = types.SimpleNamespace(T=T, d=D, V=V, hidden=hidden, weight=_mat(V), teacher=_mat(T, V), tau=1.0, n_loss=T,
                                  cu_seqlens=None, loss_mask=None, labels=None)
    return B.KDStep(batch, grads=grads, norm=norm)


@pytest.mark.parametrize("kind", ["ce", "kd"])
def test_a_join_runs_before_and_after_the_step(calls, kind):
    step = _step(kind, _mat(), True, B.NormJoin(_mat(), _mat(), pre_weight=torch.ones(D)))
    del calls[:]
    step.run()
    name = "npd_ce_fwd_bwd" if kind == "ce" else "npd_kd_fwd_bwd"
    assert calls == ["npd_norm_fwd", name, "npd_norm_bwd"]


@pytest.mark.parametrize("kind", ["ce", "kd"])
def test_gradients_that_no_run_would_write_are_refused(calls, kind):
    with pytest.raises(B.NpdError) as e:
        _step(kind, _mat(), False, B.NormJoin(_mat(), _mat(), pre_weight=torch.ones(D)))
    assert e.value.code == B.NPD_EINVAL
    step = _step(kind, _mat(), False, B.NormJoin(_mat(), _mat(), pre_weight=torch.ones(D), grads=False))
    del calls[:]
    step.run()
    assert calls[0] == "npd_norm_fwd" and "npd_norm_bwd" not in calls
