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


@pytest.mark.parametrize("kind", ["ce", "kd"])
def test_hidden_states_over_the_branch_are_refused(calls, kind):
    # the forward could write y over x, but the backward would then read y as x
    x = _mat()
    with pytest.raises(B.NpdError) as e:
        _step(kind, x, True, B.NormJoin(x, _mat(), pre_weight=torch.ones(D)))
    assert e.value.code == B.NPD_EINVAL
    _step(kind, x, False, B.NormJoin(x, _mat(), pre_weight=torch.ones(D), grads=False)).run()
    both = _mat(T, 2 * D + 16)             # windows of one buffer, side by side, are apart
    _step(kind, both[:, :D], True, B.NormJoin(both[:, D + 8:2 * D + 8], _mat())).run()
    with pytest.raises(B.NpdError):
        _step(kind, both[:, :D], True, B.NormJoin(both[:, D - 8:2 * D - 8], _mat()))


def test_d_hidden_over_an_operand_of_the_join_is_refused(calls):
    x, gate = _mat(), torch.zeros((T, D), dtype=BF16)
    for other in (x, gate):
        with pytest.raises(B.NpdError) as e:
            _step("ce", _mat(), True, B.NormJoin(x, _mat(), gate=gate), d_hidden=other)
        assert e.value.code == B.NPD_EINVAL
    _step("ce", _mat(), True, B.NormJoin(x, _mat(), gate=gate), d_hidden=_mat()).run()


def test_touch_knows_the_rows_of_a_window():
    base = torch.zeros((8, 32))
    assert B._touch(base, base) and B._touch(base, base[3:4]) and not B._touch(base[:4], base[4:])
    assert not B._touch(base[:, :8], base[:, 8:16]) and not B._touch(base[:, 16:], base[1:, :16])
    assert B._touch(base[:, :9], base[:, 8:16]) and B._touch(base[:, 16:], base[:, 15:17])
    assert not B._touch(base, torch.zeros((8, 32))) and not B._touch(base, None) and B._touch(base[0], base[:1])


def test_the_join_writes_the_hidden_states_that_the_step_reads(calls, monkeypatch):
    # a batch object may be given other tensors later on; a step stays with those it was made for
    hidden, weight = _mat(), _mat(V)
    batch = types.SimpleNamespace(T=T, d=D, V=V, hidden=hidden, weight=weight, teacher=_mat(T, V), tau=1.0, n_loss=T,
                                  cu_seqlens=None, loss_mask=None, labels=None)
    step = B.KDStep(batch, norm=B.NormJoin(_mat(), _mat(), pre_weight=torch.ones(D)))
    batch.hidden = _mat()
    written = []
    monkeypatch.setattr(B, "npd_norm_fwd", lambda x, r, y, **kw: written.append(y.data_ptr()))
    step.run()
    assert written == [step.args.hidden] == [hidden.data_ptr()]
