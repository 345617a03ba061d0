"""What a call does with the `stream` it is given (binding._scope).  The first tests need no GPU: torch's stream
objects are replaced."""

import types

import pytest
import torch

from paper_2605_05940_b200 import binding as B


def _fake_streams(monkeypatch):
    entered = []
    made = lambda handle, dev: types.SimpleNamespace(cuda_stream=handle, device=torch.device("cuda", dev))
    # torch takes a handle of 0 as none at all and gives a stream of its pool (here: handle 77)
    monkeypatch.setattr(torch.cuda, "ExternalStream", lambda handle, device: made(handle if handle else 77, device))
    monkeypatch.setattr(torch.cuda, "default_stream", lambda dev: made(0, dev))
    monkeypatch.setattr(torch.cuda, "stream", lambda s: entered.append(s) or s)
    return entered


@pytest.mark.parametrize("handle", [0, 1, 2, 0x7f0000001000])
def test_a_raw_handle_names_the_stream_itself(monkeypatch, handle):
    entered = _fake_streams(monkeypatch)
    B._scope(3, handle)
    assert [s.cuda_stream for s in entered] == [handle] and entered[0].device.index == 3


def test_a_stream_of_another_device_is_refused(monkeypatch):
    _fake_streams(monkeypatch)
    with pytest.raises(B.NpdError):
        B._scope(0, types.SimpleNamespace(cuda_stream=5, device=torch.device("cuda", 1)))


@pytest.mark.gpu
def test_calls_on_handle_zero_follow_the_default_stream():
    # the values arrive behind a long wait on the default stream; a call that ran elsewhere would read the old ones
    g = torch.Generator(device="cuda").manual_seed(1)
    new = torch.randn((64, 256), device="cuda", generator=g).to(torch.bfloat16)
    w = torch.randn((128, 256), device="cuda", generator=g).to(torch.bfloat16)
    labels = torch.randint(0, 128, (64,), device="cuda", generator=g, dtype=torch.int32)
    want = (B.npd_norm_fwd(new)[1], B.npd_linear_fwd(new, w)[0], B.npd_cross_entropy(new, w, labels)[0])
    torch.cuda.synchronize()
    x = torch.zeros_like(new)
    with torch.cuda.stream(torch.cuda.default_stream()):
        torch.cuda._sleep(20_000_000)
        x.copy_(new)
    got = (B.npd_norm_fwd(x, stream=0)[1], B.npd_linear_fwd(x, w, stream=0)[0],
           B.npd_cross_entropy(x, w, labels, stream=0)[0])
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(got, want))
