"""What a call does with the `stream` and the `workspace` it is given.  The tests that are not marked need no GPU:
torch's stream objects, or the library behind the binding, are replaced."""

import contextlib

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


class _Elsewhere(torch.Tensor):
    """A tensor that says it lies on another GPU."""
    def get_device(self):
        return 1


def _calls_with(workspace):
    """The calls that take a workspace, on CPU tensors."""
    bf16 = torch.bfloat16
    x, w = torch.zeros((8, 64), dtype=bf16), torch.zeros((16, 64), dtype=bf16)
    return {
        "norm": lambda: B.npd_norm_bwd(x, x, x, pre_weight=torch.ones(64), workspace=workspace),
        "linear": lambda: B.npd_linear_bwd(torch.zeros((8, 16), dtype=bf16), x, w, workspace=workspace),
        "ce": lambda: B.CEStep(x, w, torch.zeros(8, dtype=torch.int32), workspace=workspace).run(),
    }


@pytest.mark.parametrize("op", ["norm", "linear", "ce"])
@pytest.mark.parametrize("kind", ["dense", "elsewhere", "strided"])
def test_a_workspace_elsewhere_or_with_gaps_is_refused(monkeypatch, op, kind):
    # the address would go to the kernels as it is
    launched = []
    done = lambda args, stream: launched.append(args.workspace) or B.NPD_OK
    monkeypatch.setattr(B, "lib", lambda: types.SimpleNamespace(npd_norm_bwd=done, npd_linear_bwd=done, npd_ce_fwd_bwd=done,
                                                                npd_strerror=lambda code: b""))
    monkeypatch.setattr(B, "_device_of", lambda t, where: t.get_device())
    monkeypatch.setattr(B, "_scope", lambda dev, stream: contextlib.nullcontext())
    monkeypatch.setattr(B, "_current", lambda dev: 0)
    room = torch.zeros(1 << 16, dtype=torch.uint8)
    ws = {"dense": room, "elsewhere": room.as_subclass(_Elsewhere), "strided": room[::2]}[kind]
    call = _calls_with(ws)[op]
    if kind == "dense":
        call()
        assert launched == [room.data_ptr()]
        return
    with pytest.raises(B.NpdError) as e:
        call()
    assert e.value.code == B.NPD_EWORKSPACE and not launched


@pytest.mark.gpu
def test_a_workspace_in_host_memory_is_refused():
    bf16 = torch.bfloat16
    x, w = torch.zeros((8, 64), dtype=bf16, device="cuda"), torch.zeros((16, 64), dtype=bf16, device="cuda")
    host = torch.zeros(1 << 24, dtype=torch.uint8)
    for call in (lambda: B.npd_norm_bwd(x, x, x, pre_weight=torch.ones(64, device="cuda"), workspace=host),
                 lambda: B.npd_linear_bwd(torch.zeros((8, 16), dtype=bf16, device="cuda"), x, w, workspace=host),
                 lambda: B.CEStep(x, w, torch.zeros(8, dtype=torch.int32, device="cuda"), workspace=host)):
        with pytest.raises(B.NpdError) as e:
            call()
        assert e.value.code == B.NPD_EWORKSPACE
