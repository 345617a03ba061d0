"""npd_norm_fwd / npd_norm_bwd where every block goes through three or more rows (sets of rows, where several share a
block): the row held ahead, the ring's stages filled again, the two sets of reduction buffers in turn, and the sums over a
block's successive rows.  Against 64 bits on the GPU.

Tolerances as in test_gpu_norm.py: 80 fp32 roundings of what a row's results are made of (160 for dx, which stands
behind two norms).  The sums over tokens are taken per thread over the rows of its block (at most 9 here), over the
threads that share a column (at most 2 shuffles and 8 warps), over at most 1184 / 128 < 10 partial rows per thread and 128 such
threads (2 + 5 steps): 36 roundings, 64 counted."""

import pytest
import torch

from paper_2605_05940_b200 import binding as B

import _device_reference as ref

pytestmark = pytest.mark.gpu
DEV, BF16, F32 = "cuda", torch.bfloat16, torch.float32
F, SUM = 80, 64

# 148 SMs: blocks per SM times rows per block, three times over and a remainder
SHAPES = [(60011, 64), (30005, 121), (30000, 128), (15013, 249), (15000, 256), (7507, 300), (5003, 520), (4003, 1001), (2500, 1536),
          (1901, 2048), (1203, 3333), (1000, 4096), (700, 4104), (467, 6001), (461, 8192), (453, 8200), (451, 12288), (449, 16381)]


def _mat(g, rows, cols, dtype=BF16, pad=0, std=1.0):
    ld = (cols + 7) // 8 * 8 + pad
    buf = torch.full((rows, ld), float("nan"), device=DEV, dtype=dtype)
    buf[:, :cols] = (torch.randn((rows, cols), device=DEV, generator=g) * std).to(dtype)
    return buf[:, :cols]


def _copy(t):
    """The same values in rows that start on 16-byte boundaries."""
    out = torch.empty_strided(t.shape, ((t.shape[1] + 7) // 8 * 8, 1), dtype=t.dtype, device=DEV)
    return out.copy_(t)


def _case(T, d, sd, gate, post, wd=F32):
    g = torch.Generator(device=DEV).manual_seed(17 * T + d)
    x, r = _mat(g, T, d, pad=8), _mat(g, T, d, sd, std=2.0)
    how = dict(gate={"none": None, "shared": torch.randn(d, device=DEV, generator=g).to(BF16), "token": _mat(g, T, d)}[gate],
               post_weight=torch.randn(d, device=DEV, generator=g).to(wd) if post else None,
               pre_weight=torch.randn(d, device=DEV, generator=g).to(wd), post_norm=post, eps=1e-5, weight_offset=0.5,
               residual_scale=0.75, branch_scale=1.25)
    return g, x, r, how


def _check_forward(x, r, how, h, y):
    wh, sh, wy, sy = ref.norm_forward(x, r, **how)
    if h is not None:
        ref.near(h, wh, sh, F, "h")
    if y is not None:
        ref.near(y, wy, sy, F, "y")


def _check_backward(dy, h, x, dh, how, got):
    want = ref.norm_backward(dy, h, x, dh=dh, **how)
    gate = how["gate"]
    for name, t in zip(("dx", "dresidual", "d_post_weight", "d_pre_weight", "d_gate"), got):
        if t is None:
            continue
        v, size = want[name]
        if name == "d_gate" and gate.dim() == 1:
            v, size = v.sum(0), size.sum(0)
        steps = 2 * F if name == "dx" else F if t.dim() == 2 else F + SUM
        ref.near(t, v, size, steps, name)


@pytest.mark.parametrize("T,d", SHAPES)
@pytest.mark.parametrize("sd", [BF16, F32])
@pytest.mark.parametrize("gate,post", [("none", True), ("shared", True), ("token", True), ("token", False)])
def test_many_rows_per_block(T, d, sd, gate, post):
    g, x, r, how = _case(T, d, sd, gate, post, BF16 if T % 2 else F32)
    h, y = B.npd_norm_fwd(x, r, **how)
    _check_forward(x, r, how, h, y)
    dy, dh = _mat(g, T, d), _mat(g, T, d, sd, pad=16)
    _check_backward(dy, h, x, dh, how, B.npd_norm_bwd(dy, h, x, dh=dh, **how))


@pytest.mark.parametrize("T,d", [(30000, 128), (15013, 249), (5003, 520), (4003, 1001), (2500, 1536), (1000, 4096), (700, 4104),
                                 (461, 8192), (451, 12288)])
@pytest.mark.parametrize("sd", [BF16, F32])
def test_many_rows_with_parts_missing(T, d, sd):
    # what a plain norm, a final norm (nothing else arrives at h) and a join without a norm behind it leave out
    for gate, post in (("none", False), ("none", True), ("shared", True), ("token", True)):
        g, x, r, how = _case(T, d, sd, gate, post)
        dy, dh = _mat(g, T, d), _mat(g, T, d, sd)
        h, y = B.npd_norm_fwd(x, r, **how)
        for a, b in ((dy, None), (None, dh)):
            _check_backward(a, h, x, b, how, B.npd_norm_bwd(a, h, x, dh=b, **how))
        got = B.npd_norm_bwd(dy, h, x, dh=dh, want_dresidual=False, want_dweights=False, **how)
        assert got[1] is None and got[2] is None and got[3] is None
        _check_backward(dy, h, x, dh, how, got)
    how = dict(pre_weight=how["pre_weight"], eps=1e-5)
    h, y = B.npd_norm_fwd(None, r, **how)
    _check_forward(None, r, how, h, y)
    _check_backward(dy, h, None, None, dict(how, gate=None), B.npd_norm_bwd(dy, h, None, **how))
    h, y = B.npd_norm_fwd(x, None, want_h=False, **how)
    _check_forward(x, None, how, h, y)


@pytest.mark.parametrize("T,d", [(30000, 128), (7507, 300), (5003, 520), (2500, 1536), (700, 4104), (451, 12288)])
@pytest.mark.parametrize("sd", [BF16, F32])
def test_in_place_with_rows_ahead(T, d, sd):
    # the next rows are loaded before this row's results take their operands' place
    g, x, r, how = _case(T, d, sd, "token", True)
    h, y = B.npd_norm_fwd(x, r, **how)
    x1, r1 = _copy(x), _copy(r)
    B.npd_norm_fwd(x1, r1, h=r1, y=x1, **how)
    assert torch.equal(r1, h) and torch.equal(x1, y)
    dy, dh = _mat(g, T, d), _mat(g, T, d, sd)
    want = B.npd_norm_bwd(dy, h, x, dh=dh, **how)
    dy1, dh1, gate1 = _copy(dy), _copy(dh), _copy(how["gate"])
    got = B.npd_norm_bwd(dy1, h, x, dh=dh1, dx=dy1, dresidual=dh1, d_gate=gate1, **dict(how, gate=gate1))
    assert all(torch.equal(a, b) for a, b in zip(got, want))
    again = B.npd_norm_bwd(dy, h, x, dh=dh, **how)
    assert all(torch.equal(a, b) for a, b in zip(again, want))


@pytest.mark.parametrize("d", [64, 520, 1001, 4104])
@pytest.mark.parametrize("sd", [BF16, F32])
def test_backward_offsets_pass_32_bits(d, sd):
    # operands and results are column windows of buffers of more than 2^31 elements
    T, ld = 70, 1 << 25
    step = (d + 7) // 8 * 8
    narrow = torch.empty(T * ld, dtype=BF16, device=DEV)
    wide = torch.empty(T * ld, dtype=F32, device=DEV) if sd == F32 else narrow
    place = iter(range(8))
    window = lambda dt: torch.as_strided(narrow if dt == BF16 else wide, (T, d), (ld, 1), next(place) * step)
    g, x, r, how = _case(T, d, sd, "token", True)
    dy, dh = _mat(g, T, d), _mat(g, T, d, sd)
    h, _ = B.npd_norm_fwd(x, r, **how)
    want = B.npd_norm_bwd(dy, h, x, dh=dh, **how)
    far = []
    for t in (dy, h, x, dh, how["gate"]):
        far.append(window(t.dtype))
        far[-1].copy_(t)
    dx, dres, dgate = window(BF16), window(sd), window(BF16)
    got = B.npd_norm_bwd(far[0], far[1], far[2], dh=far[3], dx=dx, dresidual=dres, d_gate=dgate, **dict(how, gate=far[4]))
    assert all(torch.equal(a, b) for a, b in zip(got, want))
