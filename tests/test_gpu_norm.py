"""npd_norm_fwd / npd_norm_bwd against the fp64 oracle.

Tolerances: a result is off by the rounding of its type plus fp32 roundings of what was added up.  The
reductions run over d elements in a tree (at most 16 or 32 in a thread, then the warp and the block): fewer
than 64 roundings, of sums of squares (all of one sign) or of the absolute sum; rsqrt is good to 2 ulp.  So 64 + a few
elementwise steps: F = 80.  The sums over tokens add up to ceil(T / CTAs) + 64 values in a row."""

import numpy as np
import pytest
import torch

from oracle import npd_oracle as orc
from paper_2605_05940_b200 import binding as B

from _tolerance import assert_rounded, host

pytestmark = pytest.mark.gpu
DEV = "cuda"
F = 80


def _mat(g, rows, cols, dtype=torch.bfloat16, pad=0, std=1.0):
    ld = (cols + 7) // 8 * 8 + pad
    buf = torch.full((rows, ld), float("nan"), device=DEV, dtype=dtype)
    buf[:, :cols] = (torch.randn((rows, cols), device=DEV, generator=g) * std).to(dtype)
    return buf[:, :cols]


def _case(T, d, sd, wd, gate, post, seed=0, pad=0, eps=1e-5, offset=0.0):
    g = torch.Generator(device=DEV).manual_seed(seed + 31 * T + d)
    x, r = _mat(g, T, d, pad=pad), _mat(g, T, d, sd, pad=2 * pad, std=2.0)
    how = dict(gate={"none": None, "shared": torch.randn(d, device=DEV, generator=g).to(torch.bfloat16),
                     "token": _mat(g, T, d, pad=pad)}[gate],
               post_weight=torch.randn(d, device=DEV, generator=g).to(wd) if post else None,
               pre_weight=torch.randn(d, device=DEV, generator=g).to(wd), post_norm=post, eps=eps,
               weight_offset=offset, residual_scale=0.75, branch_scale=1.25)
    return x, r, how


def _host(how):
    return {k: host(v) if torch.is_tensor(v) else v for k, v in how.items()}


def _check_forward(x, r, how, h, y):
    wh, wy = orc.norm_join(None if x is None else host(x), None if r is None else host(r), **_host(how))
    scale = 0.0 if r is None else np.abs(0.75 * host(r))
    scale = scale + np.abs(wh - (0.0 if r is None else 0.75 * host(r)))      # |residual part| + |branch part|
    if h is not None:
        assert_rounded(h, wh, scale, F, "h")
    if y is not None:
        assert_rounded(y, wy, np.abs(wy / np.where(wh == 0, 1, wh)) * scale + np.abs(wy), F, "y")


def _check_backward(dy, h, x, dh, how, got):
    hh = _host(how)
    w = orc.norm_join_backward(None if dy is None else host(dy), host(h), None if x is None else host(x),
                               dh=None if dh is None else host(dh), **hh)
    dx, dres, d_post, d_pre, d_gate = got
    T, d = host(h).shape
    # the absolute size of what dh is made of: |dh_in| + r (|g| + |h| r^2 mean |g h|)
    H = host(h)
    r = 1 / np.sqrt(np.mean(H * H, 1, keepdims=True) + how["eps"])
    big = 0.0 if dh is None else np.abs(host(dh))
    if dy is not None:
        G = np.abs(host(dy) * (1.0 if hh["pre_weight"] is None else hh["pre_weight"] + how["weight_offset"]))
        big = big + r * (G + np.abs(H) * r * r * np.mean(G * np.abs(H), 1, keepdims=True))
    if dres is not None:
        assert_rounded(dres, w["dresidual"], 0.75 * big, F, "dresidual")
    rows = 64 + T                                  # additions in a sum over tokens, at most
    if d_pre is not None:
        assert_rounded(d_pre, w["d_pre_weight"], np.sum(np.abs(host(dy) * H * r), 0), rows + F, "d_pre_weight")
    if x is None:
        return
    X = host(x)
    rx = 1 / np.sqrt(np.mean(X * X, 1, keepdims=True) + how["eps"]) if how["post_norm"] else 1.0
    gain = np.abs(hh["post_weight"] + how["weight_offset"]) if hh["post_weight"] is not None else 1.0
    bd = 1.25 * big
    if how["gate"] is not None:
        if d_gate.dim() == 2:
            assert_rounded(d_gate, w["d_gate"], bd * np.abs(X) * rx * gain, F, "d_gate")
        else:
            assert_rounded(d_gate, w["d_gate"].sum(0), np.sum(bd * np.abs(X) * rx * gain, 0), rows + F, "d_gate")
    dn = bd * (1.0 if how["gate"] is None else np.abs(hh["gate"]))
    if d_post is not None:
        assert_rounded(d_post, w["d_post_weight"], np.sum(dn * np.abs(X) * rx, 0), rows + F, "d_post_weight")
    v = dn * gain
    size = rx * (v + np.abs(X) * rx * rx * np.mean(v * np.abs(X), 1, keepdims=True)) if how["post_norm"] else v
    assert_rounded(dx, w["dx"], size, 2 * F, "dx")


@pytest.mark.parametrize("T,d", [(1, 1), (1, 7), (3, 8), (5, 33), (2, 256), (700, 264), (33, 1536), (9, 4096), (6, 4104),
                                 (3, 8192), (2, 8200), (2, 16384), (2500, 100)])
@pytest.mark.parametrize("sd", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("gate,post", [("none", False), ("shared", True), ("token", True), ("token", False)])
def test_forward_and_backward(T, d, sd, gate, post):
    wd = torch.float32 if (T + d) % 2 else torch.bfloat16
    x, r, how = _case(T, d, sd, wd, gate, post, pad=8 * (T % 3), offset=float(d % 2))
    h, y = B.npd_norm_fwd(x, r, **how)
    assert h.dtype == sd and y.dtype == torch.bfloat16
    _check_forward(x, r, how, h, y)
    g = torch.Generator(device=DEV).manual_seed(1)
    dy, dh = _mat(g, T, d, pad=8), _mat(g, T, d, sd)
    got = B.npd_norm_bwd(dy, h, x, dh=dh, **how)
    _check_backward(dy, h, x, dh, how, got)


def test_parts_of_the_join():
    # a plain norm, a join without a norm behind it, no residual, no branch, no gains
    x, r, how = _case(17, 72, torch.float32, torch.float32, "none", False)
    plain = dict(how, pre_weight=None)
    for xx, rr in ((x, None), (None, r), (x, r)):
        for kw in (how, plain):
            h, y = B.npd_norm_fwd(xx, rr, **kw)
            _check_forward(xx, rr, kw, h, y)
            h2, y2 = B.npd_norm_fwd(xx, rr, want_h=False, **kw)
            assert h2 is None and torch.equal(y2, y)
            h3, y3 = B.npd_norm_fwd(xx, rr, want_y=False, **kw)
            assert y3 is None and torch.equal(h3, h)
            g = torch.Generator(device=DEV).manual_seed(2)
            dy, dh = _mat(g, 17, 72), _mat(g, 17, 72, h.dtype)
            for a, b in ((dy, dh), (dy, None), (None, dh)):
                _check_backward(a, h, xx, b, kw, B.npd_norm_bwd(a, h, xx, dh=b, **kw))


def test_rows_are_independent_and_bad_values_stay_in_their_row():
    x, r, how = _case(9, 104, torch.bfloat16, torch.float32, "token", True)
    h, y = B.npd_norm_fwd(x, r, **how)
    x2 = x.clone()
    x2[3, 5], x2[6, 0] = float("nan"), float("inf")
    h2, y2 = B.npd_norm_fwd(x2, r, **how)
    keep = [t for t in range(9) if t not in (3, 6)]
    assert torch.equal(h2[keep], h[keep]) and torch.equal(y2[keep], y[keep])
    assert torch.isnan(y2[3]).all() and torch.isnan(y2[6]).any()
    # a row of zeros: eps alone keeps it finite
    z = torch.zeros_like(x)
    h0, y0 = B.npd_norm_fwd(z, torch.zeros_like(r), **how)
    assert not h0.any() and not y0.any()
    got = B.npd_norm_bwd(torch.ones_like(x), h0, z, **how)
    assert all(torch.isfinite(t).all() for t in got)


def test_in_place_and_windows_of_a_wider_buffer():
    x, r, how = _case(50, 136, torch.bfloat16, torch.bfloat16, "token", True)
    h, y = B.npd_norm_fwd(x, r, **how)
    x1, r1 = x.clone(), r.clone()
    B.npd_norm_fwd(x1, r1, h=r1, y=x1, **how)
    assert torch.equal(r1, h) and torch.equal(x1, y)
    wide = torch.full((50, 400), 7.0, device=DEV, dtype=torch.bfloat16)
    B.npd_norm_fwd(x, r, h=wide[:, 8:144], y=wide[:, 200:336], **how)
    assert torch.equal(wide[:, 8:144], h) and torch.equal(wide[:, 200:336], y)
    assert (wide[:, :8] == 7).all() and (wide[:, 144:200] == 7).all() and (wide[:, 336:] == 7).all()
    g = torch.Generator(device=DEV).manual_seed(3)
    dy, dh = _mat(g, 50, 136), _mat(g, 50, 136)
    want = B.npd_norm_bwd(dy, h, x, dh=dh, **how)
    dy1, dh1 = dy.clone(), dh.clone()
    got = B.npd_norm_bwd(dy1, h, x, dh=dh1, dx=dy1, dresidual=dh1, **how)
    assert all(torch.equal(a, b) for a, b in zip(got, want))
    with pytest.raises(B.NpdError):
        B.npd_norm_fwd(x, r, h=wide[:, 0:136], y=wide[:, 128:264], **how)
    with pytest.raises(B.NpdError):
        B.npd_norm_fwd(x[:, 1:], r[:, 1:])                     # rows off their 16-byte boundary
    with pytest.raises(B.NpdError):
        B.npd_norm_fwd(x, r, gate=how["gate"][:1].expand(50, 136))
    with pytest.raises(B.NpdError):
        B.npd_norm_fwd(x.float(), r)


def test_large_offsets_pass_32_bits():
    # the last rows of a tensor of more than 2^31 elements, reached through a large row stride
    T, d, ld = 70, 64, 1 << 25
    buf = torch.empty(T * ld, dtype=torch.bfloat16, device=DEV)
    x = torch.as_strided(buf, (T, d), (ld, 1))
    g = torch.Generator(device=DEV).manual_seed(9)
    dense = _mat(g, T, d)
    x.copy_(dense)
    h, y = B.npd_norm_fwd(x, None)
    h1, y1 = B.npd_norm_fwd(dense, None)
    assert torch.equal(h, h1) and torch.equal(y, y1)


def test_same_bits_every_time_on_another_stream_and_from_a_graph():
    x, r, how = _case(3000, 520, torch.float32, torch.float32, "shared", True)
    g = torch.Generator(device=DEV).manual_seed(4)
    dy, dh = _mat(g, 3000, 520), _mat(g, 3000, 520, torch.float32)
    h, y = B.npd_norm_fwd(x, r, **how)
    want = B.npd_norm_bwd(dy, h, x, dh=dh, **how)
    again = B.npd_norm_bwd(dy, h, x, dh=dh, **how)
    assert all(torch.equal(a, b) for a, b in zip(want, again))
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    h2, y2 = B.npd_norm_fwd(x, r, stream=side, **how)
    got = B.npd_norm_bwd(dy, h2, x, dh=dh, stream=side, **how)
    side.synchronize()
    assert torch.equal(h2, h) and torch.equal(y2, y) and all(torch.equal(a, b) for a, b in zip(want, got))
    graph = torch.cuda.CUDAGraph()
    xs = x.clone()
    with torch.cuda.graph(graph):
        hg, yg = B.npd_norm_fwd(xs, r, **how)
        gg = B.npd_norm_bwd(dy, hg, xs, dh=dh, **how)
    xs.copy_(x)
    for _ in range(2):
        graph.replay()
    torch.cuda.synchronize()
    assert torch.equal(hg, h) and torch.equal(yg, y) and all(torch.equal(a, b) for a, b in zip(want, gg))


# Rows of at most 256 elements share a block (4 or 2 of them a warp up to 64 and 128 elements): numbers of rows around
# a block's, widths around the limits; wider ones that end inside a vector of eight, in every size of block.
@pytest.mark.parametrize("T,d", [(1, 64), (31, 64), (33, 8), (70, 63), (129, 65), (4097, 128), (257, 121), (9, 249), (7, 255),
                                 (40, 729), (301, 1001), (5, 2051), (3, 3333), (4, 4099), (3, 6001), (2, 8190)])
@pytest.mark.parametrize("sd", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("gate,post", [("none", True), ("shared", True), ("token", True)])
def test_narrow_and_ragged_rows(T, d, sd, gate, post):
    x, r, how = _case(T, d, sd, torch.float32, gate, post, pad=8 * (T % 2))
    h, y = B.npd_norm_fwd(x, r, **how)
    _check_forward(x, r, how, h, y)
    g = torch.Generator(device=DEV).manual_seed(2)
    dy, dh = _mat(g, T, d), _mat(g, T, d, sd, pad=16)
    _check_backward(dy, h, x, dh, how, B.npd_norm_bwd(dy, h, x, dh=dh, **how))


@pytest.mark.parametrize("T,d", [(37, 40), (50, 128), (19, 250), (12, 729), (5, 4104)])
@pytest.mark.parametrize("sd", [torch.bfloat16, torch.float32])
def test_calls_with_parts_missing_at_every_size_of_block(T, d, sd):
    for gate in ("none", "shared", "token"):
        x, r, how = _case(T, d, sd, torch.bfloat16, gate, True)
        h, y = B.npd_norm_fwd(x, r, **how)
        g = torch.Generator(device=DEV).manual_seed(3)
        dy, dh = _mat(g, T, d), _mat(g, T, d, sd)
        for a, b in ((dy, None), (None, dh)):
            _check_backward(a, h, x, b, how, B.npd_norm_bwd(a, h, x, dh=b, **how))
        got = B.npd_norm_bwd(dy, h, x, dh=dh, want_dresidual=False, **how)
        assert got[1] is None
        _check_backward(dy, h, x, dh, how, got)


def test_rows_that_do_not_exist_add_nothing_without_eps():
    # a block takes more rows than the call has; their zeros have no finite reciprocal norm when eps is 0
    for T, d in ((3, 64), (9, 100), (5, 256)):
        x, r, how = _case(T, d, torch.bfloat16, torch.float32, "shared", True, eps=0.0)
        h, y = B.npd_norm_fwd(x, r, **how)
        _check_forward(x, r, how, h, y)
        g = torch.Generator(device=DEV).manual_seed(4)
        dy, dh = _mat(g, T, d), _mat(g, T, d)
        _check_backward(dy, h, x, dh, how, B.npd_norm_bwd(dy, h, x, dh=dh, **how))


def test_narrow_rows_behind_the_last_one_and_in_place():
    x, r, how = _case(21, 72, torch.float32, torch.bfloat16, "token", True)
    buf = torch.full((32, 72), 7.0, device=DEV)
    yb = torch.full((32, 72), 7.0, device=DEV, dtype=torch.bfloat16)
    h, y = B.npd_norm_fwd(x, r, **how)
    B.npd_norm_fwd(x, r, h=buf[:21], y=yb[:21], **how)
    assert torch.equal(buf[:21], h) and torch.equal(yb[:21], y) and (buf[21:] == 7).all() and (yb[21:] == 7).all()
    g = torch.Generator(device=DEV).manual_seed(5)
    dy, dh = _mat(g, 21, 72), _mat(g, 21, 72, torch.float32)
    want = B.npd_norm_bwd(dy, h, x, dh=dh, **how)
    dy1, dh1, gate1 = dy.clone(), dh.clone(), how["gate"].clone()
    got = B.npd_norm_bwd(dy1, h, x, dh=dh1, dx=dy1, dresidual=dh1, d_gate=gate1, **dict(how, gate=gate1))
    assert all(torch.equal(a, b) for a, b in zip(got, want))
