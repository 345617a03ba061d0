"""npd_linear_fwd / npd_linear_bwd against the fp64 oracle.

Tolerances.  A pre-activation is a sum of K exact products of bf16 numbers: the tensor core cuts its partial sums,
at most one unit per group of 16 addends, so it is off by at most 2 u32 (K/16 + 16) of the sum of the absolute products
(A = |x| |w|^T + |bias|).  An activation's slope is at most 1.13, and evaluating it (one exponential or erfc, a
handful of operations, arguments rounded to fp32) adds less than 64 u32 (1 + |z|) |z|-free units; then the result's
own rounding.  Products of dz (rounded to bf16) with bf16 operands: u(bf16) of each product on top."""

import numpy as np
import pytest
import torch

from oracle import npd_oracle as orc
from paper_2605_05940_b200 import binding as B

from _tolerance import host, u

pytestmark = pytest.mark.gpu
DEV = "cuda"
F32, BF16 = torch.float32, torch.bfloat16
ACTS = {"none": B.NPD_ACT_NONE, "relu": B.NPD_ACT_RELU, "gelu": B.NPD_ACT_GELU, "gelu_tanh": B.NPD_ACT_GELU_TANH,
        "silu": B.NPD_ACT_SILU}


def _mat(g, rows, cols, dtype=BF16, pad=0, std=1.0):
    ld = (cols + 7) // 8 * 8 + pad
    buf = torch.full((rows, ld), float("nan"), device=DEV, dtype=dtype)
    buf[:, :cols] = (torch.randn((rows, cols), device=DEV, generator=g) * std).to(dtype)
    return buf[:, :cols]


def _out(rows, cols, dtype, pad=8):
    return torch.full((rows, (cols + 7) // 8 * 8 + pad), float("nan"), device=DEV, dtype=dtype)


def _check_forward(x, w, b, r, act, y, z):
    X, W = host(x), host(w)
    wy, wz = orc.linear(X, W, None if b is None else host(b), None if r is None else host(r), act)
    A = np.abs(X) @ np.abs(W).T + (0.0 if b is None else np.abs(host(b)))
    ez = 2 * u(F32) * (X.shape[1] / 16 + 16) * A
    ey = 1.13 * ez + 64 * u(F32) * (1 + np.abs(wz)) + (0.0 if r is None else 4 * u(F32) * np.abs(host(r)))
    err = np.abs(host(y) - wy)
    assert np.all(err <= ey + u(y.dtype) * (np.abs(wy) + ey)), float(np.max(err / (ey + u(y.dtype) * np.abs(wy) + 1e-300)))
    if z is not None:
        assert np.all(np.abs(host(z) - wz) <= ez + u(BF16) * (np.abs(wz) + ez))


def _check_backward(dy, x, w, z, act, got, base=None):
    D, X, W = host(dy), None if x is None else host(x), host(w)
    wx, ww, wb, dz = orc.linear_backward(D, np.zeros((D.shape[0], W.shape[1])) if X is None else X, W,
                                         None if z is None else host(z), act)
    edz = 0.0 * D if act == "none" else 64 * u(F32) * np.abs(D) * (1 + np.abs(host(z)))
    rz = (0.0 if act == "none" else u(BF16)) * 1.01
    dx, dw, db = got
    if dx is not None:
        t = u(BF16) * 1.01 * np.abs(wx) + (rz + 2 * u(F32) * (D.shape[1] / 16 + 16)) * (np.abs(dz) @ np.abs(W)) + edz @ np.abs(W)
        assert np.all(np.abs(host(dx) - wx) <= t + 1e-30)
    if dw is not None:
        ref = ww if base is None else ww + base
        t = u(dw.dtype) * 1.01 * np.abs(ref) + (rz + 2 * u(F32) * (D.shape[0] / 16 + 16)) * (np.abs(dz).T @ np.abs(X)) \
            + edz.T @ np.abs(X) + (0 if base is None else 4 * u(F32) * np.abs(base))
        assert np.all(np.abs(host(dw) - ref) <= t + 1e-30)
    if db is not None:
        t = u(F32) * (D.shape[0] + 64) * np.sum(np.abs(dz), 0) + edz.sum(0)
        assert np.all(np.abs(host(db) - wb) <= t + 1e-30)


SHAPES = [(1, 1, 1), (1, 64, 64), (1, 300, 1000), (2, 17, 33), (8, 16, 31), (9, 40, 512), (16, 257, 72), (17, 15, 2000),
          (32, 1000, 264), (33, 5, 7), (33, 264, 64), (64, 256, 128), (130, 33, 200), (256, 256, 65), (257, 520, 1000),
          (300, 1001, 456), (900, 700, 520)]


@pytest.mark.parametrize("M,N,K", SHAPES)
@pytest.mark.parametrize("act", list(ACTS))
def test_forward_and_backward(M, N, K, act):
    g = torch.Generator(device=DEV).manual_seed(M * 5 + N * 3 + K)
    pad = 8 * (M % 3)
    yd = F32 if (M + N) % 3 == 0 else BF16
    x, w = _mat(g, M, K, pad=pad), _mat(g, N, K, pad=pad, std=1.5 / np.sqrt(K))
    b = torch.randn(N, device=DEV, generator=g).to(F32 if N % 2 else BF16) if M % 4 else None
    r = _mat(g, M, N, yd, pad=pad) if N % 4 else None
    ybuf, zbuf = _out(M, N, yd), _out(M, N, BF16)
    st = torch.zeros(1, dtype=torch.int32, device=DEV)
    y, z = B.npd_linear_fwd(x, w, bias=b, activation=ACTS[act], residual=r, y=ybuf[:, :N], preact=zbuf[:, :N], status=st)
    _check_forward(x, w, b, r, act, y, z)
    # nothing is written beyond the results
    assert torch.isnan(ybuf[:, N:]).all() and torch.isnan(zbuf[:, N:]).all() and int(st) == 0
    y2, none = B.npd_linear_fwd(x, w, bias=b, activation=ACTS[act], residual=r, y_dtype=yd)
    assert none is None and torch.equal(y2, y)
    dy = _mat(g, M, N, pad=8)
    dw = F32 if K % 2 else BF16
    dwb, dxb = _out(N, K, dw), _out(M, K, BF16)
    got = B.npd_linear_bwd(dy, x, w, preact=z, activation=ACTS[act], want_dbias=True, dw=dwb[:, :K], dx=dxb[:, :K])
    _check_backward(dy, x, w, z, act, got)
    assert torch.isnan(dwb[:, K:]).all() and torch.isnan(dxb[:, K:]).all()


def test_parts_of_the_backward():
    g = torch.Generator(device=DEV).manual_seed(8)
    x, w, dy, z = _mat(g, 500, 200), _mat(g, 300, 200), _mat(g, 500, 300), _mat(g, 500, 300)
    for act, zz in (("none", None), ("silu", z)):
        full = B.npd_linear_bwd(dy, x, w, preact=zz, activation=ACTS[act], want_dbias=True)
        _check_backward(dy, x, w, zz, act, full)
        kw = dict(preact=zz, activation=ACTS[act])
        dx = B.npd_linear_bwd(dy, None, w, want_dw=False, **kw)
        dw = B.npd_linear_bwd(dy, x, w, want_dx=False, **kw)
        db = B.npd_linear_bwd(dy, None, w, want_dx=False, want_dw=False, want_dbias=True, **kw)
        assert torch.equal(dx[0], full[0]) and dx[1] is None and torch.equal(dw[1], full[1]) and torch.equal(db[2], full[2])
        base = torch.randn((300, 200), device=DEV, generator=g)
        acc = base.clone()
        got = B.npd_linear_bwd(dy, x, w, dw=acc, accumulate_dw=True, **kw)
        _check_backward(dy, x, w, zz, act, got, base=host(base))
    for bad in (dict(activation=B.NPD_ACT_SILU), dict(want_dx=False, want_dw=False), dict(dw=torch.zeros_like(w), accumulate_dw=True),
                dict(dx=x)):
        with pytest.raises(B.NpdError):
            B.npd_linear_bwd(dy, x, w, **bad)


@pytest.mark.parametrize("M", [3, 200])
def test_in_place_residual_and_refusals(M):
    g = torch.Generator(device=DEV).manual_seed(M)
    x, w, r = _mat(g, M, 96), _mat(g, 136, 96), _mat(g, M, 136)
    y, _ = B.npd_linear_fwd(x, w, residual=r, activation=B.NPD_ACT_GELU)
    r1 = r.clone()
    y1, _ = B.npd_linear_fwd(x, w, residual=r1, activation=B.NPD_ACT_GELU, y=r1)
    assert y1 is r1 and torch.equal(r1, y)
    square = _mat(g, M, 136)
    for kw in (dict(y=square[:, 8:104], residual=square[:, :96]), dict(y=x), dict(preact=r, residual=r), dict(activation=5),
               dict(bias=torch.zeros(7, device=DEV)), dict(bias=torch.zeros(136, device=DEV, dtype=torch.float16)),
               dict(residual=r.float(), y=y)):
        with pytest.raises(B.NpdError):
            B.npd_linear_fwd(x, w, **kw)


@pytest.mark.parametrize("M", [1, 20, 300])
def test_bad_values_stay_in_their_row(M):
    g = torch.Generator(device=DEV).manual_seed(M)
    x, w = _mat(g, M, 200), _mat(g, 90, 200)
    y, _ = B.npd_linear_fwd(x, w, activation=B.NPD_ACT_GELU_TANH)
    x2 = x.clone()
    x2[M // 2, 7] = float("nan")
    y2, _ = B.npd_linear_fwd(x2, w, activation=B.NPD_ACT_GELU_TANH)
    keep = torch.arange(M, device=DEV) != M // 2
    assert torch.isnan(y2[M // 2]).all() and torch.equal(y2[keep], y[keep])


@pytest.mark.parametrize("act", ["gelu", "gelu_tanh", "silu", "relu"])
def test_activations_far_out(act):
    # one weight of 1: z takes the values themselves, from the smallest to the largest
    v = torch.tensor([0.0, -0.0, 1e-30, -1e-30, 1e-3, -1e-3, 1, -1, 3, -3, 6, -6, 9, -9, 14, -14, 40, -40, 200, -200, 1e4, -1e4,
                      1e19, -1e19, 3e38, -3e38], device=DEV).to(BF16)
    for rows in (1, 40):
        x = torch.zeros((rows, 8), device=DEV, dtype=BF16)
        x[:, 0] = 1
        w = torch.zeros((v.numel(), 8), device=DEV, dtype=BF16)
        w[:, 0] = v
        y, z = B.npd_linear_fwd(x, w, activation=ACTS[act], y_dtype=F32, want_preact=True)
        want, slope = orc.activation(host(v), act)
        err = np.abs(host(y) - want)
        assert np.all(err <= 64 * u(F32) * (1e-30 + np.minimum(np.abs(host(v)), 1e3) + np.abs(want))), (act, host(v)[np.argmax(err)])
        assert torch.equal(z[0], v)
        dy = torch.ones((rows, 32), device=DEV, dtype=BF16)[:, :v.numel()]
        _, _, db = B.npd_linear_bwd(dy, x, w, preact=z, activation=ACTS[act], want_dbias=True)
        assert np.all(np.abs(host(db) / rows - slope) <= 64 * u(F32) * (1 + np.minimum(np.abs(host(v)), 1e2)))


def test_same_bits_other_stream_and_graph():
    g = torch.Generator(device=DEV).manual_seed(11)
    for M in (4, 700):
        x, w, r, dy = _mat(g, M, 520), _mat(g, 600, 520), _mat(g, M, 600), _mat(g, M, 600)
        b = torch.randn(600, device=DEV, generator=g)
        kw = dict(activation=B.NPD_ACT_SILU)
        y, z = B.npd_linear_fwd(x, w, bias=b, residual=r, want_preact=True, **kw)
        want = B.npd_linear_bwd(dy, x, w, preact=z, want_dbias=True, **kw)
        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        y2, z2 = B.npd_linear_fwd(x, w, bias=b, residual=r, want_preact=True, stream=side, **kw)
        got = B.npd_linear_bwd(dy, x, w, preact=z2, want_dbias=True, stream=side, **kw)
        side.synchronize()
        assert torch.equal(y, y2) and torch.equal(z, z2) and all(torch.equal(p, q) for p, q in zip(want, got))
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            y3, z3 = B.npd_linear_fwd(x, w, bias=b, residual=r, want_preact=True, **kw)
            got = B.npd_linear_bwd(dy, x, w, preact=z3, want_dbias=True, **kw)
        graph.replay()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(y, y3) and all(torch.equal(p, q) for p, q in zip(want, got))


def test_offsets_pass_32_bits():
    # more than 2^31 results: the last rows and columns against fp64
    g = torch.Generator(device=DEV).manual_seed(13)
    M, N, K = 40011, 60008, 64
    x, w = _mat(g, M, K), _mat(g, N, K, std=0.1)
    y, z = B.npd_linear_fwd(x, w, activation=B.NPD_ACT_SILU, want_preact=True)
    for rows, cols in ((slice(M - 40, M), slice(N - 300, N)), (slice(35000, 35040), slice(0, 300))):
        _check_forward(x[rows], w[cols], None, None, "silu", y[rows, cols], z[rows, cols])
    dy = y                                    # any values: its gradient of the inputs at sampled places
    dx, _, db = B.npd_linear_bwd(dy, None, w, preact=z, activation=B.NPD_ACT_SILU, want_dw=False, want_dbias=True)
    D, Z = dy[M - 20:].double(), z[M - 20:].double()
    s = torch.sigmoid(Z)
    dz = D * s * (1 + Z * (1 - s))
    ref, big = dz @ w.double(), dz.abs() @ w.double().abs()
    # the rounding of dz, the accumulation over N, the result's rounding
    bound = u(BF16) * 1.01 * ref.abs() + (u(BF16) * 1.01 + 2 * u(F32) * (N / 16 + 64)) * big
    assert bool(((dx[M - 20:].double() - ref).abs() <= bound).all())


def test_a_large_case_against_fp64_on_the_gpu():
    g = torch.Generator(device=DEV).manual_seed(12)
    x, w, r = _mat(g, 4100, 1000), _mat(g, 2300, 1000, std=0.03), _mat(g, 4100, 2300)
    y, z = B.npd_linear_fwd(x, w, residual=r, activation=B.NPD_ACT_GELU, want_preact=True)
    Z = x.double() @ w.double().t()
    assert float((z.double() - Z).abs().max()) <= float(Z.abs().max()) * u(BF16) + 1e-4
    Y = torch.nn.functional.gelu(Z) + r.double()
    assert bool(((y.double() - Y).abs() <= u(BF16) * Y.abs() * 1.01 + 1e-4).all())
    dy = _mat(g, 4100, 2300)
    dx, dw, _ = B.npd_linear_bwd(dy, x, w)
    rel = lambda a, ref: float((a.double() - ref).norm() / ref.norm())
    assert rel(dx, dy.double() @ w.double()) < u(BF16) and rel(dw, dy.double().t() @ x.double()) < u(BF16)


def test_plain_product_leaves_what_lies_beyond_its_last_column():
    g = torch.Generator(device=DEV).manual_seed(14)
    for M, N, K in ((70, 5, 40), (300, 515, 72), (33, 1, 8)):
        a, b = _mat(g, M, K), _mat(g, N, K)
        ref = host(a) @ host(b).T
        for mode, dt in ((B.NPD_GEMM_STORE_F32, F32), (B.NPD_GEMM_ADD_F32, F32), (B.NPD_GEMM_STORE_BF16, BF16)):
            buf = _out(M, N, dt)
            buf[:, :N] = 0
            B.npd_gemm_bf16(a, b, buf[:, :N], out_mode=mode)
            assert torch.isnan(buf[:, N:]).all()
            bound = u(dt) * np.abs(ref) * 1.01 + 2 * u(F32) * (K / 16 + 16) * (np.abs(host(a)) @ np.abs(host(b)).T)
            assert np.all(np.abs(host(buf[:, :N]) - ref) <= bound)


def test_accumulation_into_a_new_dw_starts_at_zero():
    g = torch.Generator(device=DEV).manual_seed(31)
    M, N, K = 200, 264, 136
    dy, x, w = ((torch.randn(s, device=DEV, generator=g)).to(BF16) for s in ((M, N), (M, K), (N, K)))
    junk = torch.full((N, K), float("nan"), device=DEV)   # its memory is what the next tensor of this size gets
    del junk
    _, dw, _ = B.npd_linear_bwd(dy, x, w, want_dx=False, dw_dtype=torch.float32, accumulate_dw=True)
    _, plain, _ = B.npd_linear_bwd(dy, x, w, want_dx=False, dw_dtype=torch.float32)
    assert torch.equal(dw, plain)                         # one add to zero per element


@pytest.mark.parametrize("rows", [1, 40])
def test_gelu_is_right_relative_to_itself_far_out(rows):
    # z Phi(z) and its slope from z = -12.5 on, where Phi(z) is about 4e-36 and still a normal number.  Tolerance, relative to
    # the value: e^(-z^2/2) has an argument with three roundings, so z^2/2 * 3 u <= 1.5 z^2 u (2 z^2 u with the exponential's
    # own), 4 u more from the exponential instruction; the factor t P(t) beside it a fit of 1e-7 (1.7 u), the coefficients'
    # roundings (1.8 u) and the multiply-adds' (their partial sums add up to 3 P(t): 3 u), t from a denominator with two
    # roundings and a reciprocal good to 2 units (6 u, on which t P(t) depends with a power of at most 2.62: 15.7 u), three
    # products (3 u): 29.2 u, below 32 u.  u = 2^-24.
    v = torch.cat([torch.linspace(-12.5, -0.5, 97, device=DEV), torch.tensor([-12.25, -8.0, -6.0, -5.0, -4.0, -0.25, -1e-3], device=DEV)]).to(BF16)
    x = torch.zeros((rows, 8), device=DEV, dtype=BF16)
    x[:, 0] = 1
    w = torch.zeros((v.numel(), 8), device=DEV, dtype=BF16)
    w[:, 0] = v
    V = host(v)
    want, slope = orc.activation(V, "gelu")
    rel = (32 + 2 * V * V) * u(F32)
    for dt in (F32, BF16):
        y, z = B.npd_linear_fwd(x, w, activation=B.NPD_ACT_GELU, y_dtype=dt, want_preact=True)
        assert torch.equal(z[0], v)
        assert np.all(np.abs(host(y) - want) <= np.abs(want) * (rel + u(dt) * (1 + rel))), dt
    _, _, db = B.npd_linear_bwd(torch.ones((1, 104), device=DEV, dtype=BF16), x[:1], w, preact=z[:1], activation=B.NPD_ACT_GELU,
                                want_dbias=True)
    # Phi(z) and z phi(z) have opposite signs
    phi = np.exp(-0.5 * V * V) / np.sqrt(2 * np.pi)
    assert np.all(np.abs(host(db) - slope) <= rel * (want / V + np.abs(V) * phi) + u(F32) * np.abs(slope))
