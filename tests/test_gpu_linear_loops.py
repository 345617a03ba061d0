"""npd_linear_fwd / npd_linear_bwd at sizes that reach what small ones do not: tiles of every width with bias, residual
and both result types, several rows per warp in the pass that forms dz, and more tiles than CTA pairs in both
products of the backward.  Against 64 bits on the GPU; tolerances as derived in test_gpu_linear.py."""

import pytest
import torch

from paper_2605_05940_b200 import binding as B

from _device_reference import activation, u

pytestmark = pytest.mark.gpu
DEV, BF16, F32 = "cuda", torch.bfloat16, torch.float32
ACTS = {"none": B.NPD_ACT_NONE, "relu": B.NPD_ACT_RELU, "gelu": B.NPD_ACT_GELU, "gelu_tanh": B.NPD_ACT_GELU_TANH,
        "silu": B.NPD_ACT_SILU}


def _mat(g, rows, cols, dtype=BF16, pad=0, std=1.0):
    ld = (cols + 7) // 8 * 8 + pad
    buf = torch.full((rows, ld), float("nan"), device=DEV, dtype=dtype)
    buf[:, :cols] = (torch.randn((rows, cols), device=DEV, generator=g) * std).to(dtype)
    return buf[:, :cols]


def _out(rows, cols, dtype):
    return torch.full((rows, (cols + 7) // 8 * 8 + 8), float("nan"), device=DEV, dtype=dtype)


def _inside(got, want, bound, what):
    err = (got.double() - want).abs()
    bad = ~(err <= bound + 1e-30)
    assert not bool(bad.any()), (what, int(bad.sum()), tuple(int(v) for v in bad.nonzero()[0]), float((err / (bound + 1e-30)).max()))


def _check_forward(x, w, b, r, act, y, z):
    X, W = x.double(), w.double()
    wz, A = X @ W.t(), X.abs() @ W.abs().t()
    if b is not None:
        wz, A = wz + b.double(), A + b.double().abs()
    wy = activation(wz, act)[0]
    ez = 2 * u(F32) * (X.shape[1] / 16 + 16) * A
    ey = 1.13 * ez + 64 * u(F32) * (1 + wz.abs())
    if r is not None:
        wy, ey = wy + r.double(), ey + 4 * u(F32) * r.double().abs()
    _inside(y, wy, ey + u(y.dtype) * (wy.abs() + ey), "y")
    if z is not None:
        _inside(z, wz, ez + u(BF16) * (wz.abs() + ez), "z")


def _check_backward(dy, x, w, z, act, got):
    D, W = dy.double(), w.double()
    dz, edz = D, 0.0 * D
    if act != "none":
        dz = D * activation(z.double(), act)[1]
        edz = 64 * u(F32) * D.abs() * (1 + z.double().abs())
    rz = 0.0 if act == "none" else u(BF16) * 1.01
    M, N = D.shape
    dx, dw, db = got
    if dx is not None:
        want = dz @ W
        _inside(dx, want, u(BF16) * 1.01 * want.abs() + (rz + 2 * u(F32) * (N / 16 + 16)) * (dz.abs() @ W.abs()) + edz @ W.abs(), "dx")
    if dw is not None:
        X = x.double()
        want = dz.t() @ X
        _inside(dw, want, u(dw.dtype) * 1.01 * want.abs() + (rz + 2 * u(F32) * (M / 16 + 16)) * (dz.abs().t() @ X.abs())
                + edz.t() @ X.abs(), "dw")
    if db is not None:
        # per thread over at most M / 8 rows of its block, then 8 warps and the blocks of rows: at most M / 8 + 64
        _inside(db, dz.sum(0), u(F32) * (M / 8 + 64) * dz.abs().sum(0) + edz.sum(0), "dbias")


# with 74 CTA pairs the first takes tiles 64 columns wide, the second and third 128, the others 256
@pytest.mark.parametrize("M,N,K", [(300, 1500, 520), (500, 3000, 200), (129, 9001, 72), (1000, 9000, 72), (4100, 2300, 136),
                                   (4097, 2315, 65)])
@pytest.mark.parametrize("yd", [BF16, F32])
@pytest.mark.parametrize("keep", [False, True])
def test_every_tile_width_with_bias_and_residual(M, N, K, yd, keep):
    g = torch.Generator(device=DEV).manual_seed(M + N + K)
    x, w = _mat(g, M, K, pad=8), _mat(g, N, K, std=1.5 / K ** 0.5)
    for act in ACTS:
        for bd, res in ((F32, True), (BF16, True), (F32, False)):
            b = torch.randn(N, device=DEV, generator=g).to(bd)
            r = _mat(g, M, N, yd) if res else None
            ybuf, zbuf = _out(M, N, yd), _out(M, N, BF16)
            y, z = B.npd_linear_fwd(x, w, bias=b, activation=ACTS[act], residual=r, y=ybuf[:, :N], preact=zbuf[:, :N] if keep else None)
            _check_forward(x, w, b, r, act, y, z)
            assert torch.isnan(ybuf[:, N:]).all() and torch.isnan(zbuf[:, N:]).all()


@pytest.mark.parametrize("M,N,K", [(20011, 1001, 72), (20000, 1024, 64), (60001, 130, 40)])
@pytest.mark.parametrize("act", list(ACTS))
def test_many_rows_per_warp_of_the_slopes(M, N, K, act):
    g = torch.Generator(device=DEV).manual_seed(M)
    dy, x, w, z = _mat(g, M, N, pad=8), _mat(g, M, K), _mat(g, N, K, std=0.3), _mat(g, M, N, std=2.0)
    kw = dict(preact=z if act != "none" else None, activation=ACTS[act])
    got = B.npd_linear_bwd(dy, x, w, want_dbias=True, dw_dtype=F32, **kw)
    _check_backward(dy, x, w, z, act, got)
    alone = B.npd_linear_bwd(dy, None, w, want_dx=False, want_dw=False, want_dbias=True, **kw)
    assert torch.equal(alone[2], got[2])


# tiles of 256 x 512 for more than one round of the 74 CTA pairs, the longer contraction in dw or in dx; some pairs take one
# more of the long tiles and fewer of the short ones (the last case: 24 long tiles, 632 short ones)
@pytest.mark.parametrize("M,N,K", [(6000, 5000, 2056), (5001, 6003, 2500), (9000, 2100, 5000), (2100, 9000, 5000), (20000, 600, 4000)])
@pytest.mark.parametrize("act", ["none", "silu"])
def test_more_tiles_than_pairs_in_the_backward(M, N, K, act):
    g = torch.Generator(device=DEV).manual_seed(M + N)
    dy, x, w, z = _mat(g, M, N), _mat(g, M, K, pad=8), _mat(g, N, K, std=0.03), _mat(g, M, N)
    dxb, dwb = _out(M, K, BF16), _out(N, K, BF16)
    got = B.npd_linear_bwd(dy, x, w, preact=z if act != "none" else None, activation=ACTS[act], want_dbias=True, dx=dxb[:, :K],
                           dw=dwb[:, :K])
    _check_backward(dy, x, w, z, act, got)
    assert torch.isnan(dxb[:, K:]).all() and torch.isnan(dwb[:, K:]).all()


@pytest.mark.parametrize("M", [1, 8, 9, 16, 17, 32])
@pytest.mark.parametrize("N,K", [(1536, 6144), (6144, 1536), (4099, 4104), (40, 16384)])
def test_few_rows_with_long_contractions(M, N, K):
    g = torch.Generator(device=DEV).manual_seed(M + N + K)
    x, w, r = _mat(g, M, K), _mat(g, N, K, std=1.0 / K ** 0.5), _mat(g, M, N)
    b = torch.randn(N, device=DEV, generator=g)
    y, z = B.npd_linear_fwd(x, w, bias=b, activation=B.NPD_ACT_GELU, residual=r, want_preact=True)
    _check_forward(x, w, b, r, "gelu", y, z)
