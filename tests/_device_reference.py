"""Plain 64-bit forms of the operators around the loss step, on the GPU: for sizes at which a block goes through its loop
several times.  Written from the definitions; beside each value stands the size of what was added up for it.

`near` counts as tests/_tolerance.py does: the result's own rounding, and `steps` fp32 roundings of that size."""

import torch

F32 = torch.float32


def u(dtype):
    return torch.finfo(dtype).eps / 2


def f64(t):
    return None if t is None else t.double()


def near(got, want, size, steps, what="", extra=0.0):
    err = (got.double() - want).abs()
    bound = u(got.dtype) * want.abs() * (1 + 2 * steps * u(F32)) + steps * u(F32) * size + extra
    bound = bound + torch.finfo(got.dtype).smallest_normal * torch.finfo(got.dtype).eps
    bad = ~(err <= bound)
    if bool(bad.any()):
        at = tuple(int(v) for v in bad.nonzero()[0])
        raise AssertionError(f"{what}: {int(bad.sum())} of {bad.numel()} outside, first at {at}: got {float(got[at])!r}, want "
                             f"{float(want[at])!r}, bound {float(torch.as_tensor(bound).expand_as(err)[at]):.3e}")


def _recip(v, eps):
    return 1.0 / torch.sqrt((v * v).mean(1, keepdim=True) + eps)


def norm_forward(x, residual, *, gate=None, post_weight=None, pre_weight=None, post_norm=False, eps=1e-6, weight_offset=0.0,
                 residual_scale=1.0, branch_scale=1.0):
    """(h, size of h's addends, y, size of y)."""
    n = torch.zeros(1, dtype=torch.float64, device="cuda")
    if x is not None:
        n = f64(x)
        if post_norm:
            n = n * _recip(n, eps) * (1.0 if post_weight is None else f64(post_weight) + weight_offset)
        n = branch_scale * n * (1.0 if gate is None else f64(gate))
    r = torch.zeros(1, dtype=torch.float64, device="cuda") if residual is None else residual_scale * f64(residual)
    h = r + n
    size = r.abs() + n.abs()
    q = _recip(h, eps) * (1.0 if pre_weight is None else f64(pre_weight) + weight_offset)
    return h, size, h * q, size * q.abs() + (h * q).abs()


def norm_backward(dy, h, x, *, dh=None, gate=None, post_weight=None, pre_weight=None, post_norm=False, eps=1e-6,
                  weight_offset=0.0, residual_scale=1.0, branch_scale=1.0):
    """{name: (value, size)}; d_gate per token."""
    out = {}
    zero = torch.zeros(1, dtype=torch.float64, device="cuda")
    total, big = (zero, zero) if dh is None else (f64(dh), f64(dh).abs())
    if dy is not None:
        H, D = f64(h), f64(dy)
        r = _recip(H, eps)
        g = D * (1.0 if pre_weight is None else f64(pre_weight) + weight_offset)
        total = total + r * (g - H * r * r * (g * H).mean(1, keepdim=True))
        big = big + r * (g.abs() + H.abs() * r * r * (g * H).abs().mean(1, keepdim=True))
        out["d_pre_weight"] = ((D * H * r).sum(0), (D * H * r).abs().sum(0))
    out["dresidual"] = (residual_scale * total, abs(residual_scale) * big)
    if x is None:
        return out
    X = f64(x)
    rx = _recip(X, eps) if post_norm else 1.0
    w = 1.0 if post_weight is None or not post_norm else f64(post_weight) + weight_offset
    b = branch_scale
    a = lambda t: t.abs() if torch.is_tensor(t) else abs(t)
    out["d_gate"] = (b * total * X * rx * w, abs(b) * big * (X * rx).abs() * a(w))
    G = 1.0 if gate is None else f64(gate)
    out["d_post_weight"] = ((b * total * G * X * rx).sum(0), (abs(b) * big * a(G) * (X * rx).abs()).sum(0))
    v, vs = b * total * G * w, abs(b) * big * a(G) * a(w)
    if post_norm:
        out["dx"] = (rx * (v - X * rx * rx * (v * X).mean(1, keepdim=True)),
                     rx * (vs + X.abs() * rx * rx * (vs * X.abs()).mean(1, keepdim=True)))
    else:
        out["dx"] = (v, vs)
    return out


def activation(z, name):
    """Value and slope."""
    if name == "none":
        return z, torch.ones_like(z)
    if name == "relu":
        return z.clamp(min=0.0), (z > 0).double()
    if name == "silu":
        s = torch.sigmoid(z)
        return z * s, s * (1 + z * (1 - s))
    if name == "gelu":
        c = 0.5 * torch.special.erfc(-z * 0.5 ** 0.5)
        return z * c, c + z * torch.exp(-0.5 * z * z) * 0.3989422804014327
    k = 0.7978845608028654
    t = torch.tanh(k * (z + 0.044715 * z ** 3))
    return 0.5 * z * (1 + t), 0.5 * (1 + t) + 0.5 * z * (1 - t * t) * k * (1 + 3 * 0.044715 * z * z)
