"""Tolerances of the tests of the operators around the loss step, from the arithmetic.

u(t) = torch.finfo(t).eps / 2 is the most a rounding to type t is off, relative to the value.
A result stored in type t is off by u(t) of itself; before that it was computed in fp32, whose error is
counted as F32 fp32 roundings of the largest quantities that were added up (`scale`, given by the test:
for a sum, the sum of the absolute values).  Elementwise: |got - want| <= u(t) |want| + F32 u(f32) scale.
"""

import numpy as np
import torch


def u(dtype):
    return torch.finfo(dtype).eps / 2


def host(t):
    return t.detach().to(torch.float64).cpu().numpy()


def assert_rounded(got, want, scale, f32_steps, what=""):
    """`got` (a tensor) is `want` (fp64) up to its own type's rounding and `f32_steps` fp32 roundings of `scale`."""
    g, want = host(got), np.asarray(want, np.float64)
    bound = u(got.dtype) * np.abs(want) * (1 + 2 * f32_steps * u(torch.float32)) + \
        f32_steps * u(torch.float32) * np.broadcast_to(np.asarray(scale, np.float64), want.shape)
    # below the smallest normal value of the type a rounding is off by half of the smallest subnormal
    bound = bound + torch.finfo(got.dtype).smallest_normal * torch.finfo(got.dtype).eps
    bad = ~(np.abs(g - want) <= bound)
    assert not bad.any(), (f"{what}: {int(bad.sum())} of {bad.size} outside; first at "
                           f"{tuple(int(v[0]) for v in np.nonzero(bad))}, got {g[bad][0]!r}, want {want[bad][0]!r}, "
                           f"bound {bound[bad][0]:.3e}")
