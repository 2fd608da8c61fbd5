"""Group norm, label log probabilities and AdamW on the GPU at values (not shapes) where they can go wrong.

Tolerances count roundings as in test_gpu_operators.py."""
import numpy as np
import pytest
import torch

from tests import plain_ops as po
from tests.test_gpu_operators import U, assert_near, dat, gn_check_backward, gn_check_forward, gn_inputs, half, host, randn  # noqa: F401 (dat: fixture)

pytestmark = pytest.mark.gpu


# ---- group norm -------------------------------------------------------------------------------------------------------
def silu_check_backward(x, dy, gamma, beta, mean, rstd, G, out):
    """As gn_check_backward, with a bound for SiLU that holds element by element: z = xhat gamma + beta is off by 4 U (|xhat gamma| +
    |beta|) and moves SiLU' by at most half of that; s, 1 - s and their products in s (1 + z (1 - s)) lose at most 16 roundings of
    1 + |z| (bf16's exponent is rounded, |z| U of e^-z, which s (1 - s) (1 + |z|) |z| <= 1 outweighs)."""
    B, H, W, C = x.shape
    xs, ds, g, b, m, r = (host(t) for t in (x, dy, gamma, beta, mean, rstd))
    dx, dg, db, size, sg, sb = po.gn_backward(xs, ds, g, b, m, r, G, 2)
    m, r = (po._spread(t, C) for t in (m, r))
    xhat = (xs - m) * r
    dz = np.abs(ds) * (16 + 18 * (np.abs(xhat * g) + np.abs(b))) * U

    def group_mean(v):
        return po._spread(v.reshape(B, -1, G, C // G).mean(axis=(1, 3)), C)

    h = np.abs(g) * dz
    moved = r * (h + group_mean(h) + np.abs(xhat) * group_mean(h * np.abs(xhat)))
    K = H * W * C // G / 64 + 32
    assert_near(host(out[0]), dx, moved + K * size * U + half(x.dtype) * 1.01 * (np.abs(dx) + moved), "dx")
    K = B * H * W / 64 + B + 32
    assert_near(host(out[1]), dg, (dz * np.abs(xhat)).sum(axis=(0, 1, 2)) + K * sg * U, "dgamma")
    assert_near(host(out[2]), db, dz.sum(axis=(0, 1, 2)) + K * sb * U, "dbeta")


# resident in vectors (with pixels left over for the last round), split in vectors, single elements
SILU_SHAPES = [(2, 9, 9, 40, 5), (3, 15, 15, 512, 32), (1, 128, 128, 64, 2), (2, 9, 9, 35, 7)]


@pytest.mark.parametrize("gamma_size", [3.0, 30.0])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("shape", SILU_SHAPES)
def test_group_norm_silu_far_from_zero(dat, shape, dtype, gamma_size):  # noqa: F811
    """z from -200 to 200 (and what gamma adds): beside e^-z that is no fp32 number, and beside a sigmoid that is below the least."""
    C, G = shape[3], shape[4]
    x, gamma, _, dy = gn_inputs(shape, dtype, 300)
    gamma, beta = gamma * gamma_size, torch.linspace(-200, 200, C, device="cuda")[torch.randperm(C, generator=torch.Generator().manual_seed(1)).cuda()]
    out = dat.group_norm_forward(x, gamma, beta, G, 2)
    gn_check_forward(dat, x, gamma, beta, G, 2, out)
    silu_check_backward(x, dy, gamma, beta, out[1], out[2], G, dat.group_norm_backward(x, dy, gamma, beta, out[1], out[2], G, 2))


def test_group_norm_silu_of_huge_values(dat):  # noqa: F811
    """SiLU of a z of any size: z for a large one, nothing for a small one."""
    x = torch.tensor([-1.0, 1.0], device="cuda").repeat(32).view(1, 4, 4, 4)
    for dtype in (torch.float32, torch.bfloat16):
        for size in (89.0, 104.0, 130.0, 1e4, 1e20, 1e38):
            gamma = torch.full((4,), size, device="cuda")
            y = host(dat.group_norm_forward(x.to(dtype), gamma, torch.zeros_like(gamma), 1, 2)[0]).reshape(-1)
            # (mean 0, variance 1: z = +-size, but for eps and roundings, 1e-5 of it)
            assert (np.abs(y[0::2]) <= size * 2.0 ** -100).all() and (np.abs(y[1::2] - size) <= (1e-5 + half(dtype)) * size).all(), (dtype, size)


# (all resident, all with threads beyond the last pixel)
@pytest.mark.parametrize("shape", [(2, 9, 9, 40, 5), (3, 15, 15, 512, 32), (1, 1, 1, 64, 8), (2, 30, 30, 64, 16), (5, 7, 7, 64, 32)])
@pytest.mark.parametrize("act", [0, 1, 2])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_group_norm_backward_with_far_means(dat, shape, act, dtype):  # noqa: F811
    """Means of many spreads, where z of a zero lies far from every value's: threads beyond the last pixel hold zeros."""
    B, H, W, C, G = shape
    _, gamma, beta, dy = gn_inputs(shape, dtype, 400)
    for means in (90.0, 95.0, 110.0, 125.0, 1000.0):
        for sign in (1, -1):
            x = (sign * means + randn(401, B, H, W, C)).to(dtype)
            _, mean, rstd = dat.group_norm_forward(x, gamma, beta, G, act)
            out = dat.group_norm_backward(x, dy, gamma, beta, mean, rstd, G, act)
            if act == 2:
                silu_check_backward(x, dy, gamma, beta, mean, rstd, G, out)
            else:
                gn_check_backward(dat, x, dy, gamma, beta, mean, rstd, G, act, out)


@pytest.mark.parametrize("act", [0, 1, 2])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_group_norm_backward_of_large_constants(dat, dtype, act):  # noqa: F811
    """Every value 2^120: xhat = 0 and rstd = 1/sqrt(eps), but mean rstd is no fp32 number."""
    shape, G = (2, 1, 2, 64, 8), 8
    _, gamma, beta, dy = gn_inputs(shape, dtype, 410)
    for sign in (1.0, -1.0):
        x = torch.full(shape[:4], sign * 2.0 ** 120, device="cuda").to(dtype)
        _, mean, rstd = dat.group_norm_forward(x, gamma, beta, G, act)
        assert (mean == sign * 2.0 ** 120).all()
        out = dat.group_norm_backward(x, dy, gamma, beta, mean, rstd, G, act)
        if act == 2:
            silu_check_backward(x, dy, gamma, beta, mean, rstd, G, out)
        else:
            gn_check_backward(dat, x, dy, gamma, beta, mean, rstd, G, act, out)
