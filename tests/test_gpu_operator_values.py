"""Group norm, label log probabilities and AdamW on the GPU at values (not shapes) where they can go wrong: activations far from
zero, means far from the values' spread, sums next to the end of the range, logits with a large common offset.

Tolerances count roundings as in test_gpu_operators.py."""
import numpy as np
import pytest
import torch

from tests import plain_ops as po
from tests.test_gpu_operators import U, assert_near, dat, gn_check_backward, gn_check_forward, gn_inputs, half, host, lp_check, lp_rows, randn  # noqa: F401 (dat: fixture)

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


@pytest.mark.parametrize("shape", [(2, 9, 9, 40, 5), (3, 28, 28, 64, 32), (2, 8, 8, 64, 64), (1, 128, 128, 64, 2), (2, 9, 9, 35, 7), (1, 300, 300, 3, 1)])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_group_norm_sums_stay_in_range(dat, shape, dtype):  # noqa: F811
    """Values of 1e37 and 3e38, all alike: their sums are no fp32 numbers, their mean is, and nothing is left of their deviations from it but
    the mean's rounding, whose square is none either: rstd = 0 (or 1/sqrt(eps) where the mean is exact), and y = beta both times."""
    B, H, W, C, G = shape
    _, gamma, beta, _ = gn_inputs(shape, dtype, 420)
    for size in (1e37, -3e38):
        x = torch.full(shape[:4], size, device="cuda").to(dtype)
        y, mean, rstd = dat.group_norm_forward(x, gamma, beta, G, 0)
        want = float(x.view(-1)[0])
        assert_near(host(mean), np.full((B, G), want), (H * W * C // G / 64 + 32) * U * abs(want), "mean")
        assert torch.equal(y, beta.expand(shape[:4]).to(dtype)) and torch.isfinite(rstd).all()


@pytest.mark.parametrize("shape", [(2, 9, 9, 40, 5), (3, 28, 28, 64, 32), (3, 20, 20, 64, 16), (2, 56, 56, 64, 8), (2, 56, 56, 64, 32), (1, 56, 56, 256, 4),
                                   (2, 100, 100, 64, 8), (1, 128, 128, 32, 1)])
@pytest.mark.parametrize("offset", [0.0, 1.0, 1.8, 1.99, 2.01, 2.2])
def test_group_norm_bf16_variance_of_large_groups(dat, shape, offset):  # noqa: F811
    """Statistics within what a thread really adds: 16 vectors (a dot product of a pair rounds twice), then at most 64 terms in LDS and
    trees of 6 and 6 lanes, 4 for shares and the square; both sides of the change from E x^2 - mean^2, which multiplies the sums' relative
    error by (var + mean^2) / var + 2 |mean| E|x| / var <= 5 + 4 sqrt 5 < 14."""
    B, H, W, C, G = shape
    Cg = C // G
    entries = 1 if Cg % 8 == 0 else 8 // Cg if Cg > 1 and 8 % Cg == 0 else 8
    K = 128 / entries + 64 + 16
    x = (randn(430, B, H, W, C) + offset).to(torch.bfloat16)
    _, mean, rstd = dat.group_norm_forward(x, None, None, G, 0)
    m, r = po.gn_stats(host(x), G, 1e-5)
    size = np.abs(host(x)).reshape(B, -1, G, Cg).mean(axis=(1, 3))
    assert_near(host(mean), m, K * U * size, "mean")
    assert_near(host(rstd), r, (14 * K / 2 + 4) * U * r, "rstd")


@pytest.mark.parametrize("shape", [(40, 9, 9, 40, 5), (40, 28, 28, 64, 32), (40, 56, 56, 64, 8), (40, 56, 56, 64, 32), (40, 15, 17, 96, 4), (40, 100, 100, 64, 8),
                                   (40, 128, 128, 32, 1), (40, 23, 29, 35, 7), (40, 100, 101, 6, 2)])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_group_norm_counts_every_value(dat, shape, dtype):  # noqa: F811
    """Groups of zeros with a single one, at another pixel of every image (the first and last ones among them): what a sum leaves out or
    counts twice is all of it.  eps = 0: rstd = 1 / sqrt((1 - 1/n) / n)."""
    B, H, W, C, G = shape
    P, Cg = H * W, C // G
    n = P * Cg
    gen = torch.Generator().manual_seed(3)
    pixel = torch.cat([torch.arange(10), torch.arange(P - 10, P), torch.randint(0, P, (B - 20,), generator=gen)])
    channel = torch.randint(0, Cg, (B, G), generator=gen) + Cg * torch.arange(G)[None, :]
    x = torch.zeros(B, P, C)
    x[torch.arange(B)[:, None], pixel[:, None], channel] = 1.0
    x = x.view(shape[:4]).cuda().to(dtype)
    _, mean, rstd = dat.group_norm_forward(x, None, None, G, 0, eps=0.0)
    assert_near(host(mean), np.full((B, G), 1.0 / n), 4 * U / n, "mean")
    want = 1 / np.sqrt((1 - 1 / n) / n)
    # (the zeros' deviations have 1/n of the sum: their roundings, at most n of them, are U of it)
    assert_near(host(rstd), np.full((B, G), want), 16 * U * want, "rstd")
    _, dgamma, dbeta = dat.group_norm_backward(x, x, None, None, mean, rstd, G, 0)
    count = x.float().sum(dim=(0, 1, 2))
    assert torch.equal(dbeta, count)                                     # (small whole numbers: exact)
    assert_near(host(dgamma), host(count) * (1 - 1 / n) * want, (B + 16) * U * host(count) * want, "dgamma")


@pytest.mark.parametrize("shape", [(3, 14, 14, 64, 16), (1, 128, 128, 64, 2), (2, 9, 9, 35, 7)])
def test_group_norm_gradient_in_place_of_the_input(dat, shape):  # noqa: F811
    G = shape[4]
    x, gamma, beta, dy = gn_inputs(shape, torch.bfloat16, 440)
    _, mean, rstd = dat.group_norm_forward(x, gamma, beta, G, 2)
    want = dat.group_norm_backward(x, dy, gamma, beta, mean, rstd, G, 2)
    own = x.clone()
    got = dat.group_norm_backward(own, dy, gamma, beta, mean, rstd, G, 2, dx=own)
    assert got[0] is own and all(torch.equal(a, b) for a, b in zip(got, want))


@pytest.mark.parametrize("shape", [(5, 1, 1, 64, 64), (98, 1, 1, 320, 320), (5, 1, 1, 35, 35)])
@pytest.mark.parametrize("act", [0, 1, 2])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_group_norm_of_single_values(dat, shape, act, dtype):  # noqa: F811
    """A group of one value: y = act(beta) whatever the value, so its gradient is 0, and the scale's."""
    x, gamma, beta, dy = gn_inputs(shape, dtype, 460)
    y, mean, rstd = dat.group_norm_forward(x, gamma, beta, shape[4], act)
    assert_near(host(y), np.broadcast_to(po.gn_act(host(beta), act), shape[:4]), (half(dtype) + 16 * U) * (np.abs(host(beta)) + 1), "y")
    dx, dgamma, dbeta = dat.group_norm_backward(x, dy, gamma, beta, mean, rstd, shape[4], act)
    assert int(torch.count_nonzero(dx)) == 0 and int(torch.count_nonzero(dgamma)) == 0 and torch.isfinite(dx).all()
    slope = torch.ones_like(beta) if act == 0 else (beta > 0).float() if act == 1 else torch.sigmoid(beta) * (1 + beta * (1 - torch.sigmoid(beta)))
    terms = dy.float()[:, 0, 0] * slope
    assert_near(host(dbeta), host(terms.double().sum(dim=0)), 64 * U * host(terms.abs().sum(dim=0)) + 32 * U, "dbeta")
    x[1, 0, 0, 3], x[2, 0, 0, 4] = float("nan"), float("inf")
    y, mean, rstd = dat.group_norm_forward(x, gamma, beta, shape[4], act)
    dx = dat.group_norm_backward(x, dy, gamma, beta, mean, rstd, shape[4], act)[0]
    bad = torch.zeros(shape[:4], dtype=torch.bool, device="cuda")
    bad[1, 0, 0, 3] = bad[2, 0, 0, 4] = True
    assert torch.isnan(dx[bad]).all() and int(torch.count_nonzero(dx[~bad])) == 0


# ---- log probabilities ---------------------------------------------------------------------------------------------
def lp_check_gradient(x, labels, a, b, dx):
    """Against the softmax's own gradient.  log p is off by (K + 4 log V) U from the sum, by 2 U |lse| where it comes from an lse of at
    most 64 in size, and by 4 U of itself; p by that and 4 U."""
    want, p, q, H = po.softmax_gradient(host(x), labels.cpu().numpy(), host(a), host(b))
    V = x.shape[1]
    hot = np.arange(V)[None, :] == labels.cpu().numpy()[:, None]
    a, b, H = np.abs(host(a))[:, None], np.abs(host(b))[:, None], H[:, None]
    K = V / 64 + 24 + 4 * np.log(V) + 4
    with np.errstate(invalid="ignore"):
        q = np.where(p > 0, np.abs(q), 0.0)
    off = (K + 128 + 4 * q) * U
    tol = a * (p * off + 2 * U * (hot + p)) + b * p * (off * (q + H + 1) + 3 * (K + 4) * (np.log(V) + 1) * U + 2 * U * (q + H))
    tol += (a + 200 * b) * 2.0 ** -126 + half(dx.dtype) * 1.01 * (np.abs(want) + tol)
    assert_near(host(dx), want, tol, "dlogits")


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("N,V", [(41, 1), (41, 2), (300, 5), (41, 16), (41, 17), (41, 64), (41, 65), (41, 128), (41, 129), (41, 256), (41, 257), (41, 1000),
                                 (41, 4099), (41, 9001), (41, 70001)])
def test_log_probs_gradient_beside_large_offsets(dat, N, V, dtype):  # noqa: F811
    """Rows that a common offset moves far from zero, up to rows of the type's lowest and largest value: p is that of the softmax."""
    low, high, inf = torch.finfo(dtype).min, torch.finfo(dtype).max, float("inf")
    x = randn(500 + V, N, V)
    offsets = [0.0, 30.0, 57.0, 63.9, 64.1, 90.0, 1e3, 3e4, 1e6, 1e12, 1e30]
    for n in range(N):
        o = offsets[(n // 2) % len(offsets)]
        step = max(o * (half(dtype) * 2), 2.0 ** -6) if o >= 1e3 else 1.0       # values that differ by a few steps of the type
        x[n] = (x[n] * step + o) * (1 if n % 2 else -1)
    x[22], x[23], x[24], x[25] = low, high, 3e38, -3e38
    x[26], x[27], x[28] = 1e6, -1e6, 65.0                                       # all alike
    x[29] = torch.where(torch.arange(V, device="cuda") % 3 == 1, low, 1e5)      # masked by the lowest value, by -inf
    x[30] = torch.where(torch.arange(V, device="cuda") % 3 == 1, -inf, 1e5)
    x[31] = torch.where(torch.arange(V, device="cuda") % 3 == 1, -inf, low)
    x[32] = torch.where(torch.arange(V, device="cuda") % 2 == 1, low, high)
    x[33] = -inf
    x[34, V // 2], x[35, 0] = float("nan"), inf
    labels = torch.randint(0, V, (N,), dtype=torch.int32, device="cuda", generator=torch.Generator(device="cuda").manual_seed(1))
    a, b = randn(501, N), randn(502, N)
    for ld in (V, V + 5):
        z = torch.full((N, ld), 7.0, dtype=dtype, device="cuda")[:, :V].copy_(x)
        _, H, lse, _, _ = dat.log_probs(z, labels)
        dx = dat.log_probs_backward(z, labels, lse, H, a, b)
        lp_check_gradient(z, labels, a, b, dx)
        assert float(dx[33].abs().max()) == 0.0 and torch.isnan(dx[34:36]).all()
        zero = torch.zeros_like(a)
        lp_check_gradient(z, labels, a, zero, dat.log_probs_backward(z, labels, lse, None, a, None))
        lp_check_gradient(z, labels, zero, b, dat.log_probs_backward(z, None, lse, H, None, b))
        own = torch.full((N, ld), 7.0, dtype=dtype, device="cuda")              # in place, rows apart
        own[:, :V] = z
        dat.log_probs_backward(own[:, :V], labels, lse, H, a, b, dlogits=own[:, :V])
        assert torch.equal(own[:, :V].nan_to_num(5.0), dx.nan_to_num(5.0)) and (own[:, V:] == 7.0).all()


@pytest.mark.parametrize("V", [3, 700, 9001, 70000])
def test_log_probs_special_rows_both_directions(dat, V):  # noqa: F811
    """Rows that hold nothing, one class, NaN, infinities, the lowest and the largest values, and labels out of range."""
    inf, nan = float("inf"), float("nan")
    x, labels = lp_rows(77, 10, V, torch.float32)
    x[0] = x[1] = -inf
    x[1, V // 2] = -3.0
    x[2, V - 1], x[3, 0] = nan, inf
    x[4] = torch.finfo(torch.float32).min
    x[5, : V - 1] = torch.finfo(torch.float32).min
    x[6, labels[6]] = -inf
    x[7], x[8] = 3e38, -1e-40
    labels[1] = V // 2
    for outside in (V, -1):
        labels[9] = outside
        for top in (2, min(V, 6)):
            out = dat.log_probs(x, labels, top)
            lp_check(x, labels, top, out)
        a, b = randn(5, 10), randn(6, 10)
        dx = dat.log_probs_backward(x, labels, out[2], out[1], a, b)
        lp_check_gradient(x, labels, a, b, dx)
        assert float(dx[0].abs().max()) == 0.0 and torch.isnan(dx[2:4]).all()


@pytest.mark.parametrize("V", [10, 16, 17, 63, 64, 65, 256, 257, 1000, 1025, 8193, 50021, 131075])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_log_probs_counts_every_logit(dat, V, dtype):  # noqa: F811
    """One logit of 0 among logits of -64 (e^-64 < 2^-92), at the first and last places and elsewhere: it is the whole sum, in few rows
    (parts of a row, a workgroup) and in many (lanes of a wavefront)."""
    at = torch.cat([torch.arange(min(V, 17)), torch.arange(max(0, V - 17), V), torch.randint(0, V, (30,), generator=torch.Generator().manual_seed(V))])
    few = len(at)
    for repeat in (1, 20 if V <= 1024 else 1):
        where = at.repeat(repeat).cuda()
        N = few * repeat
        for ld in (V, V + 3):
            x = torch.full((N, ld), 7.0, dtype=dtype, device="cuda")[:, :V].fill_(-64.0)
            x[torch.arange(N, device="cuda"), where] = 0.0
            labels = where.to(torch.int32)
            logp, H, lse, tl, ti = dat.log_probs(x, labels, 1)
            for t in (logp, lse, tl):
                assert float(t.abs().max()) <= 2 * U
            assert torch.equal(ti[:, 0], labels) and float(H.abs().max()) <= 2 * U
            dx = dat.log_probs_backward(x, ((where + 1) % V).to(torch.int32), lse, None, torch.ones(N, device="cuda"), None)
            want = torch.zeros_like(x)                                   # the other label: 1 there, -1 at the only likely class
            want[torch.arange(N, device="cuda"), (where + 1) % V] = 1.0
            want[torch.arange(N, device="cuda"), where] = -1.0
            assert float((dx - want).abs().max()) <= 8 * U


def test_log_probs_gradient_between_the_rows_of_the_logits(dat):  # noqa: F811
    for N, V in ((5, 10), (300, 77), (3, 9001)):
        buf = torch.full((N, 2 * V + 3), 7.0, device="cuda")
        x, labels = lp_rows(450, N, V, torch.float32)
        buf[:, 1:V + 1] = x
        out = dat.log_probs(buf[:, 1:V + 1], labels)
        a = randn(451, N)
        dat.log_probs_backward(buf[:, 1:V + 1], labels, out[2], None, a, None, dlogits=buf[:, V + 1:2 * V + 1])
        assert torch.equal(buf[:, 1:V + 1], x) and (buf[:, 0] == 7.0).all() and (buf[:, 2 * V + 1:] == 7.0).all()
        assert torch.equal(buf[:, V + 1:2 * V + 1], dat.log_probs_backward(x, labels, out[2], None, a, None))
        with pytest.raises(dat.DatError):
            dat.log_probs_backward(buf[:, 1:V + 1], labels, out[2], None, a, None, dlogits=buf[:, V:2 * V])
