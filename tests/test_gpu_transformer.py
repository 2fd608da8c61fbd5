"""Norm and rotation of queries and keys, gradient clipping, and a transformer's training step made of them with attention, the label
log probabilities and AdamW, on the GPU against plain forms in 64 bits.

Tolerances count roundings: U = 2^-24 is half a step of fp32, half(t) that of the stored type relative to the value.  cos and sin are
4 U off (angle in 64 bits, its rest rounded once, a polynomial of 6 operations)."""
import math

import numpy as np
import pytest
import torch

from tests import plain_transformer as pt
from tests.test_gpu_attention import assert_near, half, host, randn

pytestmark = pytest.mark.gpu
U = pt.U
F32, BF16 = torch.float32, torch.bfloat16


@pytest.fixture(scope="module")
def dat():
    import paper_2206_06257_amd as dat
    return dat


# ---- norm and rotation ------------------------------------------------------------------------------------------------
# T, H, Hkv, D, sections: one token, no keys, no queries, no pair, all pairs, a part of the pairs, pairs that are no multiple of a vector, one
# to four axes, an axis without pairs, few heads (several tokens a wave) and many
ROT = [(1, 1, 1, 64, [32]), (7, 12, 12, 64, [16, 16]), (33, 3, 0, 72, [18, 18]), (65, 0, 5, 80, [20, 20]), (130, 8, 2, 128, [28, 18, 18]), (9, 2, 1, 8, [2, 2]),
       (50, 4, 4, 96, [0, 12, 24, 12]), (21, 2, 2, 40, [6, 4]), (13, 1, 1, 80, [10]), (5, 30, 7, 256, [64, 32, 32]), (300, 1, 0, 16, [8]), (17, 3, 1, 32, []), (4, 2, 2, 256, [1, 1]), (1000, 5, 3, 24, [12])]


def rot_inputs(seed, T, H, Hkv, D, sections, dtype, far=0):
    x = (randn(seed, T, H + Hkv, D) * torch.exp(0.5 * randn(seed + 1, T, H + Hkv, 1))).to(dtype)
    dy = randn(seed + 2, T, H + Hkv, D).to(dtype)
    pos = torch.randint(-50, 1000, (T, len(sections)), device="cuda", dtype=torch.int32, generator=torch.Generator(device="cuda").manual_seed(seed)) + far
    gq, gk = 1 + 0.3 * randn(seed + 3, D), 1 + 0.3 * randn(seed + 4, D)
    part = lambda t: (t[:, :H] if H else None, t[:, H:] if Hkv else None)  # noqa: E731
    return part(x), part(dy), pos, gq, gk


def tolerance(want, size, D, dtype, extra=0):
    # a head's sum of squares or products: D / 8 in a lane, then a tree; r; two products; two more and a sum with cos and sin 4 U off
    # (numbers below 2^-126 have the steps of those from there on: half of one is half * 2^-126)
    return (D / 8 + 40 + extra) * U * size + (half(dtype) + 2 * U) * np.maximum(np.abs(want), 2.0 ** -126) * 1.01


def check_rotary(dat, x, dy, pos, gq, gk, sections, layout, eps=1e-6, norm=True, freq=None):
    freq = dat.rotary_frequencies(sections) if freq is None else freq
    w = pt.angles(pos.cpu().numpy(), freq.cpu().numpy(), sections)
    halves = layout == dat.ROTARY_HALVES
    y = dat.norm_rotary_forward(*x, gq, gk, pos, freq, sections, layout, eps, norm)
    g = dat.norm_rotary_backward(*x, gq, gk, pos, freq, sections, *dy, layout, eps, norm)
    for n in range(2):
        if x[n] is None:
            assert y[n] is None and g[n] is None and g[2 + n] is None
            continue
        D, gamma = x[n].shape[-1], (gq, gk)[n]
        gh = None if gamma is None else host(gamma)
        want, size = pt.norm_rotary(host(x[n]), gh, w, halves, eps, norm)
        assert_near(host(y[n]), want, tolerance(want, size, D, x[n].dtype), "y")
        dx, dg, size, gsize = pt.norm_rotary_backward(host(x[n]), host(dy[n]), gh, w, halves, eps, norm)
        assert_near(host(g[n]), dx, tolerance(dx, size, D, x[n].dtype, D / 8), "dx")
        if norm and gamma is not None:
            T, H = x[n].shape[:2]
            terms = T * H / 64 + 1100        # of a wave's lane (at most all that a wave takes), 64 lanes and 4 waves, 1024 workgroups / 16
            assert_near(host(g[2 + n]), dg, (terms + D / 8 + 40) * U * gsize, "dgamma")
        else:
            assert g[2 + n] is None
    again = dat.norm_rotary_backward(*x, gq, gk, pos, freq, sections, *dy, layout, eps, norm)
    assert all(a is None or torch.equal(a, b) for a, b in zip(g, again))
    return y, g


@pytest.mark.parametrize("layout", [0, 1])
@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("shape", ROT)
def test_norm_rotary(dat, shape, dtype, layout):
    T, H, Hkv, D, sections = shape
    x, dy, pos, gq, gk = rot_inputs(10, *shape, dtype)
    check_rotary(dat, x, dy, pos, gq, gk, sections, layout)
    check_rotary(dat, x, dy, pos, gq, None, sections, layout)
    check_rotary(dat, x, dy, pos, None, None, sections, layout, norm=False)


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("shape", ROT + [(20011, 6, 3, 80, [20, 20]), (70001, 2, 1, 64, [32])])
def test_gradients_of_scales_by_the_sums_they_are(dat, shape, dtype):
    """At most 512 workgroups of four waves: a lane adds up the heads of every 2048th token, a workgroup the lanes of an element (1024 / D of a wave
    at most hold the same one), then eight workgroups a thread and 64 threads."""
    T, H, Hkv, D, sections = shape
    x, dy, pos, gq, gk = rot_inputs(70, *shape, dtype)
    freq = dat.rotary_frequencies(sections)
    w = pt.angles(pos.cpu().numpy(), freq.cpu().numpy(), sections)
    for layout in (dat.ROTARY_HALVES, dat.ROTARY_PAIRS):
        g = dat.norm_rotary_backward(*x, gq, gk, pos, freq, sections, *dy, layout)
        for n, gamma in enumerate((gq, gk)):
            if x[n] is None:
                continue
            _, dg, _, gsize = pt.norm_rotary_backward(host(x[n]), host(dy[n]), host(gamma), w, layout == dat.ROTARY_HALVES, 1e-6)
            chain = math.ceil(T / 2048) * x[n].shape[1] + 4096 / D + 8 + 64
            assert_near(host(g[2 + n]), dg, (chain + D / 8 + 40) * U * gsize, "dgamma")


@pytest.mark.parametrize("far", [10**6, 2**31 - 1001, -(2**31) + 50])
def test_far_positions(dat, far):
    x, dy, pos, gq, gk = rot_inputs(20, 40, 2, 2, 64, [20, 12], F32, far)
    # angles of up to 2^31 radians have lost 31 + 53 - 53 bits in 64 bits: 2^-22 of a quarter turn = 4 U more, at a million none
    check_rotary(dat, x, dy, pos, gq, gk, [20, 12], 0, freq=torch.cat([dat.rotary_frequencies([20]), dat.rotary_frequencies([12], 100.0)]))
    y = dat.norm_rotary_forward(x[0], None, None, None, pos, torch.full((32,), 1234.5, device="cuda"), [32, 0], norm=False)[0]
    w = pt.angles(pos.cpu().numpy(), np.full(32, 1234.5, np.float32), [32, 0])
    want, size = pt.norm_rotary(host(x[0]), None, w, True, 0, False)
    # 2^31 * 1234.5 radians: the product has 2^42 steps of 2^-11; in 64 bits its rounding is 2^-53 of it, and so is that of 2 / pi
    assert_near(host(y), want, size * (20 * U + 2.0 ** 42 * 2.0 ** -52) + 4 * U * np.abs(want), "y")


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("scale", [1e-30, 1e-22, 1e18, 1e25, 1e36])
def test_heads_of_every_size(dat, dtype, scale):
    """Squares beyond fp32's range, and below it without an eps to stand in for them."""
    (q, k), dy, pos, gq, gk = rot_inputs(30, 20, 2, 1, 64, [32], F32)
    eps = 0.0 if scale < 1 else 1e-6
    x = ((q * scale).to(dtype), (k * 1.0).to(dtype))
    y, _ = check_rotary(dat, x, tuple((d * (1.0 if scale > 1 else scale)).to(dtype) for d in dy), pos, gq, gk, [32], 0, eps=eps)
    assert bool(torch.isfinite(y[0].float()).all()) and float(y[0].float().abs().max()) > 0.1


def test_zero_heads(dat):
    x, dy, pos, gq, gk = rot_inputs(40, 20, 2, 1, 64, [32], F32)
    x[0][3] = 0.0
    check_rotary(dat, x, dy, pos, gq, gk, [32], 0)
    y = dat.norm_rotary_forward(*x, gq, gk, pos, dat.rotary_frequencies([32]), [32], eps=0.0)[0]
    assert bool(torch.isnan(y[3]).all()) and bool(torch.isfinite(y[:3]).all()) and bool(torch.isfinite(y[4:]).all())


@pytest.mark.parametrize("bad", [math.nan, math.inf])
@pytest.mark.parametrize("D", [64, 72])
def test_what_is_not_finite_stays_in_its_head(dat, bad, D):
    x, dy, pos, gq, gk = rot_inputs(50, 20, 3, 2, D, [D // 2], BF16)
    freq = dat.rotary_frequencies([D // 2])
    y = dat.norm_rotary_forward(*x, gq, gk, pos, freq, [D // 2])
    g = dat.norm_rotary_backward(*x, gq, gk, pos, freq, [D // 2], *dy)
    x2 = (x[0].clone(), x[1])
    x2[0][4, 1, 9] = bad
    y2 = dat.norm_rotary_forward(*x2, gq, gk, pos, freq, [D // 2])
    g2 = dat.norm_rotary_backward(*x2, gq, gk, pos, freq, [D // 2], *dy)
    keep = torch.ones(20, 3, dtype=torch.bool, device="cuda")
    keep[4, 1] = False
    assert torch.equal(y2[0][keep], y[0][keep]) and torch.equal(y2[1], y[1]) and not bool(torch.isfinite(y2[0][4, 1]).all())
    assert torch.equal(g2[0][keep], g[0][keep]) and torch.equal(g2[1], g[1]) and torch.equal(g2[3], g[3]) and not bool(torch.isfinite(g2[0][4, 1]).all())


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_rotary_strides_and_buffers(dat, dtype):
    """Heads of one projection, [B, S, H, D], in place, gradients over what they come from, outputs into parts of one tensor."""
    B, S, H, Hkv, D = 3, 11, 4, 2, 72
    qkv = randn(60, B, S, H + 2 * Hkv, D).to(dtype)
    q, k, _ = torch.split(qkv, [H, Hkv, Hkv], dim=2)
    pos = torch.randint(0, 99, (B, S, 2), device="cuda", dtype=torch.int32)
    freq, gq, gk = dat.rotary_frequencies([20, 16]), 1 + 0.2 * randn(61, D), 1 + 0.2 * randn(62, D)
    flat = lambda t: t.reshape(B * S, -1, D)  # noqa: E731
    want = dat.norm_rotary_forward(flat(q).contiguous(), flat(k).contiguous(), gq, gk, pos.view(-1, 2), freq, [20, 16])
    got = dat.norm_rotary_forward(q, k, gq, gk, pos, freq, [20, 16])
    assert all(torch.equal(flat(a), b) for a, b in zip(got, want))
    heads_first = tuple(t.transpose(1, 2).contiguous().transpose(1, 2) for t in (q, k))
    got = dat.norm_rotary_forward(*heads_first, gq, gk, pos, freq, [20, 16])
    assert all(torch.equal(flat(a), b) for a, b in zip(got, want))
    dy = tuple(randn(63 + n, *t.shape).to(dtype) for n, t in enumerate((q, k)))
    gwant = dat.norm_rotary_backward(q, k, gq, gk, pos, freq, [20, 16], *dy)
    whole = torch.zeros_like(qkv)
    parts = torch.split(whole, [H, Hkv, Hkv], dim=2)
    dat.norm_rotary_backward(q, k, gq, gk, pos, freq, [20, 16], *dy, dq=parts[0], dk=parts[1])
    assert torch.equal(parts[0], gwant[0]) and torch.equal(parts[1], gwant[1]) and bool((parts[2] == 0).all())
    dat.norm_rotary_backward(q, k, gq, gk, pos, freq, [20, 16], *dy, dq=dy[0], dk=dy[1])
    assert torch.equal(dy[0], gwant[0]) and torch.equal(dy[1], gwant[1])
    dat.norm_rotary_forward(q, k, gq, gk, pos, freq, [20, 16], yq=q, yk=k)
    assert torch.equal(flat(q), want[0]) and torch.equal(flat(k), want[1])
    with pytest.raises(RuntimeError):
        dat.norm_rotary_forward(q, k, gq, gk, pos, freq, [20, 16], yq=qkv[:, :, 1:H + 1], yk=k)
    empty = q[:, :0]
    y = dat.norm_rotary_forward(empty, None, gq, None, pos[:, :0], freq, [20, 16])[0]
    g = dat.norm_rotary_backward(empty, None, gq, None, pos[:, :0], freq, [20, 16], empty, None)
    assert y.shape == empty.shape and bool((g[2] == 0).all())


def test_rotary_beyond_32_bit_offsets(dat):
    T, H, D = 70000, 250, 128
    x = torch.empty(T, H, D, dtype=BF16, device="cuda")
    assert x.numel() > 1 << 31
    x[-3:].normal_()
    pos, freq = torch.arange(T, device="cuda", dtype=torch.int32)[:, None], dat.rotary_frequencies([64])
    want = dat.norm_rotary_forward(x[-3:].clone(), None, None, None, pos[-3:].contiguous(), freq, [64])[0]
    gwant = dat.norm_rotary_backward(x[-3:].clone(), None, None, None, pos[-3:].contiguous(), freq, [64], x[-3:].clone(), None)[0]
    y = dat.norm_rotary_forward(x, None, None, None, pos, freq, [64])[0]
    assert torch.equal(y[-3:], want)
    dat.norm_rotary_backward(x, None, None, None, pos, freq, [64], x, None, dq=y)
    assert torch.equal(y[-3:], gwant)


# ---- clipping --------------------------------------------------------------------------------------------------------------
def gradients(seed, sizes, kinds, scale=1e-2):
    """Views of one vector for each type, so that a tensor starts at any element."""
    flat = {k: (randn(seed + n, max(1, sum(s for s, kk in zip(sizes, kinds) if kk == k)) + 3) * scale).to(k) for n, k in enumerate((F32, BF16))}
    at, out = {F32: 1, BF16: 1}, []
    for s, k in zip(sizes, kinds):
        out.append(flat[k][at[k]:at[k] + s])
        at[k] += s
    return out, flat


SIZES = [[1], [0, 5, 0], [432, 16, 4608, 32, 320, 10], [8192], [8191, 8193, 1, 16384], [40000], [70001, 3, 0, 12345, 8192], [3] * 200, [100000, 1] * 3, [5_000_001],
         [8192, 0, 0, 0], [8190, 1, 1, 3], [4096] * 8, [101] * 16, [101] * 17]          # (the last five about one launch or two)


@pytest.mark.parametrize("mixed", [0, 1, 2])
@pytest.mark.parametrize("sizes", SIZES)
def test_clip_gradients(dat, sizes, mixed):
    kinds = [(F32, BF16)[(n + mixed) % 2 if mixed < 2 and len(sizes) > 1 else mixed % 2] for n in range(len(sizes))]
    for factor in (0.3, 0.9999, 1.0001, math.inf, 0.0):
        tensors, flat = gradients(5, sizes, kinds)
        before, table = {k: v.clone() for k, v in flat.items()}, dat.gradient_table(tensors)
        norm, _, _ = pt.clip([host(t) for t in tensors], math.inf)
        largest = float(np.float32(norm * factor)) if factor < math.inf else factor
        norm, want, c = pt.clip([host(t) for t in tensors], largest)
        got = dat.clip_gradients(table, largest)
        assert_near(host(got), [norm], 1.01 * U * norm, "norm")
        for t, w in zip(tensors, want):       # c rounded to fp32, the product to fp32 and then to the type
            assert_near(host(t), w, (half(t.dtype) + 3 * U) * np.abs(w) * 1.01 if c != 1 else 0.0, "g")
        inside = sum(sizes)
        for k, v in flat.items():             # nothing around the tensors is written
            n = sum(s for s, kk in zip(sizes, kinds) if kk == k)
            assert torch.equal(v[:1], before[k][:1]) and torch.equal(v[1 + n:], before[k][1 + n:]), inside


def test_clip_extremes(dat):
    """Squares beyond fp32 and below it, gradients that are not finite."""
    for scale in (1e-30, 1e30):
        g = randn(1, 50000) * scale
        norm, want, _ = pt.clip([host(g)], 1e-31)
        got = dat.clip_gradients(dat.gradient_table([g]), 1e-31)
        assert_near(host(got), [norm], 1.01 * U * norm, "norm")
        assert_near(host(g), want[0], 3 * U * np.abs(want[0]) + 2.0 ** -149, "g")
    for n in (100, 50000):
        g = randn(2, n)
        g[n // 2] = math.inf
        assert float(dat.clip_gradients(dat.gradient_table([g]), 1.0)) == math.inf
        assert bool(torch.isnan(g[n // 2])) and bool((g[:n // 2] == 0).all()) and bool((g[n // 2 + 1:] == 0).all())
        g = randn(3, n)
        g[n // 3] = math.nan
        assert math.isnan(float(dat.clip_gradients(dat.gradient_table([g]), 1.0))) and bool(torch.isnan(g).all())
        g = torch.zeros(n, device="cuda")
        assert float(dat.clip_gradients(dat.gradient_table([g]), 0.0)) == 0.0 and bool((g == 0).all())


def test_clip_is_repeatable_and_beyond_32_bits(dat):
    big = torch.empty((1 << 31) + 12345, dtype=BF16, device="cuda")
    big.normal_()
    small = randn(7, 1001)
    table = dat.gradient_table([small[:500], big, small[500:]])
    a, b = dat.clip_gradients(table, math.inf), dat.clip_gradients(table, math.inf)
    want = math.sqrt(sum(float(p.double().square().sum()) for p in big.split(1 << 28)) + float(small.double().square().sum()))
    assert torch.equal(a, b) and abs(float(a) - want) <= 2 * U * want
    tail = big[-5:].clone()
    dat.clip_gradients(table, want / 2)
    assert_near(host(big[-5:]), host(tail) / 2, (half(BF16) + 4 * U) * np.abs(host(tail)), "tail")


def test_gradient_table_keeps_its_memory(dat):
    """A tensor that is given other memory afterwards: the table works on what it was made for."""
    g = torch.full((1000,), 3.0, device="cuda")
    old, table = g.detach(), dat.gradient_table([g])
    g.data = torch.ones(1000, device="cuda")
    assert abs(float(dat.clip_gradients(table, 1.0)) - math.sqrt(9000.0)) < 1e-4
    assert bool((g == 1).all()) and bool((old == old[0]).all()) and abs(float(old[0]) - 1 / math.sqrt(1000.0)) < 1e-8


def test_gradient_table_dropped_while_another_stream_uses_it(dat):
    """A table made for one call on a side stream: its memory is not handed out again before that stream has passed the call."""
    g, x = randn(1, 1000), randn(2, 8192, 8192)
    before, side = g.clone(), torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        for _ in range(10):                       # several milliseconds each
            x @ x
    table = dat.gradient_table([g[:500], g[500:]])
    sizes = [t.numel() * t.element_size() for t in (table.pointers, table.types, table.offsets)]
    places = {t.data_ptr() for t in (table.pointers, table.types, table.offsets)}
    norm = dat.clip_gradients(table, 1.0, stream=side)
    del table
    others = [torch.empty(n, dtype=torch.uint8, device="cuda") for n in sizes for _ in range(4)]
    assert not side.query(), "the side stream has to be busy here"
    assert not places & {t.data_ptr() for t in others}
    torch.cuda.synchronize()
    want = math.sqrt(float(before.double().square().sum()))
    assert abs(float(norm) - want) < 1e-6 * want
    assert_near(host(g), host(before) / want, 4 * U * np.abs(host(before)) / want, "g")


def test_clip_refuses_a_norm_among_the_gradients(dat):
    g = randn(1, 100)
    before, table = g.clone(), dat.gradient_table([g[:50], g[:0], g[60:]])
    for at in (0, 49, 60, 99):
        with pytest.raises(ValueError, match="norm"):
            dat.clip_gradients(table, 1.0, norm=g[at:at + 1])
    assert torch.equal(g, before)
    dat.clip_gradients(table, math.inf, norm=g[55:56])
    assert abs(float(g[55]) - math.sqrt(float(torch.cat([before[:50], before[60:]]).double().square().sum()))) < 1e-5


def test_gradient_table_refuses(dat):
    g = randn(1, 100)
    for bad in ([], [g.cpu()], [g.half()], [g[::2]], [g, g], [g[:50], g[40:]], [g, None]):
        with pytest.raises((ValueError, AttributeError)):
            dat.gradient_table(bad)
    table = dat.gradient_table([g[:50], g[50:], g[:0]])
    for call in (lambda: dat.clip_gradients(table, -1.0), lambda: dat.clip_gradients(table, math.nan), lambda: dat.clip_gradients(table, 1.0, norm=g[:2])):
        with pytest.raises((ValueError, RuntimeError)):
            call()


# ---- together -----------------------------------------------------------------------------------------------------------------
def plain_step(x, w, out, head, gq, gk, labels, angle, H, Hkv, D, window):
    """A layer in 64 bits with autograd: x [T, C] -> heads -> norm and rotation -> attention -> classes -> mean of -log p(label)."""
    T = x.shape[0]
    qkv = (x @ w).view(T, H + 2 * Hkv, D)
    q, k, v = torch.split(qkv, [H, Hkv, Hkv], dim=1)

    def one(z, gamma):
        n = z / torch.sqrt(z.square().mean(-1, keepdim=True) + 1e-6) * gamma
        a, b = n[..., :D // 2], n[..., D // 2:]
        c, s = torch.cos(angle)[:, None], torch.sin(angle)[:, None]
        return torch.cat([a * c - b * s, a * s + b * c], -1)
    q, k = one(q, gq), one(k, gk)
    see = torch.from_numpy(pt.seen(T, T, window))
    s = torch.einsum("ihd,jhd->hij", q, k.repeat_interleave(H // Hkv, 1)) / math.sqrt(D)
    p = torch.softmax(s.masked_fill(~see, -math.inf), -1)
    o = torch.einsum("hij,jhd->ihd", p, v.repeat_interleave(H // Hkv, 1)).reshape(T, H * D)
    z = (o @ out) @ head
    return -(z - torch.logsumexp(z, 1, keepdim=True))[torch.arange(T), labels].mean()


@pytest.mark.parametrize("capture", [False, True])
def test_training_step_of_a_layer(dat, capture):
    """Projection, norm and rotation, attention, log probabilities; gradients by input and by every parameter; clipping and AdamW; in fp32 against
    autograd in 64 bits, eager and captured, with several replays and eager work between."""
    T, C, H, Hkv, D, V, window = 90, 48, 4, 2, 32, 10, (-1, 0)
    g = torch.Generator().manual_seed(0)
    sizes = [C * (H + 2 * Hkv) * D, H * D * C, C * V, D, D]
    offsets = torch.tensor(np.concatenate([[0], np.cumsum(sizes)]), device="cuda")
    theta = torch.cat([torch.randn(n, generator=g) * s + m for n, s, m in zip(sizes, (0.2, 0.1, 0.3, 0.1, 0.1), (0, 0, 0, 1, 1))]).cuda()
    x0 = torch.randn(T, C, generator=g).cuda()
    labels = torch.randint(0, V, (T,), generator=g, dtype=torch.int32).cuda()
    pos = torch.stack([torch.arange(T) // 9, torch.arange(T) % 9], 1).int().cuda()
    sections = [8, 8]
    freq = dat.rotary_frequencies(sections)
    grad = torch.zeros_like(theta)
    m, v, _ = dat.adamw_state(theta.numel(), len(sizes))
    # the two scales' gradients are written straight into the flat vector; the rest as torch's products give them
    table = dat.gradient_table([grad[a:b] for a, b in zip(offsets[:-1].tolist(), offsets[1:].tolist())])
    x, dx, norm = x0.clone(), torch.empty_like(x0), torch.empty(1, device="cuda")

    def parts(t):
        w, out, head, gq, gk = torch.split(t, sizes)
        return w.view(C, -1), out.view(H * D, C), head.view(C, V), gq, gk

    def step():
        w, out, head, gq, gk = parts(theta)
        dw, dout, dhead, dgq, dgk = parts(grad)
        qkv = (x @ w).view(T, H + 2 * Hkv, D)
        q, k, val = torch.split(qkv, [H, Hkv, Hkv], dim=1)
        yq, yk = dat.norm_rotary_forward(q, k, gq, gk, pos, freq, sections)
        o, lse = dat.attention_forward(yq[None], yk[None], val[None], window=window)
        mid = o.view(T, H * D) @ out
        z = mid @ head
        lp = dat.log_probs(z, labels)
        dz = dat.log_probs_backward(z, labels, lp[2], dlogp=torch.full((T,), -1.0 / T, device="cuda"))
        torch.mm(mid.t(), dz, out=dhead)
        dmid = dz @ head.t()
        torch.mm(o.view(T, H * D).t(), dmid, out=dout)
        do = (dmid @ out.t()).view(1, T, H, D)
        dqkv = torch.empty_like(qkv)
        pq, pk, pv = torch.split(dqkv, [H, Hkv, Hkv], dim=1)
        dat.attention_backward(yq[None], yk[None], val[None], o, lse, do, window=window, dq=pq[None], dk=pk[None], dv=pv[None])
        dat.norm_rotary_backward(q, k, gq, gk, pos, freq, sections, pq, pk, dq=pq, dk=pk, dgamma_q=dgq, dgamma_k=dgk)
        torch.mm(x.t(), dqkv.view(T, -1), out=dw)
        torch.mm(dqkv.view(T, -1), w.t(), out=dx)
        dat.clip_gradients(table, 0.05, norm=norm)

    def check():
        theta64 = theta.double().cpu().requires_grad_(True)
        x64 = x.double().cpu().requires_grad_(True)
        angle = torch.from_numpy(pt.angles(pos.cpu().numpy(), freq.cpu().numpy(), sections))
        w, out, head, gq, gk = parts(theta64)
        plain_step(x64, w, out, head, gq, gk, labels.long().cpu(), angle, H, Hkv, D, window).backward()
        n64 = float(theta64.grad.norm())
        assert n64 > 0.05 and abs(float(norm) - n64) < 1e-5 * n64
        # every stage's relative error of about a hundred roundings, through six stages: 600 U = 4e-5 of the gradient's size
        for a, b in zip(parts(grad.double().cpu()), parts(theta64.grad)):
            assert float((a * n64 / 0.05 - b).norm()) < 4e-5 * n64
        assert float((dx.double().cpu() - x64.grad).norm()) < 4e-5 * float(x64.grad.norm())

    if not capture:
        step()
        check()
        before = theta.clone()
        dat.adamw_update(theta, grad, m, v, offsets, 1e-3, 1)
        assert not torch.equal(before, theta)
        step()
        check()
        return
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step()
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for n in range(3):
        x.copy_(x0 + 0.1 * n)
        graph.replay()
        torch.cuda.synchronize()
        check()
        again = [t.clone() for t in (grad, dx, norm)]
        step()                                    # eager, into the same buffers: the same bits
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(again, (grad, dx, norm)))


def test_attack_on_a_layer(dat):
    """An attack's steps through the operators: the gradient by the input of a layer (projection, norm and rotation, attention, log probabilities)
    moves the start point by dat.pgd_update; each step's gradient against autograd in 64 bits at the GPU's own point."""
    B, S, C, H, Hkv, D, V, eps, alpha = 3, 20, 24, 4, 2, 32, 10, 8 / 255, 3 / 255
    g = torch.Generator().manual_seed(1)
    T, sizes = B * S, [C * (H + 2 * Hkv) * D, H * D * C, C * V]
    w, out, head = (t.view(a, -1) for t, a in zip([torch.randn(n, generator=g).cuda() * s for n, s in zip(sizes, (0.3, 0.2, 0.4))], (C, H * D, C)))
    gq, gk = 1 + 0.1 * randn(2, D), 1 + 0.1 * randn(3, D)
    x, labels = torch.rand(B, S, C, generator=g).cuda(), torch.randint(0, V, (T,), generator=g, dtype=torch.int32).cuda()
    pos = torch.stack([torch.arange(S) // 5, torch.arange(S) % 5], 1).int().cuda().expand(B, S, 2).contiguous()
    freq = dat.rotary_frequencies([8, 8])
    angle = torch.from_numpy(pt.angles(pos[0].cpu().numpy(), freq.cpu().numpy(), [8, 8]))
    delta = dat.pgd_init(x, eps, dat.INIT_UNIFORM, seed=5)

    def gradient(z):
        qkv = (z.view(T, C) @ w).view(B, S, H + 2 * Hkv, D)
        q, k, v = torch.split(qkv, [H, Hkv, Hkv], dim=2)
        yq, yk = dat.norm_rotary_forward(q, k, gq, gk, pos, freq, [8, 8])
        o, lse = dat.attention_forward(yq, yk, v)
        logits = (o.view(T, H * D) @ out) @ head
        lp = dat.log_probs(logits, labels)
        dz = dat.log_probs_backward(logits, labels, lp[2], dlogp=torch.full((T,), -1.0 / T, device="cuda"))
        do = ((dz @ head.t()) @ out.t()).view(B, S, H, D)
        dqkv = torch.empty_like(qkv)
        dq, dk, dv = torch.split(dqkv, [H, Hkv, Hkv], dim=2)
        dat.attention_backward(yq, yk, v, o, lse, do, dq=dq, dk=dk, dv=dv)
        dat.norm_rotary_backward(q, k, gq, gk, pos, freq, [8, 8], dq, dk, dq=dq, dk=dk)
        return (dqkv.view(T, -1) @ w.t()).view_as(z)

    p64 = [t.double().cpu() for t in (w, out, head, gq, gk)]
    for _ in range(3):
        z = dat.make_xadv(x, delta)
        got = gradient(z)
        z64 = z.double().cpu().requires_grad_(True)
        sum(plain_step(z64[n], *p64, labels.long().cpu().view(B, S)[n], angle, H, Hkv, D, (-1, -1)) / B for n in range(B)).backward()
        # every stage's relative error of about a hundred roundings, through six stages: 600 U = 4e-5 of the gradient's size
        assert float((got.double().cpu() - z64.grad).norm()) < 4e-5 * float(z64.grad.norm())
        want = torch.clamp(delta.double() + alpha * torch.sign(got.double()), -eps, eps)
        want = torch.clamp(x.double() + want, 0, 1) - x.double()
        before = delta.clone()
        dat.pgd_update(x, got, delta, eps, alpha)
        assert float((delta.double() - want).abs().max()) < 4 * U and not torch.equal(before, delta)


def test_two_graphs_do_not_share_workspaces(dat):
    """Two captured graphs of the calls that need workspaces, replayed one after the other and on two streams at once."""
    def inputs(seed):
        return [randn(seed + n, 2, 140, 4, 64).to(BF16) for n in range(4)] + [randn(seed + 9, 60000)]
    sets, graphs, outs = [inputs(1), inputs(50)], [], []
    pos = torch.arange(280, device="cuda", dtype=torch.int32).view(2, 140, 1)
    freq, gamma = dat.rotary_frequencies([32]), 1 + 0.1 * randn(5, 64)
    tables = [dat.gradient_table([s[4]]) for s in sets]

    def call(s, table):
        yq, yk = dat.norm_rotary_forward(s[0], s[1], gamma, gamma, pos, freq, [32])
        o, lse = dat.attention_forward(yq, yk, s[2])
        g = dat.attention_backward(yq, yk, s[2], o, lse, s[3])
        return list(g) + list(dat.norm_rotary_backward(s[0], s[1], gamma, gamma, pos, freq, [32], g[0], g[1])) + [dat.clip_gradients(table, math.inf)]
    for s, table in zip(sets, tables):
        call(s, table)
        torch.cuda.synchronize()
        graphs.append(torch.cuda.CUDAGraph())
        with torch.cuda.graph(graphs[-1]):
            outs.append(call(s, table))
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    for n in range(3):
        for s in sets:
            for t in s[:4]:
                t.mul_(0.9)
        torch.cuda.synchronize()
        for graph, st in zip(graphs, streams):
            with torch.cuda.stream(st):
                graph.replay()
        torch.cuda.synchronize()
        for s, table, out in zip(sets, tables, outs):
            assert all(torch.equal(a, b) for a, b in zip(out, call(s, table)))


def test_calls_on_two_streams_at_once(dat):
    sets = [[randn(seed + n, 2, 300, 4, 64).to(BF16) for n in range(4)] for seed in (1, 50)]
    want = []
    for q, k, v, do in sets:
        o, lse = dat.attention_forward(q, k, v, window=(-1, 0))
        want.append((o, lse) + dat.attention_backward(q, k, v, o, lse, do, window=(-1, 0)))
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    torch.cuda.synchronize()
    got = []
    for st, (q, k, v, do) in zip(streams, sets):
        o, lse = dat.attention_forward(q, k, v, window=(-1, 0), stream=st)
        got.append((o, lse) + dat.attention_backward(q, k, v, o, lse, do, window=(-1, 0), stream=st))
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for x, y in zip(want, got) for a, b in zip(x, y))
