"""Refusals of the group norm, label log probability and AdamW calls (no GPU needed: nothing is launched), their plain forms against
finite differences, and the 8-bit moment format."""
import numpy as np
import pytest
import torch

import paper_2206_06257_amd.binding as b
from tests import plain_ops as po

lib = b._lib
P = 4096          # a non-null, aligned address that no refused call looks at


def gn_fwd(x=P, gamma=P, beta=P, dtype=0, B=2, H=4, W=4, C_=16, groups=4, eps=1e-5, act=0, y=P, mean=P, rstd=P, ws=None, size=0):
    return lib.dat_group_norm_forward(x, gamma, beta, dtype, B, H, W, C_, groups, eps, act, y, mean, rstd, ws, size, None)


def gn_bwd(x=P, dy=P, gamma=P, beta=P, mean=P, rstd=P, dtype=0, B=2, H=4, W=4, C_=16, groups=4, act=0, dx=P, dgamma=P, dbeta=P, ws=P, size=1 << 20):
    return lib.dat_group_norm_backward(x, dy, gamma, beta, mean, rstd, dtype, B, H, W, C_, groups, act, dx, dgamma, dbeta, ws, size, None)


@pytest.mark.parametrize("status,kw", [
    (1, dict(x=None)), (1, dict(y=None)), (1, dict(mean=None)), (1, dict(rstd=None)), (1, dict(gamma=None)), (1, dict(beta=None)), (1, dict(dtype=2)),
    (1, dict(B=-1)), (1, dict(H=0)), (1, dict(W=0)), (1, dict(C_=0)), (1, dict(groups=0)), (1, dict(groups=3)), (1, dict(groups=32)), (1, dict(eps=-1.0)),
    (1, dict(eps=float("nan"))), (1, dict(act=3)), (1, dict(act=-1)), (1, dict(x=P + 2)), (1, dict(dtype=1, y=P + 1)), (1, dict(mean=P + 2)),
    (2, dict(H=1 << 16, W=1 << 16)), (2, dict(H=1 << 14, W=1 << 14)), (2, dict(B=1 << 30))])
def test_group_norm_forward_refuses(status, kw):
    assert gn_fwd(**kw) == status


@pytest.mark.parametrize("status,kw", [
    (1, dict(x=None)), (1, dict(dy=None)), (1, dict(dx=None)), (1, dict(mean=None)), (1, dict(rstd=None)), (1, dict(gamma=None)), (1, dict(dgamma=None)),
    (1, dict(dbeta=None)), (1, dict(groups=5)), (1, dict(act=7)), (1, dict(ws=None)), (1, dict(size=4)), (1, dict(ws=P + 8)), (1, dict(dy=P + 1)),
    (2, dict(B=1 << 28, C_=64))])
def test_group_norm_backward_refuses(status, kw):
    assert gn_bwd(**kw) == status


def test_group_norm_workspace_needs():
    assert lib.dat_group_norm_workspace(0, 0, -1, 4, 4, 16, 4) == 0 and lib.dat_group_norm_workspace(1, 0, 2, 4, 4, 16, 3) == 0
    need = lib.dat_group_norm_workspace(1, 0, 2, 4, 4, 16, 4)
    assert gn_bwd(size=need - 1) == 1 and need >= 2 * 2 * 16 * 4


def lp(x=P, dtype=0, N=3, V=10, ld=10, labels=P, top=2, logp=P, entropy=P, lse=P, tl=P, ti=P, ws=P, size=1 << 40):
    return lib.dat_log_probs(x, dtype, N, V, ld, labels, top, logp, entropy, lse, tl, ti, ws, size, None)


def lp_bwd(x=P, dtype=0, N=3, V=10, ld=10, labels=P, lse=P, entropy=P, dlogp=P, dentropy=P, dx=2 * P, ldd=10):
    return lib.dat_log_probs_backward(x, dtype, N, V, ld, labels, lse, entropy, dlogp, dentropy, dx, ldd, None)


@pytest.mark.parametrize("status,kw", [
    (1, dict(x=None)), (1, dict(dtype=5)), (1, dict(N=-1)), (1, dict(V=0)), (1, dict(ld=9)), (1, dict(labels=None)), (1, dict(top=-1)), (1, dict(top=33)),
    (1, dict(tl=None)), (1, dict(ti=None)), (1, dict(x=P + 2)), (1, dict(dtype=1, x=P + 1)), (1, dict(lse=P + 1)), (1, dict(ti=P + 2)),
    (2, dict(V=(1 << 30) + 1, ld=(1 << 30) + 1)), (2, dict(N=1 << 31)), (2, dict(N=1 << 30, ld=1 << 40)),
    (1, dict(N=1, V=1 << 20, ld=1 << 20, size=0, ws=None)), (1, dict(N=1, V=1 << 20, ld=1 << 20, ws=P + 8))])
def test_log_probs_refuses(status, kw):
    if "ws" in kw and not lib.dat_log_probs_workspace(1, 1 << 20, 2):
        pytest.skip("needs no workspace")
    assert lp(**kw) == status


@pytest.mark.parametrize("status,kw", [
    (1, dict(x=None)), (1, dict(dx=None)), (1, dict(lse=None)), (1, dict(labels=None)), (1, dict(dlogp=None)), (1, dict(entropy=None)),
    (1, dict(dentropy=None)), (1, dict(ldd=9)), (1, dict(dx=P, ldd=12)), (1, dict(dx=P + 2)), (1, dict(dlogp=P + 1)), (2, dict(N=1 << 31))])
def test_log_probs_backward_refuses(status, kw):
    assert lp_bwd(**kw) == status


def adamw(theta=P, g=P, dtype=0, off=P, T=2, d=10, bits=32, m=P, v=P, scales=P, lr=0.1, b1=0.9, b2=0.99, eps=1e-8, wd=0.0, decay=None, t=1, copy=None):
    return lib.dat_adamw_update(theta, g, dtype, off, T, d, bits, m, v, scales, 0, lr, b1, b2, eps, wd, decay, t, copy, None)


@pytest.mark.parametrize("kw", [
    dict(theta=None), dict(g=None), dict(off=None), dict(m=None), dict(v=None), dict(bits=8, scales=None), dict(T=0), dict(d=-1), dict(dtype=3), dict(bits=16),
    dict(lr=-1.0), dict(lr=float("nan")), dict(b1=1.0), dict(b1=-0.1), dict(b2=1.0), dict(b2=float("nan")), dict(eps=-1.0), dict(wd=-1.0), dict(t=0),
    dict(theta=P + 2), dict(g=P + 2), dict(dtype=1, g=P + 1), dict(off=P + 4), dict(m=P + 1), dict(decay=P + 2), dict(copy=P + 1), dict(d=1 << 42)])
def test_adamw_refuses(kw):
    assert adamw(**kw) == 1


def test_more_threads_than_a_launch_has_are_refused():
    assert lp(N=1 << 30) == 2 and lp(N=1 << 28, V=100, ld=100) == 2 and lp(N=1 << 23, V=20000, ld=20000) == 2
    assert lp_bwd(N=1 << 30) == 2 and lp_bwd(N=1 << 24, V=2000, ld=2000, ldd=2000) == 2
    assert adamw(d=1 << 34) == 1 and lib.dat_adamw_moments(P, P, P, P, 2, 1 << 34, P, P, None) == 1
    small = dict(B=1 << 24, H=1, W=1, C_=64, groups=32, ws=P, size=1 << 40)
    assert gn_fwd(**small) == 2 and gn_bwd(**small) == 2


def test_nothing_to_do_is_no_error():
    assert adamw(d=0, theta=None, g=None, m=None, v=None) == 0
    assert lp(N=0, x=None, labels=None, logp=None, entropy=None, lse=None, tl=None, ti=None, ws=None, size=0) == 0
    assert lp_bwd(N=0, x=None, dx=None, lse=None) == 0
    assert gn_fwd(B=0, x=None, y=None, mean=None, rstd=None) == 0
    assert gn_bwd(B=0, x=None, dy=None, dx=None, mean=None, rstd=None, dgamma=None, dbeta=None, ws=None, size=0) == 0


def test_model_update_refuses():
    assert lib.dat_model_adamw_update(None, P, 32, 0, 0.1, 0.9, 0.99, 1e-8, 0.0, 1, None) == 1
    assert lib.dat_adamw_moments(None, P, P, P, 1, 10, P, P, None) == 1 and lib.dat_adamw_moments(P, P, P, P, 0, 10, P, P, None) == 1
    assert lib.dat_adamw_slots(-1, 3) == 0 and lib.dat_adamw_slots(1000, 4) == 7


def test_binding_refuses_shapes_types_and_places():
    f, h = torch.zeros(4, 10), torch.zeros(4, 10, dtype=torch.float16)
    y = torch.zeros(4, dtype=torch.int32)
    for call in (lambda: b.log_probs(h, y), lambda: b.log_probs(f, y.long()), lambda: b.log_probs(f, y[:3]), lambda: b.log_probs(f.t(), y), lambda: b.log_probs(f, y),
                 lambda: b.log_probs(f[0], y), lambda: b.log_probs(f.expand(4, 10)[:1].expand(4, 10), y),
                 lambda: b.log_probs_backward(f, y, f[:, 0]), lambda: b.log_probs_backward(f, None, torch.zeros(4), None, torch.zeros(4)),
                 lambda: b.log_probs_backward(f, y, torch.zeros(4), torch.zeros(3), None, torch.zeros(4))):
        with pytest.raises((ValueError, AttributeError)):
            call()
    x, c = torch.zeros(2, 4, 4, 16), torch.zeros(16)
    for call in (lambda: b.group_norm_forward(x[0], c, c, 4), lambda: b.group_norm_forward(x.permute(0, 3, 1, 2), c, c, 4), lambda: b.group_norm_forward(x, c[:8], c, 4),
                 lambda: b.group_norm_forward(x, c, c, 4), lambda: b.group_norm_forward(x, c, c, 4, y=x.bfloat16()),
                 lambda: b.group_norm_backward(x, x.bfloat16(), c, c, torch.zeros(2, 4), torch.zeros(2, 4), 4),
                 lambda: b.group_norm_backward(x, x, c, c, torch.zeros(2, 3), torch.zeros(2, 4), 4)):
        with pytest.raises(ValueError):
            call()
    th, off = torch.zeros(10), torch.tensor([0, 4, 10])
    m, v, s = b.adamw_state(10, 2, 8, device="cpu")
    for call in (lambda: b.adamw_update(th, th[:9], th, th, off, 0.1, 1), lambda: b.adamw_update(th, th, m, v, off, 0.1, 1), lambda: b.adamw_update(th, th, m, th, off, 0.1, 1),
                 lambda: b.adamw_update(th, th, m, v, off, 0.1, 1, scales=s[:1]), lambda: b.adamw_update(th, th, m, v, off.int(), 0.1, 1, scales=s),
                 lambda: b.adamw_update(th, th, m, v, off, 0.1, 1, scales=s, decay=th), lambda: b.adamw_update(th, th, m, v, off, 0.1, 1, scales=s),
                 lambda: b.adamw_state(10, 2, 4), lambda: b.adamw_moments(th, v, s, off)):
        with pytest.raises(ValueError):
            call()


# ---- the plain forms themselves ----------------------------------------------------------------------------------------
@pytest.mark.parametrize("act", [0, 1, 2])
def test_plain_group_norm_gradient_against_differences(act):
    rng = np.random.default_rng(act)
    x, gamma, beta, w = rng.standard_normal((2, 3, 3, 6)), 1 + 0.2 * rng.standard_normal(6), 0.3 * rng.standard_normal(6), rng.standard_normal((2, 3, 3, 6))
    mean, rstd = po.gn_stats(x, 3, 1e-5)
    dx, dg, db = po.gn_backward(x, w, gamma, beta, mean, rstd, 3, act)[:3]
    f = lambda x, g, be: (po.gn_forward(x, g, be, 3, act, 1e-5)[0] * w).sum()  # noqa: E731
    for k, grad in enumerate((dx, dg, db)):
        at = [x, gamma, beta]
        for _ in range(5):
            u = rng.standard_normal(grad.shape)
            ends = [f(*[a + s * 1e-6 * u if i == k else a for i, a in enumerate(at)]) for s in (1, -1)]
            assert abs((ends[0] - ends[1]) / 2e-6 - (grad * u).sum()) < 1e-7 * np.abs(grad * u).sum() + 1e-7


def test_plain_log_probs_gradient_against_differences():
    rng = np.random.default_rng(0)
    x, y, a, c = rng.standard_normal((4, 7)), np.array([0, 6, 3, -1]), rng.standard_normal(4), rng.standard_normal(4)
    a[3] = 0.0
    x[1, 2] = -np.inf
    _, H, lse, _, _ = po.log_probs(x, y, 0)
    dx, _ = po.log_probs_backward(x, y, lse, H, a, c)

    def f(x):
        lp_, H_, _, _, _ = po.log_probs(x, y, 0)
        return np.where(a != 0, a * np.nan_to_num(lp_), 0).sum() + (c * H_).sum()

    for _ in range(5):
        u = rng.standard_normal(x.shape)
        assert abs((f(x + 1e-6 * u) - f(x - 1e-6 * u)) / 2e-6 - (dx * u).sum()) < 1e-7 * np.abs(dx * u).sum() + 1e-7


def test_plain_moment_format():
    off = np.array([0, 0, 300, 301, 900], np.int64)
    slots = b.adamw_slots(900, 4)
    slot, place = po.adamw_places(off)
    assert len(set(zip(slot, place))) == 900 and slot.max() < slots          # no two tensors share a block
    rng = np.random.default_rng(2)
    x = (rng.standard_normal(900) * 10.0 ** rng.uniform(-6, 0, 900)).astype(np.float32)
    x[:4] = [0.0, -0.0, 1e-30, -2.0]
    for top, val in ((127, x), (255, np.abs(x))):
        r = rng.integers(0, 1 << 16, 900)
        code, scale = po.adamw_encode(val, r, off, slots, top, np.zeros(slots, np.int64))
        got = po.adamw_decode(code, scale, off, top).astype(np.float64)
        largest = np.zeros(slots)
        np.maximum.at(largest, slot, np.abs(val))
        kept = np.abs(val) >= largest[slot] * 2.0 ** (-15 if top == 127 else -31)
        assert (np.abs(got - val)[kept] <= np.abs(val)[kept] / 8).all() and (np.sign(got) == np.sign(val))[kept].all()
        assert (np.abs(got)[~kept] <= largest[slot][~kept] * 2.0 ** (-14.5 if top == 127 else -30.5)).all()
        if top == 255:
            assert (got[val > 0] > 0).all()
        # the mean over the random numbers is the value
        j = 1 if top == 127 else 3
        reps = [po.adamw_decode(*po.adamw_encode(val, np.full(900, k), off, slots, top, np.zeros(slots, np.int64)), off, top)[100] for k in range(0, 1 << 16, 16)]
        assert abs(np.mean(reps, dtype=np.float64) / val[100] - 1) < 1e-4, j


def test_buffer_stores_keep_their_data():
    """The group norm kernels' buffer stores have their whole offset in a vector register and wait states behind them (gfx950 reads
    the data of other stores late: what is computed into the same registers next can come out in memory)."""
    import os
    import re
    import subprocess
    from tests.test_kernel_resources import _code_objects
    objdump = os.path.join(os.environ.get("ROCM_PATH", "/opt/rocm"), "llvm", "bin", "llvm-objdump")
    seen = 0
    for i, elf in enumerate(_code_objects()):
        r = subprocess.run([objdump, "-d", "--no-show-raw-insn", "-"], input=elf, stdout=subprocess.PIPE, check=True)
        for name, body in re.findall(r"^[0-9a-f]+ <(\S+)>:\n(.*?)(?=^[0-9a-f]+ <|\Z)", r.stdout.decode(), re.S | re.M):
            if "gn_" not in name:
                continue
            lines = [x.split("//")[0].split() for x in body.splitlines()]
            for k, x in enumerate(lines):
                if x and x[0].startswith("buffer_store"):
                    seen += 1
                    assert x[-2:] == ["0", "offen"] and lines[k + 1][:2] == ["s_nop", "3"], (name, x, lines[k + 1])
    assert seen >= 100


def test_plain_softmax_gradient():
    """Against the gradient from an exact lse, and rows of equal logits of any size: p = 1/V, and the gradient of a log probability sums
    to zero over its row."""
    rng = np.random.default_rng(1)
    x, y, a, c = rng.standard_normal((4, 7)) * 3, np.array([0, 6, 3, -1]), rng.standard_normal(4), rng.standard_normal(4)
    x[1, 2] = -np.inf
    _, H, lse, _, _ = po.log_probs(x, y, 0)
    got, p, q, h = po.softmax_gradient(x, y, a, c)
    assert np.abs(got - po.log_probs_backward(x, y, lse, H, a, c)[0]).max() < 1e-13 and np.abs(h - H).max() < 1e-13
    same = np.array([np.finfo(np.float32).min, -1e6, 3e38])[:, None] * np.ones((1, 5))
    got, p, q, h = po.softmax_gradient(same, np.array([1, 2, 3]), np.ones(3), np.ones(3))
    assert np.abs(p - 0.2).max() < 1e-15 and np.abs(got.sum(axis=1)).max() < 1e-14 and np.abs(h - np.log(5)).max() < 1e-14
    assert np.abs(got[0] - [-0.2, 0.8, -0.2, -0.2, -0.2]).max() < 1e-14


def test_outputs_that_overlap_inputs_are_refused():
    n = 2 * 4 * 4 * 16 * 4
    for d in (4, 16, n - 4):
        assert gn_fwd(y=P * 4 + d, x=P * 4) == 1 and gn_fwd(y=P * 4 - d, x=P * 4) == 1
        assert gn_bwd(dx=P * 4 + d, x=P * 4, dy=P * 9) == 1 and gn_bwd(dx=P * 4 - d, dy=P * 4, x=P * 9) == 1
    for d in (4, 36, 40, 44, 3 * 40 - 4):                  # three rows of ten, one behind the other
        assert lp_bwd(dx=P + d) == 1 and lp_bwd(x=P + d, dx=P) == 1
    for d in (4, 36, 48, 52, 88 + 4, 2 * 84 + 36):         # rows apart: 40 of 84 bytes
        assert lp_bwd(dx=P + d, ld=21, ldd=21) == 1 and lp_bwd(x=P + d, dx=P, ld=21, ldd=21) == 1
    assert lp_bwd(N=1, dx=P + 36, ld=1000, ldd=1000) == 1 and lp_bwd(dtype=1, dx=P + 2) == 1


@pytest.mark.parametrize("seed", range(4))
def test_rows_overlap_agrees_with_sets(seed):
    """The refusals of interleaved rows, against the sets of elements (a copy of the rule: nothing may be launched here)."""
    rng = np.random.default_rng(seed)
    for _ in range(2000):
        N, row = int(rng.integers(1, 5)), int(rng.integers(1, 7))
        step, d = row + int(rng.integers(0, 8)), int(rng.integers(0, 60))
        one = {n * step + i for n in range(N) for i in range(row)}
        share = d != 0 and bool(one & {e + d for e in one})
        rule = d != 0 and d < (N - 1) * step + row and (d % step < row or (step - d % step < row and d < (N - 1) * step))
        assert share == rule, (N, row, step, d)


def test_binding_names_what_is_missing():
    f, y, n, x, c = torch.zeros(4, 10), torch.zeros(4, dtype=torch.int32), torch.zeros(4), torch.zeros(2, 4, 4, 16), torch.zeros(16)
    for name, call in (("labels", lambda: b.log_probs_backward(f, None, n, None, n)), ("entropy", lambda: b.log_probs_backward(f, y, n, None, None, n)),
                       ("lse", lambda: b.log_probs_backward(f, y, None, None, n)), ("dy", lambda: b.group_norm_backward(x, None, c, c, c, c, 4)),
                       ("mean", lambda: b.group_norm_backward(x, x, c, c, None, c, 4)), ("grads", lambda: b.adamw_update(n, None, n, n, y, 0.1, 1))):
        with pytest.raises(ValueError, match=name):
            call()
