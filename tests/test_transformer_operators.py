"""Refusals of the attention, norm-and-rotation and clipping calls (no GPU needed: nothing is launched), and their plain forms against differences."""
import math

import numpy as np
import pytest
import torch

import paper_2206_06257_amd.binding as b
from tests import plain_transformer as pt

lib = b._lib
P = 1 << 20       # a non-null, aligned address that no refused call looks at
FAR = 1 << 40     # between the addresses of tensors that do not overlap


# ---- attention ---------------------------------------------------------------------------------------------------------
BASE = dict(dtype=0, B=2, Sq=10, Sk=12, H=4, Hkv=2, D=16, scale=0.25, left=-1, right=-1, offsets_q=None, offsets_k=None)


def heads(n, S, H, D, **kw):
    h = dict(data=P + n * FAR, batch=S * H * D, token=H * D, head=D)
    h.update(kw)
    return b._Heads(**h)


def attn(backward=False, lse=P, ws=P, size=1 << 40, stream=None, t=None, **kw):
    """The C call with one tensor's fields changed by t = (name, fields)."""
    d = dict(BASE, **kw)
    shape = b._Attention(**d)
    tensors = {}
    for n, name in enumerate(("q", "k", "v", "o", "do", "dq", "dk", "dv")):
        S, H = (d["Sq"], d["H"]) if name in ("q", "o", "do", "dq") else (d["Sk"], d["Hkv"])
        tensors[name] = heads(n, S, H, d["D"], **(t[1] if t and t[0] == name else {}))
    x = tensors
    if not backward:
        return lib.dat_attention_forward(shape, x["q"], x["k"], x["v"], x["o"], lse, ws, size, stream)
    return lib.dat_attention_backward(shape, x["q"], x["k"], x["v"], x["o"], lse, x["do"], x["dq"], x["dk"], x["dv"], ws, size, stream)


SHARED = [(1, dict(dtype=2)), (1, dict(B=-1)), (1, dict(Sq=-1)), (1, dict(Sk=-1)), (1, dict(H=0)), (1, dict(Hkv=0)), (1, dict(H=3)), (1, dict(D=0)),
          (1, dict(scale=0.0)), (1, dict(scale=-1.0)), (1, dict(scale=math.nan)), (1, dict(scale=math.inf)), (1, dict(scale=3e38)), (1, dict(left=-2)), (1, dict(right=-7)),
          (1, dict(offsets_q=P)), (1, dict(offsets_k=P)), (1, dict(offsets_q=P + 2, offsets_k=P)), (2, dict(D=12)), (2, dict(D=136)), (2, dict(Sq=1 << 30)), (2, dict(Sk=1 << 30)),
          (1, dict(t=("q", dict(data=None)))), (1, dict(t=("k", dict(data=P + 8)))), (1, dict(t=("v", dict(token=30)))), (1, dict(t=("o", dict(head=2)))),
          (1, dict(t=("q", dict(batch=-16)))), (2, dict(t=("k", dict(token=1 << 21)))), (1, dict(lse=None)), (1, dict(lse=P + 2)), (1, dict(dtype=1, t=("q", dict(token=4))))]


@pytest.mark.parametrize("status,kw", SHARED + [
    (1, dict(t=("o", dict(token=0)))), (1, dict(t=("o", dict(head=8)))), (1, dict(t=("o", dict(data=P)))), (1, dict(t=("o", dict(data=P + FAR + 64)))),
    (2, dict(B=1 << 20, H=1 << 12, Hkv=1 << 12))])
def test_attention_forward_refuses(status, kw):
    assert attn(**kw) == status


@pytest.mark.parametrize("status,kw", SHARED + [
    (1, dict(ws=None)), (1, dict(ws=P + 8)), (1, dict(size=2 * 2 * 4 * 10 * 4 - 1)), (1, dict(t=("dq", dict(data=P)))), (1, dict(t=("dk", dict(data=P + 7 * FAR)))),
    (1, dict(t=("dv", dict(token=0)))), (1, dict(t=("do", dict(data=P + 4)))), (1, dict(t=("dv", dict(data=P + 6 * FAR + 32 * 4 * 3))))])
def test_attention_backward_refuses(status, kw):
    assert attn(backward=True, **kw) == status


def test_attention_refuses_null_structs_and_has_nothing_to_do():
    h, s = heads(0, 10, 4, 16), b._Attention(**BASE)
    assert lib.dat_attention_forward(None, h, h, h, h, P, None, 0, None) == 1 and lib.dat_attention_forward(s, None, h, h, h, P, None, 0, None) == 1
    assert lib.dat_attention_forward(s, h, h, h, None, P, None, 0, None) == 1
    assert lib.dat_attention_backward(s, h, h, h, h, P, h, h, h, None, P, 1 << 20, None) == 1
    assert attn(B=0) == 0 and attn(backward=True, B=0, lse=None, ws=None, size=0) == 0 and attn(Sq=0, lse=None) == 0
    assert attn(B=0, offsets_q=P, offsets_k=P) == 0 and attn(backward=True, Sq=0, Sk=0, ws=None, size=0) == 0


def test_attention_workspace():
    s = b._Attention(**BASE)
    assert lib.dat_attention_workspace(1, s) >= 2 * 4 * 2 * 4 * 10 and lib.dat_attention_workspace(1, None) == 0
    assert lib.dat_attention_workspace(1, b._Attention(**dict(BASE, D=7))) == 0 and lib.dat_attention_workspace(2, s) == 0


def test_attention_parts_of_one_tensor_do_not_overlap():
    """Outputs between one another and beside inputs: told apart by strides, refused where an element is shared.  (What is allowed is asked of
    a call that is refused for another reason, so that nothing is launched.)"""
    B, S, H, Hkv, D = 2, 12, 4, 2, 16
    w, W = 4, (H + 2 * Hkv) * D
    kw = dict(batch=S * W, token=W, head=D)
    d = dict(BASE, Sq=S, Sk=S)
    part = lambda first: b._Heads(data=P + first * D * w, **kw)  # noqa: E731
    h = [heads(n + 1, S, H, D) for n in range(8)]
    hk = [heads(n + 20, S, Hkv, D) for n in range(3)]

    def call(dq, dk, dv, ws):
        return lib.dat_attention_backward(b._Attention(**d), h[0], hk[0], hk[1], h[1], P, h[2], dq, dk, dv, ws, 1 << 20, None)
    # all parts apart: only the missing workspace is refused, and that is looked at last
    assert call(part(0), part(H), part(H + Hkv), None) == 1
    for dq, dk, dv in ((part(0), part(H - 1), part(H + Hkv)), (part(0), part(H), part(H + 1)), (part(1), part(H), part(H + Hkv))):
        assert call(dq, dk, dv, P) == 1


def test_attention_binding_refuses():
    q, k = torch.zeros(2, 5, 4, 16), torch.zeros(2, 7, 2, 16)
    off = torch.zeros(3, dtype=torch.int32)
    lse = torch.zeros(2, 4, 5)
    for call in (lambda: b.attention_forward(q, k, k), lambda: b.attention_forward(q.half(), k.half(), k.half()), lambda: b.attention_forward(q, k.bfloat16(), k),
                 lambda: b.attention_forward(q, k, k[:, :6]), lambda: b.attention_forward(q[0], k, k), lambda: b.attention_forward(q, k[:1], k[:1]),
                 lambda: b.attention_forward(q, k[..., :8], k[..., :8]), lambda: b.attention_forward(q.transpose(2, 3).contiguous().transpose(2, 3), k, k),
                 lambda: b.attention_forward(q, k, k, offsets_q=off), lambda: b.attention_forward(q, k, k, offsets_q=off, offsets_k=off),
                 lambda: b.attention_forward(q[0], k[0], k[0], offsets_q=off.long(), offsets_k=off), lambda: b.attention_forward(q[0], k[0], k[0], offsets_q=off, offsets_k=off[:2]),
                 lambda: b.attention_forward(q, k, k, o=q[:, :4]), lambda: b.attention_forward(q, k, None), lambda: b.attention_forward(q, k, k, window=(1,)), lambda: b.attention_forward(q, k, k, window=((1 << 32) + 5, 0)),
                 lambda: b.attention_forward(q, k, k, window=(-1, -2)), lambda: b.attention_forward(q[:1].expand(1 << 31, *q.shape[1:]), k[:1].expand(1 << 31, *k.shape[1:]), k),
                 lambda: b.attention_backward(q, k, k, q, lse[:1], q), lambda: b.attention_backward(q, k, k, q, lse, k), lambda: b.attention_backward(q, k, k, q, lse, q, dk=q),
                 lambda: b.attention_backward(q, k, k, q, lse, q)):
        with pytest.raises((ValueError, AttributeError)):
            call()


def test_attention_binding_refuses_sizes_beyond_its_types():
    q, k = torch.zeros(2, 5, 4, 16), torch.zeros(2, 7, 2, 16)
    for window in (((1 << 32) + 5, 0), (-1, 1 << 31), (-2, 0)):
        with pytest.raises(ValueError, match="window"):
            b.attention_forward(q, k, k, window=window)
    with pytest.raises(ValueError, match="below 2"):
        b.attention_forward(*(t[:1].expand((1 << 32) + 1, *t.shape[1:]) for t in (q, k, k)))
    with pytest.raises(ValueError, match="below 2"):
        b.norm_rotary_forward(q[:1].expand((1 << 32) + 1, *q.shape[1:]), None, None, None, None, None, [])


def test_numbers_are_taken_by_value():
    """A scale, a window or sections held in tensors that change: each call goes by what they hold then."""
    q, k = torch.zeros(2, 5, 4, 16), torch.zeros(2, 7, 2, 16)
    scale, side, layout = torch.tensor(0.5), torch.tensor(3), torch.tensor(0)
    pos, f = torch.zeros(2, 5, 2, dtype=torch.int32), torch.zeros(8)
    sections, eps = [torch.tensor(4), torch.tensor(4)], torch.tensor(0.5)
    for s, n, e in ((0.5, 4, 0.5), (0.25, 2, 0.125), (2.0, 0, 1.0)):
        scale.fill_(s), side.fill_(n), sections[0].fill_(n), eps.fill_(e), layout.fill_(n // 4)
        shape = b._attention(q, k, scale, (side, side), None, None)[0]
        assert (shape.scale, shape.left, shape.right) == (s, n, n)
        for given in (sections, torch.stack(sections)):
            shape = b._rotary(q, k[:, :5], None, None, pos, f[:n + 4], given, layout, eps, True)[0]
            assert list(shape.sections) == [n, 4, 0, 0] and shape.eps == e and shape.layout == n // 4
        with pytest.raises(ValueError, match="frequencies"):
            b._rotary(q, k[:, :5], None, None, pos, f[:n + 3], sections, layout, eps, True)
    for window in ((1.5, 0), (0, 1.0), ("1", 0)):
        with pytest.raises((TypeError, ValueError)):
            b._attention(q, k, None, window, None, None)
    with pytest.raises((TypeError, ValueError)):
        b._rotary(q, k[:, :5], None, None, pos, f[:8], [4.0, 4.0], 0, 1e-6, True)


def test_group_norm_workspace_is_taken_by_value():
    x, groups, size = torch.zeros(1, 7, 7, 64), torch.tensor(8), {}
    for n in (8, 2, 64, 1):
        groups.fill_(n)
        size[n] = b._gn_workspace(1, x, groups)[1]
        assert size[n] == int(b._lib.dat_group_norm_workspace(1, b.F32, *x.shape, n))
    assert len(set(size.values())) > 1


@pytest.mark.parametrize("window", [(-1, -1), (-1, 0), (2, 1)])
@pytest.mark.parametrize("Lq,Lk", [(5, 7), (7, 4), (1, 1)])
def test_plain_attention_gradient_against_differences(Lq, Lk, window):
    rng = np.random.default_rng(Lq)
    q, k, v, w = rng.standard_normal((Lq, 4, 6)), rng.standard_normal((Lk, 2, 6)), rng.standard_normal((Lk, 2, 6)), rng.standard_normal((Lq, 4, 6))
    o, lse = pt.attention(q, k, v, 0.7, window)[:2]
    grads = pt.attention_backward(q, k, v, o, lse, w, 0.7, window, 0.0)[0]
    f = lambda *t: (pt.attention(*t, 0.7, window)[0] * w).sum()  # noqa: E731
    for n in range(3):
        for _ in range(4):
            u = rng.standard_normal(grads[n].shape)
            ends = [f(*[t + s * 1e-6 * u if i == n else t for i, t in enumerate((q, k, v))]) for s in (1, -1)]
            assert abs((ends[0] - ends[1]) / 2e-6 - (grads[n] * u).sum()) < 1e-7 * (1 + np.abs(grads[n] * u).sum())


# ---- norm and rotation ---------------------------------------------------------------------------------------------------
ROT = dict(dtype=0, B=2, S=10, H=4, Hkv=2, D=32, axes=2, sections=(8, 8, 0, 0), layout=0, norm=1, eps=1e-6)


def rot(backward=False, positions=P, freq=P, gq=P, gk=P, dgq=P, dgk=P, ws=P, size=1 << 40, t=None, null=(), **kw):
    d = dict(ROT, **kw)
    shape = b._Rotary(d["dtype"], d["B"], d["S"], d["H"], d["Hkv"], d["D"], d["axes"], (b.C.c_int32 * 4)(*d["sections"]), d["layout"], d["norm"], d["eps"])
    x = {}
    for n, name in enumerate(("q", "k", "yq", "yk", "dq", "dk")):
        H = d["H"] if name in ("q", "yq", "dq") else d["Hkv"]
        x[name] = None if name in null else heads(n, d["S"], H, d["D"], **(t[1] if t and t[0] == name else {}))
    if not backward:
        return lib.dat_norm_rotary_forward(shape, x["q"], x["k"], gq, gk, positions, freq, x["yq"], x["yk"], None)
    return lib.dat_norm_rotary_backward(shape, x["q"], x["k"], gq, gk, positions, freq, x["yq"], x["yk"], x["dq"], x["dk"], dgq, dgk, ws, size, None)


ROT_REFUSED = [(1, dict(dtype=2)), (1, dict(B=-1)), (1, dict(S=-1)), (1, dict(H=-1)), (1, dict(H=0, Hkv=0)), (1, dict(D=0)), (1, dict(axes=-1)), (1, dict(axes=5)),
               (1, dict(sections=(-8, 8, 0, 0))), (1, dict(sections=(8, 9, 0, 0))), (1, dict(layout=2)), (1, dict(norm=2)), (1, dict(eps=-1.0)), (1, dict(eps=math.nan)), (1, dict(eps=math.inf)),
               (2, dict(D=36)), (2, dict(D=264)), (2, dict(sections=(8, 7, 0, 0))), (2, dict(B=1 << 16, S=1 << 15)), (2, dict(H=1 << 20)),
               (1, dict(positions=None)), (1, dict(freq=None)), (1, dict(positions=P + 2)), (1, dict(freq=P + 1)), (1, dict(gq=P + 2)), (1, dict(gk=P + 1)),
               (1, dict(null=("q",))), (1, dict(null=("yk",))), (1, dict(t=("q", dict(data=P + 8)))), (1, dict(t=("k", dict(token=33)))), (1, dict(t=("yq", dict(head=-32)))),
               (1, dict(dtype=1, t=("q", dict(head=36))))]


@pytest.mark.parametrize("status,kw", ROT_REFUSED + [(1, dict(t=("yq", dict(token=0)))), (1, dict(t=("yq", dict(data=P + 16)))), (1, dict(t=("yk", dict(data=P + 2 * FAR + 64)))),
                                                      (1, dict(t=("yk", dict(data=P)))), (1, dict(t=("yq", dict(data=P, token=256))))])
def test_norm_rotary_forward_refuses(status, kw):
    assert rot(**kw) == status


@pytest.mark.parametrize("status,kw", ROT_REFUSED + [(1, dict(ws=None)), (1, dict(ws=P + 8)), (1, dict(size=100)), (1, dict(dgq=P + 2)), (1, dict(dgk=P + 1)), (1, dict(null=("dq",))),
                                                      (1, dict(t=("dq", dict(token=0)))), (1, dict(t=("dq", dict(data=P + 16)))), (1, dict(t=("dk", dict(data=P + 4 * FAR)))),
                                                      (1, dict(t=("dk", dict(data=P + 2 * FAR))))])
def test_norm_rotary_backward_refuses(status, kw):
    assert rot(backward=True, **kw) == status


def test_norm_rotary_has_nothing_to_do():
    assert rot(B=0) == 0 and rot(S=0, positions=None, freq=None) == 0 and rot(backward=True, S=0, dgq=None, dgk=None, ws=None, size=0) == 0
    shape = b._Rotary(0, 2, 10, 4, 2, 32, 2, (b.C.c_int32 * 4)(8, 8, 0, 0), 0, 1, 1e-6)
    assert lib.dat_norm_rotary_workspace(0, shape) == 0 and lib.dat_norm_rotary_workspace(1, shape) >= 2 * 32 * 4 and lib.dat_norm_rotary_workspace(1, None) == 0
    assert lib.dat_norm_rotary_forward(None, None, None, None, None, None, None, None, None, None) == 1


def test_norm_rotary_binding_refuses():
    q, k, g = torch.zeros(5, 4, 32), torch.zeros(5, 2, 32), torch.ones(32)
    pos, f = torch.zeros(5, 2, dtype=torch.int32), torch.zeros(16)
    for call in (lambda: b.norm_rotary_forward(q, k, g, g, pos, f, [8, 8]), lambda: b.norm_rotary_forward(q, k, g[:8], g, pos, f, [8, 8]), lambda: b.norm_rotary_forward(q, k, g, g, pos.long(), f, [8, 8]),
                 lambda: b.norm_rotary_forward(q, k, g, g, pos[:4], f, [8, 8]), lambda: b.norm_rotary_forward(q, k, g, g, pos, f, [16]), lambda: b.norm_rotary_forward(q, k, g, g, pos, f[:8], [8, 8]),
                 lambda: b.norm_rotary_forward(q, k[:4], g, g, pos, f, [8, 8]), lambda: b.norm_rotary_forward(q, k.bfloat16(), g, g, pos, f, [8, 8]), lambda: b.norm_rotary_forward(None, None, g, g, pos, f, [8, 8]),
                 lambda: b.norm_rotary_forward(q, k, g, g, None, f, [8, 8]), lambda: b.norm_rotary_forward(q, k, g, g, pos, f, [2, 2, 4, 4, 4]), lambda: b.norm_rotary_forward(q[0], k[0], g, g, pos, f, [8, 8]),
                 lambda: b.norm_rotary_forward(q.half(), None, g, g, pos, f, [8, 8]), lambda: b.norm_rotary_forward(q, k, g, g, pos, f, [8, 8], yq=k),
                 lambda: b.norm_rotary_backward(None, k, g, g, pos, f, [8, 8], q, k), lambda: b.norm_rotary_backward(q, k, g, g, pos, f, [8, 8], k, k),
                 lambda: b.norm_rotary_backward(q, k, g, g, pos, f, [8, 8], q, k, dgamma_q=g[:3]), lambda: b.norm_rotary_backward(q, k, g, g, pos, f, [8, 8], q, k)):
        with pytest.raises((ValueError, AttributeError)):
            call()


def test_rotary_frequencies():
    f = b.rotary_frequencies([2, 4], 100.0, device="cpu")
    assert torch.allclose(f, torch.tensor([1.0, 0.1, 1.0, 100 ** -0.25, 0.1, 100 ** -0.75])) and b.rotary_frequencies([], device="cpu").numel() == 0


@pytest.mark.parametrize("halves", [True, False])
@pytest.mark.parametrize("norm", [True, False])
def test_plain_rotation_gradient_against_differences(halves, norm):
    rng = np.random.default_rng(3)
    x, gamma, dy, w = rng.standard_normal((3, 2, 12)), 1 + 0.2 * rng.standard_normal(12), rng.standard_normal((3, 2, 12)), rng.uniform(-9, 9, (3, 5))
    dx, dg = pt.norm_rotary_backward(x, dy, gamma, w, halves, 1e-3, norm)[:2]
    f = lambda x, g: (pt.norm_rotary(x, g, w, halves, 1e-3, norm)[0] * dy).sum()  # noqa: E731
    for n, grad in enumerate((dx, dg) if norm else (dx,)):
        for _ in range(4):
            u = rng.standard_normal(grad.shape)
            ends = [f(*[t + s * 1e-6 * u if i == n else t for i, t in enumerate((x, gamma))]) for s in (1, -1)]
            assert abs((ends[0] - ends[1]) / 2e-6 - (grad * u).sum()) < 1e-7 * (1 + np.abs(grad * u).sum())


# ---- clipping --------------------------------------------------------------------------------------------------------------
def clip(pointers=P, types=P, off=P, T=3, total=100, largest=1.0, norm=P, ws=P, size=1 << 30):
    return lib.dat_clip_gradients(pointers, types, off, T, total, largest, norm, ws, size, None)


@pytest.mark.parametrize("status,kw", [
    (1, dict(pointers=None)), (1, dict(types=None)), (1, dict(off=None)), (1, dict(norm=None)), (1, dict(ws=None)), (1, dict(T=0)), (1, dict(total=-1)), (1, dict(largest=-1.0)),
    (1, dict(largest=math.nan)), (1, dict(pointers=P + 4)), (1, dict(off=P + 4)), (1, dict(norm=P + 2)), (1, dict(ws=P + 4)), (1, dict(size=3)), (2, dict(total=1 << 45))])
def test_clip_gradients_refuses(status, kw):
    assert clip(**kw) == status


def test_clip_gradients_binding_refuses():
    assert lib.dat_clip_gradients_workspace(0, 5) == 0 and lib.dat_clip_gradients_workspace(3, -1) == 0 and lib.dat_clip_gradients_workspace(3, 100) >= 8
    for bad in ([], [torch.zeros(3)], [torch.zeros(3, dtype=torch.float16)], [None]):
        with pytest.raises(ValueError):
            b.gradient_table(bad)


class Place:
    """A device tensor as clip_gradients looks at it, which notes the streams that it is recorded for."""

    def __init__(self):
        self.device, self.streams = torch.device("cpu"), []

    def data_ptr(self):
        return P

    def record_stream(self, stream):
        self.streams.append(stream)


@pytest.mark.parametrize("made,used", [(7, 7), (7, 9), (0, 5), (5, 0)])
def test_gradient_table_is_recorded_for_the_stream_it_is_used_on(monkeypatch, made, used):
    """The table's memory goes back to the stream that it was made on, so every other one that reads it has to be known."""
    table = b.GradientTable.__new__(b.GradientTable)
    table.tensors, table.total, table.stream, table.places = [None], 100, made, []
    table.pointers, table.types, table.offsets = places = Place(), Place(), Place()

    class On:
        def __init__(self, *args):
            pass

        def __enter__(self):
            return used

        def __exit__(self, *exc):
            pass
    monkeypatch.setattr(b, "_On", On)
    monkeypatch.setattr(torch.cuda, "current_stream", lambda device=None: "the stream")
    monkeypatch.setattr(b._lib, "dat_clip_gradients", lambda *args: 0)
    b.clip_gradients(table, 1.0, norm=torch.zeros(1))
    assert all(p.streams == ([] if made == used else ["the stream"]) for p in places)


def test_plain_clip():
    norm, out, c = pt.clip([np.array([3.0]), np.array([0.0, 4.0])], 2.5)
    assert norm == 5.0 and c == 0.5 and out[1][1] == 2.0 and pt.clip([np.array([3.0])], 3.0)[2] == 1.0


# Calls that are refused for their launch (DAT_ERR_SHAPE), which is looked at behind the overlaps (DAT_ERR_ARG): nothing is launched.
def places_in(layout, S, W, D):
    """Strides of parts of one tensor [B, S, W, D], or [B, W, S, D] with heads before tokens, and the bytes from head to head."""
    kw = dict(batch=W * S * D, token=W * D, head=D) if layout == "tokens" else dict(batch=W * S * D, token=D, head=S * D)
    return kw, 4 * kw["head"]


A = 1 << 46       # an address that nothing else has
PARTS = [(S, B, H, Hkv, layout) for B, H, Hkv in ((1 << 22, 1 << 10, 1), (1 << 22, 1 << 10, 2), (1 << 24, 1, 1), (1 << 23, 2, 1), (1, 1 << 24, 1), (1, 1 << 24, 1 << 23))
         for S in (1, 2) for layout in ("tokens", "heads") if not (layout == "tokens" and S > 1 and B == 1)]       # (token strides stay below 2^23 bytes)


@pytest.mark.parametrize("S,B,H,Hkv,layout", PARTS)
def test_attention_tells_parts_of_one_tensor_apart(S, B, H, Hkv, layout):
    D, W = 16, H + 2 * Hkv
    kw, step = places_in(layout, S, W, D)
    part = lambda first: b._Heads(data=P + first * step, **kw)  # noqa: E731
    h, hk = [b._Heads(data=P + (n + 1) * FAR, **kw) for n in range(3)], [b._Heads(data=P + (n + 20) * FAR, **kw) for n in range(2)]

    def call(dq, dk, dv):
        return lib.dat_attention_backward(b._Attention(**dict(BASE, B=B, Sq=S, Sk=S, H=H, Hkv=Hkv)), h[0], hk[0], hk[1], h[1], A, h[2], dq, dk, dv, P, 1 << 62, None)
    assert call(part(0), part(H), part(H + Hkv)) == 2 and call(part(2 * Hkv), part(0), part(Hkv)) == 2 and call(part(Hkv), part(0), part(H + Hkv)) == 2
    for dq, dk, dv in ((0, H - 1, H + Hkv), (0, H, H + Hkv - 1), (1, H, H + Hkv), (0, 0, H), (0, H, H)):
        assert call(part(dq), part(dk), part(dv)) == 1, (dq, dk, dv)
    # parts of it as inputs beside outputs in the others
    assert lib.dat_attention_forward(b._Attention(**dict(BASE, B=B, Sq=S, Sk=S, H=H, Hkv=Hkv)), h[0], part(H), part(H + Hkv), part(0), A, P, 1 << 62, None) == 2
    assert lib.dat_attention_forward(b._Attention(**dict(BASE, B=B, Sq=S, Sk=S, H=H, Hkv=Hkv)), h[0], part(H - 1), part(H + Hkv), part(0), A, P, 1 << 62, None) == 1


def test_attention_tells_parts_along_tokens_and_batches_apart():
    """dk and dv behind dq's tokens, with heads before tokens; other strides: by their extents."""
    B, H, Hkv, S, Sk, D = 1 << 22, 1 << 10, 2, 2, 3, 16
    T = S + 2 * Sk
    kw = dict(batch=H * T * D, token=D, head=T * D)
    h, hk = [b._Heads(data=P + (n + 1) * 4 * FAR, **kw) for n in range(3)], [b._Heads(data=P + (n + 10) * 4 * FAR, **kw) for n in range(2)]
    part = lambda first, **other: b._Heads(data=P + first * D * 4, **dict(kw, **other))  # noqa: E731

    def call(dq, dk, dv):
        return lib.dat_attention_backward(b._Attention(**dict(BASE, B=B, Sq=S, Sk=Sk, H=H, Hkv=Hkv)), h[0], hk[0], hk[1], h[1], A, h[2], dq, dk, dv, P, 1 << 62, None)
    assert call(part(0), part(S), part(S + Sk)) == 2
    assert call(part(0), part(S - 1), part(S + Sk)) == 1 and call(part(0), part(S), part(S + Sk - 1)) == 1
    assert call(part(0), part(S), part(S + Sk, token=2 * D)) == 1          # (a stride unlike dq's, within its extent)


@pytest.mark.parametrize("layout", ["tokens", "heads"])
@pytest.mark.parametrize("H,Hkv", [(4, 1), (4, 2), (1, 4), (1, 1)])
@pytest.mark.parametrize("B,S", [(2, 1 << 27), (1 << 27, 2), (1, 1 << 28), (1 << 28, 1)])
def test_norm_rotary_tells_parts_of_one_tensor_apart(B, S, H, Hkv, layout):
    D = 256
    kw, step = places_in(layout, S, H + Hkv, D)
    part = lambda first: b._Heads(data=P + first * step, **kw)  # noqa: E731
    d = dict(ROT, B=B, S=S, H=H, Hkv=Hkv, D=D, sections=(2, 2, 0, 0))
    shape = b._Rotary(d["dtype"], B, S, H, Hkv, D, d["axes"], (b.C.c_int32 * 4)(*d["sections"]), 0, 1, 1e-6)
    q, k, far = part(0), part(H), [b._Heads(data=P + (n + 1) * 16 * FAR, **kw) for n in range(4)]
    forward = lambda yq, yk: lib.dat_norm_rotary_forward(shape, q, k, A, A, A, A, yq, yk, None)  # noqa: E731
    assert forward(q, k) == 2 and forward(q, far[0]) == 2 and forward(far[0], k) == 2 and forward(far[0], far[1]) == 2
    assert forward(k, far[0]) == 1 and forward(far[0], q) == 1 and forward(far[0], far[0]) == 1
    assert lib.dat_norm_rotary_backward(shape, far[0], far[1], A, A, A, A, far[2], far[3], q, k, A, A + 4096, P, 1 << 62, None) == 2
    assert lib.dat_norm_rotary_backward(shape, far[0], far[1], A, A, A, A, far[2], far[3], k, k, A, A + 4096, P, 1 << 62, None) == 1


# ---- buffers beside the tensors of heads ---------------------------------------------------------------------------------

@pytest.mark.parametrize("name", ["q", "k", "v", "o"])
def test_attention_forward_refuses_lse_over_a_tensor(name):
    B, H, Hkv, S, D = 1 << 22, 1 << 10, 2, 2, 16
    sizes = dict(q=H, k=Hkv, v=Hkv, o=H)
    t = {n: b._Heads(data=P + i * 4 * FAR, batch=S * h * D, token=h * D, head=D) for i, (n, h) in enumerate(sizes.items())}
    call = lambda lse: lib.dat_attention_forward(b._Attention(**dict(BASE, B=B, Sq=S, Sk=S, H=H, Hkv=Hkv)), *t.values(), lse, P, 1 << 62, None)  # noqa: E731
    first, bytes_, lse = t[name].data, 4 * B * S * sizes[name] * D, 4 * B * H * S
    assert call(A) == 2 and call(first + bytes_) == 2 and call(first + bytes_ - 4) == 1 and call(first) == 1
    assert call(first - lse + 4) == 1 if first > lse else True


@pytest.mark.parametrize("name", ["dq", "dk", "dv"])
def test_attention_backward_refuses_gradients_over_lse(name):
    B, H, Hkv, S, D = 1 << 22, 1 << 10, 2, 2, 16
    sizes = dict(q=H, k=Hkv, v=Hkv, o=H, do=H, dq=H, dk=Hkv, dv=Hkv)
    t = {n: b._Heads(data=P + i * 4 * FAR, batch=S * h * D, token=h * D, head=D) for i, (n, h) in enumerate(sizes.items())}
    x = list(t.values())
    call = lambda lse: lib.dat_attention_backward(b._Attention(**dict(BASE, B=B, Sq=S, Sk=S, H=H, Hkv=Hkv)), *x[:4], lse, *x[4:], P, 1 << 62, None)  # noqa: E731
    first, bytes_, lse = t[name].data, 4 * B * S * sizes[name] * D, 4 * B * H * S
    assert call(A) == 2 and call(first + bytes_) == 2 and call(first - lse) == 2
    assert call(first + bytes_ - 4) == 1 and call(first) == 1 and call(first - lse + 4) == 1
    assert call(t["q"].data) == 2 and call(t["o"].data) == 2                 # (both are read)


def test_norm_rotary_refuses_outputs_over_what_it_reads_or_writes_beside_them():
    """Scales' gradients that share elements with each other or with a tensor; outputs over scales, positions or frequencies."""
    B, S, H, Hkv, D, axes, pairs = 2, 1 << 27, 4, 2, 256, 2, 4
    d = dict(ROT, B=B, S=S, H=H, Hkv=Hkv, D=D, sections=(2, 2, 0, 0))
    shape = b._Rotary(d["dtype"], B, S, H, Hkv, D, axes, (b.C.c_int32 * 4)(*d["sections"]), 0, 1, 1e-6)
    sizes = dict(q=H, k=Hkv, yq=H, yk=Hkv, dq=H, dk=Hkv)
    t = {n: b._Heads(data=P + i * 4 * FAR, batch=S * h * D, token=h * D, head=D) for i, (n, h) in enumerate(sizes.items())}
    end = {n: t[n].data + 4 * B * S * h * D for n, h in sizes.items()}
    small = dict(gq=A, gk=A + 4096, positions=A + 8192, freq=A + 4096 + 16 * B * S)
    more = dict(dgq=A + (1 << 40), dgk=A + (1 << 40) + 4 * D)

    def forward(**kw):
        s = dict(small, **kw)
        return lib.dat_norm_rotary_forward(shape, t["q"], t["k"], s["gq"], s["gk"], s["positions"], s["freq"], t["yq"], t["yk"], None)

    def backward(norm=1, **kw):
        s = dict(small, **more, **{})
        s.update(kw)
        sh = b._Rotary(d["dtype"], B, S, H, Hkv, D, axes, (b.C.c_int32 * 4)(*d["sections"]), 0, norm, 1e-6)
        return lib.dat_norm_rotary_backward(sh, t["q"], t["k"], s["gq"], s["gk"], s["positions"], s["freq"], t["yq"], t["yk"], t["dq"], t["dk"], s["dgq"], s["dgk"],
                                            P, 1 << 62, None)
    assert forward() == 2 and forward(gq=t["q"].data) == 2 and forward(gq=A, gk=A) == 2 and forward(gq=None, gk=None) == 2
    assert backward() == 2 and backward(dgq=None) == 2 and backward(dgk=None) == 2 and backward(dgq=A, dgk=A + 4 * D) == 2     # (a scale's gradient over the scale)
    for name, bytes_ in (("gq", 4 * D), ("gk", 4 * D), ("positions", 4 * B * S * axes), ("freq", 4 * pairs)):
        for out in ("yq", "yk"):
            assert forward(**{name: end[out] - 4}) == 1 and forward(**{name: end[out]}) == 2
            assert forward(**{name: t[out].data - bytes_ + 4}) == 1 or t[out].data < bytes_
        for out in ("dq", "dk"):
            assert backward(**{name: end[out] - 4}) == 1 and backward(**{name: end[out]}) == 2
    for name in ("dgq", "dgk"):
        for over in t:
            assert backward(**{name: t[over].data}) == 1 and backward(**{name: end[over] - 4}) == 1 and backward(**{name: end[over]}) == 2, (name, over)
    assert backward(dgq=more["dgk"]) == 1 and backward(dgq=more["dgk"] + 4 * D - 4) == 1 and backward(dgq=more["dgk"] - 4 * D + 4) == 1
    assert backward(norm=0, dgq=more["dgk"]) == 2                             # (not written)


def test_gradient_table_knows_what_it_holds():
    table = b.GradientTable.__new__(b.GradientTable)
    table.places = [(100, 140), (200, 204), (204, 300)]
    for at, held in ((90, False), (96, False), (98, True), (100, True), (136, True), (140, False), (196, False), (200, True), (296, True), (300, False), (1 << 40, False)):
        assert table.holds(at, 4) is held, at
    table.places = []
    assert table.holds(5, 4) is False


def test_attention_refuses_outputs_over_offsets():
    """Packed sequences: more heads than a launch takes, so that what is allowed is refused for that."""
    T, H, Hkv, D, B = 64, 1 << 24, 2, 8, 5
    sizes = dict(q=H, k=Hkv, v=Hkv, o=H, do=H, dq=H, dk=Hkv, dv=Hkv)
    t = {n: b._Heads(data=P + i * FAR, batch=0, token=D, head=T * D) for i, n in enumerate(sizes)}
    x, end = list(t.values()), {n: t[n].data + 4 * T * D * h for n, h in sizes.items()}

    def call(backward, lse=A, **offsets):
        shape = b._Attention(**dict(BASE, B=B, Sq=T, Sk=T, H=H, Hkv=Hkv, D=D, **dict(dict(offsets_q=A + FAR, offsets_k=A + FAR + 64), **offsets)))
        if backward:
            return lib.dat_attention_backward(shape, *x[:4], lse, *x[4:], P, 1 << 62, None)
        return lib.dat_attention_forward(shape, *x[:4], lse, P, 1 << 62, None)
    for name in ("offsets_q", "offsets_k"):
        for backward, outs, ins in ((False, ("o",), ("q", "k", "v")), (True, ("dq", "dk", "dv"), ("q", "k", "v", "o", "do"))):
            assert call(backward) == 2
            for n in outs:
                assert call(backward, **{name: end[n] - 4}) == 1 and call(backward, **{name: end[n]}) == 2
                assert call(backward, **{name: t[n].data - 4 * B}) == 1 and call(backward, **{name: t[n].data - 4 * B - 4}) == 2
            for n in ins:
                assert call(backward, **{name: t[n].data}) == 2
        assert call(False, lse=A + FAR - 4 * T * H) == 2 and call(False, lse=A + FAR - 4 * T * H + 4) == 1 and call(True, lse=A + FAR) == 2


# ---- what the binding refuses, by the text it says; the first of each list has nothing to refuse but that its tensors are on the CPU ----------
def refused(call, text):
    with pytest.raises(ValueError, match=text):
        call()


Q, K, OFF, LSE = torch.zeros(2, 5, 4, 16), torch.zeros(2, 7, 2, 16), torch.zeros(3, dtype=torch.int32), torch.zeros(2, 4, 5)
PQ, PK, PLSE = Q.flatten(0, 1), K.flatten(0, 1), torch.zeros(4, 10)            # packed
APART = torch.zeros(2, 5, 4, 32)[..., ::2]                                       # elements of a head apart
ON_CPU = "belong on a GPU"


@pytest.mark.parametrize("text,args,kw", [
    (ON_CPU, (Q, K, K), {}), (ON_CPU, (Q, K, K), dict(o=Q)), (ON_CPU, (Q, K[:, :0], K[:, :0]), {}), (ON_CPU, (PQ, PK, PK), dict(offsets_q=OFF, offsets_k=OFF)),
    ("^q: torch.float16", (Q.half(), K, K), {}), ("^q: torch.float64", (Q.double(), K.double(), K.double()), {}), ("^k: torch.bfloat16", (Q, K.bfloat16(), K), {}),
    ("^v: torch.bfloat16", (Q, K, K.bfloat16()), {}), ("^v: .*expected", (Q, K, K[:, :6]), {}), ("^v: .*expected", (Q, K, K[:, :, :1]), {}), ("^v: .*expected", (Q, K, K[..., :8]), {}),
    ("^v: .*expected", (Q, K, K[:1]), {}), ("^q: expected .B, S, H, D.", (PQ, K, K), {}), ("^q: expected .T, H, D.", (Q, K, K), dict(offsets_q=OFF, offsets_k=OFF)),
    ("^k: .*does not go with", (Q, PK, PK), {}), ("^k: .*does not go with", (Q, K[:1], K[:1]), {}), ("^k: .*does not go with", (Q, K[..., :8], K[..., :8]), {}),
    ("^q: the elements", (APART, K, K), {}), ("^k: the elements", (Q, APART, APART), {}), ("^v: the elements", (Q, Q, APART), {}), ("^o: the elements", (Q, K, K), dict(o=APART)),
    ("^o: .*expected", (Q, K, K), dict(o=Q[:, :4])), ("^o: torch.bfloat16", (Q, K, K), dict(o=Q.bfloat16())), ("^v: needed", (Q, K, None), {}),
    ("^offsets_q and offsets_k", (Q, K, K), dict(offsets_q=OFF)), ("^offsets_q and offsets_k", (Q, K, K), dict(offsets_k=OFF)),
    ("^offsets_q: torch.int64", (PQ, PK, PK), dict(offsets_q=OFF.long(), offsets_k=OFF)), ("^offsets_k: torch.int64", (PQ, PK, PK), dict(offsets_q=OFF, offsets_k=OFF.long())),
    ("^offsets_k: .*expected", (PQ, PK, PK), dict(offsets_q=OFF, offsets_k=OFF[:2])), ("^offsets_q: .*not contiguous", (PQ, PK, PK), dict(offsets_q=torch.zeros(6, dtype=torch.int32)[::2], offsets_k=OFF)),
    ("^offsets_k: .*not contiguous", (PQ, PK, PK), dict(offsets_q=OFF, offsets_k=torch.zeros(6, dtype=torch.int32)[::2])),
    ("^offsets_q: expected .B . 1.", (PQ, PK, PK), dict(offsets_q=OFF[:0], offsets_k=OFF[:0])), ("^offsets_q: expected .B . 1.", (PQ, PK, PK), dict(offsets_q=OFF.view(1, 3), offsets_k=OFF.view(1, 3))),
    ("^window: ", (Q, K, K), dict(window=(-2, 0))), ("^window: ", (Q, K, K), dict(window=(-1, -2)))])
def test_attention_forward_binding_says_what_it_refuses(text, args, kw):
    refused(lambda: b.attention_forward(*args, **kw), text)


@pytest.mark.parametrize("text,args,kw", [
    (ON_CPU, (Q, K, K, Q, LSE, Q), {}), (ON_CPU, (Q, K, K, Q, LSE, Q), dict(dq=Q, dk=K, dv=K)), (ON_CPU, (PQ, PK, PK, PQ, PLSE, PQ), dict(offsets_q=OFF, offsets_k=OFF)),
    ("^k: .*does not go with", (Q, K[:1], K, Q, LSE, Q), {}), ("^v: .*expected", (Q, K, K[:, :6], Q, LSE, Q), {}), ("^v: torch.bfloat16", (Q, K, K.bfloat16(), Q, LSE, Q), {}),
    ("^o: .*expected", (Q, K, K, Q[:, :4], LSE, Q), {}), ("^o: torch.bfloat16", (Q, K, K, Q.bfloat16(), LSE, Q), {}), ("^o: the elements", (Q, K, K, APART, LSE, Q), {}),
    ("^o: needed", (Q, K, K, None, LSE, Q), {}), ("^lse: .*expected", (Q, K, K, Q, LSE[:1], Q), {}), ("^lse: .*expected", (Q, K, K, Q, LSE[:, :, :4], Q), {}),
    ("^lse: .*expected", (PQ, PK, PK, PQ, PLSE.t().contiguous(), PQ), dict(offsets_q=OFF, offsets_k=OFF)), ("^lse: torch.bfloat16", (Q, K, K, Q, LSE.bfloat16(), Q), {}),
    ("^lse: .*not contiguous", (Q, K, K, Q, torch.zeros(2, 5, 4).transpose(1, 2), Q), {}), ("^lse: needed", (Q, K, K, Q, None, Q), {}),
    ("^do: .*expected", (Q, K, K, Q, LSE, K), {}), ("^do: torch.bfloat16", (Q, K, K, Q, LSE, Q.bfloat16()), {}), ("^do: the elements", (Q, K, K, Q, LSE, APART), {}), ("^do: needed", (Q, K, K, Q, LSE, None), {}),
    ("^dq: .*expected", (Q, K, K, Q, LSE, Q), dict(dq=K)), ("^dk: .*expected", (Q, K, K, Q, LSE, Q), dict(dk=Q)), ("^dv: .*expected", (Q, K, K, Q, LSE, Q), dict(dv=K[:, :6])),
    ("^dq: torch.bfloat16", (Q, K, K, Q, LSE, Q), dict(dq=Q.bfloat16())), ("^dq: the elements", (Q, K, K, Q, LSE, Q), dict(dq=APART)),
    ("^offsets_q and offsets_k", (Q, K, K, Q, LSE, Q), dict(offsets_q=OFF))])
def test_attention_backward_binding_says_what_it_refuses(text, args, kw):
    refused(lambda: b.attention_backward(*args, **kw), text)


RQ, RK, G, POS, FREQ = torch.zeros(5, 4, 32), torch.zeros(5, 2, 32), torch.ones(32), torch.zeros(5, 2, dtype=torch.int32), torch.zeros(16)
ROT_SHARED = [      # (text, what is given in place of the usual)
    ("^gamma_q: .*expected", dict(gq=G[:8])), ("^gamma_k: .*expected", dict(gk=G[:8])), ("^gamma_q: torch.bfloat16", dict(gq=G.bfloat16())), ("^gamma_k: torch.float64", dict(gk=G.double())),
    ("^gamma_q: .*not contiguous", dict(gq=torch.ones(64)[::2])), ("^gamma_k: .*not contiguous", dict(gk=torch.ones(64)[::2])),
    ("^positions: torch.int64", dict(pos=POS.long())), ("^positions: .*expected", dict(pos=POS[:4])), ("^positions: .*expected", dict(pos=POS[:, :1])), ("^positions: needed", dict(pos=None)),
    ("^positions: .*expected", dict(sections=[16])), ("^positions: .*not contiguous", dict(pos=torch.zeros(2, 5, dtype=torch.int32).t())), ("^frequencies: .*expected", dict(freq=FREQ[:8])),
    ("^frequencies: torch.float64", dict(freq=FREQ.double())), ("^frequencies: needed", dict(freq=None)), ("^frequencies: .*not contiguous", dict(freq=torch.zeros(32)[::2])),
    ("^sections: at most 4", dict(sections=[2, 2, 4, 4, 4])), ("^q or k: one of them", dict(q=None, k=None)), ("^q: expected", dict(q=RQ[0], k=None)),
    ("^k: .*does not go with", dict(k=RK[:4])), ("^k: .*does not go with", dict(k=RK[..., :16])), ("^k: .*does not go with", dict(k=RK[None])), ("^q: torch.float16", dict(q=RQ.half())),
    ("^k: torch.float16", dict(q=None, k=RK.half()))]


def rot_args(kw):
    d = dict(q=RQ, k=RK, gq=G, gk=G, pos=POS, freq=FREQ, sections=[8, 8])
    d.update(kw)
    return d


@pytest.mark.parametrize("text,kw", [(ON_CPU, {}), (ON_CPU, dict(q=None)), (ON_CPU, dict(k=None, gq=None)), (ON_CPU, dict(sections=[], pos=None, freq=None)), (ON_CPU, dict(yq=RQ, yk=RK))] + ROT_SHARED + [
    ("^k: torch.bfloat16", dict(k=RK.bfloat16())), ("^q: the elements", dict(q=torch.zeros(5, 4, 64)[..., ::2])), ("^k: the elements", dict(k=torch.zeros(5, 2, 64)[..., ::2])),
    ("^yq: .*expected", dict(yq=RK)), ("^yk: .*expected", dict(yk=RQ)), ("^yq: torch.bfloat16", dict(yq=RQ.bfloat16())), ("^yk: the elements", dict(yk=torch.zeros(5, 2, 64)[..., ::2]))])
def test_norm_rotary_forward_binding_says_what_it_refuses(text, kw):
    d = rot_args(kw)
    refused(lambda: b.norm_rotary_forward(d["q"], d["k"], d["gq"], d["gk"], d["pos"], d["freq"], d["sections"], yq=d.get("yq"), yk=d.get("yk")), text)


@pytest.mark.parametrize("text,kw", [(ON_CPU, {}), (ON_CPU, dict(q=None)), (ON_CPU, dict(k=None)), (ON_CPU, dict(xq=None, xk=None, norm=False)), (ON_CPU, dict(dq=RQ, dk=RK, dgq=G, dgk=G + 0))] + [
    (text, kw) for text, kw in ROT_SHARED] + [
    ("^dyk: torch.bfloat16", dict(k=RK.bfloat16())), ("^dyq: the elements", dict(q=torch.zeros(5, 4, 64)[..., ::2])), ("^q: needed", dict(xq=None)), ("^k: needed", dict(xk=None)),
    ("^q: .*expected", dict(xq=RK)), ("^k: .*expected", dict(xk=RQ)), ("^q: torch.bfloat16", dict(xq=RQ.bfloat16())), ("^k: the elements", dict(xk=torch.zeros(5, 2, 64)[..., ::2])),
    ("^dq: .*expected", dict(dq=RK)), ("^dk: .*expected", dict(dk=RQ)), ("^dq: torch.bfloat16", dict(dq=RQ.bfloat16())), ("^dgamma_q: .*expected", dict(dgq=G[:3])), ("^dgamma_k: torch.bfloat16", dict(dgk=G.bfloat16())),
    ("^dgamma_q: .*not contiguous", dict(dgq=torch.ones(64)[::2]))])
def test_norm_rotary_backward_binding_says_what_it_refuses(text, kw):
    """(q and k of rot_args stand for the incoming gradients here, as which the sizes are taken; xq and xk for what was normed.)"""
    d = rot_args(kw)
    refused(lambda: b.norm_rotary_backward(d.get("xq", RQ), d.get("xk", RK), d["gq"], d["gk"], d["pos"], d["freq"], d["sections"], d["q"], d["k"], norm=d.get("norm", True),
                                           dq=d.get("dq"), dk=d.get("dk"), dgamma_q=d.get("dgq"), dgamma_k=d.get("dgk")), text)


@pytest.mark.parametrize("text,tensors", [
    ("needs a tensor", []), ("tensor 0: all tensors belong on one GPU", [torch.zeros(3)]), ("^tensor 0: torch.float16", [torch.zeros(3, dtype=torch.float16)]),
    ("^tensor 0: .*not contiguous", [torch.zeros(6)[::2]]), ("^tensor 0: needed", [None])])
def test_gradient_table_says_what_it_refuses(text, tensors):
    refused(lambda: b.gradient_table(tensors), text)


@pytest.mark.parametrize("norm", [torch.zeros(2), torch.zeros(1, dtype=torch.float64), torch.zeros(1, dtype=torch.bfloat16), torch.zeros(())])
def test_clip_gradients_says_what_it_refuses(norm):
    table = b.GradientTable.__new__(b.GradientTable)
    table.places, table.pointers = [], Place()
    refused(lambda: b.clip_gradients(table, 1.0, norm=norm), "^norm: .*expected")
