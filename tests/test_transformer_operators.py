"""Refusals of the attention calls (no GPU needed: nothing is launched) and their plain forms against differences."""
import ctypes as C
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
        return lib.dat_attention_forward(shape, x["q"], x["k"], x["v"], x["o"], lse, stream)
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
    assert lib.dat_attention_forward(None, h, h, h, h, P, None) == 1 and lib.dat_attention_forward(s, None, h, h, h, P, None) == 1
    assert lib.dat_attention_forward(s, h, h, h, None, P, None) == 1
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
                 lambda: b.attention_forward(q, k, k, o=q[:, :4]), lambda: b.attention_forward(q, k, None), lambda: b.attention_forward(q, k, k, window=(1,)),
                 lambda: b.attention_backward(q, k, k, q, lse[:1], q), lambda: b.attention_backward(q, k, k, q, lse, k), lambda: b.attention_backward(q, k, k, q, lse, q, dk=q),
                 lambda: b.attention_backward(q, k, k, q, lse, q)):
        with pytest.raises((ValueError, AttributeError)):
            call()


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
