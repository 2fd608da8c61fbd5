"""What the binding allocates does not depend on torch's default type: the library writes 32-bit numbers into it."""
import ast
import inspect

import pytest
import torch

import paper_2206_06257_amd.binding as b

MAKERS = ("empty", "zeros", "ones", "full", "tensor", "arange", "rand", "randn", "linspace")


def test_every_new_tensor_names_its_type():
    calls = [n for n in ast.walk(ast.parse(inspect.getsource(b))) if isinstance(n, ast.Call) and isinstance(n.func, ast.Attribute)
             and isinstance(n.func.value, ast.Name) and n.func.value.id == "torch" and n.func.attr in MAKERS]
    assert len(calls) > 20
    without = [n.lineno for n in calls if not any(k.arg == "dtype" for k in n.keywords)]
    assert not without, "binding.py, lines %s" % without


@pytest.mark.parametrize("default", [torch.float64, torch.bfloat16])
def test_frequencies_and_moments_are_fp32(default):
    try:
        torch.set_default_dtype(default)
        made = [b.rotary_frequencies([2, 4], device="cpu"), b.rotary_frequencies([], device="cpu")] + list(b.adamw_state(10, 2, device="cpu")[:2])
    finally:
        torch.set_default_dtype(torch.float32)
    assert all(t.dtype == torch.float32 for t in made)


@pytest.mark.gpu
@pytest.mark.parametrize("default", [torch.float64, torch.bfloat16])
def test_calls_under_another_default_type(default):
    """Every call that allocates: results of the same types and bits as under fp32."""
    g = torch.Generator(device="cuda").manual_seed(1)
    randn = lambda *shape: torch.randn(*shape, device="cuda", generator=g, dtype=torch.float32)  # noqa: E731
    q, k, x, logits, grads = randn(1, 70, 4, 256), randn(1, 70, 2, 256), randn(2, 6, 6, 64), randn(50, 1000), randn(3000)
    gamma, labels = randn(256), torch.arange(50, dtype=torch.int32, device="cuda")
    pos = torch.arange(70, dtype=torch.int32, device="cuda").view(1, 70, 1)
    m, v, scales = b.adamw_state(3000, 1, bits=8)
    offsets = torch.tensor([0, 3000], device="cuda")

    def calls():
        freq = b.rotary_frequencies([128])
        out = list(b.norm_rotary_forward(q, k, gamma, gamma, pos, freq, [128])) + list(b.norm_rotary_backward(q, k, gamma, gamma, pos, freq, [128], q, k))
        h = [t[..., :128] for t in (q, k, k)]
        o, lse = b.attention_forward(*h)
        out += [o, lse] + list(b.attention_backward(*h, o, lse, o))
        y, mean, rstd = b.group_norm_forward(x, None, None, 8)
        out += [y, mean, rstd] + list(b.group_norm_backward(x, x, None, None, mean, rstd, 8))
        out += list(b.log_probs(logits, labels, 3)) + list(b.adamw_moments(m, v, scales, offsets))
        return out + list(b.adamw_state(10, 1)[:2]) + [b.clip_gradients(b.gradient_table([grads.clone()]), 1.0)]

    want = calls()
    try:
        torch.set_default_dtype(default)
        got = calls()
    finally:
        torch.set_default_dtype(torch.float32)
    assert len(got) == len(want)
    for n, (a, c) in enumerate(zip(got, want)):
        assert a.dtype == c.dtype and torch.equal(a, c), n
