"""Gradients that start anywhere in memory: a program that lays outputs end to end hands their nodes views of one tensor, and such a view need not start on 16 bytes."""
import pytest
import torch

from paper_2205_14135_amd import autograd
from paper_2205_14135_amd.autograd import flash_attention, norm_rotary_embedding, rotary_embedding
from paper_2205_14135_amd.rotary import HeadNorm, Rotary

pytestmark = pytest.mark.gpu


def _tensors(*heads, N=150, d=64, dtype=torch.bfloat16):
    gen = torch.Generator(device="cuda").manual_seed(31)
    return [torch.randn(2, h, N, d, generator=gen, device="cuda").to(dtype) for h in heads]


def _moved(x, elements):
    """The same numbers, sizes and strides, `elements` behind a start on 16 bytes."""
    y = torch.empty(x.numel() + elements, dtype=x.dtype, device=x.device)[elements:].view(x.shape).copy_(x)
    assert y.stride() == x.stride() and y.data_ptr() % 16 == 2 * elements % 16
    return y


def _window(leaves, node, window, **kw):
    if node == "native":
        return flash_attention(*leaves, causal=True, window=window, sinks=3, softmax_scale=0.125, **kw)
    return autograd._WindowAttention.apply(*leaves, 0.125, 0.0, 0, 0, kw.get("key_lengths"), window, 3)


# (a window of 200 hides nothing of 150 keys)
@pytest.mark.parametrize("window", [40, 200])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("node", ["native", "python"])
def test_window(node, dtype, window):
    q, k, v, do = _tensors(2, 2, 2, 2, dtype=dtype)
    leaves = [x.requires_grad_(True) for x in (q, k, v)]
    lengths = torch.tensor([150, 77], dtype=torch.int32, device="cuda")
    out = _window(leaves, node, window, key_lengths=lengths)
    want = torch.autograd.grad(out, leaves, do, retain_graph=True)
    for elements in (1, 4, 7, 8):
        got = torch.autograd.grad(out, leaves, _moved(do, elements), retain_graph=True)
        assert all(torch.equal(a, b) for a, b in zip(got, want)), elements


@pytest.mark.parametrize("node", ["native", "python"])
def test_window_behind_a_concatenation(node):
    """(the concatenation's gradient is cut into views with the output's own strides)"""
    q, k, v, do = _tensors(2, 2, 2, 2)
    leaves = [x.requires_grad_(True) for x in (q, k, v)]
    want = torch.autograd.grad(_window(leaves, node, 40), leaves, do)
    first = torch.zeros(3, dtype=q.dtype, device="cuda")
    out = _window(leaves, node, 40)
    got = torch.autograd.grad(torch.cat([first, out.flatten()]), leaves, torch.cat([first, do.flatten()]))
    assert all(torch.equal(a, b) for a, b in zip(got, want))


def _turned(q, k, weights, node, normed):
    if normed:
        norm, rotary = HeadNorm(*weights), Rotary.make(64)
        if node == "native":
            return norm_rotary_embedding(q, k, norm, rotary)
        return autograd._NormRotaryEmbedding.apply(q, k, *weights, norm.eps, rotary.frequencies, False, 1.0, None)
    rotary = Rotary.make(64)
    if node == "native":
        return rotary_embedding(q, k, rotary)
    return autograd._RotaryEmbedding.apply(q, k, rotary.frequencies, False, 1.0, None, False)


@pytest.mark.parametrize("normed", [False, True])
@pytest.mark.parametrize("node", ["native", "python"])
def test_rotation(node, normed):
    q, k, gq, gk = _tensors(3, 1, 3, 1)
    weights = [torch.linspace(0.5, 1.5, 64, device="cuda", requires_grad=normed) for _ in range(2)]
    leaves = [q.requires_grad_(True), k.requires_grad_(True)] + (weights if normed else [])
    ys = _turned(q, k, weights, node, normed)
    want = torch.autograd.grad(ys, leaves, (gq, gk), retain_graph=True)
    for elements in (1, 4, 7, 8):
        got = torch.autograd.grad(ys, leaves, [_moved(g, elements) for g in (gq, gk)], retain_graph=True)
        assert all(torch.equal(a, b) for a, b in zip(got, want)), elements
