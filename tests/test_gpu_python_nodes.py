"""The nodes in Python of the norm with the rotation and of windowed attention, which functorch's transforms, forward-mode differentiation, tracing and compilation get: the native nodes' bits and rules."""
import pytest
import torch
from torch.autograd import forward_ad

from paper_2205_14135_amd import autograd
from paper_2205_14135_amd.autograd import flash_attention, norm_rotary_embedding
from paper_2205_14135_amd.rotary import HeadNorm, Rotary

pytestmark = pytest.mark.gpu


def _leaves(kind=torch.float32, requires_grad=True):
    gen = torch.Generator(device="cuda").manual_seed(12)
    q, k, gq, gk = (torch.randn(2, 45, h, 64, generator=gen, device="cuda").to(torch.bfloat16).transpose(1, 2) for h in (3, 1, 3, 1))
    wq, wk = ((1.0 + 0.25 * torch.randn(64, generator=gen, device="cuda")).to(kind) for _ in range(2))
    return [x.requires_grad_(requires_grad) for x in (q, k, wq, wk)], (gq, gk)


@pytest.mark.parametrize("kind", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("r,interleaved", [(0, False), (64, False), (20, False), (32, True)])
@pytest.mark.parametrize("given", [False, True])
def test_the_same_bits(kind, r, interleaved, given):
    leaves, grads = _leaves(kind)
    q, k, wq, wk = leaves
    rotary = Rotary.make(r, interleaved=interleaved, scaling="parts", factor=4.0) if r else None
    positions = torch.arange(100, 145, dtype=torch.int32, device="cuda") if given and r else None
    norm = HeadNorm(wq, wk, eps=1e-4)
    f, i, m = (None, False, 1.0) if rotary is None else (rotary.frequencies, rotary.interleaved, rotary.magnitude)
    native = norm_rotary_embedding(q, k, norm, rotary, positions)
    python = autograd._NormRotaryEmbedding.apply(q, k, wq, wk, norm.eps, f, i, m, positions)
    assert all(torch.equal(a, b) for a, b in zip(native, python))
    a, b = (torch.autograd.grad(ys, leaves, grads, retain_graph=True) for ys in (native, python))
    assert all(torch.equal(x, y) and x.dtype == y.dtype for x, y in zip(a, b))
    # of one output: the other one's gradient is none, or zeros
    a, b = (torch.autograd.grad(ys[1], (k, wk), grads[1]) for ys in (native, python))
    assert all(torch.equal(x, y) for x, y in zip(a, b))


def test_no_second_gradients_and_no_changed_inputs():
    leaves, grads = _leaves()
    q, k, wq, wk = leaves
    run = lambda: autograd._NormRotaryEmbedding.apply(q, k, wq, wk, 1e-6, None, False, 1.0, None)  # noqa: E731
    dq, = torch.autograd.grad(run()[0], q, grads[0], create_graph=True)
    with pytest.raises(RuntimeError):
        torch.autograd.grad(dq.float().sum(), wq)
    for x in (q, wq):
        ys = run()
        with torch.no_grad():
            x.add_(1)
        with pytest.raises(RuntimeError, match="inplace"):
            torch.autograd.grad(ys, leaves, grads)


def test_transforms_keep_it():
    (q, k, wq, wk), grads = _leaves(requires_grad=False)
    norm, rotary = HeadNorm(wq, wk), Rotary.make(64)
    with pytest.raises(RuntimeError, match="setup_context"):
        torch.func.vmap(lambda x, y: norm_rotary_embedding(x, y, norm, rotary))(q.unsqueeze(0), k.unsqueeze(0))
    with pytest.raises(RuntimeError, match="setup_context"):
        torch.func.grad(lambda x: norm_rotary_embedding(x, k, norm, rotary)[0].float().sum())(q)
    with forward_ad.dual_level():
        with pytest.raises(NotImplementedError):
            norm_rotary_embedding(forward_ad.make_dual(q, grads[0]), k, norm, rotary)
    traced = torch.jit.trace(lambda x, y: norm_rotary_embedding(x, y, norm, rotary), (q, k), check_trace=False)
    others = [x.flip(2).contiguous() for x in (q, k)]
    assert all(torch.equal(a, b) for a, b in zip(traced(*others), norm_rotary_embedding(*others, norm, rotary)))


def test_windowed_attention_under_transforms_keeps_its_node_in_python():
    gen = torch.Generator(device="cuda").manual_seed(3)
    q, k, v, g = (torch.randn(1, 2, 90, 64, generator=gen, device="cuda").to(torch.bfloat16) for _ in range(4))
    run = lambda x, y, z: flash_attention(x, y, z, causal=True, window=20, sinks=2)  # noqa: E731
    with pytest.raises(RuntimeError, match="setup_context"):
        torch.func.vmap(run)(*(x.unsqueeze(0) for x in (q, k, v)))
    with forward_ad.dual_level():
        with pytest.raises(NotImplementedError):
            run(forward_ad.make_dual(q, g), k, v)
    traced = torch.jit.trace(run, (q, k, v), check_trace=False)
    others = [x.flip(2).contiguous() for x in (q, k, v)]
    assert torch.equal(traced(*others), run(*others))


@pytest.mark.parametrize("node", ["native", "python"])
def test_key_lengths_that_change_before_the_backward_pass_are_noticed(node):
    gen = torch.Generator(device="cuda").manual_seed(4)
    leaves = [torch.randn(2, 2, 90, 64, generator=gen, device="cuda").to(torch.bfloat16).requires_grad_(True) for _ in range(3)]
    lengths = torch.tensor([90, 40], dtype=torch.int32, device="cuda")
    if node == "native":
        out = flash_attention(*leaves, causal=True, window=20, sinks=2, softmax_scale=0.125, key_lengths=lengths)
    else:
        out = autograd._WindowAttention.apply(*leaves, 0.125, 0.0, 0, 0, lengths, 20, 2)
    lengths.sub_(10)
    with pytest.raises(RuntimeError, match="inplace"):
        torch.autograd.grad(out, leaves, torch.ones_like(out))
