"""The node in Python of windowed attention, which functorch's transforms, forward-mode differentiation, tracing and compilation get."""
import pytest
import torch

from paper_2205_14135_amd import autograd
from paper_2205_14135_amd.autograd import flash_attention

pytestmark = pytest.mark.gpu


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
