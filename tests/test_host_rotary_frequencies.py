"""Frequencies that require a gradient (no GPU needed: refused before anything else is looked at)."""
import pytest
import torch

from paper_2205_14135_amd.autograd import flash_attention, rotary_embedding
from paper_2205_14135_amd.rotary import Rotary, rotary_frequencies


def test_frequencies_that_require_a_gradient_are_refused():
    """There is none for them, and a program that learns them would not notice."""
    f = rotary_frequencies(64)[0].requires_grad_(True)
    q = torch.zeros(1, 2, 8, 64, dtype=torch.bfloat16)
    with pytest.raises(ValueError, match="frequencies require a gradient"):
        rotary_embedding(q, q, Rotary(f))
    for call in (lambda: rotary_embedding(q, q, Rotary(f.detach())), lambda: flash_attention(q, q, q, rotary=Rotary(f))):
        with pytest.raises(RuntimeError, match="GPU only"):     # (tensors on the CPU)
            call()
    with torch.no_grad(), pytest.raises(RuntimeError, match="GPU only"):
        rotary_embedding(q, q, Rotary(f))


@pytest.mark.gpu
def test_frequencies_that_require_a_gradient_on_the_gpu():
    f = rotary_frequencies(64)[0].cuda().requires_grad_(True)
    q, k, v = (torch.randn(1, 2, 8, 64, device="cuda").to(torch.bfloat16) for _ in range(3))
    with pytest.raises(ValueError, match="frequencies require a gradient"):
        flash_attention(q, k, v, rotary=Rotary(f))
    with torch.no_grad():
        got = rotary_embedding(q, k, Rotary(f))
    assert all(torch.equal(a, b) for a, b in zip(got, rotary_embedding(q, k, Rotary(f.detach()))))
