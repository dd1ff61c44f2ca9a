"""Outputs that the paged calls make by themselves hold what they are and no gaps of their inputs."""
import pytest
import torch

from paper_2205_14135_amd import binding
from paper_2205_14135_amd.rotary import Rotary

pytestmark = pytest.mark.gpu


def _layouts():
    """[5, 4, 64] rows of Q: packed, a part of a projection's rows, one token of each sequence of a long tensor, heads in front of tokens, one row for all tokens."""
    gen = torch.Generator(device="cuda").manual_seed(1)
    normal = lambda *shape: torch.randn(shape, generator=gen, device="cuda").to(torch.bfloat16)
    return {"packed": normal(5, 4, 64), "fused": normal(5, 12, 64)[:, :4], "token": normal(5, 100, 4, 64)[:, 17], "heads": normal(4, 5, 64).transpose(0, 1),
            "heads_part": normal(4, 9, 64).transpose(0, 1)[2:7], "repeated": normal(1, 4, 64).expand(5, 4, 64)}


@pytest.mark.parametrize("layout", ["packed", "fused", "token", "heads", "heads_part", "repeated"])
def test_outputs_have_no_gaps(layout):
    q = _layouts()[layout]
    rotary = Rotary.make(64)
    kc, vc = (torch.randn(5, 2, 16, 64, device="cuda").to(torch.bfloat16) for _ in range(2))
    table = torch.arange(5, dtype=torch.int32, device="cuda").view(5, 1)
    lengths = torch.tensor([3, 1, 16, 9, 2], dtype=torch.int32, device="cuda")
    k, v = (torch.randn(5, 2, 64, device="cuda").to(torch.bfloat16) for _ in range(2))
    turned = binding.attn_paged_append(k, v, kc, vc, table, lengths, Q=q, rotary=rotary)
    out, lse = binding.attn_paged_fwd(q, kc, vc, table, lengths, softmax_scale=0.125)
    given = torch.empty(5, 4, 64, dtype=torch.bfloat16, device="cuda"), torch.empty(5, 4, 64, dtype=torch.bfloat16, device="cuda")
    binding.attn_paged_append(k, v, kc, vc, table, lengths, Q=q, rotary=rotary, out=given[0])
    _, want_l = binding.attn_paged_fwd(q, kc, vc, table, lengths, softmax_scale=0.125, out=given[1])
    assert torch.equal(lse, want_l)
    for got, want in zip((turned, out), given):
        assert torch.equal(got, want)
        assert got.untyped_storage().nbytes() == 2 * got.numel()
        assert got.stride() == ((64, 5 * 64, 1) if layout.startswith("heads") else (4 * 64, 64, 1))
