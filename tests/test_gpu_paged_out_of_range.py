"""Starts beyond what there is mean the same to the append and to the attention: a token has one position."""
import pytest
import torch

from paper_2205_14135_amd import binding
from paper_2205_14135_amd.rotary import Rotary, rotary_frequencies
from tests import paged_helpers as ph

pytestmark = pytest.mark.gpu


def ints(x):
    return torch.tensor(x, dtype=torch.int32).cuda()


# starts, and which rows belong to which sequence once they are forced into 0 .. T
@pytest.mark.parametrize("starts,forced", [([0, 5, 400], [0, 5, 40]), ([-9, 5, 30], [0, 5, 30]), ([-2 ** 31, 33, 2 ** 31 - 1], [0, 33, 40]), ([0, 40, 2 ** 31 - 1], [0, 40, 40])])
@pytest.mark.parametrize("d", [32, 128])
def test_starts_outside_the_rows(starts, forced, d):
    """T = 40 rows.  What the append writes and turns, and what the attention sees, are those of the starts forced into range, bit by bit."""
    T, Hq, Hk, page = 40, 4, 2, 16
    gen = torch.Generator().manual_seed(d)
    q, k, v = (torch.randn(T, h, d, generator=gen).to(torch.bfloat16).cuda() for h in (Hq, Hk, Hk))
    rotary = Rotary(rotary_frequencies(d)[0].cuda())
    held = [torch.randn(12, Hk, page, d, generator=gen).to(torch.bfloat16).cuda() for _ in range(2)]
    table, lengths = torch.randperm(12, generator=gen).to(torch.int32).view(2, 6).cuda(), ints([70, 90])

    def run(s):
        kc, vc = (c.clone() for c in held)
        turned = torch.full_like(q, 7.0)
        binding.attn_paged_append(k, v, kc, vc, table, lengths, ints(s), Q=q, rotary=rotary, out=turned)
        out, lse = torch.full_like(q, 7.0), torch.full((Hq, T), 7.0, device="cuda")
        binding.attn_paged_fwd(turned, kc, vc, table, lengths, ints(s), softmax_scale=d ** -0.5, out=out, lse=lse)
        return kc, vc, turned, out, lse

    for got, want in zip(run(starts), run(forced)):
        assert torch.equal(got, want)


def test_starts_that_fall_write_no_row_behind_a_length():
    """Starts are documented as rising; others give unspecified rows, but nothing behind a sequence's length, whose rows may be another one's."""
    T, Hk, page, d = 40, 2, 16, 64
    gen = torch.Generator().manual_seed(3)
    k, v = (torch.randn(T, Hk, d, generator=gen).to(torch.bfloat16).cuda() for _ in range(2))
    table, lengths = torch.arange(18, dtype=torch.int32).view(3, 6).cuda(), [70, 90, 50]
    for starts in ([0, 10, 2, 3], [0, 30, 5, 6], [20, 10, 30, 11]):
        kc, vc = (torch.full((18, Hk, page, d), 7.0, dtype=torch.bfloat16, device="cuda") for _ in range(2))
        binding.attn_paged_append(k, v, kc, vc, table, ints(lengths), ints(starts))
        for c in (kc, vc):
            rows = c.view(3, 6, Hk, page, d).transpose(2, 3).reshape(3, 6 * page, Hk, d)
            assert all(bool((rows[b, n:] == 7.0).all()) for b, n in enumerate(lengths))
