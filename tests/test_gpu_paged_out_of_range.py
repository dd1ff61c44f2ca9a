"""Lengths and starts beyond what there is mean the same to the append and to the attention: a token has one position."""
import copy

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


@pytest.mark.parametrize("d,page", [(32, 16), (64, 32), (128, 16)])
@pytest.mark.parametrize("new", [1, 20, 150])
@pytest.mark.parametrize("over", [1, 9, 1000, 2 ** 30])
def test_lengths_beyond_the_table(new, over, d, page):
    """A length `over` tokens beyond what a row of the table holds, causal: token i stands at position length - new + i, as in the append, and sees the keys
    up to its own that there are."""
    capacity = 320
    batch = ph.Batch([capacity - new, 100], [new, 3], 4, 2, d, "bf16", page, seed=d + new)
    q, kc, vc, table, lengths, starts = batch.gpu()
    lengths[0] += over
    assert table.shape[1] * page == capacity
    out, lse = binding.attn_paged_fwd(q, kc, vc, table, lengths, starts, softmax_scale=batch.tau)
    # every token a sequence of its own, as long as it sees
    plain = copy.copy(batch)
    positions = [capacity + over - new + i for i in range(new)] + [100, 101, 102]
    plain.B, plain.new, plain.starts = batch.tokens, [1] * batch.tokens, torch.arange(batch.tokens + 1)
    plain.lengths = [min(p + 1, capacity) for p in positions]
    plain.table = torch.cat([batch.table[:1].expand(new, -1), batch.table[1:].expand(3, -1)])
    want, want_l, bound, bound_l = ph.attention(plain, True)
    ph.assert_within(out, want, bound, "O")
    ph.assert_within(lse, want_l, bound_l, "LSE")


@pytest.mark.parametrize("T,d,Hq,Hk", [(64, 64, 8, 2), (2000, 64, 8, 2), (4000, 128, 4, 4)])
def test_starts_that_share_rows_are_not_begun(T, d, Hq, Hk):
    """Every second sequence would have all rows: many times the work of any rising starts."""
    B, page, width = 64, 16, 40
    q = torch.randn(T, Hq, d, device="cuda").to(torch.bfloat16)
    kc, vc = (torch.randn(8, Hk, page, d, device="cuda").to(torch.bfloat16) for _ in range(2))
    table, lengths = torch.zeros(B, width, dtype=torch.int32, device="cuda"), ints([page * width] * B)
    out, lse = torch.full_like(q, 7.0), torch.full((Hq, T), 7.0, device="cuda")
    for causal in (True, False):
        binding.attn_paged_fwd(q, kc, vc, table, lengths, ints([0, T] * (B // 2) + [0]), softmax_scale=0.1, causal=causal, out=out, lse=lse)
        assert bool((out == 7.0).all()) and bool((lse == 7.0).all())


@pytest.mark.parametrize("B,width", [(1 << 16, 1024), (1 << 13, 512)])
def test_starts_that_share_rows_beyond_what_doubles_hold(B, width):
    """(2^57 and 2^51 units of work, where rising starts give 2^45 at most)"""
    T, Hq, Hk, d, page = 1 << 16, 64, 8, 16, 4096
    q = torch.zeros(T, Hq, d, dtype=torch.bfloat16, device="cuda")
    kc, vc = (torch.zeros(1, Hk, page, d, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    table, lengths = torch.zeros(1, width, dtype=torch.int32, device="cuda").expand(B, width), ints([page * width] * B)
    out, lse = torch.full_like(q, 7.0), torch.full((Hq, T), 7.0, device="cuda")
    binding.attn_paged_fwd(q, kc, vc, table, lengths, ints([0, T] * (B // 2) + [0]), softmax_scale=0.1, causal=False, out=out, lse=lse)
    assert bool((out == 7.0).all()) and bool((lse == 7.0).all())
