"""Attention of new tokens over a paged cache with a sliding window and first tokens that stay visible, against the same in 64 bits."""
import math
import threading

import pytest
import torch

from paper_2205_14135_amd import binding
from paper_2205_14135_amd.autograd import flash_attention
from paper_2205_14135_amd.paged import PageTable
from paper_2205_14135_amd.rotary import HeadNorm, Rotary
from tests import paged_helpers as ph

pytestmark = pytest.mark.gpu


def _seen(batch, b, window, sinks):
    """[new tokens, keys] of sequence b.  (A length below the number of new tokens leaves the first ones at negative positions.)"""
    m = batch.new[b]
    n = batch.lengths[b]
    pos, key = torch.arange(n - m, n).unsqueeze(1), torch.arange(n).unsqueeze(0)
    return (key <= pos) & ((key > pos - window) | (key < sinks))


def attention(batch, window, sinks, tau=None):
    """As paged_helpers.attention, bounds and all, with another rule of what is seen."""
    u = torch.finfo(batch.dtype).eps / 2
    tau = batch.tau if tau is None else tau
    O, L = torch.zeros(batch.tokens, batch.Hq, batch.d, dtype=torch.float64), torch.full((batch.Hq, batch.tokens), -math.inf, dtype=torch.float64)
    bO, bL = torch.zeros_like(O), torch.zeros_like(L)
    G = batch.Hq // batch.Hk
    for b in range(batch.B):
        m, n, at = batch.new[b], batch.lengths[b], int(batch.starts[b])
        if m == 0 or n == 0:
            continue
        seen = _seen(batch, b, window, sinks)
        some = seen.any(-1)
        k, v = batch.rows(batch.kc, b), batch.rows(batch.vc, b)
        used = seen.any(0)
        k, v = (torch.where(used.view(-1, 1, 1), x, torch.zeros_like(x)) for x in (k, v))      # (the others may be NaN)
        for h in range(batch.Hq):
            q, kh, vh = batch.q[at:at + m, h].double(), k[:, h // G], v[:, h // G]
            s = (tau * (q @ kh.t())).masked_fill(~seen, -math.inf)
            size = (tau * (q.abs() @ kh.abs().t())).masked_fill(~seen, 0.0)
            lse = torch.logsumexp(s, -1)
            w = torch.exp(s - lse.unsqueeze(-1)).masked_fill(~seen, 0.0)
            o = w @ vh
            rho = (batch.d + 32) * 2.0 ** -24 * (size.amax(-1) + 8.0)
            spread = w @ vh.abs() + o.abs()
            bound = (u + 2 * rho).unsqueeze(-1) * spread + u * o.abs() + 2.0 ** -24
            if batch.dtype == torch.float16:
                bound = bound + n * 2.0 ** -17 * 2.0 ** -8 * vh.abs().amax()
            O[at:at + m, h] = torch.where(some.unsqueeze(-1), o, torch.zeros_like(o))
            bO[at:at + m, h] = torch.where(some.unsqueeze(-1), bound, torch.zeros_like(bound))
            L[h, at:at + m] = torch.where(some, lse, torch.full_like(lse, -math.inf))
            bL[h, at:at + m] = rho + (n / 32 + 16) * 2.0 ** -24 + 2.0 ** -22 * lse.abs().clamp(max=1e9)
    return O, L, bO, bL


def check(batch, window, sinks, single=False, tau=None, give_away=True, workspace=None):
    if give_away:   # pages that no new token sees a key of: of another sequence by now (here: NaN), or of none
        for b in range(batch.B):
            if batch.lengths[b] == 0 or batch.new[b] == 0:
                continue
            used = _seen(batch, b, window, sinks).any(0)
            for t in range(-(-batch.lengths[b] // batch.page)):
                if not used[t * batch.page:(t + 1) * batch.page].any():
                    number = int(batch.table[b, t])
                    if t % 2 or not 0 <= number < batch.pages:
                        batch.table[b, t] = (-1, 10 ** 9)[t // 2 % 2]
                    else:
                        batch.kc[number], batch.vc[number] = math.nan, math.nan
    q, kc, vc, table, lengths, starts = batch.gpu(single)
    before = [x.clone() for x in (kc, vc)]
    out = torch.empty_strided(q.size(), q.stride(), dtype=q.dtype, device="cuda").fill_(7.0)
    lse = torch.full((batch.Hq, q.shape[0]), 5.0, device="cuda")
    o, l = binding.attn_paged_fwd(q, kc, vc, table, lengths, starts, softmax_scale=tau or batch.tau, out=out, lse=lse, window=window, sinks=sinks, workspace=workspace)
    assert o is out and l is lse
    want, want_l, bound, bound_l = attention(batch, window, sinks, tau)
    ph.assert_within(out[:batch.tokens], want, bound, "O")
    ph.assert_within(lse[:, :batch.tokens], want_l, bound_l, "LSE")
    assert (out[batch.tokens:] == 7.0).all() and (lse[:, batch.tokens:] == 5.0).all()
    for x, y in zip((kc, vc), before):
        assert torch.equal(torch.nan_to_num(x, 3.0), torch.nan_to_num(y, 3.0))
    return out, lse


WINDOWS = [(1, 0), (16, 0), (33, 4), (64, 1), (100, 70), (300, 16)]


@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
@pytest.mark.parametrize("d,page", [(16, 16), (32, 64), (64, 16), (64, 128), (128, 16), (128, 256)])
@pytest.mark.parametrize("Hq,Hk", [(4, 4), (6, 2), (7, 1)])
@pytest.mark.parametrize("window,sinks", WINDOWS)
def test_single_tokens(dtype, d, page, Hq, Hk, window, sinks):
    n = [1, 16, 17, 63, 64, 65, 333, 1000]
    check(ph.Batch([x - 1 for x in n], [1] * len(n), Hq, Hk, d, dtype, page, seed=d + page), window, sinks, single=True)


@pytest.mark.parametrize("d", [32, 64, 128])
@pytest.mark.parametrize("lengths,window,sinks", [([9000], 4000, 4), ([4097, 1, 2500, 700], 2049, 0), ([128 * i + 3 for i in range(1, 12)], 500, 33), ([9000, 30], 5000, 3000)])
def test_long_windows_are_divided(d, lengths, window, sinks):
    check(ph.Batch([x - 1 for x in lengths], [1] * len(lengths), 8, 2, d, "bf16", 16, seed=d), window, sinks, single=True)


@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
@pytest.mark.parametrize("d,page,Hq,Hk", [(16, 32, 4, 2), (32, 16, 3, 3), (64, 64, 8, 2), (64, 16, 5, 1), (128, 16, 4, 4), (128, 128, 6, 2)])
@pytest.mark.parametrize("window,sinks", WINDOWS)
def test_chunks(dtype, d, page, Hq, Hk, window, sinks):
    check(ph.Batch([0, 40, 100, 0, 700, 33], [1, 0, 5, 130, 64, 257], Hq, Hk, d, dtype, page, pad=19, seed=page), window, sinks)


@pytest.mark.parametrize("d", [32, 64, 128])
@pytest.mark.parametrize("window,sinks", [(200, 4), (1000, 0), (70, 1100), (1, 1030)])
def test_long_chunks(d, window, sinks):
    """Blocks of many tiles, in front of them sinks of less and of more than sixteen tiles, whose page numbers come by sixteens."""
    check(ph.Batch([4000, 0, 1500], [700, 900, 1], 4, 2, d, "bf16", 16, pad=3, seed=d), window, sinks)


def test_a_chunk_among_single_tokens():
    check(ph.Batch([900, 0, 2000, 31, 64], [1, 300, 1, 1, 1], 8, 2, 64, "bf16", 16, pad=3, seed=5), 150, 4)


@pytest.mark.parametrize("new", [[1, 500, 1, 16, 17, 0, 1, 9], [40, 33, 300, 64], [1] * 7 + [900]])
def test_few_rows_are_worked_on_apart(new):
    """Long windows, wide tables, d = 128: sequences of at most 32 rows (16 tokens of two heads a group) go to the kernel for single tokens, the others to that for chunks."""
    B = len(new)
    batch = ph.Batch([(b * 1237) % 3000 for b in range(B)], new, 32, 16, 128, "bf16", 16, pad=3, seed=30)
    wide = torch.full((B, 400), -1, dtype=torch.int32)
    wide[:, :batch.table.shape[1]] = batch.table
    batch.table = wide
    assert 16 * (B - 1) * min(6400, 4500) >= 3000 * 64       # (the rule's bound)
    check(batch, 4500, 0)
    check(ph.Batch([(b * 1237) % 3000 for b in range(B)], new, 32, 16, 128, "fp16", 256, pad=3, seed=31), 2600, 1900)


@pytest.mark.parametrize("new", [[1, 500, 1, 16, 17, 0, 1, 9], [40, 33, 300, 64], [1] * 7 + [900]])
@pytest.mark.parametrize("dtype,page,window,sinks", [("fp16", 256, 2600, 1900), ("bf16", 64, 100, 4400), ("fp16", 16, 4096, 4)])
def test_few_rows_apart_with_many_sinks(new, dtype, page, window, sinks):
    """The same two passes over wide pages, and with sinks of many tiles."""
    B = len(new)
    batch = ph.Batch([(b * 1237) % 3000 for b in range(B)], new, 32, 16, 128, dtype, page, pad=3, seed=31)
    wide = torch.full((B, 5120 // page), -1, dtype=torch.int32)
    wide[:, :batch.table.shape[1]] = batch.table
    batch.table = wide
    assert sum(new) * 2 > 32 * B and 16 * (B - 1) * min(5120, window + sinks) >= 3000 * 64       # (larger blocks, and the rule's bound)
    check(batch, window, sinks)


@pytest.mark.parametrize("new", [[2, 3, 1], [1, 1, 1]])
def test_few_tokens_with_starts(new):
    check(ph.Batch([600, 20, 2100], new, 8, 2, 128, "bf16", 16, pad=2, seed=6), 250, 3)


@pytest.mark.parametrize("single", [True, False])
@pytest.mark.parametrize("d,page,Hq,Hk", [(16, 16, 66, 2), (32, 32, 12, 12), (64, 16, 33, 1), (128, 64, 8, 8)])
@pytest.mark.parametrize("window,sinks", [(1, 0), (31, 33), (95, 1), (577, 0), (1500, 65), (6000, 3)])
def test_single_tokens_of_mixed_lengths(d, page, Hq, Hk, window, sinks, single):
    """Without `starts` up to a number of tiles by a workgroup for each, beyond that, and with them, divided."""
    n = [5, 0, 1, 97, 1600, 32, 0, 6400]
    check(ph.Batch([x - 1 if single else max(x - 1, 0) for x in n], [1 if single else min(x, 1) for x in n], Hq, Hk, d, "bf16", page, seed=d + window), window, sinks, single=single)


@pytest.mark.parametrize("B,Hq,Hk,d", [(63, 1, 1, 64), (64, 1, 1, 64), (128, 4, 4, 16), (171, 3, 3, 32), (129, 4, 4, 128), (9, 33 * 32, 32, 64)])
def test_either_side_of_a_number_of_workgroups(B, Hq, Hk, d):
    check(ph.Batch([(37 * i) % 1400 for i in range(B)], [1] * B, Hq, Hk, d, "fp16", 16, seed=B), 1300, 2, single=True)


@pytest.mark.parametrize("Hq,d", [(40, 64), (71, 64), (128, 128)])
def test_many_heads_share_one(Hq, d):
    check(ph.Batch([900, 10, 64], [1, 1, 1], Hq, 1, d, "bf16", 16, seed=7), 100, 2, single=True)
    check(ph.Batch([300, 10], [3, 2], Hq, 1, d, "bf16", 16, seed=8), 100, 2)


@pytest.mark.parametrize("single", [True, False])
@pytest.mark.parametrize("B", [64, 65, 200])
def test_many_sequences(B, single):
    new = [1] * B if single else [(b * 7) % 4 for b in range(B)]
    check(ph.Batch([(b * 37) % 150 for b in range(B)], new, 2, 1, 64, "bf16", 16, seed=B), 40, 3, single=single)


@pytest.mark.parametrize("d", [16, 128])
def test_rows_that_see_nothing(d):
    batch = ph.Batch([-3, -5, -2, 0, -200], [5, 5, 2, 3, 150], 4, 2, d, "bf16", 16, seed=9)
    out, lse = check(batch, 3, 1)
    assert (out[5:10] == 0).all() and torch.isinf(lse[:, 5:10]).all()
    check(ph.Batch([-1, 5, -1], [1, 1, 1], 4, 2, d, "fp16", 16, seed=10), 2, 0, single=True)


@pytest.mark.parametrize("token_major,fused", [(True, False), (False, True), (True, True)])
@pytest.mark.parametrize("new", [[1, 1, 1], [70, 1, 33]])
def test_strides(token_major, fused, new):
    check(ph.Batch([30, 400, 1000], new, 8, 4, 64, "bf16", 32, pad=2, token_major=token_major, fused=fused, seed=11), 90, 5)


@pytest.mark.parametrize("single", [True, False])
@pytest.mark.parametrize("d", [16, 64, 128])
def test_numbers_that_are_no_page_read_as_zeros(d, single):
    batch = ph.Batch([200, 90, 70], [1, 1, 1] if single else [3, 40, 1], 4, 2, d, "bf16", 16, seed=12)
    for b, t, number in ((0, 10, -1), (0, 12, batch.pages), (1, 0, 2 ** 31 - 1), (1, 5, -2 ** 31), (2, 4, batch.pages + 1)):
        batch.table[b, t] = number
    check(batch, 60, 3, single=single)


@pytest.mark.parametrize("scale", [8.0, 30.0])
def test_peaked_rows(scale):
    check(ph.Batch([900, 64, 2000], [1, 1, 1], 8, 2, 64, "bf16", 16, seed=14), 300, 4, single=True, tau=scale / 8.0)
    check(ph.Batch([900, 64], [33, 90], 4, 2, 128, "bf16", 16, seed=15), 300, 4, tau=scale / 11.0)


@pytest.mark.parametrize("new", [[1, 1, 1], [40, 1, 130]])
@pytest.mark.parametrize("window,sinks", [(10 ** 9, 0), (2 ** 31 - 1, 2 ** 31 - 1), (1, 10 ** 12), (700, 700)])
def test_a_window_that_hides_nothing(new, window, sinks):
    """The same as without one, to the bounds of both (the tiles of blocks are the same, so that the order of sums is)."""
    batch = ph.Batch([600, 30, 0], new, 8, 2, 64, "bf16", 16, seed=17)
    q, kc, vc, table, lengths, starts = batch.gpu()
    o, l = binding.attn_paged_fwd(q, kc, vc, table, lengths, starts, softmax_scale=batch.tau, window=window, sinks=sinks)
    want, want_l, bound, bound_l = ph.attention(batch, True)
    ph.assert_within(o, want, bound, "O")
    ph.assert_within(l, want_l, bound_l, "LSE")


def test_lengths_and_starts_out_of_range_stay_inside():
    batch = ph.Batch([47, 20], [1, 4], 4, 2, 64, "bf16", 16, pad=5, seed=13)
    q, kc, vc, table, lengths, starts = batch.gpu()
    kc, vc = torch.nan_to_num(kc), torch.nan_to_num(vc)
    for window, sinks in ((1, 0), (20, 3), (2 ** 31 - 1, 0)):
        for n, s in (([2 ** 31 - 1, -2 ** 31], [0, 1, 5]), ([48, 24], [-9, 2 ** 31 - 1, 3]), ([48, 24], [7, 3, 1]), ([0, -1], [2 ** 31 - 1] * 3)):
            out = torch.full_like(q, 7.0)
            binding.attn_paged_fwd(q, kc, vc, table, torch.tensor(n, dtype=torch.int32).cuda(), torch.tensor(s, dtype=torch.int32).cuda(), softmax_scale=0.1, out=out, window=window, sinks=sinks)
    torch.cuda.synchronize()
    # a length beyond the table: the token keeps its position, 60, and sees keys 41 .. 47 and the three sinks
    n = torch.tensor([61, 24], dtype=torch.int32).cuda()
    out, lse = binding.attn_paged_fwd(q, kc, vc, table, n, starts, softmax_scale=batch.tau, window=20, sinks=3)
    k, v = (torch.nan_to_num(batch.rows(torch.nan_to_num(c), 0)) for c in (batch.kc, batch.vc))
    rows = [0, 1, 2, *range(41, 48)]
    for h in range(4):
        s = batch.tau * (k[rows, h // 2] @ batch.q[0, h].double())
        want = torch.softmax(s, 0) @ v[rows, h // 2]
        assert (out[0, h].cpu().double() - want).abs().max() <= 2.0 ** -7 * v.abs().max()
        assert abs(float(lse[h, 0]) - float(torch.logsumexp(s, 0))) <= 1e-4
    # and one far beyond it sees the sinks alone
    out, lse = binding.attn_paged_fwd(q, kc, vc, table, torch.tensor([500, 24], dtype=torch.int32).cuda(), starts, softmax_scale=batch.tau, window=20, sinks=1)
    assert torch.equal(out[0], vc[int(table[0, 0]), :, 0].repeat_interleave(2, 0))


@pytest.mark.parametrize("d", [16, 64, 128])
@pytest.mark.parametrize("window,sinks", [(20, 3), (1, 0), (2 ** 31 - 1, 0)])
def test_lengths_out_of_range_of_single_tokens(d, window, sinks):
    """More than the table holds, none, and what is no length: a token keeps its position and sees the keys that there are."""
    lengths = [61, 2 ** 31 - 1, 0, -5, -2 ** 31, 48]
    batch = ph.Batch([47] * 6, [1] * 6, 4, 2, d, "bf16", 16, seed=d)
    q, kc, vc, table, _, _ = batch.gpu(True)
    out, lse = binding.attn_paged_fwd(q, kc, vc, table, torch.tensor(lengths, dtype=torch.int32).cuda(), softmax_scale=batch.tau, window=window, sinks=sinks)
    u = torch.finfo(batch.dtype).eps / 2
    for b, n in enumerate(lengths):
        k, v = batch.rows(batch.kc, b), batch.rows(batch.vc, b)
        rows = [j for j in range(min(n, 48)) if j > n - 1 - window or j < sinks]
        for h in range(4):
            if not rows:
                assert (out[b, h] == 0).all() and float(lse[h, b]) == -math.inf
                continue
            s = batch.tau * (k[rows, h // 2] @ batch.q[b, h].double())
            w = torch.softmax(s, 0)
            want, spread = w @ v[rows, h // 2], w @ v[rows, h // 2].abs()
            # (the rounding of O, that of the probabilities in numerator and denominator, and logits in 32 bits)
            assert ((out[b, h].cpu().double() - want).abs() <= u * want.abs() + (u + 2.0 ** -16) * (spread + want.abs()) + 2.0 ** -24).all()
            assert abs(float(lse[h, b]) - float(torch.logsumexp(s, 0))) <= 1e-4


def test_caches_beyond_32_bit_offsets():
    """More than 4 GiB of K: pages at both ends of the cache."""
    pages, Hk, page, d = 9000, 8, 256, 128
    kc, vc = (torch.zeros(pages, Hk, page, d, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    batch = ph.Batch([700, 1000], [1, 60], 16, Hk, d, "bf16", page, seed=18)
    q, sk, sv, table, lengths, starts = batch.gpu()
    where = torch.tensor([(i * 8999) // max(batch.pages - 1, 1) for i in range(batch.pages)], device="cuda")
    kc[where], vc[where] = torch.nan_to_num(sk), torch.nan_to_num(sv)
    moved = torch.where(table >= 0, where[table.clamp(min=0).long()].to(torch.int32), table)
    out, lse = binding.attn_paged_fwd(q, kc, vc, moved, lengths, starts, softmax_scale=batch.tau, window=300, sinks=4)
    want, want_l, bound, bound_l = attention(batch, 300, 4)
    ph.assert_within(out, want, bound, "O")
    ph.assert_within(lse, want_l, bound_l, "LSE")


def test_the_same_bits_from_threads_and_streams():
    batches = [ph.Batch([3000, 70, 900], new, 8, 2, 64, "bf16", 16, seed=20 + i) for i, new in enumerate(([1, 1, 1], [200, 1, 60]))]
    args = [b.gpu() for b in batches]
    kw = dict(softmax_scale=batches[0].tau, window=700, sinks=5)
    want = [binding.attn_paged_fwd(*a, **kw) for a in args]
    torch.cuda.synchronize()
    got, errors = [None, None], []

    def worker(i):
        try:
            with torch.cuda.stream(torch.cuda.Stream()):
                for _ in range(10):
                    got[i] = binding.attn_paged_fwd(*args[i], **kw)
                torch.cuda.current_stream().synchronize()
        except Exception as e:  # noqa: BLE001
            errors.append(e)

    threads = [threading.Thread(target=worker, args=(i,)) for i in range(2)]
    for t in threads:
        t.start()
    for t in threads:
        t.join(60.0)
    assert not errors
    for g, w in zip(got, want):
        assert all(torch.equal(a, b) for a, b in zip(g, w))


def test_steps_in_a_captured_graph():
    """A step of a running batch, captured: lengths, pages and tokens change between replays; one workspace with an eager call of another shape in between."""
    Hq, Hk, d, page, window, sinks = 8, 2, 64, 16, 50, 4
    gen = torch.Generator(device="cuda").manual_seed(1)
    rand = lambda *s: torch.randn(s, generator=gen, device="cuda").to(torch.bfloat16)  # noqa: E731
    kc, vc = (torch.zeros(64, Hk, page, d, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    table = torch.randperm(64, generator=torch.Generator().manual_seed(2)).to(torch.int32).view(2, 32).cuda()
    n = torch.tensor([20, 130], dtype=torch.int32, device="cuda")
    q, k, v = rand(2, Hq, d), rand(2, Hk, d), rand(2, Hk, d)
    norm, rotary = HeadNorm(rand(d), rand(d)), Rotary.make(d)
    out, turned, lse = torch.zeros_like(q), torch.zeros_like(q), torch.zeros(Hq, 2, device="cuda")
    ws = binding.attn_paged_workspace(q, kc, 2)

    def step(k_cache, v_cache, out, lse, ws):
        n.add_(1)
        binding.attn_paged_append(k, v, k_cache, v_cache, table, n, Q=q, rotary=rotary, norm=norm, out=turned)
        binding.attn_paged_fwd(turned, k_cache, v_cache, table, n, softmax_scale=0.125, window=window, sinks=sinks, out=out, lse=lse, workspace=ws)

    kc[:], vc[:] = rand(*kc.shape), rand(*vc.shape)
    eager = [kc.clone(), vc.clone()]
    start = n.clone()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step(kc.clone(), vc.clone(), out, lse, ws)
    torch.cuda.current_stream().wait_stream(side)
    n.copy_(start)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step(kc, vc, out, lse, ws)
    n.copy_(start)
    for i in range(6):
        for t in (q, k, v):
            t.copy_(rand(*t.shape))
        before = n.clone()
        graph.replay()
        torch.cuda.synchronize()
        got = [x.clone() for x in (out, lse, kc, vc)]
        n.copy_(before)
        step(*eager, out, lse, ws)
        assert all(torch.equal(a, b) for a, b in zip(got, (out, lse, *eager))), i
        big = ph.Batch([700], [300], Hq, Hk, d, "bf16", page, seed=i)
        binding.attn_paged_fwd(*big.gpu(), softmax_scale=0.125, window=window, workspace=ws)


@pytest.mark.parametrize("d", [64, 128])
def test_a_prompt_by_chunks_and_tokens_equals_the_dense_window(d):
    """Norm, rotation, append and attention with a window through a PageTable, against flash_attention over the whole text: two results within a rounding of the weights and of O each."""
    H, N, window, sinks = 4, 500, 96, 4
    gen = torch.Generator(device="cuda").manual_seed(3)
    q, k, v = (torch.randn(1, N, H, d, generator=gen, device="cuda").to(torch.bfloat16).transpose(1, 2) for _ in range(3))
    norm, rotary = HeadNorm(torch.rand(d, device="cuda") + 0.5, torch.rand(d, device="cuda") + 0.5), Rotary.make(d)
    want = flash_attention(q, k, v, causal=True, norm=norm, rotary=rotary, window=window, sinks=sinks)
    table = PageTable(pages=40, page_size=16)
    kc, vc = (torch.zeros(40, H, 16, d, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    seq, at, got = table.add(), 0, []
    for n in (130, 1, 1, 200, 1, 167):
        table.extend([seq], [n])
        block, lengths = table.batch([seq])
        starts = torch.tensor([0, n], dtype=torch.int32, device="cuda")
        rows = [x[0, :, at:at + n].transpose(0, 1) for x in (q, k, v)]
        turned = binding.attn_paged_append(rows[1], rows[2], kc, vc, block, lengths, starts, Q=rows[0], rotary=rotary, norm=norm)
        got.append(binding.attn_paged_fwd(turned, kc, vc, block, lengths, starts, softmax_scale=d ** -0.5, window=window, sinks=sinks)[0])
        at += n
    got = torch.cat(got).transpose(0, 1).double()
    # both within (2 u) (max |v| + |O|) of the exact result
    assert (got - want[0].double()).abs().max() <= 4 * 2.0 ** -8 * (v.double().abs().max() + want.double().abs().max())
    assert ((got - want[0].double()).norm() / want.double().norm()) <= 2.0 ** -7
