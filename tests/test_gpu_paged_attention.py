"""Attention of new tokens over a paged cache against the same in 64 bits."""
import math

import pytest
import torch

from paper_2205_14135_amd import binding
from tests import paged_helpers as ph

pytestmark = pytest.mark.gpu


def check(batch, causal=True, single=False, tau=None, workspace=None):
    q, kc, vc, table, lengths, starts = batch.gpu(single)
    before = [x.clone() for x in (kc, vc)]
    out = torch.empty_strided(q.size(), q.stride(), dtype=q.dtype, device="cuda").fill_(7.0)
    lse = torch.full((batch.Hq, q.shape[0]), 5.0, device="cuda")
    o, l = binding.attn_paged_fwd(q, kc, vc, table, lengths, starts, softmax_scale=tau or batch.tau, causal=causal, out=out, lse=lse, workspace=workspace)
    assert o is out and l is lse
    want, want_l, bound, bound_l = ph.attention(batch, causal, tau)
    ph.assert_within(out[:batch.tokens], want, bound, "O")
    ph.assert_within(lse[:, :batch.tokens], want_l, bound_l, "LSE")
    assert (out[batch.tokens:] == 7.0).all() and (lse[:, batch.tokens:] == 5.0).all()          # rows behind the last sequence
    for x, y in zip((kc, vc), before):
        assert torch.equal(torch.nan_to_num(x, 3.0), torch.nan_to_num(y, 3.0))
    return out, lse


@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
@pytest.mark.parametrize("d,page", [(16, 16), (32, 64), (64, 16), (64, 128), (128, 16), (128, 32), (128, 256)])
@pytest.mark.parametrize("Hq,Hk", [(4, 4), (8, 2), (6, 2), (7, 1)])
def test_single_tokens(dtype, d, page, Hq, Hk):
    n = [1, 16, 17, 63, 64, 65, 333]
    check(ph.Batch([x - 1 for x in n], [1] * len(n), Hq, Hk, d, dtype, page, seed=d + page), single=True)


@pytest.mark.parametrize("d", [32, 64, 128])
@pytest.mark.parametrize("lengths", [[5000], [4097, 1, 2500, 700], [128 * i + 3 for i in range(1, 12)]])
def test_long_contexts_are_divided(d, lengths):
    check(ph.Batch([x - 1 for x in lengths], [1] * len(lengths), 8, 2, d, "bf16", 16, seed=d), single=True)


@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
@pytest.mark.parametrize("d,page,Hq,Hk", [(16, 32, 4, 2), (32, 16, 3, 3), (64, 64, 8, 2), (64, 16, 5, 1), (128, 16, 4, 4), (128, 128, 6, 2)])
def test_chunks(causal, dtype, d, page, Hq, Hk):
    check(ph.Batch([0, 40, 100, 0, 700, 33], [1, 0, 5, 130, 64, 257], Hq, Hk, d, dtype, page, pad=19, seed=page), causal)


@pytest.mark.parametrize("causal", [True, False])
def test_a_chunk_among_single_tokens(causal):
    check(ph.Batch([900, 0, 2000, 31, 64], [1, 300, 1, 1, 1], 8, 2, 64, "bf16", 16, pad=3, seed=5), causal)


@pytest.mark.parametrize("new", [[2, 3, 1], [1, 1, 1]])
def test_few_tokens_with_starts(new):
    check(ph.Batch([600, 20, 2100], new, 8, 2, 128, "bf16", 16, pad=2, seed=6))


@pytest.mark.parametrize("Hq,d", [(40, 64), (71, 64), (128, 128)])
def test_many_heads_share_one(Hq, d):
    check(ph.Batch([900, 10, 64], [1, 1, 1], Hq, 1, d, "bf16", 16, seed=7), single=True)
    check(ph.Batch([300, 10], [3, 2], Hq, 1, d, "bf16", 16, seed=8))


@pytest.mark.parametrize("single", [True, False])
@pytest.mark.parametrize("B", [63, 64, 65, 130, 200])
def test_many_sequences(B, single):
    new = [1] * B if single else [(b * 7) % 4 for b in range(B)]
    check(ph.Batch([(b * 37) % 150 for b in range(B)], new, 2, 1, 64, "bf16", 16, seed=B), single=single)


@pytest.mark.parametrize("single", [True, False])
def test_very_many_sequences(single):
    B = 1500
    check(ph.Batch([(b * 37) % 70 for b in range(B)], [1] * B if single else [(b * 7) % 3 for b in range(B)], 2, 1, 32, "bf16", 16, pad=0 if single else 5, seed=4), single=single)


def test_single_tokens_of_a_padded_batch():
    """More rows of Q than sequences: those behind are left as they were."""
    check(ph.Batch([30, 400, 7], [1, 1, 1], 8, 2, 64, "bf16", 16, pad=5, seed=40), single=True)


def test_rows_in_front_of_the_first_sequence_and_a_part_of_a_table():
    batch = ph.Batch([30, 400], [3, 70], 8, 2, 64, "bf16", 16, seed=41)
    q, kc, vc, table, lengths, starts = batch.gpu()
    q = torch.cat([torch.full((4, 8, 64), math.nan, dtype=q.dtype, device="cuda"), q])
    wide = torch.full((2, table.shape[1] + 9), 10 ** 9, dtype=torch.int32, device="cuda")
    wide[:, 3:3 + table.shape[1]] = table
    out, lse = torch.full_like(q, 7.0), torch.full((8, q.shape[0]), 5.0, device="cuda")
    binding.attn_paged_fwd(q, kc, vc, wide[:, 3:3 + table.shape[1]], lengths, starts + 4, softmax_scale=batch.tau, out=out, lse=lse)
    want, want_l, bound, bound_l = ph.attention(batch, True)
    ph.assert_within(out[4:], want, bound, "O")
    ph.assert_within(lse[:, 4:], want_l, bound_l, "LSE")
    assert (out[:4] == 7.0).all() and (lse[:, :4] == 5.0).all()


@pytest.mark.parametrize("d", [16, 128])
@pytest.mark.parametrize("causal", [True, False])
def test_rows_that_see_nothing(d, causal):
    """Lengths below the number of new tokens leave the first ones at negative positions; a length of 0 leaves all."""
    batch = ph.Batch([-3, -5, -2, 0, -200], [5, 5, 2, 3, 150], 4, 2, d, "bf16", 16, seed=9)
    out, lse = check(batch, causal)
    assert (out[5:10] == 0).all() and torch.isinf(lse[:, 5:10]).all()
    check(ph.Batch([-1, 5, -1], [1, 1, 1], 4, 2, d, "fp16", 16, seed=10), causal, single=True)


@pytest.mark.parametrize("token_major,fused", [(True, False), (False, True), (True, True)])
@pytest.mark.parametrize("new", [[1, 1, 1], [70, 1, 33]])
def test_strides(token_major, fused, new):
    check(ph.Batch([30, 400, 1000], new, 8, 4, 64, "bf16", 32, pad=2, token_major=token_major, fused=fused, seed=11))


@pytest.mark.parametrize("single", [True, False])
@pytest.mark.parametrize("d", [16, 64, 128])
def test_numbers_that_are_no_page_read_as_zeros(d, single):
    batch = ph.Batch([200, 90, 70], [1, 1, 1] if single else [3, 40, 1], 4, 2, d, "bf16", 16, seed=12)
    for b, t, number in ((0, 2, -1), (0, 5, batch.pages), (1, 0, 2 ** 31 - 1), (1, 5, -2 ** 31), (2, 4, batch.pages + 1)):
        batch.table[b, t] = number
    check(batch, single=single)


def test_lengths_and_starts_out_of_range_stay_inside():
    """No more than the table holds, no rows behind the last of Q; what they give is not specified, except that sequences in order are right."""
    batch = ph.Batch([47, 20], [1, 4], 4, 2, 64, "bf16", 16, pad=5, seed=13)
    q, kc, vc, table, lengths, starts = batch.gpu()
    kc, vc = torch.nan_to_num(kc), torch.nan_to_num(vc)
    for n, s in (([2 ** 31 - 1, -2 ** 31], [0, 1, 5]), ([48, 24], [-9, 2 ** 31 - 1, 3]), ([48, 24], [7, 3, 1]), ([0, -1], [2 ** 31 - 1] * 3)):
        out = torch.full_like(q, 7.0)
        binding.attn_paged_fwd(q, kc, vc, table, torch.tensor(n, dtype=torch.int32).cuda(), torch.tensor(s, dtype=torch.int32).cuda(), softmax_scale=0.1, out=out)
    torch.cuda.synchronize()
    batch.lengths = [48, 24]
    out, _ = binding.attn_paged_fwd(q, kc, vc, table, torch.tensor([2 ** 30, 24], dtype=torch.int32).cuda(), starts, softmax_scale=batch.tau)
    want, _, bound, _ = ph.attention(batch, True)    # the first sequence fills its 3 pages
    ph.assert_within(out[:batch.tokens], want, bound, "O")


@pytest.mark.parametrize("scale", [8.0, 30.0])
def test_peaked_rows(scale):
    check(ph.Batch([900, 64, 2000], [1, 1, 1], 8, 2, 64, "bf16", 16, seed=14), single=True, tau=scale / 8.0)
    check(ph.Batch([900, 64], [33, 90], 4, 2, 128, "bf16", 16, seed=15), tau=scale / 11.0)


def test_a_row_that_is_not_finite_stays_alone():
    batch = ph.Batch([300, 80], [4, 3], 4, 2, 64, "bf16", 16, seed=16)
    want, want_l, bound, bound_l = ph.attention(batch, True)
    batch.q[2, 1, 5] = math.nan
    batch.q[5, 0, 0] = math.inf
    q, kc, vc, table, lengths, starts = batch.gpu()
    out, lse = binding.attn_paged_fwd(q, kc, vc, table, lengths, starts, softmax_scale=batch.tau)
    assert torch.isnan(out[2, 1]).all() and torch.isnan(lse[1, 2]) and torch.isnan(out[5, 0]).all()
    for x in (bound, ):
        x[2, 1], x[5, 0] = math.inf, math.inf
    bound_l[1, 2], bound_l[0, 5] = math.inf, math.inf
    ph.assert_within(torch.nan_to_num(out), want, bound, "O")
    ph.assert_within(torch.nan_to_num(lse), want_l, bound_l, "LSE")


def test_caches_beyond_32_bit_offsets():
    """More than 4 GiB of K: pages at both ends of the cache."""
    page, Hk, d = 64, 8, 128
    pages = (5 << 30) // (2 * page * Hk * d)
    batch = ph.Batch([700, 90], [1, 1], 16, Hk, d, "bf16", page, seed=17, extra_pages=0)
    q, small_k, small_v, table, lengths, _ = batch.gpu(single=True)
    place = torch.tensor([i if i % 2 else pages - 1 - i for i in range(batch.pages)], device="cuda")
    caches = []
    for small in (small_k, small_v):
        big = torch.empty(pages, Hk, page, d, dtype=small.dtype, device="cuda")
        big[place] = small
        caches.append(big)
    moved = torch.where(table >= 0, place[table.clamp(min=0).long()].to(torch.int32), table)
    out, lse = binding.attn_paged_fwd(q, *caches, moved, lengths, softmax_scale=batch.tau)
    want, want_l, bound, bound_l = ph.attention(batch, True)
    ph.assert_within(out, want, bound, "O")
    ph.assert_within(lse, want_l, bound_l, "LSE")


def test_the_same_in_every_call():
    batch = ph.Batch([6000, 50, 900, 3000], [1, 1, 1, 1], 8, 2, 128, "bf16", 16, seed=18)
    args = batch.gpu(single=True)
    first = binding.attn_paged_fwd(*args, softmax_scale=batch.tau)
    for _ in range(5):
        junk = torch.full((1 << 22,), math.nan, device="cuda")     # (memory of the workspaces that are made here)
        del junk
        again = binding.attn_paged_fwd(*args, softmax_scale=batch.tau)
        assert all(torch.equal(x, y) for x, y in zip(first, again))


def test_graph_follows_the_lengths():
    """A captured step reads lengths, table and tokens when it is replayed; eager calls run between the replays."""
    n = [900, 1, 64, 2000]
    batches = [ph.Batch([x - 1 for x in n], [1] * 4, 8, 2, 64, "bf16", 16, seed=20 + i) for i in range(2)]
    short = [3, 700, 65, 128]
    batches.append(ph.Batch([x - 1 for x in short], [1] * 4, 8, 2, 64, "bf16", 16, seed=23))
    width, pages = max(b.table.shape[1] for b in batches), max(b.pages for b in batches)
    q, kc, vc = batches[0].gpu(single=True)[:3]
    kc, vc = (torch.zeros(pages, *kc.shape[1:], dtype=kc.dtype, device="cuda") for _ in range(2))
    table = torch.zeros(4, width, dtype=torch.int32, device="cuda")
    lengths = torch.ones(4, dtype=torch.int32, device="cuda")
    out, lse, ws = torch.zeros_like(q), torch.zeros(8, 4, device="cuda"), binding.attn_paged_workspace(q, kc, 4)

    def load(b):
        g = b.gpu(single=True)
        q.copy_(g[0])
        kc[:b.pages], vc[:b.pages] = g[1], g[2]
        table.zero_()
        table[:, :b.table.shape[1]] = g[3]
        lengths.copy_(g[4])

    def call():
        binding.attn_paged_fwd(q, kc, vc, table, lengths, softmax_scale=batches[0].tau, out=out, lse=lse, workspace=ws)

    load(batches[0])
    call()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call()
    for b in (*batches, batches[0]):
        load(b)
        graph.replay()
        torch.cuda.synchronize()
        replayed = out.clone(), lse.clone()
        call()
        torch.cuda.synchronize()
        assert torch.equal(replayed[0], out) and torch.equal(replayed[1], lse)
        want, _, bound, _ = ph.attention(b, True)
        ph.assert_within(replayed[0], want, bound, "O")


def test_two_streams_with_workspaces_of_their_own():
    batches = [ph.Batch([3000 + i, 40, 900], [1, 1, 1], 8, 2, 128, "bf16", 16, seed=30 + i) for i in range(2)]
    args = [b.gpu(single=True) for b in batches]
    want = [binding.attn_paged_fwd(*a, softmax_scale=batches[0].tau) for a in args]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(2)]
    got = [None, None]
    for _ in range(4):
        for i, s in enumerate(streams):
            with torch.cuda.stream(s):
                got[i] = binding.attn_paged_fwd(*args[i], softmax_scale=batches[0].tau)
    torch.cuda.synchronize()
    for g, w in zip(got, want):
        assert torch.equal(g[0], w[0]) and torch.equal(g[1], w[1])


def test_graphs_of_whole_steps_share_a_workspace():
    """Two captured steps, appending and attending, of one token a sequence: the lengths count on inside the graph; replayed in turn on one workspace, against eager steps
    of the same tokens on a second cache."""
    from paper_2205_14135_amd.rotary import Rotary
    Hq, Hk, d, page, B, before = 8, 2, 64, 16, 3, 600
    rotary = Rotary.make(d)
    gen = torch.Generator(device="cuda").manual_seed(50)
    normal = lambda *shape: torch.randn(shape, generator=gen, device="cuda").to(torch.bfloat16)
    pages = B * 48
    caches = [[normal(pages, Hk, page, d) for _ in range(2)] for _ in range(2)]          # of the two graphs
    eager = [[c.clone() for c in pair] for pair in caches]
    table = torch.randperm(pages, generator=gen, device="cuda").to(torch.int32).view(B, 48)
    q, k, v = normal(B, Hq, d), normal(B, Hk, d), normal(B, Hk, d)
    ws = binding.attn_paged_workspace(q, caches[0][0], B)
    lengths = [torch.tensor([before, before + 5, 3], dtype=torch.int32, device="cuda") for _ in range(2)]
    outs = [(torch.zeros_like(q), torch.zeros(Hq, B, device="cuda"), torch.zeros_like(q)) for _ in range(2)]

    def step(pair, n, out, lse, turned):
        binding.attn_paged_append(k, v, *pair, table, n, Q=q, rotary=rotary, out=turned)
        binding.attn_paged_fwd(turned, *pair, table, n, softmax_scale=d ** -0.5, out=out, lse=lse, workspace=ws)

    graphs = []
    for i in range(2):
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            lengths[i] += 1
            step(caches[i], lengths[i], *outs[i])
        graphs.append(graph)
    seen = [n.clone() for n in lengths]
    for rep in range(4):
        for i in range(2):
            for x in (q, k, v):
                x.copy_(normal(*x.shape))
            graphs[i].replay()
            torch.cuda.synchronize()
            got = [x.clone() for x in outs[i]]
            seen[i] += 1
            want = tuple(torch.zeros_like(x) for x in outs[i])
            step(eager[i], seen[i], *want)
            torch.cuda.synchronize()
            assert all(torch.equal(a, b) for a, b in zip(got, want)), (rep, i)
            assert all(torch.equal(a, b) for a, b in zip(caches[i], eager[i]))


def test_two_host_threads():
    import threading
    batches = [ph.Batch([2000 + i, 40], [1, 60], 8, 2, 64, "bf16", 16, seed=60 + i) for i in range(2)]
    args = [b.gpu() for b in batches]
    want = [binding.attn_paged_fwd(*a, softmax_scale=batches[0].tau) for a in args]
    torch.cuda.synchronize()
    got, errors = [None, None], []

    def worker(i):
        try:
            with torch.cuda.stream(torch.cuda.Stream()):
                for _ in range(20):
                    got[i] = binding.attn_paged_fwd(*args[i], softmax_scale=batches[0].tau)
                torch.cuda.current_stream().synchronize()
        except Exception as e:  # noqa: BLE001
            errors.append(e)

    threads = [threading.Thread(target=worker, args=(i,)) for i in range(2)]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    assert not errors
    for g, w in zip(got, want):
        assert torch.equal(g[0], w[0]) and torch.equal(g[1], w[1])


# ---- the larger blocks (many rows a sequence): more than sixteen tiles of page numbers, cuts, bad numbers, rows that are no numbers

BLOCKS = pytest.mark.parametrize("d,page,Hq,Hk", [(16, 16, 4, 2), (32, 32, 4, 4), (64, 16, 8, 2), (64, 256, 3, 3), (128, 16, 8, 2), (128, 64, 4, 4)])


@pytest.mark.parametrize("causal", [True, False])
@BLOCKS
def test_chunks_on_long_contexts(causal, d, page, Hq, Hk):
    check(ph.Batch([2500, 1023, 0, 1500, 4000], [300, 129, 511, 1, 70], Hq, Hk, d, "bf16", page, pad=7, seed=100 + d), causal)


@BLOCKS
def test_chunks_and_numbers_that_are_no_page(d, page, Hq, Hk):
    batch = ph.Batch([1300, 400], [260, 200], Hq, Hk, d, "fp16", page, seed=110 + d)
    last = (1560 - 1) // page
    for b, t, number in ((0, 0, -1), (0, 2, batch.pages), (0, last, 2 ** 31 - 1), (1, 1, -2 ** 31), (1, 599 // page, batch.pages + 1)):
        batch.table[b, t] = number
    check(batch)


@BLOCKS
def test_rows_of_chunks_that_see_nothing(d, page, Hq, Hk):
    """More new tokens than the sequence is long: the first of them stand in front of it."""
    check(ph.Batch([-250, -300, 200], [400, 300, 40], Hq, Hk, d, "bf16", page, seed=120 + d))


@pytest.mark.parametrize("d", [64, 128])
def test_rows_of_a_chunk_that_are_no_numbers_stay_alone(d):
    batch = ph.Batch([300, 80], [200, 150], 4, 2, d, "bf16", 16, seed=130)
    want, want_l, bound, bound_l = ph.attention(batch, True)
    batch.q[2, 1, 5] = math.nan
    batch.q[205, 0, 0] = math.inf
    q, kc, vc, table, lengths, starts = batch.gpu()
    out, lse = binding.attn_paged_fwd(q, kc, vc, table, lengths, starts, softmax_scale=batch.tau)
    assert torch.isnan(out[2, 1]).all() and torch.isnan(lse[1, 2])
    bound[2, 1], bound[205, 0] = math.inf, math.inf
    bound_l[1, 2], bound_l[0, 205] = math.inf, math.inf
    ph.assert_within(torch.nan_to_num(out), want, bound, "O")
    ph.assert_within(torch.nan_to_num(lse), want_l, bound_l, "LSE")


@pytest.mark.parametrize("d", [64, 128])
def test_lengths_and_starts_of_chunks_out_of_range_stay_inside(d):
    batch = ph.Batch([47, 20], [300, 200], 4, 2, d, "bf16", 16, pad=5, seed=140)
    q, kc, vc, table, lengths, starts = batch.gpu()
    kc, vc = torch.nan_to_num(kc), torch.nan_to_num(vc)
    for n, s in (([2 ** 31 - 1, -2 ** 31], [0, 300, 500]), ([347, 220], [-9, 2 ** 31 - 1, 3]), ([347, 220], [400, 3, 1]), ([0, -1], [2 ** 31 - 1] * 3), ([347, 220], [-2 ** 31, 505, 2 ** 31 - 1])):
        out = torch.full_like(q, 7.0)
        binding.attn_paged_fwd(q, kc, vc, table, torch.tensor(n, dtype=torch.int32).cuda(), torch.tensor(s, dtype=torch.int32).cuda(), softmax_scale=0.1, out=out)
    torch.cuda.synchronize()
    out, _ = binding.attn_paged_fwd(q, kc, vc, table, lengths, starts, softmax_scale=batch.tau)
    want, _, bound, _ = ph.attention(batch, True)
    ph.assert_within(out[:batch.tokens], want, bound, "O")


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("scale", [8.0, 30.0])
def test_peaked_rows_of_chunks(scale, d):
    check(ph.Batch([900, 64, 1500], [133, 290, 200], 4, 2, d, "bf16", 16, seed=150), tau=scale / math.sqrt(d))


@pytest.mark.parametrize("d,interleaved", [(64, False), (128, True)])
def test_chunks_in_views_of_a_projection_and_another_order_of_axes(d, interleaved):
    check(ph.Batch([500, 0, 1200], [170, 330, 1], 6, 2, d, "fp16", 32, pad=4, seed=160, token_major=interleaved, fused=True))


@pytest.mark.parametrize("Hk,d", [(16, 64), (8, 128)])
def test_chunks_in_caches_beyond_32_bit_offsets(Hk, d):
    """More than 4 GiB of K: pages at both ends of the cache."""
    page = 64
    pages = (5 << 30) // (2 * page * Hk * d)
    batch = ph.Batch([700, 90], [150, 300], Hk, Hk, d, "bf16", page, seed=170, extra_pages=0)
    q, small_k, small_v, table, lengths, starts = batch.gpu()
    place = torch.tensor([i if i % 2 else pages - 1 - i for i in range(batch.pages)], device="cuda")
    caches = []
    for small in (small_k, small_v):
        big = torch.empty(pages, Hk, page, d, dtype=small.dtype, device="cuda")
        big[place] = small
        caches.append(big)
    moved = torch.where(table >= 0, place[table.clamp(min=0).long()].to(torch.int32), table)
    out, lse = binding.attn_paged_fwd(q, *caches, moved, lengths, starts, softmax_scale=batch.tau)
    want, want_l, bound, bound_l = ph.attention(batch, True)
    ph.assert_within(out, want, bound, "O")
    ph.assert_within(lse, want_l, bound_l, "LSE")
