"""Appending to a paged cache and copying its pages, and a run of all of it together."""
import math

import pytest
import torch

from paper_2205_14135_amd import binding
from paper_2205_14135_amd.autograd import flash_attention
from paper_2205_14135_amd.rotary import Rotary, rotary_frequencies
from tests import paged_helpers as ph

pytestmark = pytest.mark.gpu


def _append(batch, rotary, f, single=False, in_place=False):
    """Appends the batch's new tokens and compares the whole caches: written rows, and every other row as it was."""
    q, kc, vc, table, lengths, starts = batch.gpu(single)
    k, v = (torch.empty_strided(x.size(), x.stride(), dtype=x.dtype, device="cuda").copy_(x) for x in (batch.k, batch.v))
    out = None
    if rotary is not None:
        out = q if in_place else torch.full_like(q, 7.0)
    got = binding.attn_paged_append(k, v, kc, vc, table, lengths, starts, Q=None if rotary is None else q, rotary=rotary, out=out)
    assert got is out
    want_k, want_v = batch.kc.double(), batch.vc.double()
    bound_k = torch.zeros_like(want_k)
    want_q, bound_q = (batch.q.double() if in_place else torch.full(batch.q.shape, 7.0, dtype=torch.float64)), torch.zeros(batch.q.shape, dtype=torch.float64)
    capacity = batch.table.shape[1] * batch.page
    for b in range(batch.B):
        at, m, n = int(batch.starts[b]), batch.new[b], batch.lengths[b]
        for i in range(m):
            pos = n - m + i
            row_k, row_q = batch.k[at + i].double(), batch.q[at + i].double()
            bk = bq = None
            if rotary is not None:
                p = torch.tensor([pos])
                row_k, bk = ph.turned(batch.k[at + i:at + i + 1], p, f, rotary.interleaved, rotary.magnitude)
                row_q, bq = ph.turned(batch.q[at + i:at + i + 1], p, f, rotary.interleaved, rotary.magnitude)
                row_k, row_q, bk, bq = row_k[0], row_q[0], bk[0] + ph.rounding(row_k[0], batch.dtype), bq[0] + ph.rounding(row_q[0], batch.dtype)
                want_q[at + i], bound_q[at + i] = row_q, bq
            if pos < 0 or pos >= capacity:
                continue
            number = int(batch.table[b, pos // batch.page])
            if not 0 <= number < batch.pages:
                continue
            want_k[number, :, pos % batch.page] = row_k
            want_v[number, :, pos % batch.page] = batch.v[at + i].double()
            if bk is not None:
                bound_k[number, :, pos % batch.page] = bk
    ph.assert_within(torch.nan_to_num(kc, 99.0), torch.nan_to_num(want_k, 99.0), bound_k, "K cache")
    ph.assert_within(torch.nan_to_num(vc, 99.0), torch.nan_to_num(want_v, 99.0), torch.zeros_like(want_v), "V cache")
    if rotary is not None:
        ph.assert_within(torch.nan_to_num(out, 99.0), torch.nan_to_num(want_q, 99.0), bound_q, "Q")


@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
@pytest.mark.parametrize("d,r,interleaved", [(16, 16, False), (16, 4, True), (32, 32, False), (64, 64, False), (64, 32, True), (64, 12, False), (128, 128, False), (128, 96, True)])
@pytest.mark.parametrize("new", [[1, 1, 1, 1], [5, 0, 130, 17]])
def test_append(dtype, d, r, interleaved, new):
    f, m = rotary_frequencies(r, scaling="parts", factor=4.0)
    _append(ph.Batch([0, 15, 16, 900], new, 6, 2, d, dtype, 16, pad=9, seed=d + r), Rotary(f.cuda(), interleaved=interleaved, magnitude=m), f)


@pytest.mark.parametrize("token_major,fused", [(False, False), (True, True)])
@pytest.mark.parametrize("in_place", [False, True])
def test_append_layouts(token_major, fused, in_place):
    f, m = rotary_frequencies(64)
    rotary = Rotary(f.cuda())
    _append(ph.Batch([30, 64, 0], [1, 1, 1], 8, 2, 64, "bf16", 32, pad=2, token_major=token_major, fused=fused, seed=1), rotary, f, single=False, in_place=in_place)
    _append(ph.Batch([30, 64, 0], [1, 1, 1], 8, 8, 64, "bf16", 64, pad=2, token_major=token_major, fused=fused, seed=2), rotary, f, single=True, in_place=in_place)
    _append(ph.Batch([30, 64, 0], [7, 70, 1], 8, 2, 64, "bf16", 256, token_major=token_major, fused=fused, seed=3), None, None)


@pytest.mark.parametrize("B", [1, 64, 65, 300])
@pytest.mark.parametrize("d", [16, 128])
def test_append_many_sequences(B, d):
    f, _ = rotary_frequencies(d)
    _append(ph.Batch([(b * 11) % 50 for b in range(B)], [(b * 5) % 3 for b in range(B - 1)] + [1], 2, 1, d, "bf16", 16, pad=4, seed=B), Rotary(f.cuda()), f)


def test_append_writes_nothing_outside():
    """Negative positions, positions behind the table, numbers that are no page."""
    f, _ = rotary_frequencies(64)
    batch = ph.Batch([-3, 40, 20, 10], [5, 30, 2, 1], 4, 2, 64, "bf16", 16, seed=4)
    batch.table[1, 3], batch.table[2, 1], batch.table[3, 0] = -1, batch.pages, 2 ** 31 - 1
    batch.lengths[1] += 1000     # (the last ones behind what a row of the table holds)
    _append(batch, Rotary(f.cuda()), f)


@pytest.mark.parametrize("dtype,d,page,Hk", [("bf16", 128, 16, 8), ("fp16", 64, 64, 3), ("bf16", 16, 32, 1), ("bf16", 32, 4096, 2)])
@pytest.mark.parametrize("layers", [0, 3])
@pytest.mark.parametrize("token_major", [False, True])
def test_copy(dtype, d, page, Hk, layers, token_major):
    gen = torch.Generator().manual_seed(page)
    pages = 9
    shape = ((layers,) if layers else ()) + ((pages, page, Hk, d) if token_major else (pages, Hk, page, d))
    caches = [torch.randn(shape, generator=gen).to(ph.DTYPES[dtype]).cuda() for _ in range(2)]
    if token_major:
        caches = [c.transpose(-3, -2) for c in caches]
    want = [c.clone() for c in caches]
    pairs = [(3, 0), (3, 8), (5, 1)]
    for w in want:
        x = w if layers else w.unsqueeze(0)
        for s, t in pairs:
            x[:, t] = x[:, s]
    binding.attn_paged_copy(*caches, pairs)
    assert all(torch.equal(a, b) for a, b in zip(caches, want))
    binding.attn_paged_copy(*caches, [])
    assert all(torch.equal(a, b) for a, b in zip(caches, want))


def test_copy_of_more_pages_than_one_launch_takes():
    gen = torch.Generator(device="cuda").manual_seed(1)
    kc, vc = (torch.randn(3000, 2, 16, 32, generator=gen, device="cuda").to(torch.bfloat16) for _ in range(2))
    order = torch.randperm(3000)
    pairs = torch.stack([order[:1400], order[1400:2800]], 1).to(torch.int32)
    want = [c.clone() for c in (kc, vc)]
    for w in want:
        w[pairs[:, 1].cuda().long()] = w[pairs[:, 0].cuda().long()]
    binding.attn_paged_copy(kc, vc, pairs)
    assert torch.equal(kc, want[0]) and torch.equal(vc, want[1])


def test_copy_replays_its_list():
    kc, vc = (torch.randn(8, 2, 16, 64, device="cuda").to(torch.bfloat16) for _ in range(2))
    pairs = torch.tensor([[0, 4], [1, 5]], dtype=torch.int32)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        binding.attn_paged_copy(kc, vc, pairs)
    pairs.fill_(7)     # the graph has its own
    for _ in range(3):
        kc.normal_()
        vc.normal_()
        want = [c.clone() for c in (kc, vc)]
        for w in want:
            w[4:6] = w[0:2]
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(kc, want[0]) and torch.equal(vc, want[1])


@pytest.mark.parametrize("d,Hq,Hk,interleaved", [(64, 8, 2, False), (128, 4, 4, True)])
def test_prompt_fork_and_single_tokens_together(d, Hq, Hk, interleaved):
    """A prompt read in by two chunks, forked, and both copies continued token by token, each with tokens of its own, against flash_attention with
    rotary positions over the whole sequences: the cache's path and the training path give the same attention.

    Both outputs are within the bounds of attention over rotated and rounded Q and K (which both compute with the same arithmetic), so they differ by twice
    that bound at most: for unit normal values weights sum to 1 and |v| < 6, (u + u) (6 + 6) + the outputs' own rounding u 6, twice."""
    page, tokens, steps = 16, 100, 20
    gen = torch.Generator(device="cuda").manual_seed(d)
    rotary = Rotary.make(d // 2, interleaved=interleaved)
    total = tokens + steps
    q, k, v = (torch.randn(2, total, h, d, generator=gen, device="cuda").to(torch.bfloat16) for h in (Hq, Hk, Hk))
    for x in (q, k, v):
        x[1, :tokens] = x[0, :tokens]     # the prompt is shared
    kc, vc = (torch.full((40, Hk, page, d), math.nan, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    table = torch.full((2, -(-total // page)), -1, dtype=torch.int32, device="cuda")
    free = list(range(39, -1, -1))
    ints = lambda *x: torch.tensor(x, dtype=torch.int32, device="cuda")
    got = torch.zeros_like(q)
    ws = binding.attn_paged_workspace(torch.empty(64, Hq, d, dtype=torch.bfloat16, device="cuda"), kc, 1)

    held = 0
    for n in (64, tokens - 64):      # the prompt, sequence 0 alone
        while held + n > page * int((table[0] >= 0).sum()):
            table[0, int((table[0] >= 0).sum())] = free.pop()
        rows = slice(held, held + n)
        held += n
        turned = binding.attn_paged_append(k[0, rows], v[0, rows], kc, vc, table[:1], ints(held), ints(0, n), Q=q[0, rows], rotary=rotary)
        got[0, rows], _ = binding.attn_paged_fwd(turned, kc, vc, table[:1], ints(held), ints(0, n), softmax_scale=1 / math.sqrt(d), workspace=ws)
    got[1, :tokens] = got[0, :tokens]
    table[1] = table[0]               # the fork shares full pages and gets a copy of the last one
    last = tokens // page
    table[1, last] = free.pop()
    binding.attn_paged_copy(kc, vc, [(int(table[0, last]), int(table[1, last]))])
    for i in range(tokens, total):
        if i % page == 0:
            table[0, i // page], table[1, i // page] = free.pop(), free.pop()
        n = ints(i + 1, i + 1)
        turned = binding.attn_paged_append(k[:, i], v[:, i], kc, vc, table, n, Q=q[:, i], rotary=rotary)
        got[:, i], _ = binding.attn_paged_fwd(turned, kc, vc, table, n, softmax_scale=1 / math.sqrt(d), workspace=ws)
    spread = lambda x: x.repeat_interleave(Hq // Hk, 2).transpose(1, 2).contiguous()
    want = flash_attention(q.transpose(1, 2).contiguous(), spread(k), spread(v), causal=True, rotary=rotary).transpose(1, 2)
    assert torch.isfinite(got).all()
    u = 2.0 ** -8
    assert (got.float() - want.float()).abs().max().item() <= 2 * (2 * u * 12 + 6 * u)
    assert (got.float() - want.float()).pow(2).mean().sqrt().item() <= 2 * u     # (rms of values below 1: two roundings of each)


def test_sequences_forked_ended_and_compacted():
    """Three prompts in a cache of two layers through `PageTable`: forked, continued apart, one ended, the cache compacted, continued; every step's attention against the same
    in 64 bits over all tokens that the sequence was given (turned and rounded as the cache holds them)."""
    from paper_2205_14135_amd.paged import PageTable
    Hq, Hk, d, page, layers = 4, 2, 64, 16, 2
    gen = torch.Generator().manual_seed(3)
    table = PageTable(30, page)
    kc, vc = (torch.full((layers, table.pages, Hk, page, d), math.nan, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    given = {}      # sequence -> per layer, K and V rows on the CPU

    def step(seqs, new):
        pairs = table.extend(seqs, new)
        binding.attn_paged_copy(kc, vc, pairs)
        block, lengths = table.batch(seqs)
        starts = torch.tensor([sum(new[:i]) for i in range(len(new) + 1)], dtype=torch.int32, device="cuda")
        T = sum(new)
        for l in range(layers):
            q, k, v = (torch.randn(T, h, d, generator=gen).to(torch.bfloat16) for h in (Hq, Hk, Hk))
            binding.attn_paged_append(k.cuda(), v.cuda(), kc[l], vc[l], block, lengths, starts)
            out, lse = binding.attn_paged_fwd(q.cuda(), kc[l], vc[l], block, lengths, starts, softmax_scale=d ** -0.5)
            at = 0
            for s, n in zip(seqs, new):
                given[s][l][0].append(k[at:at + n])
                given[s][l][1].append(v[at:at + n])
                at += n
            # the same batch on plain rows: pages in order
            plain = ph.Batch([table.length(s) - n for s, n in zip(seqs, new)], new, Hq, Hk, d, "bf16", page)
            plain.q = q
            for cache, i in ((plain.kc, 0), (plain.vc, 1)):
                for b, s in enumerate(seqs):
                    rows = torch.cat(given[s][l][i])
                    for t in range(-(-len(rows) // page)):
                        part = rows[t * page:(t + 1) * page]
                        cache[int(plain.table[b, t]), :, :len(part)] = part.transpose(0, 1)
            want, want_l, bound, bound_l = ph.attention(plain, True)
            ph.assert_within(out, want, bound, "O")
            ph.assert_within(lse, want_l, bound_l, "LSE")

    def fork(s):
        t = table.fork(s)
        given[t] = [[list(x) for x in layer] for layer in given[s]]
        return t

    a, b, c = (table.add() for _ in range(3))
    for s in (a, b, c):
        given[s] = [[[], []] for _ in range(layers)]
    step([a, b, c], [37, 5, 64])
    e, f = fork(a), fork(c)
    step([e, a, f], [3, 1, 2])
    step([b, c, e], [1, 1, 20])
    table.free(a)
    table.free(f)
    pairs = table.compact()
    assert pairs
    binding.attn_paged_copy(kc, vc, pairs)
    kc[:, table.pages - table.free_pages:] = math.nan
    vc[:, table.pages - table.free_pages:] = math.nan
    step([e, b, c], [1, 1, 1])
    g = fork(e)
    step([g, e, b, c], [1, 1, 30, 1])


def test_append_of_very_many_heads():
    """Position 0 turns nothing: K, V and Q arrive as they are."""
    H = 65536
    f, _ = rotary_frequencies(16)
    gen = torch.Generator().manual_seed(90)
    q, k, v = (torch.randn(1, H, 16, generator=gen).to(torch.bfloat16).cuda() for _ in range(3))
    kc, vc = (torch.full((2, H, 16, 16), 3.0, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    table, lengths = torch.tensor([[1]], dtype=torch.int32).cuda(), torch.tensor([1], dtype=torch.int32).cuda()
    out = binding.attn_paged_append(k, v, kc, vc, table, lengths, Q=q, rotary=Rotary(f.cuda()))
    assert torch.equal(out, q)
    for cache, x in ((kc, k), (vc, v)):
        assert torch.equal(cache[1, :, 0], x[0])
        cache[1, :, 0] = 3.0
        assert bool((cache == 3.0).all())


def test_append_and_copy_beyond_32_bit_offsets():
    """More than 4 GiB of K: the last page is written, and copied to the front and back; its neighbours stay."""
    page, Hk, d = 64, 8, 128
    pages = (5 << 30) // (2 * page * Hk * d)
    kc, vc = (torch.empty(pages, Hk, page, d, dtype=torch.float16, device="cuda") for _ in range(2))
    for c in (kc, vc):
        c[:4] = 3.0
        c[-4:] = 3.0
    gen = torch.Generator().manual_seed(91)
    k, v = (torch.randn(10, Hk, d, generator=gen).half().cuda() for _ in range(2))
    table, lengths, starts = (torch.tensor(x, dtype=torch.int32).cuda() for x in ([[pages - 1]], [60], [0, 10]))
    binding.attn_paged_append(k, v, kc, vc, table, lengths, starts)
    binding.attn_paged_copy(kc, vc, [(pages - 1, 1), (0, pages - 3)])
    for c, x in ((kc, k), (vc, v)):
        want = torch.full((Hk, page, d), 3.0, dtype=torch.float16, device="cuda")
        want[:, 50:60] = x.transpose(0, 1)
        assert torch.equal(c[-1], want) and torch.equal(c[1], want)
        assert all(bool((c[i] == 3.0).all()) for i in (0, 2, 3, -2, -3, -4))
