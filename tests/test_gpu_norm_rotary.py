"""Norm of Q and K with the rotation in the same pass, forward and backward, against the formula in 64 bits; the append of new tokens with both."""
import math

import pytest
import torch
from torch.utils.checkpoint import checkpoint

from paper_2205_14135_amd import binding
from paper_2205_14135_amd.autograd import flash_attention, norm_rotary_embedding
from paper_2205_14135_amd.rotary import HeadNorm, Rotary, rotary_frequencies
from tests import norm_helpers as nh
from tests import paged_helpers as ph

pytestmark = pytest.mark.gpu
EPS = 1e-5


def _tensor(B, H, N, d, dtype, seed, layout="head"):
    gen = torch.Generator().manual_seed(seed)
    x = torch.randn((B, N, H, d) if layout != "head" else (B, H, N, d), generator=gen).to(ph.DTYPES[dtype])
    if layout == "fused":     # a part of a projection's rows
        big = torch.zeros(B, N, 3 * H, d, dtype=x.dtype)
        big[:, :, H:2 * H] = x
        return big.cuda()[:, :, H:2 * H].transpose(1, 2)
    return x.cuda() if layout == "head" else x.cuda().transpose(1, 2)


def _weights(d, dtype, kind, seed):
    gen = torch.Generator().manual_seed(seed)
    w = [1.0 + 0.5 * torch.randn(d, generator=gen) for _ in range(2)]
    return [x.to(ph.DTYPES[dtype]) if kind == "same" else x for x in w]


def _check(B, N, Hq, Hk, d, dtype, r, interleaved, kind="float32", layout="head", magnitude=1.0, positions=None, scale=1.0):
    f = rotary_frequencies(r)[0] if r else None
    rotary = Rotary(f.cuda(), interleaved=interleaved, magnitude=magnitude) if r else None
    q, k, gq, gk = (_tensor(B, H, N, d, dtype, 10 + i, layout) * s for i, (H, s) in enumerate(((Hq, scale), (Hk, scale), (Hq, 1), (Hk, 1))))
    wq, wk = _weights(d, dtype, kind, 5)
    norm = HeadNorm(wq.cuda(), wk.cuda(), eps=EPS)
    pos = torch.arange(N) if positions is None else positions
    on = None if positions is None else positions.to(torch.int32).cuda()
    kw = dict(f=f, interleaved=interleaved, magnitude=magnitude)
    eps = float(torch.tensor(EPS, dtype=torch.float32))
    got = binding.attn_norm_rotary(q, k, norm, rotary, positions=on)
    for x, w, y, what in ((q, wq, got[0], "q"), (k, wk, got[1], "k")):
        want, bound = nh.over_batch(nh.forward, x, w, eps, positions=pos, **kw)
        ph.assert_within(y, want, bound, what)
        assert y.stride() == x.stride()
    dq, dk, dwq, dwk = binding.attn_norm_rotary_bwd(q, k, gq, gk, norm, rotary, positions=on)
    for x, w, g, dx, dw, what in ((q, wq, gq, dq, dwq, "q"), (k, wk, gk, dk, dwk, "k")):
        want, bound, want_w, bound_w = nh.over_batch(nh.gradients, x, w, eps, positions=pos, dy=g, **kw)
        ph.assert_within(dx, want, bound, "d" + what)
        if kind == "same":
            bound_w = bound_w + ph.rounding(want_w.abs() + bound_w, w.dtype)
        assert dw.dtype == w.dtype
        ph.assert_within(dw, want_w, bound_w, "weights of " + what)


@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
@pytest.mark.parametrize("d,r,interleaved", [(16, 16, False), (16, 6, False), (16, 6, True), (32, 32, False), (32, 8, True), (64, 64, False), (64, 20, False), (64, 0, False),
                                             (64, 64, True), (128, 128, False), (128, 64, True), (128, 126, False), (128, 16, False)])
@pytest.mark.parametrize("layout", ["head", "token", "fused"])
def test_forward_and_gradients(dtype, d, r, interleaved, layout):
    _check(2, 37, 5, 2, d, dtype, r, interleaved, "same" if layout == "head" else "float32", layout, 1.25 if r else 1.0)


@pytest.mark.parametrize("B,N,Hq,Hk", [(1, 1, 1, 1), (1, 1, 17, 3), (3, 2, 9, 9), (1, 197, 12, 12), (5, 64, 1, 13), (1, 33, 70, 1)])
@pytest.mark.parametrize("d", [16, 128])
def test_sizes(B, N, Hq, Hk, d):
    _check(B, N, Hq, Hk, d, "bf16", d, False)


def test_more_rows_than_one_round_of_workgroups():
    """d = 128: 32 tokens to a workgroup, 2048 workgroups."""
    _check(1, 70001, 1, 1, 128, "fp16", 128, False)


@pytest.mark.parametrize("positions", [torch.tensor([0, -1, 2 ** 31 - 1, -2 ** 31, 1000003, 7, 7, 131072]), torch.arange(16).view(2, 8) * 12345])
def test_positions(positions):
    _check(2, 8, 3, 1, 64, "bf16", 64, False, positions=positions)


@pytest.mark.parametrize("scale", [2.0 ** -12, 2.0 ** 9])
def test_small_and_large_rows(scale):
    """Rows whose mean square is far below eps, and such as fill most of fp16."""
    _check(1, 50, 3, 2, 64, "fp16", 64, False, scale=scale)


def test_rows_of_zeros():
    q = torch.zeros(1, 2, 5, 64, dtype=torch.bfloat16, device="cuda")
    g = torch.ones_like(q)
    norm = HeadNorm(torch.full((64,), 2.0, device="cuda"), eps=1e-4)
    y, none = binding.attn_norm_rotary(q, None, norm)
    assert none is None and (y == 0).all()
    dq, _, dw, _ = binding.attn_norm_rotary_bwd(q, None, g, None, norm)
    assert torch.equal(dq, torch.full_like(q, 200.0)) and (dw == 0).all()     # w / sqrt(eps) = 200 exactly in bf16


def test_formula_against_differences():
    """The gradients that the tests above compare with, against central differences of the forward formula: h = 2^-16, off by h^2 of a third derivative and 2^-52 / h."""
    gen = torch.Generator().manual_seed(3)
    x, dy = (torch.randn(4, 2, 16, generator=gen, dtype=torch.float64) for _ in range(2))
    w, f, pos, h = torch.randn(16, generator=gen, dtype=torch.float64), rotary_frequencies(8)[0], torch.arange(4), 2.0 ** -16
    value = lambda x, w: float((nh.forward(x, w, 1e-3, pos, f, True, 1.5)[0] * dy).sum())  # noqa: E731
    dx, _, dw, _ = nh.gradients(x, w, dy, 1e-3, pos, f, True, 1.5)
    for i in range(0, x.numel(), 5):
        e = torch.zeros(x.numel(), dtype=torch.float64)
        e[i] = h
        assert dx.reshape(-1)[i] == pytest.approx((value(x + e.view(x.shape), w) - value(x - e.view(x.shape), w)) / (2 * h), abs=1e-7)
    for i in range(16):
        e = torch.zeros(16, dtype=torch.float64)
        e[i] = h
        assert dw[i] == pytest.approx((value(x, w + e) - value(x, w - e)) / (2 * h), abs=1e-7)


@pytest.mark.parametrize("interleaved,r", [(False, 64), (False, 20), (True, 64), (False, 0)])
def test_in_place_one_tensor_and_the_same_bits_again(interleaved, r):
    rotary = Rotary.make(r, interleaved=interleaved) if r else None
    q, k = _tensor(3, 9, 301, 64, "bf16", 3, "token"), _tensor(3, 3, 301, 64, "bf16", 4, "token")
    norm = HeadNorm(*(w.cuda() for w in _weights(64, "bf16", "same", 1)))
    want = binding.attn_norm_rotary(q, k, norm, rotary)
    alone, none = binding.attn_norm_rotary(q, None, norm, rotary)
    assert none is None and torch.equal(alone, want[0])
    grads = [binding.attn_norm_rotary_bwd(q, k, *want, norm, rotary) for _ in range(2)]
    assert all(torch.equal(a, b) for a, b in zip(*grads))
    alone = binding.attn_norm_rotary_bwd(q, None, want[0], None, norm, rotary)
    assert torch.equal(alone[0], grads[0][0]) and alone[1] is None and alone[3] is None
    a, b = q.clone(), k.clone()
    got = binding.attn_norm_rotary(a, b, norm, rotary, out=(a, b))
    assert got[0] is a and got[1] is b and torch.equal(a, want[0]) and torch.equal(b, want[1])


# ---- autograd

def _leaves(N=40, kind="float32", H=(3, 1)):
    q, k, gq, gk = (_tensor(2, h, N, 64, "bf16", 20 + i, "token") for i, h in enumerate((*H, *H)))
    wq, wk = (w.cuda() for w in _weights(64, "bf16", kind, 9))
    return q, k, wq, wk, gq, gk, Rotary.make(64)


@pytest.mark.parametrize("which", range(1, 16))
def test_autograd_takes_any_of_the_four(which):
    q, k, wq, wk, gq, gk, rotary = _leaves()
    want = binding.attn_norm_rotary_bwd(q, k, gq, gk, HeadNorm(wq, wk), rotary)
    leaves = [x for i, x in enumerate((q, k, wq, wk)) if which >> i & 1]
    for x in leaves:
        x.requires_grad_(True)
    ys = norm_rotary_embedding(q, k, HeadNorm(wq, wk), rotary)
    assert all(torch.equal(a, b) for a, b in zip(ys, binding.attn_norm_rotary(q.detach(), k.detach(), HeadNorm(wq.detach(), wk.detach()), rotary)))
    got = torch.autograd.grad(ys, leaves, (gq, gk), allow_unused=True)
    assert all(torch.equal(a, b) for a, b in zip(got, [g for i, g in enumerate(want) if which >> i & 1]))


def test_autograd_of_one_output_and_of_broadcast_inputs():
    q, k, wq, wk, gq, gk, rotary = _leaves()
    for x in (q, k, wq, wk):
        x.requires_grad_(True)
    norm = HeadNorm(wq, wk)
    want = binding.attn_norm_rotary_bwd(q.detach(), k.detach(), gq, gk, HeadNorm(wq.detach(), wk.detach()), rotary)
    yq, yk = norm_rotary_embedding(q, k, norm, rotary)
    dk, dwk, dq = torch.autograd.grad(yk, (k, wk, q), gk, allow_unused=True)
    assert torch.equal(dk, want[1]) and torch.equal(dwk, want[3]) and dq is None
    # K of one head shown to three, a gradient of ones that is one number in memory
    yq, yk = norm_rotary_embedding(q, k.expand(2, 3, 40, 64), norm, rotary)
    assert torch.equal(yk[:, 0], yk[:, 2])
    dk, = torch.autograd.grad(yk.sum(), k)
    one = binding.attn_norm_rotary_bwd(q.detach(), k.detach(), gq, torch.ones_like(gk), HeadNorm(wq.detach(), wk.detach()), rotary)[1]
    # three equal bf16 gradients added up: at most two roundings of half a step, of sums of up to three times the value
    assert (dk.double() - 3 * one.double()).abs().max() <= 2 * 2.0 ** -8 * 3 * one.double().abs().max()


def test_the_gradients_have_no_gradients():
    q, k, wq, wk, gq, gk, rotary = _leaves()
    q.requires_grad_(True)
    wq.requires_grad_(True)
    yq, _ = norm_rotary_embedding(q, k, HeadNorm(wq, wk), rotary)
    dq, = torch.autograd.grad(yq, q, gq, create_graph=True)
    with pytest.raises(RuntimeError, match="cannot be differentiated again"):
        torch.autograd.grad(dq.float().sum(), wq, allow_unused=True)


def test_checkpoint_hooks_and_changed_inputs():
    q, k, wq, wk, gq, gk, rotary = _leaves()
    for x in (q, k, wq, wk):
        x.requires_grad_(True)
    norm = HeadNorm(wq, wk)
    want = torch.autograd.grad(norm_rotary_embedding(q, k, norm, rotary), (q, k, wq, wk), (gq, gk))
    ys = checkpoint(lambda a, b: norm_rotary_embedding(a, b, norm, rotary), q, k, use_reentrant=False)
    assert all(torch.equal(a, b) for a, b in zip(torch.autograd.grad(ys, (q, k, wq, wk), (gq, gk)), want))
    with torch.autograd.graph.save_on_cpu():
        ys = norm_rotary_embedding(q, k, norm, rotary)
    assert all(torch.equal(a, b) for a, b in zip(torch.autograd.grad(ys, (q, k, wq, wk), (gq, gk)), want))
    with torch.autograd.graph.saved_tensors_hooks(lambda x: x, lambda x: x[..., :32]):
        ys = norm_rotary_embedding(q, k, norm, rotary)
    with pytest.raises(ValueError, match="not those of the forward call"):
        torch.autograd.grad(ys, (q, k), (gq, gk))
    ys = norm_rotary_embedding(q, k, norm, rotary)
    with torch.no_grad():
        wq.add_(1)
    with pytest.raises(RuntimeError, match="inplace"):
        torch.autograd.grad(ys, (q, k), (gq, gk))


def test_in_front_of_attention():
    q, k, wq, wk, gq, _, rotary = _leaves(H=(3, 3))
    v = _tensor(2, 3, 40, 64, "bf16", 31, "token")
    for x in (q, k, v, wq, wk):
        x.requires_grad_(True)
    norm = HeadNorm(wq, wk)
    got = flash_attention(q, k, v, causal=True, rotary=rotary, norm=norm)
    want = flash_attention(*norm_rotary_embedding(q, k, norm, rotary), v, causal=True)
    assert torch.equal(got, want)
    assert all(torch.equal(a, b) for a, b in zip(torch.autograd.grad(got, (q, k, v, wq, wk), gq), torch.autograd.grad(want, (q, k, v, wq, wk), gq)))


def test_a_training_step_in_a_captured_graph():
    q, k, wq, wk, gq, gk, rotary = _leaves()
    for x in (q, k, wq, wk):
        x.requires_grad_(True)
    norm = HeadNorm(wq, wk)

    def step():
        ys = norm_rotary_embedding(q, k, norm, rotary)
        return [y.detach() for y in ys] + list(torch.autograd.grad(ys, (q, k, wq, wk), (gq, gk)))

    held = norm_rotary_embedding(q, k, norm, rotary)
    graph = torch.cuda.CUDAGraph()
    kept = torch.zeros(1, device="cuda")
    with torch.cuda.graph(graph):
        kept.add_(1)
        with pytest.raises(RuntimeError, match="still leads to the same leaf"):
            norm_rotary_embedding(q, k, norm, rotary)
    del held
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step()
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = step()
    for n in range(4):
        with torch.no_grad():
            q.mul_(0.75)
            gk.add_(0.5)
        graph.replay()
        torch.cuda.synchronize()
        got = [x.clone() for x in out]
        want = [*binding.attn_norm_rotary(q.detach(), k.detach(), HeadNorm(wq.detach(), wk.detach()), rotary),
                *binding.attn_norm_rotary_bwd(q.detach(), k.detach(), gq, gk, HeadNorm(wq.detach(), wk.detach()), rotary)]
        assert all(torch.equal(a, b) for a, b in zip(got, want)), n


@pytest.mark.parametrize("interleaved,r", [(False, 64), (False, 20), (True, 64)])
def test_rows_and_heads_beyond_32_bit_offsets(interleaved, r):
    """Tensors that span more than 4 GiB, by their rows and by their heads: the bits of packed ones."""
    N, H, d = 300, 2, 64
    gen = torch.Generator(device="cuda").manual_seed(r)
    packed = [torch.randn(1, H, N, d, generator=gen, device="cuda").to(torch.bfloat16) for _ in range(4)]
    norm = HeadNorm(*(1.0 + 0.25 * torch.randn(d, generator=gen, device="cuda") for _ in range(2)))
    rotary = Rotary.make(r, interleaved=interleaved)

    def run(ts):
        return [*binding.attn_norm_rotary(ts[0], ts[1], norm, rotary), *binding.attn_norm_rotary_bwd(*ts, norm, rotary)]

    want = run(packed)
    for strides in ((H * 256, 256, 1 << 23, 1), ((1 << 33), (1 << 31) + 1024, d, 1)):
        far = [torch.empty_strided(x.shape, strides, dtype=x.dtype, device="cuda").copy_(x) for x in packed]
        for got, exact in zip(run(far), want):
            assert torch.equal(got, exact)
        del far


def test_on_another_stream():
    q, k, wq, wk, gq, gk, rotary = _leaves(N=3000)
    norm = HeadNorm(wq, wk)
    want = binding.attn_norm_rotary_bwd(q, k, gq, gk, norm, rotary)
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(3)]
    got = []
    for s in streams:
        with torch.cuda.stream(s):
            got.append(binding.attn_norm_rotary_bwd(q, k, gq, gk, norm, rotary))
    torch.cuda.synchronize()
    for g in got:
        assert all(torch.equal(a, b) for a, b in zip(g, want))


# ---- the append

def _append(batch, r, interleaved, kind, with_q=True, single=False, in_place=False):
    q, kc, vc, table, lengths, starts = batch.gpu(single)
    k, v = (torch.empty_strided(x.size(), x.stride(), dtype=x.dtype, device="cuda").copy_(x) for x in (batch.k, batch.v))
    f = rotary_frequencies(r)[0] if r else None
    rotary = Rotary(f.cuda(), interleaved=interleaved, magnitude=1.1) if r else None
    dtype = "bf16" if batch.dtype == torch.bfloat16 else "fp16"
    wq, wk = _weights(batch.d, dtype, kind, 6)
    out = (q if in_place else torch.full_like(q, 7.0)) if with_q else None
    got = binding.attn_paged_append(k, v, kc, vc, table, lengths, starts, Q=q if with_q else None, rotary=rotary, norm=HeadNorm(wq.cuda(), wk.cuda(), eps=EPS), out=out)
    assert got is out
    eps = float(torch.tensor(EPS, dtype=torch.float32))
    want_k, want_v, bound_k = batch.kc.double(), batch.vc.double(), torch.zeros(batch.kc.shape, dtype=torch.float64)
    want_q = batch.q.double() if in_place else torch.full(batch.q.shape, 7.0, dtype=torch.float64)
    bound_q = torch.zeros_like(want_q)
    capacity = batch.table.shape[1] * batch.page
    for b in range(batch.B):
        at, m, n = int(batch.starts[b]), batch.new[b], batch.lengths[b]
        pos = torch.arange(n - m, n)
        rows = slice(at, at + m)
        yk, bk = nh.forward(batch.k[rows], wk, eps, pos, f, interleaved, 1.1)
        if m:
            want_q[rows], bound_q[rows] = nh.forward(batch.q[rows], wq, eps, pos, f, interleaved, 1.1)
        for i, p in enumerate(pos.tolist()):
            if not 0 <= p < capacity or not 0 <= int(batch.table[b, p // batch.page]) < batch.pages:
                continue
            at_row = int(batch.table[b, p // batch.page]), slice(None), p % batch.page
            want_k[at_row], bound_k[at_row] = yk[i], bk[i]
            want_v[at_row] = batch.v[at + i].double()
    ph.assert_within(torch.nan_to_num(kc, 99.0), torch.nan_to_num(want_k, 99.0), bound_k, "K cache")
    ph.assert_within(torch.nan_to_num(vc, 99.0), torch.nan_to_num(want_v, 99.0), torch.zeros_like(want_v), "V cache")
    if with_q:
        ph.assert_within(torch.nan_to_num(out, 99.0), torch.nan_to_num(want_q, 99.0), bound_q, "Q")


@pytest.mark.parametrize("dtype,kind", [("bf16", "same"), ("fp16", "float32")])
@pytest.mark.parametrize("d,r,interleaved", [(16, 16, False), (32, 0, False), (64, 32, True), (64, 12, False), (128, 128, False), (128, 96, True)])
@pytest.mark.parametrize("new", [[1, 1, 1, 1], [5, 0, 130, 17]])
def test_append(dtype, kind, d, r, interleaved, new):
    _append(ph.Batch([0, 15, 16, 900], new, 6, 2, d, dtype, 16, pad=9, seed=d + r), r, interleaved, kind)


@pytest.mark.parametrize("kw", [dict(single=True), dict(with_q=False), dict(in_place=True)])
def test_append_other_ways(kw):
    _append(ph.Batch([3, 15, 16, 900, 0], [1] * 5, 8, 8, 64, "bf16", 32, token_major=True, fused=True), 64, False, "float32", **kw)


def test_append_of_tokens_that_have_no_place():
    """Pages that are none, and a length beyond the table."""
    batch = ph.Batch([40, 100], [20, 30], 4, 2, 64, "bf16", 16, seed=4)
    batch.table[0, 3] = 10 ** 6
    batch.table = batch.table[:, :8].contiguous()
    _append(batch, 64, False, "float32")


def test_append_then_attend_equals_the_whole_prompt():
    """A prompt read in by chunks and single tokens through the cache, against normed attention over all of it at once: the rows of Q and K are rounded once on either way,
    so that the attention reads the same bits."""
    H, N, d = 4, 300, 64
    q, k, v = (_tensor(1, H, N, d, "bf16", 40 + i, "token") for i in range(3))
    norm, rotary = HeadNorm(*(w.cuda() for w in _weights(d, "bf16", "same", 2))), Rotary.make(d)
    want_q, want_k = binding.attn_norm_rotary(q, k, norm, rotary)
    kc, vc = (torch.zeros(32, H, 16, d, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    table = torch.randperm(32, generator=torch.Generator().manual_seed(1))[:20].to(torch.int32).view(1, 20).cuda()
    at = 0
    for n in (100, 1, 1, 150, 48):
        rows = [x[0, :, at:at + n].transpose(0, 1) for x in (q, k, v)]
        at += n
        lengths, starts = torch.tensor([at], dtype=torch.int32).cuda(), torch.tensor([0, n], dtype=torch.int32).cuda()
        turned = binding.attn_paged_append(rows[1], rows[2], kc, vc, table, lengths, starts, Q=rows[0], rotary=rotary, norm=norm)
        assert torch.equal(turned, want_q[0, :, at - n:at].transpose(0, 1))
    held = kc[table[0].long()].transpose(1, 2).reshape(-1, H, d)[:N]
    assert torch.equal(held, want_k[0].transpose(0, 1))
