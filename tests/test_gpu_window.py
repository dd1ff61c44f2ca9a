"""Attention with a sliding window and first tokens that stay visible, forward and backward, against the definition in 64 bits."""
import math

import pytest
import torch
from torch.utils.checkpoint import checkpoint

from oracle import attention_oracle as orc
from paper_2205_14135_amd import autograd, binding
from paper_2205_14135_amd.autograd import flash_attention, norm_rotary_embedding
from paper_2205_14135_amd.rotary import HeadNorm, Rotary
from tests import window_helpers as wh

pytestmark = pytest.mark.gpu
DTYPES = {"fp16": torch.float16, "bf16": torch.bfloat16}


def _inputs(B, H, N, d, dtype, seed, layout="head"):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    shape = (B, N, H, d) if layout == "token" else (B, H, N, d)
    ts = [torch.randn(shape, generator=gen, device="cuda").to(DTYPES[dtype]) for _ in range(4)]
    return [t.transpose(1, 2) for t in ts] if layout == "token" else ts


def _check(B, H, N, d, dtype, window, sinks, *, layout="head", lengths=None, p=0.0, seed=11, offset=3, times=1.0, o_fp32=False, heads=None):
    q, k, v, do = _inputs(B, H, N, d, dtype, 100 + N + d, layout)
    tau = times / math.sqrt(d)
    kl = None if lengths is None else torch.tensor(lengths, dtype=torch.int32, device="cuda")
    kw = dict(window=window, sinks=sinks, softmax_scale=tau, dropout_p=p, seed=seed, offset=offset, o_fp32=o_fp32, key_lengths=kl)
    O, L = binding.attn_window_fwd(q, k, v, **kw)
    grads = binding.attn_window_bwd(q, k, v, O, do, L, **kw)
    assert O.stride() == q.stride() and all(g.stride() == q.stride() for g in grads)
    for b in range(B):
        for h in range(H):
            if heads is not None and (b, h) not in heads:
                continue
            keep, factor = None, 1.0
            if p > 0:
                keep = torch.from_numpy(orc.dropout_keep_mask(b, h, H, N, p, seed, offset).astype("float64")).cuda()
                factor = 256.0 / (256.0 - math.floor(p * 256))
            x = wh.Head(q[b, h], k[b, h], v[b, h], do[b, h], tau, window, sinks, None if lengths is None else lengths[b], keep, factor, o_rounded=not o_fp32)
            wh.assert_within(L[b, h], x.L, x.bL, "L")
            wh.assert_within(O[b, h], x.O, x.bO32 if o_fp32 else x.bO, "O")
            for got, want, bound, name in zip(grads, (x.dQ, x.dK, x.dV), (x.bQ, x.bK, x.bV), ("dQ", "dK", "dV")):
                wh.assert_within(got[b, h], want, bound, name)
                # (the bar of the dense gradients; where few keys are visible dP and D nearly cancel and the rounding of O shows, and of one key the exact dQ and dK are zero)
                if (N if lengths is None else lengths[b]) >= 64 and window >= 16:
                    assert wh.relative(got[b, h], want) <= 2e-2, name


CASES = [(1, 1, 0), (2, 1, 0), (2, 1, 1), (5, 2, 2), (64, 63, 0), (65, 64, 0), (130, 1, 0), (130, 64, 1), (197, 64, 4), (300, 17, 33), (300, 299, 0), (300, 300, 0),
         (513, 128, 64), (640, 100, 130), (1000, 300, 0), (1000, 129, 5), (700, 31, 200), (1153, 640, 32)]


@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
@pytest.mark.parametrize("d", [16, 32, 64, 128])
@pytest.mark.parametrize("N,window,sinks", CASES)
def test_forward_and_backward(dtype, d, N, window, sinks):
    _check(1, 2, N, d, dtype, window, sinks, layout="token" if N % 2 else "head")


@pytest.mark.parametrize("d", [16, 32, 64, 128])
@pytest.mark.parametrize("window,sinks", [(100, 0), (64, 7), (33, 70)])
def test_padded_batches(d, window, sinks):
    _check(6, 2, 333, d, "bf16", window, sinks, lengths=[333, 0, 1, 128, 200, 70])


@pytest.mark.parametrize("d", [32, 64, 128])
@pytest.mark.parametrize("N,window,sinks,lengths", [(197, 64, 4, None), (700, 150, 40, [700, 333])])
def test_dropout(d, N, window, sinks, lengths):
    _check(2, 2, N, d, "bf16", window, sinks, p=0.2, lengths=lengths)


@pytest.mark.parametrize("d", [64, 128])
def test_peaked_rows_and_32_bit_outputs(d):
    _check(1, 3, 500, d, "bf16", 120, 3, times=4.0, o_fp32=True)
    _check(1, 3, 500, d, "fp16", 120, 3, o_fp32=True)


@pytest.mark.parametrize("d", [32, 64, 128])
@pytest.mark.parametrize("N,window,sinks", [(5003, 700, 70), (4096, 1024, 4), (6000, 16, 1), (3000, 50, 1500)])
def test_long(d, N, window, sinks):
    """Several stretches of queries for the sinks, and more blocks of sinks than there are compute units' shares."""
    _check(1, 1, N, d, "bf16", window, sinks)


def test_many_heads():
    """More blocks than fit at once, XCDs with unequal numbers of them; a padded batch deals its heads round."""
    _check(5, 13, 700, 64, "bf16", 200, 4, heads=[(0, 0), (2, 7), (4, 12)])
    _check(3, 11, 700, 64, "bf16", 200, 4, lengths=[700, 90, 400], heads=[(0, 0), (1, 3), (2, 10)])


@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
@pytest.mark.parametrize("N,window,sinks,kw", [(100, 20, 2, {}), (130, 40, 0, dict(layout="token")), (100, 33, 3, dict(p=0.2)), (129, 64, 1, dict(lengths=[129, 70]))])
def test_more_blocks_than_three_to_a_compute_unit(dtype, N, window, sinks, kw):
    _check(2, 400, N, 64, dtype, window, sinks, heads=[(0, 0), (0, 399), (1, 7), (1, 368), (1, 399)], **kw)


@pytest.mark.parametrize("d", [32, 64, 128])
def test_rows_and_heads_beyond_32_bit_offsets(d):
    """Tensors that span more than 4 GiB, by their rows and by their heads: the bits of packed ones."""
    N, H = 300, 2
    gen = torch.Generator(device="cuda").manual_seed(d)
    packed = [torch.randn(1, H, N, d, generator=gen, device="cuda").to(torch.bfloat16) for _ in range(4)]
    kw = dict(window=70, sinks=3, softmax_scale=d ** -0.5)

    def run(ts):
        O, L = binding.attn_window_fwd(*ts[:3], **kw)
        return [O, L, *binding.attn_window_bwd(*ts[:3], O, ts[3], L, **kw)]

    want = run(packed)
    for strides in ((H * 256, 256, 1 << 23, 1), ((1 << 33), (1 << 31) + 1024, d, 1)):
        far = [torch.empty_strided(x.shape, strides, dtype=x.dtype, device="cuda").copy_(x) for x in packed]
        assert far[0].storage_offset() + sum((n - 1) * s for n, s in zip(far[0].shape, strides)) > 1 << 31
        for got, exact in zip(run(far), want):
            assert torch.equal(got, exact)
        del far


@pytest.mark.parametrize("d", [16, 32, 64, 128])
@pytest.mark.parametrize("N,window,sinks,kw", [(300, 200, 4, {}), (300, 150, 140, {}), (333, 200, 40, dict(p=0.2)), (300, 200, 5, dict(lengths=[300, 17, 256, 129, 0, 299, 300])), (260, 130, 129, {})])
def test_sinks_that_are_swept_through(d, N, window, sinks, kw):
    """Many heads, few tiles behind the window: the blocks of keys that hold sinks take all queries."""
    _check(7, 30, N, d, "bf16", window, sinks, heads=[(0, 0), (2, 17), (3, 1), (6, 29)], **kw)


def test_more_sinks_than_segments_can_share():
    _check(4, 20, 1500, 32, "fp16", 100, 40, heads=[(0, 0), (3, 19)])


@pytest.mark.parametrize("d", [32, 64, 128])
@pytest.mark.parametrize("window,sinks", [(600, 0), (10 ** 12, 0), (500, 100), (1, 599), (1, 10 ** 12)])
def test_a_window_that_hides_nothing_is_the_causal_mask(d, window, sinks):
    q, k, v, do = _inputs(2, 3, 600, d, "bf16", 1)
    kw = dict(softmax_scale=1 / math.sqrt(d))
    O, L = binding.attn_fwd(q, k, v, causal=True, **kw)
    o, l = binding.attn_window_fwd(q, k, v, window=window, sinks=sinks, **kw)
    assert torch.equal(O, o) and torch.equal(L, l)
    want, got = binding.attn_bwd(q, k, v, O, do, L, causal=True, **kw), binding.attn_window_bwd(q, k, v, O, do, L, window=window, sinks=sinks, **kw)
    assert all(torch.equal(a, b) for a, b in zip(want, got))


@pytest.mark.parametrize("d", [64, 128])
def test_what_is_hidden_does_not_count(d):
    """Other keys and values (finite ones) behind the window: the same bits, for rows whose wavefront of 32 holds none that sees them (the reference of the softmax is moved for
    all rows of a wavefront together, so that the last bits of a row depend on the others)."""
    N, window, sinks = 900, 100, 6
    q, k, v, do = _inputs(1, 2, N, d, "bf16", 2)
    kw = dict(window=window, sinks=sinks, softmax_scale=0.1)
    O, L = binding.attn_window_fwd(q, k, v, **kw)
    k2, v2 = k.clone(), v.clone()
    k2[:, :, sinks:400] = 30.0
    v2[:, :, sinks:400] = -1e4
    o, l = binding.attn_window_fwd(q, k2, v2, **kw)
    assert torch.equal(O[:, :, 512:], o[:, :, 512:]) and torch.equal(L[:, :, 512:], l[:, :, 512:])
    assert not torch.equal(O[:, :, 300], o[:, :, 300])
    # and a query's gradients reach no key that it does not see
    do0 = torch.zeros_like(do)
    do0[:, :, 700] = do[:, :, 700]
    dq, dk, dv = binding.attn_window_bwd(q, k, v, O, do0, L, **kw)
    seen = [*range(sinks), *range(601, 701)]
    for g in (dk, dv):
        assert (g[:, :, seen] != 0).any(-1).all()
        rest = torch.ones(N, dtype=torch.bool)
        rest[seen] = False
        assert (g[:, :, rest] == 0).all()
    assert (dq[:, :, torch.arange(N) != 700] == 0).all()


@pytest.mark.parametrize("d", [16, 64, 128])
@pytest.mark.parametrize("N", [1, 77, 300, 515])
def test_nothing_outside_the_tensors(d, N):
    """Rows behind every head: NaN where the library reads, sentinels where it writes."""
    B, H, window, sinks = 2, 2, 40, 5
    ts = _inputs(B, H, N, d, "bf16", 3)
    wide = [torch.full((B, H, N + 8, d), math.nan, dtype=torch.bfloat16, device="cuda") for _ in range(9)]
    for w, t in zip(wide, ts):
        w[:, :, :N] = t
    for w in wide[4:]:
        w[:, :, N:] = 77.0
    q, k, v, do, O, dq, dk, dv, _ = (w[:, :, :N] for w in wide)
    L = torch.full((B * H * N + 8,), 55.0, device="cuda")
    kw = dict(window=window, sinks=sinks, softmax_scale=0.1)
    binding.attn_window_fwd(q, k, v, out=O, lse=L[:B * H * N].view(B, H, N), **kw)
    p = binding.make_params(q, 0.1, True)
    need = binding.attn_window_bwd_workspace_bytes(p, window, sinks)
    ws = torch.full((need + 256,), 0xFF, dtype=torch.uint8, device="cuda")      # (NaN, read as floats)
    binding.attn_window_bwd(q, k, v, O, do, L[:B * H * N].view(B, H, N), workspace=ws[:need], grads=(dq, dk, dv), **kw)
    assert (ws[need:] == 0xFF).all() and (L[B * H * N:] == 55.0).all()
    for w in wide[4:8]:
        assert (w[:, :, N:] == 77.0).all() and torch.isfinite(w[:, :, :N]).all()
    want, wl = binding.attn_window_fwd(*ts[:3], **kw)
    assert torch.equal(want, O) and torch.equal(wl, L[:B * H * N].view(B, H, N))
    for a, b in zip(binding.attn_window_bwd(*ts[:3], want, ts[3], wl, **kw), (dq, dk, dv)):
        assert torch.equal(a, b)


@pytest.mark.parametrize("d", [32, 64, 128])
def test_the_same_bits_every_time_and_on_any_stream(d):
    q, k, v, do = _inputs(2, 4, 2000, d, "bf16", 4)
    kw = dict(window=300, sinks=37, softmax_scale=0.1)
    O, L = binding.attn_window_fwd(q, k, v, **kw)
    want = binding.attn_window_bwd(q, k, v, O, do, L, **kw)
    torch.cuda.synchronize()
    streams, got = [torch.cuda.Stream() for _ in range(3)], []
    for s in streams:
        with torch.cuda.stream(s):
            o, l = binding.attn_window_fwd(q, k, v, **kw)
            got.append((o, l, *binding.attn_window_bwd(q, k, v, O, do, L, **kw)))
    torch.cuda.synchronize()
    for g in got:
        assert all(torch.equal(a, b) for a, b in zip(g, (O, L, *want)))


# ---- autograd

def test_autograd():
    q, k, v, do = _inputs(2, 3, 400, 64, "bf16", 5, "token")
    lengths = torch.tensor([400, 123], dtype=torch.int32, device="cuda")
    kw = dict(window=90, sinks=4, dropout_p=0.2, seed=9, key_lengths=lengths)
    O, L = binding.attn_window_fwd(q, k, v, softmax_scale=0.125, **kw)
    want = binding.attn_window_bwd(q, k, v, O, do, L, softmax_scale=0.125, **kw)
    leaves = [t.detach().requires_grad_(True) for t in (q, k, v)]
    out = flash_attention(*leaves, causal=True, **kw)
    assert torch.equal(out, O) and all(torch.equal(a, b) for a, b in zip(torch.autograd.grad(out, leaves, do), want))
    out = autograd._WindowAttention.apply(*leaves, 0.125, 0.2, 9, 0, lengths, 90, 4)
    assert torch.equal(out, O) and all(torch.equal(a, b) for a, b in zip(torch.autograd.grad(out, leaves, do), want))
    out = checkpoint(lambda *x: flash_attention(*x, causal=True, **kw), *leaves, use_reentrant=False)
    assert all(torch.equal(a, b) for a, b in zip(torch.autograd.grad(out, leaves, do), want))
    # a gradient that is one number in memory, and one of another layout
    out = flash_attention(*leaves, causal=True, **kw)
    got = torch.autograd.grad(out.float().sum(), leaves, retain_graph=True)
    assert all(torch.equal(a, b) for a, b in zip(got, binding.attn_window_bwd(q, k, v, O, torch.ones_like(do), L, softmax_scale=0.125, **kw)))
    got = torch.autograd.grad(out, leaves, do.contiguous())
    assert all(torch.equal(a, b) for a, b in zip(got, want))


def test_hooks_changed_inputs_and_second_gradients():
    q, k, v, do = _inputs(1, 2, 200, 64, "bf16", 15)
    leaves = [t.requires_grad_(True) for t in (q, k, v)]
    run = lambda: flash_attention(*leaves, causal=True, window=50, sinks=2)  # noqa: E731
    want = torch.autograd.grad(run(), leaves, do)
    with torch.autograd.graph.save_on_cpu():
        out = run()
    assert all(torch.equal(a, b) for a, b in zip(torch.autograd.grad(out, leaves, do, retain_graph=True), want))
    assert all(torch.equal(a, b) for a, b in zip(torch.autograd.grad(out, leaves, do), want))
    with pytest.raises(RuntimeError, match="second time"):
        torch.autograd.grad(out, leaves, do)
    for unpack in (lambda x: x[..., :32] if x.dim() == 4 else x, lambda x: x[:, :1] if x.dim() == 3 else x, lambda x: x.half() if x.dim() == 4 else x):
        with torch.autograd.graph.saved_tensors_hooks(lambda x: x, unpack):
            out = run()
        with pytest.raises(ValueError):
            torch.autograd.grad(out, leaves, do)
    out = run()
    with torch.no_grad():
        v.add_(1)
    with pytest.raises(RuntimeError, match="inplace"):
        torch.autograd.grad(out, leaves, do)
    dq, = torch.autograd.grad(run(), q, do, create_graph=True)
    for x in leaves:
        with pytest.raises(RuntimeError, match="cannot be differentiated again"):
            torch.autograd.grad(dq.float().sum(), x, retain_graph=True)
    with torch.no_grad():
        assert run().grad_fn is None
    # of one input alone
    x = q.detach().requires_grad_(True)
    got, = torch.autograd.grad(flash_attention(x, k.detach(), v.detach(), causal=True, window=50, sinks=2), x, do)
    assert torch.equal(got, torch.autograd.grad(run(), q, do)[0])


def test_formula_against_differences():
    """The gradients that the tests compare with, against central differences in 64 bits (h = 2^-16)."""
    gen = torch.Generator().manual_seed(8)
    N, d, h = 9, 4, 2.0 ** -16
    q, k, v, do = (torch.randn(N, d, generator=gen, dtype=torch.float64) for _ in range(4))

    def value(q, k, v):
        s = (0.7 * q @ k.t()).masked_fill(~wh.visible(N, 3, 2, 8, "cpu"), -math.inf)
        return float((torch.nan_to_num(torch.softmax(s, -1)) @ v * do).sum())

    x = wh.Head(q.to(torch.bfloat16), k.to(torch.bfloat16), v.to(torch.bfloat16), do.to(torch.bfloat16), 0.7, 3, 2, 8)
    q, k, v, do = (t.to(torch.bfloat16).double() for t in (q, k, v, do))
    for which, g in enumerate((x.dQ, x.dK, x.dV)):
        for i in range(N):
            for j in range(d):
                ts = [[t.clone() for t in (q, k, v)] for _ in range(2)]
                ts[0][which][i, j] += h
                ts[1][which][i, j] -= h
                assert g[i, j] == pytest.approx((value(*ts[0]) - value(*ts[1])) / (2 * h), abs=1e-7)


def test_with_norm_and_rotation():
    q, k, v, do = _inputs(1, 4, 500, 64, "bf16", 6)
    wq, wk = (torch.randn(64, device="cuda").requires_grad_(True) for _ in range(2))
    leaves = [t.requires_grad_(True) for t in (q, k, v)] + [wq, wk]
    norm, rotary = HeadNorm(wq, wk), Rotary.make(64)
    got = flash_attention(q, k, v, causal=True, norm=norm, rotary=rotary, window=128, sinks=4)
    want = flash_attention(*norm_rotary_embedding(q, k, norm, rotary), v, causal=True, window=128, sinks=4)
    assert torch.equal(got, want)
    assert all(torch.equal(a, b) for a, b in zip(torch.autograd.grad(got, leaves, do), torch.autograd.grad(want, leaves, do)))


def test_a_training_step_in_a_captured_graph():
    q, k, v, do = _inputs(1, 4, 700, 64, "bf16", 7)
    leaves = [t.requires_grad_(True) for t in (q, k, v)]
    kw = dict(window=100, sinks=40)

    def step():
        out = flash_attention(*leaves, causal=True, **kw)
        return [out.detach(), *torch.autograd.grad(out, leaves, do)]

    held = flash_attention(*leaves, causal=True, **kw)
    kept, graph = torch.zeros(1, device="cuda"), torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        kept.add_(1)
        with pytest.raises(RuntimeError, match="still leads to the same leaf"):
            flash_attention(*leaves, causal=True, **kw)
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
            q.mul_(1.25)
            v.add_(0.5)
        graph.replay()
        torch.cuda.synchronize()
        got = [x.clone() for x in out]
        O, L = binding.attn_window_fwd(q.detach(), k.detach(), v.detach(), softmax_scale=0.125, **kw)
        want = [O, *binding.attn_window_bwd(q.detach(), k.detach(), v.detach(), O, do, L, softmax_scale=0.125, **kw)]
        assert all(torch.equal(a, b) for a, b in zip(got, want)), n


def test_c_entry_points_refuse_a_short_workspace():
    q, k, v, do = _inputs(1, 1, 300, 64, "bf16", 9)
    O, L = binding.attn_window_fwd(q, k, v, window=50, sinks=2, softmax_scale=0.1)
    need = binding.attn_window_bwd_workspace_bytes(binding.make_params(q, 0.1, True), 50, 2)
    with pytest.raises(binding.AttnError):
        binding.attn_window_bwd(q, k, v, O, do, L, window=50, sinks=2, softmax_scale=0.1, workspace=torch.empty(need - 256, dtype=torch.uint8, device="cuda"))


def test_tensors_that_do_not_fit_are_refused():
    q, k, v, do = _inputs(1, 2, 100, 64, "bf16", 21)
    kw = dict(window=20, softmax_scale=0.1)
    O, L = binding.attn_window_fwd(q, k, v, **kw)
    for out, lse, error in ((O[:, :1], L, ValueError), (O.float(), L, ValueError), (O.cpu(), L, ValueError), (O, L[:, :, :50], ValueError), (O, L.double(), ValueError), (O, L.cpu(), ValueError),
                            (torch.empty(1, 2, 100, 128, dtype=torch.bfloat16, device="cuda")[..., :64], L, ValueError)):
        with pytest.raises(error):
            binding.attn_window_fwd(q, k, v, out=out, lse=lse, **kw)
        with pytest.raises(error):
            binding.attn_window_bwd(q, k, v, out, do, lse, **kw)
    with pytest.raises(ValueError):
        binding.attn_window_fwd(q, k, v, out=O, o_fp32=True, **kw)
    with pytest.raises(TypeError):
        binding.attn_window_fwd(q, k.half(), v, **kw)
    with pytest.raises(TypeError):
        flash_attention(q, k, v.float(), causal=True, window=20)
    with pytest.raises(ValueError):
        binding.attn_window_bwd(q, k, v, O, do, L, grads=(q, k, v[:, :, :50]), **kw)
    with pytest.raises(ValueError):
        binding.attn_window_bwd(q, k, v, O, do, L, workspace=torch.empty(1 << 20, dtype=torch.uint8), **kw)
    with pytest.raises(ValueError):
        binding.attn_window_fwd(q, k, v, key_lengths=torch.ones(1, dtype=torch.int32), **kw)
