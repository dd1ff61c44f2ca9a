"""Rotary positions against the rotation in 64 bits: both ways to pair columns, parts of a row, strides, in place, far positions, gradients."""
import math

import pytest
import torch

from paper_2205_14135_amd import binding
from paper_2205_14135_amd.autograd import flash_attention, rotary_embedding
from paper_2205_14135_amd.rotary import Rotary, rotary_frequencies
from tests import paged_helpers as ph

pytestmark = pytest.mark.gpu


def _tensor(B, H, N, d, dtype, seed, layout="head"):
    gen = torch.Generator().manual_seed(seed)
    x = torch.randn((B, N, H, d) if layout != "head" else (B, H, N, d), generator=gen).to(ph.DTYPES[dtype])
    if layout == "fused":     # a part of a projection's rows
        big = torch.zeros(B, N, 3 * H, d, dtype=x.dtype)
        big[:, :, H:2 * H] = x
        return big.cuda()[:, :, H:2 * H].transpose(1, 2)
    return x.cuda() if layout == "head" else x.cuda().transpose(1, 2)


def _want(x, positions, f, interleaved, magnitude, inverse=False):
    x = x.detach().cpu()
    B, H, N, d = x.shape
    pos = positions if positions.dim() == 2 else positions.expand(B, N)
    y, bound = torch.empty(x.shape, dtype=torch.float64), torch.empty(x.shape, dtype=torch.float64)
    for b in range(B):
        yb, eb = ph.turned(x[b].transpose(0, 1), pos[b], f, interleaved, magnitude, inverse)
        y[b], bound[b] = yb.transpose(0, 1), eb.transpose(0, 1)
    return y, bound + ph.rounding(y, x.dtype)


@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("d,r", [(16, 16), (16, 6), (32, 32), (32, 8), (64, 64), (64, 16), (64, 20), (128, 128), (128, 64), (128, 2), (128, 126)])
@pytest.mark.parametrize("layout", ["head", "token", "fused"])
def test_forward_and_inverse(dtype, interleaved, d, r, layout):
    f, _ = rotary_frequencies(r)
    rotary = Rotary(f.cuda(), interleaved=interleaved, magnitude=1.25)
    q, k = _tensor(2, 5, 37, d, dtype, 1, layout), _tensor(2, 2, 37, d, dtype, 2, layout)
    pos = torch.arange(37)
    for inverse in (False, True):
        got = binding.attn_rotary(q, k, rotary, inverse=inverse)
        for x, y in zip((q, k), got):
            want, bound = _want(x, pos, f, interleaved, 1.25, inverse)
            ph.assert_within(y, want, bound, "y")
            assert y.stride() == x.stride()


@pytest.mark.parametrize("interleaved,r", [(False, 64), (False, 20), (True, 64)])
def test_in_place_and_one_tensor(interleaved, r):
    f, _ = rotary_frequencies(r)
    rotary = Rotary(f.cuda(), interleaved=interleaved)
    q, k = _tensor(3, 9, 301, 64, "bf16", 3, "token"), _tensor(3, 3, 301, 64, "bf16", 4, "token")
    want = binding.attn_rotary(q, k, rotary)
    alone, none = binding.attn_rotary(q, None, rotary)
    assert none is None and torch.equal(alone, want[0])
    got = binding.attn_rotary(q, k, rotary, out=(q, k))
    assert got[0] is q and torch.equal(q, want[0]) and torch.equal(k, want[1])


@pytest.mark.parametrize("interleaved", [False, True])
def test_far_positions(interleaved):
    f, magnitude = rotary_frequencies(128, scaling="parts", factor=16.0)
    q, k = _tensor(2, 2, 8, 128, "fp16", 5), _tensor(2, 1, 8, 128, "fp16", 6)
    pos = torch.tensor([[0, 1, 4095, 131071, 1 << 20, (1 << 24) + 1, 2 ** 31 - 1, -5], [7, -2 ** 31, 3, 2, 10 ** 9, 5, 99999, 12]], dtype=torch.int32)
    got = binding.attn_rotary(q, k, Rotary(f.cuda(), interleaved=interleaved, magnitude=magnitude), positions=pos.cuda())
    for x, y in zip((q, k), got):
        want, bound = _want(x, pos, f, interleaved, magnitude)
        ph.assert_within(y, want, bound, "y")


@pytest.mark.parametrize("B,H,N", [(1, 1, 1), (1, 32, 1), (64, 40, 1), (1, 3, 4099), (5, 1, 333)])
def test_sizes(B, H, N):
    f, _ = rotary_frequencies(64)
    q, k = _tensor(B, H, N, 64, "bf16", 7), _tensor(B, max(1, H // 4), N, 64, "bf16", 8)
    for x, y in zip((q, k), binding.attn_rotary(q, k, Rotary(f.cuda()))):
        want, bound = _want(x, torch.arange(N), f, False, 1.0)
        ph.assert_within(y, want, bound, "y")


def test_positions_of_each_entry_and_a_repeated_input():
    f, _ = rotary_frequencies(32)
    q = _tensor(1, 4, 50, 64, "bf16", 9).expand(3, 4, 50, 64)
    pos = torch.randint(0, 10000, (3, 50), dtype=torch.int32)
    got, _ = binding.attn_rotary(q, None, Rotary(f.cuda()), positions=pos.cuda())
    want, bound = _want(q, pos, f, False, 1.0)
    ph.assert_within(got, want, bound, "y")


@pytest.mark.parametrize("python_node", [False, True])
@pytest.mark.parametrize("interleaved,r", [(False, 64), (True, 48), (False, 22)])
def test_gradients(interleaved, r, python_node, monkeypatch):
    """d loss / d x of sum(g . y) is the rotation of g by the negative angle; against differences too: the rotation is linear, so one step of any size will do."""
    from paper_2205_14135_amd import autograd
    if python_node:
        monkeypatch.setattr(autograd, "_node_in_python", lambda: True)
    f, _ = rotary_frequencies(r)
    rotary = Rotary(f.cuda(), interleaved=interleaved, magnitude=0.75)
    pos = torch.arange(100, 141, dtype=torch.int32)
    q, k = _tensor(2, 4, 41, 64, "fp16", 10, "token"), _tensor(2, 2, 41, 64, "fp16", 11, "fused")
    q.requires_grad_(True)
    k.requires_grad_(True)
    gq, gk = _tensor(2, 4, 41, 64, "fp16", 12), _tensor(2, 2, 41, 64, "fp16", 13, "token")
    yq, yk = rotary_embedding(q, k, rotary, pos.cuda())
    dq, dk = torch.autograd.grad((yq, yk), (q, k), (gq, gk))
    for g, got in ((gq, dq), (gk, dk)):
        want, bound = _want(g, pos, f, interleaved, 0.75, inverse=True)
        ph.assert_within(got, want, bound, "dx")
    # <g, y(x + e) - y(x)> = <dx, e>, with y in 64 bits (each element of dx is off by its rounding alone)
    e = _tensor(2, 4, 41, 64, "fp16", 14).cpu().double()
    y0, _ = _want(q, pos, f, interleaved, 0.75)
    moved = torch.empty_like(y0)
    for b in range(2):
        moved[b] = ph.turned((q[b].detach().cpu().double() + e[b]).transpose(0, 1), pos, f, interleaved, 0.75)[0].transpose(0, 1)
    left, right = (gq.cpu().double() * (moved - y0)).sum(), (dq.cpu().double() * e).sum()
    slack = ((2.0 ** -11 * dq.cpu().double().abs() + 2.0 ** -18) * e.abs()).sum()
    assert abs(left - right) <= slack


def test_gradient_of_one_output_of_a_sum_and_twice():
    f, _ = rotary_frequencies(64)
    rotary = Rotary(f.cuda())
    q, k = (_tensor(1, 2, 33, 64, "bf16", 15 + i).requires_grad_(True) for i in range(2))
    yq, yk = rotary_embedding(q, k, rotary)
    dq, = torch.autograd.grad(yq.sum(), q)                      # (an expanded gradient; none for K)
    want, bound = _want(torch.ones_like(q), torch.arange(33), f, False, 1.0, inverse=True)
    ph.assert_within(dq, want, bound, "dq")
    g = _tensor(1, 2, 33, 64, "bf16", 20).requires_grad_(True)
    yq, _ = rotary_embedding(q, k, rotary)
    dq, = torch.autograd.grad(yq, q, g, create_graph=True)
    h = _tensor(1, 2, 33, 64, "bf16", 21)
    dg, = torch.autograd.grad(dq, g, h)
    want, bound = _want(h, torch.arange(33), f, False, 1.0)
    ph.assert_within(dg, want, bound, "dg")


@pytest.mark.parametrize("interleaved", [False, True])
def test_flash_attention_with_rotary_is_rotary_then_attention(interleaved):
    f, m = rotary_frequencies(32, scaling="linear", factor=2.0)
    rotary = Rotary(f.cuda(), interleaved=interleaved, magnitude=m)
    pos = torch.arange(5, 205, dtype=torch.int32, device="cuda")
    ts = [_tensor(2, 4, 200, 64, "bf16", 30 + i, "fused").requires_grad_(True) for i in range(3)]
    g = _tensor(2, 4, 200, 64, "bf16", 40)
    out = flash_attention(*ts, causal=True, rotary=rotary, positions=pos)
    grads = torch.autograd.grad(out, ts, g)
    turned = rotary_embedding(ts[0], ts[1], rotary, pos)
    ref = flash_attention(*turned, ts[2], causal=True)
    want = torch.autograd.grad(ref, ts, g)
    assert torch.equal(out, ref) and all(torch.equal(a, b) for a, b in zip(grads, want))


def test_graph_of_forward_and_backward():
    f, _ = rotary_frequencies(64)
    rotary = Rotary(f.cuda())
    q, k = (_tensor(2, 4, 130, 64, "bf16", 50 + i).requires_grad_(True) for i in range(2))
    pos = torch.arange(130, dtype=torch.int32, device="cuda")
    g = _tensor(2, 4, 130, 64, "bf16", 52)

    def step():
        y = rotary_embedding(q, k, rotary, pos)
        return (*[t.detach() for t in y], *torch.autograd.grad(y, (q, k), (g, g)))

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step()
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        held = step()
    for shift in (0, 1000, 7):
        pos.copy_(torch.arange(130, dtype=torch.int32, device="cuda") + shift)
        graph.replay()
        torch.cuda.synchronize()
        replayed = [t.clone() for t in held]
        want = step()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(replayed, want))


@pytest.mark.parametrize("call", ["rotary", "attention", "attention_v"])
def test_capture_beside_an_eager_graph_is_refused(call):
    """The forward pass under capture is refused while an eager graph of the default stream leads to a leaf; without that graph it is not."""
    f, _ = rotary_frequencies(64)
    rotary = Rotary(f.cuda())
    q, k, v = (_tensor(1, 2, 40, 64, "bf16", 60 + i).requires_grad_(call != "attention_v" or i == 2) for i in range(3))
    run = (lambda: rotary_embedding(q, k, rotary)) if call == "rotary" else (lambda: flash_attention(q, k, v, rotary=rotary))
    held = run()
    here = torch.zeros(1, device="cuda")
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        here.add_(1)
        with pytest.raises(RuntimeError, match="still leads to the same leaf"):
            run()
    with torch.no_grad(), torch.cuda.graph(torch.cuda.CUDAGraph()):
        run()
    del held
    with torch.cuda.graph(torch.cuda.CUDAGraph()):
        run()
    graph.replay()
    torch.cuda.synchronize()
    assert here.item() == 1.0


def test_very_many_heads():
    f, _ = rotary_frequencies(16)
    rotary = Rotary(f.cuda())
    q, k = _tensor(1, 65536, 1, 16, "bf16", 70), _tensor(1, 65535, 1, 16, "bf16", 71)
    pos = torch.tensor([5], dtype=torch.int32)
    for x, y in zip((q, k), binding.attn_rotary(q, k, rotary, positions=pos.cuda())):
        want, bound = _want(x, pos, f, False, 1.0)
        ph.assert_within(y, want, bound, "y")
