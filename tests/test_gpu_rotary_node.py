"""The native autograd node of the rotation under what a program may do with a graph: saved-tensor hooks, checkpoints, threads, transforms."""
import threading

import pytest
import torch
from torch.autograd import forward_ad
from torch.utils.checkpoint import checkpoint

from paper_2205_14135_amd.autograd import flash_attention, rotary_embedding
from paper_2205_14135_amd.rotary import Rotary

pytestmark = pytest.mark.gpu


def _tensors(requires_grad=True, H=3, N=40):
    gen = torch.Generator(device="cuda").manual_seed(5)
    q, k, gq, gk = (torch.randn(2, h, N, 64, generator=gen, device="cuda").to(torch.bfloat16) for h in (H, 1, H, 1))
    pos = torch.arange(7, 7 + N, dtype=torch.int32, device="cuda")
    return q.requires_grad_(requires_grad), k.requires_grad_(requires_grad), gq, gk, Rotary.make(64), pos


def test_two_threads_do_not_unpack_the_same_node_at_once():
    """A thread that is inside the node (here: in a hook of the program, which brings back a saved tensor) keeps another one out, as the nodes of torch do; so
    none finds the saved tensors half released."""
    q, k, gq, gk, rotary, pos = _tensors()
    inside, most = [0], [0]
    entered = threading.Event()

    def unpack(x):
        inside[0] += 1
        most[0] = max(most[0], inside[0])
        entered.set()
        threading.Event().wait(0.3)      # (without the interpreter lock)
        inside[0] -= 1
        return x

    with torch.autograd.graph.saved_tensors_hooks(lambda x: x, unpack):
        yq, _ = rotary_embedding(q, k, rotary, pos)
    got, errors = [None, None], []

    def worker(i):
        try:
            got[i] = yq.grad_fn(gq, gk)
            torch.cuda.synchronize()
        except Exception as e:  # noqa: BLE001
            errors.append(e)

    threads = [threading.Thread(target=worker, args=(i,)) for i in range(2)]
    threads[0].start()
    entered.wait(5.0)
    threads[1].start()
    for t in threads:
        t.join(20.0)
    assert not errors and not any(t.is_alive() for t in threads)
    assert most[0] == 1
    assert all(torch.equal(a, b) for a, b in zip(*got))


def test_graph_rules():
    q, k, gq, gk, rotary, pos = _tensors()
    ys = rotary_embedding(q, k, rotary, pos)
    want = torch.autograd.grad(ys, (q, k), (gq, gk), retain_graph=True)
    got = torch.autograd.grad(ys, (q, k), (gq, gk))
    assert all(torch.equal(a, b) for a, b in zip(got, want))
    with pytest.raises(RuntimeError, match="second time"):
        torch.autograd.grad(ys, (q, k), (gq, gk))
    ys = rotary_embedding(q, k, rotary, pos)
    pos.add_(1)
    with pytest.raises(RuntimeError, match="inplace"):
        torch.autograd.grad(ys, (q, k), (gq, gk))
    with torch.no_grad():
        assert all(y.grad_fn is None for y in rotary_embedding(q, k, rotary, pos))


def test_backward_from_two_threads():
    """Two threads run backward through one graph: one has the gradients, and the other has them too or is told that the graph is gone."""
    for _ in range(20):
        q, k, gq, gk, rotary, pos = _tensors()
        ys = rotary_embedding(q, k, rotary, pos)
        want = torch.autograd.grad(ys, (q, k), (gq, gk), retain_graph=True)
        got, errors = [], []

        def worker():
            try:
                got.append(torch.autograd.grad(ys, (q, k), (gq, gk)))
            except RuntimeError as e:
                errors.append(str(e))

        threads = [threading.Thread(target=worker) for _ in range(2)]
        for t in threads:
            t.start()
        for t in threads:
            t.join(20.0)
        assert len(got) >= 1 and len(got) + len(errors) == 2 and all("second time" in e for e in errors)
        for g in got:
            assert all(torch.equal(a, b) for a, b in zip(g, want))


def test_gradients_have_no_gaps():
    """Gradients with the strides of a projection's part, as the attention hands them back: what comes out holds its own elements alone."""
    q, k, gq, gk, rotary, pos = _tensors()
    wide = [torch.zeros(2, 40, 3 * g.shape[1], 64, dtype=g.dtype, device="cuda")[:, :, :g.shape[1]].transpose(1, 2).copy_(g) for g in (gq, gk)]
    ys = rotary_embedding(q, k, rotary, pos)
    want = torch.autograd.grad(ys, (q, k), (gq, gk), retain_graph=True)
    got = torch.autograd.grad(ys, (q, k), wide)
    assert all(torch.equal(a, b) for a, b in zip(got, want))
    assert all(g.untyped_storage().nbytes() == 2 * g.numel() for g in got)


def test_saved_tensor_hooks_and_checkpoint():
    q, k, gq, gk, rotary, pos = _tensors()
    want = torch.autograd.grad(rotary_embedding(q, k, rotary, pos), (q, k), (gq, gk))
    seen = [0, 0]

    def pack(x):
        seen[0] += 1
        return x.cpu()

    def unpack(x):
        seen[1] += 1
        return x.cuda()

    with torch.autograd.graph.saved_tensors_hooks(pack, unpack):
        ys = rotary_embedding(q, k, rotary, pos)
    got = torch.autograd.grad(ys, (q, k), (gq, gk))
    assert seen == [2, 2] and all(torch.equal(a, b) for a, b in zip(got, want))
    for reentrant in (False, True):
        ys = checkpoint(lambda a, b: rotary_embedding(a, b, rotary, pos), q, k, use_reentrant=reentrant)
        for t in (q, k):
            t.grad = None
        torch.autograd.backward(ys, (gq, gk))
        assert torch.equal(q.grad, want[0]) and torch.equal(k.grad, want[1])


@pytest.mark.parametrize("change", [lambda x: x.cpu(), lambda x: x.float(), lambda x: x[:3]])
def test_saved_tensors_that_come_back_changed(change):
    q, k, gq, gk, rotary, pos = _tensors()
    with torch.autograd.graph.saved_tensors_hooks(lambda x: x, change):
        ys = rotary_embedding(q, k, rotary, pos)
    with pytest.raises(ValueError, match="saved frequencies or positions"):
        torch.autograd.grad(ys, (q, k), (gq, gk))


@pytest.mark.parametrize("python_node", [False, True])
def test_saved_frequencies_that_come_back_in_another_number(python_node, monkeypatch):
    """(fewer or more columns would turn than did)"""
    from paper_2205_14135_amd import autograd
    if python_node:
        monkeypatch.setattr(autograd, "_node_in_python", lambda: True)
    q, k, gq, gk, _, _ = _tensors()
    for change in (lambda x: x[:3], lambda x: torch.cat([x, x])):
        with torch.autograd.graph.saved_tensors_hooks(lambda x: x, change):
            ys = rotary_embedding(q, k, Rotary.make(32))
        with pytest.raises(ValueError, match="saved frequencies or positions"):
            torch.autograd.grad(ys, (q, k), (gq, gk))


def test_transforms_keep_the_python_node():
    q, k, gq, _, rotary, pos = _tensors(False)
    with pytest.raises(RuntimeError, match="setup_context"):
        torch.func.grad(lambda x: rotary_embedding(x, k, rotary, pos)[0].float().sum())(q)
    with forward_ad.dual_level():
        with pytest.raises(NotImplementedError):
            rotary_embedding(forward_ad.make_dual(q, gq), k, rotary, pos)
    traced = torch.jit.trace(lambda x: flash_attention(x, x, x, causal=True, rotary=rotary, positions=pos), (q,), check_trace=False)
    other = q.flip(2).contiguous()
    assert torch.equal(traced(other), flash_attention(other, other, other, causal=True, rotary=rotary, positions=pos))
