"""A captured forward pass whose gradient graph leads, through other operations, to a leaf that an eager graph of the default stream still leads to."""
import pytest
import torch

from paper_2205_14135_amd.autograd import flash_attention, rotary_embedding
from paper_2205_14135_amd.rotary import Rotary

pytestmark = pytest.mark.gpu


def _capture(run):
    """`run` in a captured graph that holds another step too."""
    here = torch.zeros(1, device="cuda")
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        here.add_(1)
        run()
    graph.replay()
    torch.cuda.synchronize()
    assert here.item() == 1.0


@pytest.mark.parametrize("call", ["rotary_q", "rotary_k", "attention_v"])
def test_leaves_behind_other_operations(call):
    """x w with a weight w whose gradient sum an eager graph holds: refused, in the forward pass; not refused without that graph, or without gradients."""
    rotary = Rotary.make(64)
    gen = torch.Generator(device="cuda").manual_seed(1)
    x = [torch.randn(1, 2, 40, 64, generator=gen, device="cuda").to(torch.bfloat16) for _ in range(3)]
    w = torch.randn(64, generator=gen, device="cuda").to(torch.bfloat16).requires_grad_(True)
    at = {"rotary_q": 0, "rotary_k": 1, "attention_v": 2}[call]

    def run():
        q, k, v = ((t * w) * 0.5 if i == at else t for i, t in enumerate(x))
        return flash_attention(q, k, v, rotary=rotary) if call == "attention_v" else rotary_embedding(q, k, rotary)

    def run_and_drop():
        run()

    def refused():
        with pytest.raises(RuntimeError, match="still leads to the same leaf"):
            run()

    run()
    _capture(run_and_drop)      # (the eager graph above is gone)
    held = run()
    _capture(refused)
    with torch.no_grad():
        _capture(run_and_drop)
    del held
    _capture(run_and_drop)


def test_an_eager_graph_made_on_another_stream_is_not_refused():
    rotary = Rotary.make(64)
    w = torch.randn(64, device="cuda").to(torch.bfloat16).requires_grad_(True)
    x = torch.randn(1, 2, 40, 64, device="cuda").to(torch.bfloat16)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        held = rotary_embedding(x * w, x, rotary)
    torch.cuda.current_stream().wait_stream(side)
    _capture(lambda: rotary_embedding(x * w, x, rotary)[0].detach())
    assert held[0].grad_fn is not None
