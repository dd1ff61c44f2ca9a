"""Attention with a sliding window over padded batches: what stands at padded positions reaches nothing, whatever its products would be."""
import math

import pytest
import torch

from paper_2205_14135_amd import binding

pytestmark = pytest.mark.gpu

N = 320
LENGTHS = [200, 320, 1, 0, 128, 257]
# "huge" is finite (2^127): its products overflow float32, with both signs
VALUES = {"huge": 2.0 ** 127, "nan": math.nan, "inf": math.inf}


def _run(ts, lengths, **kw):
    O, L = binding.attn_window_fwd(*ts[:3], key_lengths=lengths, softmax_scale=0.125, **kw)
    return [O, L, *binding.attn_window_bwd(*ts[:3], O, ts[3], L, key_lengths=lengths, softmax_scale=0.125, **kw)]


# few blocks of rows (divided among groups of wavefronts), and so many that they are not
@pytest.mark.parametrize("H", [2, 36])
@pytest.mark.parametrize("d", [16, 32, 64, 128])
@pytest.mark.parametrize("kind", VALUES)
@pytest.mark.parametrize("kw", [dict(window=70, sinks=0), dict(window=70, sinks=4), dict(window=17, sinks=140), dict(window=130, sinks=2, dropout_p=0.2, seed=5)])
def test_what_stands_at_padded_positions_does_not_count(H, d, kind, kw):
    gen = torch.Generator(device="cuda").manual_seed(d)
    ts = [torch.randn(len(LENGTHS), H, N, d, generator=gen, device="cuda").to(torch.bfloat16) for _ in range(4)]
    lengths = torch.tensor(LENGTHS, dtype=torch.int32, device="cuda")
    want = _run(ts, lengths, **kw)
    padded = torch.arange(N, device="cuda").view(1, 1, N) >= lengths.view(-1, 1, 1)
    got = _run([t.masked_fill(padded.unsqueeze(-1), VALUES[kind]) for t in ts], lengths, **kw)
    for x, y, name in zip(got, want, ("O", "L", "dQ", "dK", "dV")):
        assert torch.equal(x, y), name
        rows = x.masked_select(padded.expand(x.shape[:3]) if x.dim() == 3 else padded.unsqueeze(-1).expand(x.shape))
        assert (rows == (-math.inf if name == "L" else 0.0)).all(), name
