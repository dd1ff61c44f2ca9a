"""Columns that do not turn, and K without a rotation, arrive bit by bit: infinities, NaN of any kind, zeros with a sign, the smallest and the largest numbers, and none of
them reaches a column that turns."""
import pytest
import torch

from paper_2205_14135_amd import binding
from paper_2205_14135_amd.autograd import rotary_embedding
from paper_2205_14135_amd.rotary import Rotary, rotary_frequencies
from tests import paged_helpers as ph

pytestmark = pytest.mark.gpu

# +-infinity, a quiet and a signalling NaN, -0, the smallest subnormal, the largest number
SPECIAL = {"bf16": [0x7f80, -0x80, 0x7fc1, 0x7f81, -0x8000, 0x0001, 0x7f7f], "fp16": [0x7c00, -0x400, 0x7e01, 0x7c01, -0x8000, 0x0001, 0x7bff]}

# pairs (i, i + r / 2) by eights, pairs (i, i + r / 2) of any r, neighbours
FORMS = [(32, 16, False), (64, 16, False), (64, 48, False), (128, 64, False), (16, 6, False), (32, 8, False), (64, 20, False), (128, 2, False), (128, 126, False),
         (16, 4, True), (32, 16, True), (64, 2, True), (64, 20, True), (128, 64, True), (128, 126, True)]


def bits(x):
    return x.detach().cpu().contiguous().view(torch.int16)


def specials(shape, dtype, seed):
    gen = torch.Generator().manual_seed(seed)
    values = torch.tensor(SPECIAL[dtype], dtype=torch.int16)
    return values[torch.randint(0, len(values), shape, generator=gen)].view(ph.DTYPES[dtype])


def rows(shape, r, dtype, seed):
    """Normal numbers in the columns that turn, special ones behind them."""
    x = torch.randn(shape, generator=torch.Generator().manual_seed(seed)).to(ph.DTYPES[dtype])
    x[..., r:] = specials(x[..., r:].shape, dtype, seed + 1)
    return x


def check(got, x, positions, r, f, interleaved, magnitude, inverse=False):
    """x: [tokens, heads, d], one position a token."""
    assert torch.equal(bits(got)[..., r:], bits(x)[..., r:])
    clean = x.clone()
    clean[..., r:] = 0.0
    want, bound = ph.turned(clean, positions, f, interleaved, magnitude, inverse)
    ph.assert_within(got[..., :r], want[..., :r], (bound + ph.rounding(want, x.dtype))[..., :r], "columns that turn")


@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
@pytest.mark.parametrize("d,r,interleaved", FORMS)
def test_rotation(dtype, d, r, interleaved):
    f, _ = rotary_frequencies(r)
    rotary = Rotary(f.cuda(), interleaved=interleaved, magnitude=1.25)
    x = rows((21, 5, d), r, dtype, d + r)
    q = x.transpose(0, 1).unsqueeze(0).cuda()
    for inverse in (False, True):
        got, _ = binding.attn_rotary(q, None, rotary, inverse=inverse)
        check(got[0].transpose(0, 1), x, torch.arange(21), r, f, interleaved, 1.25, inverse)
    k = q.clone()
    binding.attn_rotary(k, None, rotary, out=(k, None))
    check(k[0].transpose(0, 1), x, torch.arange(21), r, f, interleaved, 1.25)


@pytest.mark.parametrize("d,r,interleaved", [(64, 16, False), (64, 20, False), (64, 20, True)])
def test_gradients(d, r, interleaved):
    f, _ = rotary_frequencies(r)
    rotary = Rotary(f.cuda(), interleaved=interleaved)
    q, k = (torch.randn(1, 3, 21, d, device="cuda").to(torch.bfloat16).requires_grad_(True) for _ in range(2))
    g = [rows((21, 3, d), r, "bf16", 7 + i) for i in range(2)]
    got = torch.autograd.grad(rotary_embedding(q, k, rotary), (q, k), [x.transpose(0, 1).unsqueeze(0).cuda() for x in g])
    for x, y in zip(g, got):
        check(y[0].transpose(0, 1), x, torch.arange(21), r, f, interleaved, 1.0, inverse=True)


def append(dtype, d, r, interleaved, page=16):
    """(rows of K and V as given, positions, Q, and what stands in the cache and in Q' afterwards) of one sequence of 40 tokens, 25 of them new."""
    f = rotary_frequencies(r)[0] if r else None
    q, k = rows((25, 4, d), r, dtype, 1), rows((25, 2, d), r, dtype, 3)
    v = specials((25, 2, d), dtype, 5)
    kc, vc = (torch.zeros(3, 2, page, d, dtype=ph.DTYPES[dtype], device="cuda") for _ in range(2))
    ints = lambda *x: torch.tensor(x, dtype=torch.int32, device="cuda")
    rotary = Rotary(f.cuda(), interleaved=interleaved) if r else None
    turned = binding.attn_paged_append(k.cuda(), v.cuda(), kc, vc, ints(2, 0, 1).view(1, 3), ints(40), ints(0, 25), Q=q.cuda() if r else None, rotary=rotary)
    held = lambda c: c[torch.tensor([2, 0, 1])].transpose(1, 2).reshape(48, 2, d)[15:40]
    return q, k, v, f, turned, held(kc), held(vc)


@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
@pytest.mark.parametrize("d", [16, 32, 64, 128])
def test_append_without_a_rotation(dtype, d):
    _, k, v, _, _, kc, vc = append(dtype, d, 0, False)
    assert torch.equal(bits(kc), bits(k)) and torch.equal(bits(vc), bits(v))


@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
@pytest.mark.parametrize("d,r,interleaved", FORMS)
def test_append_of_rows_that_turn_in_part(dtype, d, r, interleaved):
    q, k, v, f, turned, kc, vc = append(dtype, d, r, interleaved)
    assert torch.equal(bits(vc), bits(v))
    check(turned, q, torch.arange(15, 40), r, f, interleaved, 1.0)
    check(kc, k, torch.arange(15, 40), r, f, interleaved, 1.0)
