"""Infinities, NaN, zeros with a sign and numbers whose squares leave 32 bits in the rows, the weights and the gradients of the norm: columns that do not turn take nothing from the column beside them."""
import math

import pytest
import torch

from paper_2205_14135_amd import binding
from paper_2205_14135_amd.rotary import HeadNorm, Rotary, rotary_frequencies
from tests import norm_helpers as nh
from tests import paged_helpers as ph

pytestmark = pytest.mark.gpu

EPS = float(torch.tensor(1e-5, dtype=torch.float32))
# pairs (i, i + r / 2) by eights, pairs (i, i + r / 2) of any r, neighbours; no rotation
FORMS = [(32, 16, False), (64, 48, False), (128, 64, False), (16, 6, False), (64, 20, False), (128, 126, False), (16, 4, True), (64, 20, True), (128, 64, True), (64, 0, False)]
N, H = 37, 3
BAD = [0, 5, 20, 36]     # tokens


def _case(d, r, interleaved, dtype):
    """x, dy [N, H, d] and positive weights on the CPU, the rotation and its frequencies."""
    gen = torch.Generator().manual_seed(d + r)
    x, dy = (torch.randn(N, H, d, generator=gen).to(ph.DTYPES[dtype]) for _ in range(2))
    x[x == 0] = 1.0
    w = 0.5 + torch.rand(d, generator=gen)
    f = rotary_frequencies(r)[0] if r else None
    return x, dy, w, f, None if f is None else Rotary(f.cuda(), interleaved=interleaved)


def _gpu(x):
    return x.transpose(0, 1).unsqueeze(0).cuda()


def _cpu(y):
    return y[0].transpose(0, 1).cpu()


def _forward(x, w, rotary):
    return _cpu(binding.attn_norm_rotary(_gpu(x), None, HeadNorm(w.cuda(), eps=EPS), rotary)[0])


def _backward(x, dy, w, rotary):
    dx, _, dw, _ = binding.attn_norm_rotary_bwd(_gpu(x), None, _gpu(dy), None, HeadNorm(w.cuda(), eps=EPS), rotary)
    return _cpu(dx), dw.cpu()


def _same(got, want, what):
    """Equal numbers, NaN where NaN is."""
    assert torch.equal(torch.isnan(got), torch.isnan(want)), what
    assert torch.equal(torch.nan_to_num(got.double(), 0.5), torch.nan_to_num(want.double(), 0.5)), what


def _good():
    return [n for n in range(N) if n not in BAD]


@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
@pytest.mark.parametrize("d,r,interleaved", FORMS)
@pytest.mark.parametrize("value", [math.inf, -math.inf, math.nan])
def test_rows(dtype, d, r, interleaved, value):
    """An infinity makes the root mean square one: its own column is no number, the others are zeros.  What turns with it is no number either, what does not is a zero."""
    x, _, w, f, rotary = _case(d, r, interleaved, dtype)
    columns = sorted({0, r // 2, max(r - 1, 0), r, d - 2, d - 1} & set(range(d)))
    for c in columns:
        y = x.clone()
        y[BAD, 1, c] = value
        want, bound = nh.forward(y, w, EPS, torch.arange(N), f, interleaved)
        got = _forward(y, w, rotary)
        ph.assert_within(got[_good()], want[_good()], bound[_good()], "other rows")
        ph.assert_within(got[:, [0, 2]], want[:, [0, 2]], bound[:, [0, 2]], "other heads")
        _same(got[BAD, 1], want[BAD, 1], f"column {c}")


@pytest.mark.parametrize("d,r,interleaved", FORMS)
@pytest.mark.parametrize("value", [math.inf, math.nan])
def test_weights(d, r, interleaved, value):
    x, _, w, f, rotary = _case(d, r, interleaved, "bf16")
    want, bound = nh.forward(x, w, EPS, torch.arange(N), f, interleaved)
    for c in sorted({r, r + 1, d - 2, d - 1}):
        if not r <= c < d:
            continue
        odd = w.clone()
        odd[c] = value
        got = _forward(x, odd, rotary)
        _same(got[..., c], x[..., c].float().sign() * value, f"column {c}")
        rest = [i for i in range(d) if i != c]
        ph.assert_within(got[..., rest], want[..., rest], bound[..., rest], f"beside column {c}")


@pytest.mark.parametrize("d,r,interleaved", FORMS)
def test_zeros_keep_their_sign(d, r, interleaved):
    x, _, w, f, rotary = _case(d, r, interleaved, "bf16")
    zeros = torch.rand(x.shape, generator=torch.Generator().manual_seed(1)) < 0.5
    x[..., r:] = torch.where(zeros, x * 0.0, x)[..., r:]
    got = _forward(x, w, rotary)
    assert torch.equal(torch.signbit(got[..., r:]), torch.signbit(x[..., r:]))


@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
@pytest.mark.parametrize("d,r,interleaved", FORMS)
def test_gradients(dtype, d, r, interleaved):
    """An infinite gradient of one element: of its row nothing is finite (the mean goes through all of it), and of the weights' gradient one column."""
    x, dy, w, f, rotary = _case(d, r, interleaved, dtype)
    for c in sorted({r, r + 1, d - 2, d - 1}):
        if not r <= c < d:
            continue
        g = dy.clone()
        g[BAD[1], 1, c] = math.inf
        want, bound, want_w, bound_w = nh.gradients(x, w, g, EPS, torch.arange(N), f, interleaved)
        got, got_w = _backward(x, g, w, rotary)
        rest = [n for n in range(N) if n != BAD[1]]
        ph.assert_within(got[rest], want[rest], bound[rest], "other rows")
        _same(got[BAD[1], 1], want[BAD[1], 1], f"column {c}")
        assert got_w[c] == x[BAD[1], 1, c].float().sign() * math.inf
        rest = [i for i in range(d) if i != c]
        ph.assert_within(got_w[rest], want_w[rest], bound_w[rest], "weights")


@pytest.mark.parametrize("d,r,interleaved", FORMS)
def test_append(d, r, interleaved):
    """Rows of K with an infinity behind the columns that turn, on their way into the cache."""
    x, _, w, f, rotary = _case(d, r, interleaved, "bf16")
    if r == d:
        return
    x[BAD, 1, d - 1] = math.inf
    kc, vc = (torch.zeros(3, H, 16, d, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    ints = lambda *a: torch.tensor(a, dtype=torch.int32, device="cuda")  # noqa: E731
    out = binding.attn_paged_append(x.cuda(), x.cuda(), kc, vc, ints(2, 0, 1).view(1, 3), ints(N), ints(0, N), Q=x.cuda(), rotary=rotary, norm=HeadNorm(w.cuda(), w.cuda(), eps=EPS))
    want = _forward(x, w, rotary)
    _same(out.cpu(), want, "Q")
    _same(kc[torch.tensor([2, 0, 1])].transpose(1, 2).reshape(48, H, d)[:N].cpu(), want, "K")
    exact, _ = nh.forward(x, w, EPS, torch.arange(N), f, interleaved)
    _same(want[BAD, 1], exact[BAD, 1], "the rows with an infinity")


@pytest.mark.parametrize("d,r,interleaved", FORMS)
@pytest.mark.parametrize("exponent,columns", [(66, None), (126, None), (64, 1), (127, 1)])
def test_squares_beyond_32_bits(d, r, interleaved, exponent, columns):
    """Finite rows whose squares add up beyond float32 come out as zeros and have no gradient: not in their own elements, and not in that of the weights."""
    x, dy, w, f, rotary = _case(d, r, interleaved, "bf16")
    dy = dy * 16.0
    large, none = x.clone(), x.clone()
    large[BAD, 1, :columns] = torch.where(x[BAD, 1, :columns] < 0, -(2.0 ** exponent), 2.0 ** exponent).to(x.dtype)
    none[BAD, 1] = 0.0
    got, want = _forward(large, w, rotary), _forward(none, w, rotary)
    assert (got[BAD, 1] == 0).all() and torch.equal(got, want)
    (dx, dw), (want, want_w) = _backward(large, dy, w, rotary), _backward(none, dy, w, rotary)
    assert (dx[BAD, 1] == 0).all() and torch.equal(dw, want_w)
    want[BAD, 1] = 0.0
    assert torch.equal(dx, want)


@pytest.mark.parametrize("d,r,interleaved", FORMS)
@pytest.mark.parametrize("value", [math.inf, math.nan])
def test_rows_that_are_no_numbers_have_no_gradients_either(d, r, interleaved, value):
    """(by the formula: 0 times an infinity is in every element of such a row, and in every column of the weights' gradient that it has a part in)"""
    x, dy, w, f, rotary = _case(d, r, interleaved, "bf16")
    x[BAD[1], 1, d // 2] = value
    want, bound, want_w, bound_w = nh.gradients(x, w, dy, EPS, torch.arange(N), f, interleaved)
    got, got_w = _backward(x, dy, w, rotary)
    rest = [n for n in range(N) if n != BAD[1]]
    ph.assert_within(got[rest], want[rest], bound[rest], "other rows")
    assert torch.isnan(want[BAD[1], 1]).all() and torch.isnan(got[BAD[1], 1]).all()
    numbers = ~torch.isnan(want_w)
    assert torch.equal(~torch.isnan(got_w), numbers)
    ph.assert_within(got_w[numbers], want_w[numbers], bound_w[numbers], "weights")
