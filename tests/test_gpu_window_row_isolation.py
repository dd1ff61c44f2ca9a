"""Attention with a sliding window: a query row whose logits are not finite leaves every other row alone, and a key that is no number those rows that do not see it; each row of O and L, and of dQ,
depends on its own query only.  Dense, and over a paged cache."""
import math

import pytest
import torch

from oracle import attention_oracle as orc
from paper_2205_14135_amd import binding
from tests import paged_helpers as ph
from tests import window_helpers as wh
from tests.test_gpu_paged_window import attention

pytestmark = pytest.mark.gpu

N = 320
BAD_ROWS = [5, 48, 176, 319]
# "huge" is finite (2^127): only its products overflow float32, with both signs
VALUES = {"nan": math.nan, "inf": math.inf, "huge": 2.0 ** 127}
DTYPES = {"fp16": torch.float16, "bf16": torch.bfloat16}
# few blocks (divided among groups of wavefronts), and so many that they are not, at the head dimension
HEADS = {16: (2, 210), 32: (2, 210), 64: (2, 110), 128: (2, 60)}


def _inputs(d, dtype, many, seed=1):
    H = HEADS[d][many]
    gen = torch.Generator(device="cuda").manual_seed(seed + d)
    return [torch.randn(1, H, N, d, generator=gen, device="cuda").to(DTYPES[dtype]) for _ in range(4)], (0, H - 1)


def _head(ts, h, window, sinks, length=None, p=0.0, seed=0, offset=0):
    keep, factor, H, d = None, 1.0, ts[0].shape[1], ts[0].shape[-1]
    if p > 0:
        keep = torch.from_numpy(orc.dropout_keep_mask(0, h, H, N, p, seed, offset).astype("float64")).cuda()
        factor = 256.0 / (256.0 - math.floor(p * 256))
    return wh.Head(*(t[0, h] for t in ts), 1 / math.sqrt(d), window, sinks, length, keep, factor)


@pytest.mark.parametrize("many", [False, True])
@pytest.mark.parametrize("d,dtype,kind", [(16, "fp16", "nan"), (32, "bf16", "huge"), (64, "bf16", "huge"), (64, "fp16", "nan"), (128, "bf16", "huge"), (128, "bf16", "inf")])
@pytest.mark.parametrize("window,sinks,p", [(70, 0, 0.0), (70, 4, 0.0), (17, 40, 0.0), (70, 4, 0.1)])
def test_one_row_does_not_touch_the_others(d, dtype, kind, window, sinks, p, many):
    clean, heads = _inputs(d, dtype, many)
    q, k, v, do = clean
    q = q.clone()
    q[:, :, BAD_ROWS] = VALUES[kind]
    good = [i for i in range(N) if i not in BAD_ROWS]
    kw = dict(window=window, sinks=sinks, softmax_scale=1 / math.sqrt(d), dropout_p=p, seed=77, offset=2)
    O, L = binding.attn_window_fwd(q, k, v, **kw)
    dQ = binding.attn_window_bwd(q, k, v, O, do, L, **kw)[0]
    assert torch.isnan(O[:, :, BAD_ROWS]).all()
    for h in heads:
        x = _head(clean, h, window, sinks, p=p, seed=77, offset=2)
        wh.assert_within(O[0, h][good], x.O[good], x.bO[good], "O")
        wh.assert_within(L[0, h][good], x.L[good], x.bL[good], "L")
        wh.assert_within(dQ[0, h][good], x.dQ[good], x.bQ[good], "dQ")


@pytest.mark.parametrize("many", [False, True])
@pytest.mark.parametrize("d", [32, 64, 128])
@pytest.mark.parametrize("window,sinks,key", [(70, 0, 100), (70, 4, 100), (1, 40, 33), (64, 4, 2)])
def test_rows_that_do_not_see_a_key_that_is_not_a_number(d, window, sinks, key, many):
    clean, heads = _inputs(d, "bf16", many)
    q, k, v, do = clean
    k = k.clone()
    k[:, :, key] = math.nan
    O, L = binding.attn_window_fwd(q, k, v, window=window, sinks=sinks, softmax_scale=1 / math.sqrt(d))
    sees = wh.visible(N, window, sinks)[:, key]
    assert torch.isnan(O[:, :, sees]).all()
    for h in heads:
        x = _head(clean, h, window, sinks)
        wh.assert_within(O[0, h][~sees], x.O[~sees], x.bO[~sees], "O")
        wh.assert_within(L[0, h][~sees], x.L[~sees], x.bL[~sees], "L")


@pytest.mark.parametrize("many", [False, True])
@pytest.mark.parametrize("d", [32, 64, 128])
@pytest.mark.parametrize("kind", ["nan", "huge"])
def test_padded_queries_do_not_touch_the_valid_rows(d, kind, many):
    length = 200
    clean, heads = _inputs(d, "bf16", many)
    q, k, v, do = clean
    q = q.clone()
    q[:, :, length:] = VALUES[kind]
    O, L = binding.attn_window_fwd(q, k, v, window=70, sinks=4, softmax_scale=1 / math.sqrt(d), key_lengths=torch.tensor([length], dtype=torch.int32, device="cuda"))
    assert (O[:, :, length:] == 0).all() and (L[:, :, length:] == -math.inf).all()
    for h in heads:
        x = _head(clean, h, 70, 4, length)
        wh.assert_within(O[0, h][:length], x.O[:length], x.bO[:length], "O")
        wh.assert_within(L[0, h][:length], x.L[:length], x.bL[:length], "L")


# single tokens by a workgroup each and divided; chunks at d = 64 and 128; chunks and few rows apart
PAGED = {"short window": (dict(new=[1, 1, 1], single=True), 64, 40), "divided": (dict(new=[1, 1, 1], single=True), 64, 3000), "divided, wide": (dict(new=[1, 1, 1], single=True), 128, 3000),
         "chunks": (dict(new=[40, 1, 200]), 64, 70), "chunks, wide": (dict(new=[40, 1, 300]), 128, 70), "apart": (dict(new=[40, 1, 300, 16, 9]), 128, 3000)}


@pytest.mark.parametrize("kind", ["nan", "inf", "huge"])
@pytest.mark.parametrize("form", PAGED)
def test_over_a_paged_cache(form, kind):
    how, d, window = PAGED[form]
    new, single = how["new"], how.get("single", False)
    heads = (32, 16) if form == "apart" else (8, 2)
    batch = ph.Batch([3500, 20, 1200, 700, 60][:len(new)], new, *heads, d, "bf16", 16, seed=d)
    if form == "apart":
        wide = torch.full((batch.B, 400), -1, dtype=torch.int32)
        wide[:, :batch.table.shape[1]] = batch.table
        batch.table = wide
        assert 16 * (batch.B - 1) * min(6400, window + 4) >= 3000 * 64       # (the rule's bound)
    want, want_l, bound, bound_l = attention(batch, window, 4)
    q, kc, vc, table, lengths, starts = batch.gpu(single)
    bad = torch.zeros(batch.tokens, heads[0], dtype=torch.bool)
    bad[0, 1] = bad[batch.tokens // 2] = bad[-1, ::3] = True
    q[bad.cuda()] = VALUES[kind]
    O, L = binding.attn_paged_fwd(q, kc, vc, table, lengths, starts, softmax_scale=batch.tau, window=window, sinks=4)
    assert torch.isnan(O[bad.cuda()]).all()
    ph.assert_within(O[~bad.cuda()], want[~bad], bound[~bad], "O")
    ph.assert_within(L[~bad.cuda().t()], want_l[~bad.t()], bound_l[~bad.t()], "LSE")
