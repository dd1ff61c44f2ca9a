"""The operators around attention that a program with a paged key/value cache and rotary positions calls, as they are measured.

Four operators, through the framework's public entry points (`own`), or in elementary torch operations:

  rotary  rotation of Q and K by their tokens' positions, forward and backward (`autograd.rotary_embedding`): pairs of columns,
          (2 i, 2 i + 1) or (i, i + r / 2) of the first r, turn by position * frequency_i
  append  the new tokens of every sequence: Q rotated, K rotated and written into the pages of a cache with V (`attn_paged_append`)
  attend  softmax(tau Q K^T) V of the new tokens of every sequence over what its pages hold (`attn_paged_fwd`)
  copy    pages of a cache of several layers copied to other pages: a fork, or a compaction (`attn_paged_copy`)

A case is a dict of plain values; sizes of a ragged batch follow from its "shape" number alone.

  kind          "rotary", "append", "attend" or "copy"
  Hq, Hk, d     heads of Q, heads of K and V, head dimension;  dtype "bf16" | "fp16"
  rotary        B, N, layout "head" ([B,H,N,d] memory) | "token" (a view of [B,N,H,d]), r (columns that turn), interleaved, scaling
                (None: angles position * base^(-2 i / r); a factor: long contexts, slow pairs slowed by it and fast ones left)
  append/attend B sequences, page (tokens a page), before (lo, hi) tokens that a sequence holds already, new "single" (one token a
                sequence), "chunk" (lo, hi tokens) or "mixed" (one chunk of `hi` tokens among single ones), pad rows behind the last token
  copy          pages (of a cache), pairs (copied), layers
"""
from __future__ import annotations

import math
import random

import numpy as np
import torch

own = False

DTYPES = {"fp16": torch.float16, "bf16": torch.bfloat16}
BASE = 10000.0
ORIGINAL = 4096      # tokens that a scaled model was trained for


def _rotary(name, B, N, Hq, Hk, d, dtype, layout, r, interleaved, scaling=0.0, train=True):
    c = dict(kind="rotary", B=B, N=N, Hq=Hq, Hk=Hk, d=d, dtype=dtype, layout=layout, r=r, interleaved=interleaved, scaling=scaling, train=train)
    return dict(c, name=name) if name else c


def _batch_case(name, kind, B, Hq, Hk, d, dtype, page, before, new, q=(1, 1), pad=0, shape=1, r=0, interleaved=False, scaling=0.0, causal=True):
    c = dict(kind=kind, B=B, Hq=Hq, Hk=Hk, d=d, dtype=dtype, page=page, before_lo=before[0], before_hi=before[1], new=new, q_lo=q[0], q_hi=q[1],
             pad=pad, shape=shape, r=r, interleaved=interleaved, scaling=scaling, causal=causal)
    return dict(c, name=name) if name else c


def _copy(name, layers, pages, pairs, page, Hk, d, dtype):
    c = dict(kind="copy", layers=layers, pages=pages, pairs=pairs, page=page, Hk=Hk, d=d, dtype=dtype)
    return dict(c, name=name) if name else c


def listed():
    return [
        # one sentence through one layer, forward alone: the launch and the host path are all there is
        _rotary("rotary_sentence_fwd", 1, 197, 12, 12, 64, "fp16", "token", 64, False, train=False),
        # the layer of a GPT-2-medium training step, heads interleaved in memory as a projection leaves them
        _rotary("rotary_gpt2_train", 8, 1024, 16, 16, 64, "bf16", "token", 64, False),
        # the long end: half of a wide head turns, neighbouring columns, frequencies scaled for four times the trained length, shared K heads
        _rotary("rotary_long_train", 1, 16384, 16, 4, 128, "fp16", "head", 64, True, 4.0),
        # one step of 64 running sequences
        _batch_case("append_step", "append", 64, 32, 8, 128, "bf16", 16, (100, 1000), "single", r=128),
        # prompts of different lengths read in together, padded behind the last
        _batch_case("append_prompts", "append", 12, 16, 16, 64, "fp16", 64, (0, 300), "chunk", (50, 2048), pad=37, r=32, interleaved=True),
        # the smallest answer: one sequence, one token, two groups of heads
        _batch_case("attend_one_token", "attend", 1, 16, 2, 64, "bf16", 16, (776, 776), "single"),
        # one step of 64 running sequences of very different lengths, four Q heads to a K head
        _batch_case("attend_step", "attend", 64, 32, 8, 128, "bf16", 16, (128, 8192), "single"),
        # two long documents, one token each
        _batch_case("attend_long_documents", "attend", 2, 32, 8, 128, "bf16", 64, (65536, 131071), "single"),
        # a chunk of a long prompt, on top of what was read in before
        _batch_case("attend_chunk", "attend", 1, 32, 8, 128, "bf16", 16, (14336, 14336), "chunk", (2048, 2048)),
        # a chunk of a prompt that shares its call with running sequences, padded
        _batch_case("attend_mixed", "attend", 33, 16, 4, 64, "fp16", 32, (30, 4000), "mixed", (1000, 1000), pad=23),
        # sixteen sequences forked: their last pages, in one layer
        _copy("copy_fork", 1, 256, 16, 16, 8, 128, "bf16"),
        # a cache of 24 layers compacted
        _copy("copy_compact", 24, 1024, 400, 64, 4, 64, "fp16"),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


MAX_FLOPS = 5.1e11          # just below attend_chunk
MAX_BYTES = 0.75e9          # just below attend_long_documents


def draw(rng):
    """One more case: the kinds of the list, sizes over the logarithm of their range, odd ones among them."""
    while True:
        kind = rng.choice(["rotary", "append", "attend", "attend", "attend", "copy"])
        dtype = rng.choice(["fp16", "bf16", "bf16"])
        d = rng.choice([32, 64, 64, 128, 128])
        Hk = rng.choice([1, 2, 4, 8, 16])
        Hq = Hk * rng.choice([1, 2, 4, 8] if Hk <= 4 else [1, 2, 4])
        if kind == "rotary":
            N = _log_int(rng, 100, 16384)
            c = _rotary(None, max(1, _log_int(rng, N, 32768) // N), N, Hq, Hk, d, dtype, rng.choice(["head", "token"]),
                        rng.choice([d, d, d // 2, d // 4]), rng.random() < 0.4, rng.choice([0.0, 0.0, 4.0, 8.0]), rng.random() < 0.7)
        elif kind == "copy":
            pages, page = _log_int(rng, 64, 2000), rng.choice([16, 32, 64, 128])
            c = _copy(None, rng.choice([1, 1, 12, 24]), pages, _log_int(rng, 1, pages // 3), page, Hk, d, dtype)
        else:
            new = rng.choice(["single", "single", "chunk", "mixed"])
            B = _log_int(rng, 1, 128) if new == "single" else _log_int(rng, 1, 40)
            q_hi = _log_int(rng, 2, 3000) if new != "single" else 1
            hi = _log_int(rng, 16, 65536 if kind == "attend" else 2000)
            c = _batch_case(None, kind, B, Hq, Hk, d, dtype, rng.choice([16, 16, 32, 64, 128, 256]), (_log_int(rng, 1, hi), hi), new,
                            (max(1, q_hi // 8), q_hi), rng.choice([0, 0, 5, 41]), rng.randrange(1 << 30),
                            rng.choice([d, d // 2]) if kind == "append" else 0, kind == "append" and rng.random() < 0.4,
                            rng.choice([0.0, 4.0]) if kind == "append" else 0.0, rng.random() < 0.85 if kind == "attend" else True)
        w = work(c)
        if w["flops"] <= MAX_FLOPS and w["bytes"] <= MAX_BYTES and _cache_bytes(c) <= 3e9:
            return c


def _sizes(case):
    """(tokens held before, new tokens) of every sequence."""
    rng = random.Random(case["shape"])
    before = [_log_int(rng, case["before_lo"] + 1, case["before_hi"] + 1) - 1 for _ in range(case["B"])]
    new = [1] * case["B"]
    if case["new"] == "chunk":
        new = [_log_int(rng, case["q_lo"], case["q_hi"]) for _ in new]
    elif case["new"] == "mixed":
        new[rng.randrange(case["B"])] = case["q_hi"]
    return before, new


def _pages_of(case):
    """Pages that each sequence holds once the new tokens are in."""
    before, new = _sizes(case)
    return [-(-(b + n) // case["page"]) for b, n in zip(before, new)]


def _cache_bytes(case):
    if case["kind"] == "rotary":
        return 0
    pages = case["layers"] * case["pages"] if case["kind"] == "copy" else sum(_pages_of(case))
    return 4 * pages * case["page"] * case["Hk"] * case["d"]


def _normal(gen, shape, case):
    return torch.randn(shape, generator=gen, device="cuda", dtype=torch.float32).to(DTYPES[case["dtype"]])


def _frequencies(case):
    """Radians a position of each pair, and the factor of the rotated values.  A scaled model keeps the pairs that turn 32 times and more within
    the trained length, slows those that turn at most once by the factor, and goes over between them along the number of turns."""
    half = case["r"] // 2
    f = BASE ** (-np.arange(half, dtype=np.float64) / half)
    s = case["scaling"]
    if not s:
        return f, 1.0
    keep = np.clip((f * ORIGINAL / (2 * math.pi) - 1.0) / 31.0, 0.0, 1.0)
    return f * (keep + (1.0 - keep) / s), 0.1 * math.log(s) + 1.0


def _copy_pairs(case, seed):
    rng = random.Random(seed * 7919 + case["pairs"])
    ids = rng.sample(range(case["pages"]), 2 * case["pairs"])
    return torch.tensor([ids[:case["pairs"]], ids[case["pairs"]:]], dtype=torch.int32).t().contiguous()


def _inputs(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    kind, d = case["kind"], case["d"]
    if kind == "rotary":
        B, N = case["B"], case["N"]
        ts = {}
        for name, H in (("q", case["Hq"]), ("k", case["Hk"]), ("dq", case["Hq"]), ("dk", case["Hk"])):
            token = case["layout"] == "token"
            x = _normal(gen, (B, N, H, d) if token else (B, H, N, d), case)
            ts[name] = x.transpose(1, 2) if token else x
        # a long case is a later part of its text
        ts["positions"] = torch.arange(N, dtype=torch.int32, device="cuda") + (0 if not case["scaling"] else ORIGINAL)
        return ts
    if kind == "copy":
        shape = (case["layers"], case["pages"], case["Hk"], case["page"], d)
        return {"k_cache": _normal(gen, shape, case), "v_cache": _normal(gen, shape, case), "pairs": _copy_pairs(case, seed)}
    before, new = _sizes(case)
    counts = _pages_of(case)
    total = sum(counts)
    order = torch.randperm(total, generator=gen, device="cuda", dtype=torch.int64).to(torch.int32)
    # a sequence's row of the table ends with a number that is no page
    table = torch.full((case["B"], max(counts) + 1), -1, dtype=torch.int32, device="cuda")
    at = 0
    for b, n in enumerate(counts):
        table[b, :n] = order[at:at + n]
        at += n
    T = sum(new) + case["pad"]
    shape = (total, case["Hk"], case["page"], d)
    starts = np.concatenate([[0], np.cumsum(new)])
    return {
        "k_cache": _normal(gen, shape, case), "v_cache": _normal(gen, shape, case), "table": table,
        "lengths": torch.tensor([b + n for b, n in zip(before, new)], dtype=torch.int32, device="cuda"),
        "starts": torch.tensor(starts, dtype=torch.int32, device="cuda"),
        "q": _normal(gen, (T, case["Hq"], d), case),
        "k": _normal(gen, (T, case["Hk"], d), case), "v": _normal(gen, (T, case["Hk"], d), case),
    }


def prepare(case, seed):
    """Tensors, and what a program keeps beside them: the frequencies, output buffers, the attention's workspace."""
    st = _inputs(case, seed)
    st["case"] = case
    kind = case["kind"]
    if kind in ("rotary", "append"):
        f, st["magnitude"] = _frequencies(case)
        st["frequencies"] = torch.tensor(f, dtype=torch.float64, device="cuda")
        if own:
            from paper_2205_14135_amd.rotary import Rotary
            st["rotary"] = Rotary(st["frequencies"], interleaved=case["interleaved"], magnitude=st["magnitude"])
    if kind == "rotary" and case["train"]:
        st["q"].requires_grad_(True)
        st["k"].requires_grad_(True)
    if kind in ("append", "attend"):
        st["out"] = torch.zeros_like(st["q"])
        if case["new"] == "single" and case["pad"] == 0:
            st["single"] = True
        st["ends"] = _sizes(case)      # what the program knows on the host, for the plain form's loop over sequences
    if kind == "attend":
        del st["k"], st["v"]
        st["lse"] = torch.zeros((case["Hq"], st["q"].shape[0]), dtype=torch.float32, device="cuda")
        if own:
            from paper_2205_14135_amd import binding
            st["workspace"] = binding.attn_paged_workspace(st["q"], st["k_cache"], case["B"])
    return st


# ---------------------------------------------------------------------------------------------
# The plain forms.

def _turn(x, positions, st, inverse=False):
    """x [..., tokens, d] in 32 bits, turned by its tokens' positions [tokens]; angles in 64 bits."""
    case = st["case"]
    r = case["r"]
    angle = positions.to(torch.float64).unsqueeze(-1) * st["frequencies"]
    c, s = (torch.cos(angle) * st["magnitude"]).float(), (torch.sin(angle) * st["magnitude"]).float()
    if inverse:
        s = -s
    x = x.float()
    y = x.clone()
    a, b = (x[..., 0:r:2], x[..., 1:r:2]) if case["interleaved"] else (x[..., :r // 2], x[..., r // 2:r])
    ya, yb = a * c - b * s, b * c + a * s
    if case["interleaved"]:
        y[..., 0:r:2], y[..., 1:r:2] = ya, yb
    else:
        y[..., :r // 2], y[..., r // 2:r] = ya, yb
    return y


def _plain_rotary(st):
    names = ("q", "k")
    with torch.no_grad():
        out = [_turn(st[n], st["positions"], st).to(st[n].dtype) for n in names]
        if st["case"]["train"]:
            out += [_turn(st["d" + n], st["positions"], st, inverse=True).to(st[n].dtype) for n in names]
    return tuple(out)


def _plain_append(st):
    case = st["case"]
    before, new = st["ends"]
    page = case["page"]
    positions = torch.cat([torch.arange(b, b + n, device="cuda") for b, n in zip(before, new)])
    seq = torch.repeat_interleave(torch.arange(case["B"], device="cuda"), torch.tensor(new, device="cuda"))
    n = positions.numel()
    ids = st["table"][seq, positions // page].long()
    q = _turn(st["q"][:n].transpose(0, 1), positions, st).transpose(0, 1)
    k = _turn(st["k"][:n].transpose(0, 1), positions, st).transpose(0, 1)
    st["out"][:n] = q.to(st["q"].dtype)
    st["k_cache"][ids, :, positions % page] = k.to(st["q"].dtype)
    st["v_cache"][ids, :, positions % page] = st["v"][:n]
    return st["out"], st["k_cache"], st["v_cache"]


def _plain_attend(st):
    case = st["case"]
    before, new = st["ends"]
    Hk, G, d, page = case["Hk"], case["Hq"] // case["Hk"], case["d"], case["page"]
    at = 0
    for b in range(case["B"]):
        n, m = before[b] + new[b], new[b]
        ids = st["table"][b, :-(-n // page)].long()
        q = st["q"][at:at + m].float().view(m, Hk, G, d).permute(1, 2, 0, 3).reshape(Hk, G * m, d)
        last = torch.arange(before[b], n, device="cuda").repeat(G).unsqueeze(-1) if case["causal"] else None
        for h in range(Hk):
            k = st["k_cache"][ids, h].reshape(-1, d)[:n].float()
            v = st["v_cache"][ids, h].reshape(-1, d)[:n].float()
            s = torch.matmul(q[h], k.t().contiguous()) * (1.0 / math.sqrt(d))
            if case["causal"] and m > 1:
                s.masked_fill_(torch.arange(n, device="cuda") > last, -math.inf)
            top = s.amax(-1, keepdim=True)
            p = torch.exp(s - top)
            total = p.sum(-1, keepdim=True)
            o = torch.matmul(p, v) / total
            st["out"][at:at + m, h * G:(h + 1) * G] = o.view(G, m, d).transpose(0, 1).to(st["q"].dtype)
            st["lse"][h * G:(h + 1) * G, at:at + m] = (top + torch.log(total)).view(G, m)
        at += m
    return st["out"], st["lse"]


def _plain_copy(st):
    src, dst = st["pairs"][:, 0].to("cuda", torch.int64), st["pairs"][:, 1].to("cuda", torch.int64)
    for name in ("k_cache", "v_cache"):
        st[name][:, dst] = st[name][:, src]
    return st["k_cache"], st["v_cache"]


def run(st):
    case = st["case"]
    kind = case["kind"]
    if not own:
        return {"rotary": _plain_rotary, "append": _plain_append, "attend": _plain_attend, "copy": _plain_copy}[kind](st)
    from paper_2205_14135_amd import binding
    if kind == "rotary":
        if not case["train"]:
            return binding.attn_rotary(st["q"], st["k"], st["rotary"], positions=st["positions"])
        from paper_2205_14135_amd.autograd import rotary_embedding
        q, k = rotary_embedding(st["q"], st["k"], st["rotary"], positions=st["positions"])
        return (q.detach(), k.detach(), *torch.autograd.grad((q, k), (st["q"], st["k"]), (st["dq"], st["dk"])))
    starts = None if st.get("single") else st.get("starts")
    if kind == "append":
        binding.attn_paged_append(st["k"], st["v"], st["k_cache"], st["v_cache"], st["table"], st["lengths"], starts, Q=st["q"], rotary=st["rotary"],
                                  out=st["out"])
        return st["out"], st["k_cache"], st["v_cache"]
    if kind == "attend":
        return binding.attn_paged_fwd(st["q"], st["k_cache"], st["v_cache"], st["table"], st["lengths"], starts, softmax_scale=1.0 / math.sqrt(case["d"]),
                                      causal=case["causal"], out=st["out"], lse=st["lse"], workspace=st["workspace"])
    binding.attn_paged_copy(st["k_cache"], st["v_cache"], st["pairs"])
    return st["k_cache"], st["v_cache"]


def work(case):
    """Every input once, every output once; attention: two products over the visible (query, key) pairs; rotary: six operations a pair of columns."""
    d, kind = case["d"], case["kind"]
    if kind == "rotary":
        tokens = case["B"] * case["N"]
        passes = 2 if case["train"] else 1
        heads = case["Hq"] + case["Hk"]
        return {"bytes": passes * tokens * (heads * d * 4 + 4) + 8 * (case["r"] // 2), "flops": passes * tokens * heads * case["r"] * 3}
    if kind == "copy":
        return {"bytes": case["layers"] * case["pairs"] * case["page"] * case["Hk"] * d * 8, "flops": 0}
    before, new = _sizes(case)
    table = 4 * sum(_pages_of(case)) + 8 * case["B"]
    T = sum(new)
    if kind == "append":
        return {"bytes": T * d * 4 * (case["Hq"] + 2 * case["Hk"]) + table, "flops": T * (case["Hq"] + case["Hk"]) * case["r"] * 3}
    pairs = sum(n * b + n * (n + 1) // 2 if case["causal"] else n * (b + n) for b, n in zip(before, new))
    held = sum(b + n for b, n in zip(before, new))
    return {"bytes": held * case["Hk"] * d * 4 + T * case["Hq"] * (4 * d + 4) + table, "flops": 4 * pairs * case["Hq"] * d}


# ---------------------------------------------------------------------------------------------
# The same results in 64 bits, from the definitions.

def _exact_turn(x, angle, factor, interleaved):
    """x [tokens, H, d] in 64 bits; angle [tokens, pairs].  As a product of complex numbers."""
    r = 2 * angle.shape[-1]
    pairs = x[..., :r].unflatten(-1, (r // 2, 2)) if interleaved else x[..., :r].unflatten(-1, (2, r // 2)).transpose(-1, -2)
    z = torch.view_as_complex(pairs.contiguous()) * torch.polar(torch.full_like(angle, factor), angle).unsqueeze(-2)
    turned = torch.view_as_real(z)
    turned = turned.flatten(-2) if interleaved else turned.transpose(-1, -2).flatten(-2)
    return torch.cat([turned, x[..., r:]], dim=-1)


def exact(case, seed):
    kind = case["kind"]
    t = _inputs(case, seed)
    d = case["d"]
    if kind == "copy":
        source = list(range(case["pages"]))       # page p holds afterwards what source[p] held
        for src, dst in t["pairs"].tolist():
            source[dst] = src
        source = torch.tensor(source, device="cuda")
        return tuple(t[name].index_select(1, source).double() for name in ("k_cache", "v_cache"))
    if kind == "rotary":
        f, factor = _frequencies(case)
        angle = t["positions"].double().unsqueeze(-1) * torch.tensor(f, device="cuda")
        out = []
        for name, sign in (("q", 1), ("k", 1), ("dq", -1), ("dk", -1))[:4 if case["train"] else 2]:
            y = torch.empty(t[name].shape, dtype=torch.float64, device="cuda")
            for b in range(case["B"]):
                y[b] = _exact_turn(t[name][b].transpose(0, 1).double(), sign * angle, factor, case["interleaved"]).transpose(0, 1)
            out.append(y)
        return tuple(out)
    before, new = _sizes(case)
    page, G = case["page"], case["Hq"] // case["Hk"]
    if kind == "append":
        f, factor = _frequencies(case)
        f = torch.tensor(f, device="cuda")
        out = torch.zeros(t["q"].shape, dtype=torch.float64, device="cuda")
        caches = [t["k_cache"].double(), t["v_cache"].double()]
        at = 0
        for b in range(case["B"]):
            for i0 in range(0, new[b], 1024):
                rows = slice(at + i0, at + min(new[b], i0 + 1024))
                pos = torch.arange(before[b] + i0, before[b] + i0 + rows.stop - rows.start, device="cuda")
                angle = pos.double().unsqueeze(-1) * f
                out[rows] = _exact_turn(t["q"][rows].double(), angle, factor, case["interleaved"])
                turned = _exact_turn(t["k"][rows].double(), angle, factor, case["interleaved"])
                slot = t["table"][b, (pos // page)].long() * page + pos % page
                for cache, rows_new in zip(caches, (turned, t["v"][rows].double())):
                    flat = cache.transpose(1, 2).reshape(-1, case["Hk"], d)
                    flat[slot] = rows_new
                    cache.copy_(flat.view(-1, page, case["Hk"], d).transpose(1, 2))
            at += new[b]
        return out, caches[0], caches[1]
    out = torch.zeros(t["q"].shape, dtype=torch.float64, device="cuda")
    lse = torch.zeros((case["Hq"], t["q"].shape[0]), dtype=torch.float64, device="cuda")
    at = 0
    for b in range(case["B"]):
        n, m = before[b] + new[b], new[b]
        key = torch.arange(n, device="cuda")
        slot = t["table"][b, key // page].long() * (case["Hk"] * page) + key % page
        for h in range(case["Hk"]):
            k = t["k_cache"].view(-1, d)[slot + h * page].double()
            v = t["v_cache"].view(-1, d)[slot + h * page].double()
            for g in range(h * G, (h + 1) * G):
                for i0 in range(0, m, 1024):
                    i1 = min(m, i0 + 1024)
                    s = torch.mm(t["q"][at + i0:at + i1, g].double(), k.t()) / math.sqrt(d)
                    if case["causal"]:
                        s = s.masked_fill(key.unsqueeze(0) > torch.arange(before[b] + i0, before[b] + i1, device="cuda").unsqueeze(1), -math.inf)
                    lse[g, at + i0:at + i1] = torch.logsumexp(s, -1)
                    out[at + i0:at + i1, g] = torch.mm(torch.softmax(s, -1), v)
        at += m
    return out, lse
