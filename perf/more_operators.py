"""Operators of attention with a sliding window, and of normed queries and keys, as they are measured.

Four operators, through the framework's public entry points (`own`), or in elementary torch operations:

  norm    every row of Q and K divided by the root of its mean square, times weights, and turned by its token's position, forward and backward
          (`binding.attn_norm_rotary`, `autograd.norm_rotary_embedding`)
  append  the new tokens of every sequence: Q and K normed and turned, K written into the pages of a cache with V (`binding.attn_paged_append` with a norm)
  window  softmax attention in which a query sees the last `window` keys, its own among them, and the first `sinks` keys, forward and backward
          (`binding.attn_window_fwd`, `autograd.flash_attention` with a window)
  step    the same for the new tokens of every sequence over what its pages hold (`binding.attn_paged_fwd` with a window)

A case is a dict of plain values; sizes of a ragged batch follow from its "shape" number alone.

  kind          "norm", "append", "window" or "step"
  Hq, Hk, d     heads of Q, heads of K and V, head dimension;  dtype "bf16" | "fp16"
  norm/append   r (columns that turn), interleaved, weights "float32" | "same" (the type of the norm's weights)
  norm/window   B, N, layout "head" ([B,H,N,d] memory) | "token" (a view of [B,N,H,d]), train
  window/step   window, sinks;  window: padded (true lengths between N / 3 and N)
  append/step   B sequences, page (tokens a page), before (lo, hi) tokens that a sequence holds already, new "single" (one token a
                sequence), "chunk" (lo, hi tokens) or "mixed" (one chunk of `hi` tokens among single ones), pad rows behind the last token
"""
from __future__ import annotations

import math
import random

import numpy as np
import torch

own = False

DTYPES = {"fp16": torch.float16, "bf16": torch.bfloat16}
BASE = 10000.0
EPS = 1e-6


def _norm(name, B, N, Hq, Hk, d, dtype, layout, r, interleaved, weights, train=True):
    c = dict(kind="norm", B=B, N=N, Hq=Hq, Hk=Hk, d=d, dtype=dtype, layout=layout, r=r, interleaved=interleaved, weights=weights, train=train)
    return dict(c, name=name) if name else c


def _window(name, B, N, H, d, dtype, layout, window, sinks, padded=False, train=True, shape=1):
    c = dict(kind="window", B=B, N=N, Hq=H, Hk=H, d=d, dtype=dtype, layout=layout, window=window, sinks=sinks, padded=padded, train=train, shape=shape)
    return dict(c, name=name) if name else c


def _batch_case(name, kind, B, Hq, Hk, d, dtype, page, before, new, q=(1, 1), pad=0, shape=1, **more):
    c = dict(kind=kind, B=B, Hq=Hq, Hk=Hk, d=d, dtype=dtype, page=page, before_lo=before[0], before_hi=before[1], new=new, q_lo=q[0], q_hi=q[1],
             pad=pad, shape=shape, **more)
    return dict(c, name=name) if name else c


def listed():
    return [
        # one sentence through one layer, forward alone: the launch and the host path are all there is
        _norm("norm_sentence_fwd", 1, 197, 12, 12, 64, "fp16", "token", 64, False, "same", train=False),
        # the layer of a training step, heads interleaved in memory as a projection leaves them
        _norm("norm_train", 8, 1024, 16, 16, 64, "bf16", "token", 64, False, "float32"),
        # the long end: half of a wide head turns, neighbouring columns, shared K heads
        _norm("norm_long_train", 1, 16384, 16, 4, 128, "fp16", "head", 64, True, "same"),
        # one step of 64 running sequences
        _batch_case("append_step", "append", 64, 32, 8, 128, "bf16", 16, (100, 1000), "single", r=128, interleaved=False, weights="same"),
        # prompts of different lengths read in together, padded behind the last
        _batch_case("append_prompts", "append", 12, 16, 16, 64, "fp16", 64, (0, 300), "chunk", (50, 2048), pad=37, r=32, interleaved=True, weights="float32"),
        # one sentence, forward alone
        _window("window_sentence_fwd", 1, 197, 12, 64, "fp16", "token", 64, 4, train=False),
        # a padded batch of odd lengths, no first tokens
        _window("window_padded_train", 5, 1000, 12, 32, "fp16", "head", 300, 0, padded=True),
        # the layer of a GPT-2-medium training step with a quarter of its context in sight
        _window("window_gpt2_train", 8, 1024, 16, 64, "bf16", "token", 256, 4),
        # a long document: each token sees a sixteenth of it, and the first four tokens
        _window("window_long_train", 1, 16384, 16, 128, "bf16", "head", 1024, 4),
        # the smallest answer: one sequence, one token, two groups of heads
        _batch_case("step_one_token", "step", 1, 16, 2, 64, "bf16", 16, (7776, 7776), "single", window=512, sinks=4),
        # one step of 64 running sequences of very different lengths, some shorter than the window
        _batch_case("step_running", "step", 64, 32, 8, 128, "bf16", 16, (500, 30000), "single", window=2048, sinks=4),
        # a chunk of a long prompt among running sequences, padded
        _batch_case("step_chunk", "step", 9, 32, 8, 128, "bf16", 16, (2000, 14336), "mixed", (2048, 2048), pad=23, window=4096, sinks=16),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


MAX_FLOPS = 4.6e11          # just below window_long_train
MAX_BYTES = 5.0e8           # just below step_running


def draw(rng):
    """One more case: the kinds of the list, sizes over the logarithm of their range, odd ones among them."""
    while True:
        kind = rng.choice(["norm", "append", "window", "window", "step", "step"])
        dtype = rng.choice(["fp16", "bf16", "bf16"])
        d = rng.choice([32, 64, 64, 128, 128])
        Hk = rng.choice([1, 2, 4, 8, 16])
        Hq = Hk * rng.choice([1, 2, 4, 8] if Hk <= 4 else [1, 2, 4])
        layout = rng.choice(["head", "token"])
        window, sinks = _log_int(rng, 16, 8192), rng.choice([0, 1, 4, 4, 16, 64])
        if kind == "norm":
            N = _log_int(rng, 100, 16384)
            c = _norm(None, max(1, _log_int(rng, N, 32768) // N), N, Hq, Hk, d, dtype, layout, rng.choice([d, d, d // 2, d // 4]), rng.random() < 0.4,
                      rng.choice(["float32", "same"]), rng.random() < 0.7)
        elif kind == "window":
            N = _log_int(rng, 60, 16384)
            c = _window(None, max(1, _log_int(rng, N, 32768) // N), N, rng.choice([1, 3, 8, 12, 16]), d, dtype, layout, window, sinks, rng.random() < 0.3,
                        rng.random() < 0.7, rng.randrange(1 << 30))
        else:
            new = rng.choice(["single", "single", "chunk", "mixed"])
            B = _log_int(rng, 1, 128) if new == "single" else _log_int(rng, 1, 40)
            q_hi = _log_int(rng, 2, 3000) if new != "single" else 1
            hi = _log_int(rng, 16, 65536 if kind == "step" else 2000)
            more = dict(window=window, sinks=sinks) if kind == "step" else dict(r=rng.choice([d, d // 2]), interleaved=rng.random() < 0.4,
                                                                                weights=rng.choice(["float32", "same"]))
            c = _batch_case(None, kind, B, Hq, Hk, d, dtype, rng.choice([16, 16, 32, 64, 128, 256]), (_log_int(rng, 1, hi), hi), new,
                            (max(1, q_hi // 8), q_hi), rng.choice([0, 0, 5, 41]), rng.randrange(1 << 30), **more)
        w = work(c)
        if w["flops"] <= MAX_FLOPS and w["bytes"] <= MAX_BYTES and _cache_bytes(c) <= 6e9:
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


def _true_lengths(case):
    if not case["padded"]:
        return [case["N"]] * case["B"]
    rng = random.Random(case["shape"])
    return [rng.randint(max(1, case["N"] // 3), case["N"]) for _ in range(case["B"])]


def _pages_of(case):
    """Pages that each sequence holds once the new tokens are in."""
    before, new = _sizes(case)
    return [-(-(b + n) // case["page"]) for b, n in zip(before, new)]


def _cache_bytes(case):
    return 4 * sum(_pages_of(case)) * case["page"] * case["Hk"] * case["d"] if case["kind"] in ("append", "step") else 0


def _normal(gen, shape, case):
    return torch.randn(shape, generator=gen, device="cuda", dtype=torch.float32).to(DTYPES[case["dtype"]])


def _frequencies(case):
    """Radians a position of each pair."""
    return BASE ** (-np.arange(case["r"] // 2, dtype=np.float64) / (case["r"] // 2))


def _inputs(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    kind, d = case["kind"], case["d"]
    ts = {}
    if kind in ("norm", "append"):
        # weights as training leaves them: around one, all different
        for name in ("wq", "wk"):
            w = 1.0 + 0.25 * torch.randn(d, generator=gen, device="cuda", dtype=torch.float32)
            ts[name] = w.to(DTYPES[case["dtype"]]) if case["weights"] == "same" else w
    if kind in ("norm", "window"):
        B, N = case["B"], case["N"]
        names = (("q", case["Hq"]), ("k", case["Hk"]), ("dq", case["Hq"]), ("dk", case["Hk"])) if kind == "norm" else tuple((n, case["Hq"]) for n in ("q", "k", "v", "do"))
        for name, H in names:
            token = case["layout"] == "token"
            x = _normal(gen, (B, N, H, d) if token else (B, H, N, d), case)
            ts[name] = x.transpose(1, 2) if token else x
        if kind == "norm":
            ts["positions"] = torch.arange(N, dtype=torch.int32, device="cuda")
        elif case["padded"]:
            ts["key_lengths"] = torch.tensor(_true_lengths(case), dtype=torch.int32, device="cuda")
        return ts
    before, new = _sizes(case)
    counts = _pages_of(case)
    total = sum(counts)
    order = torch.randperm(total, generator=gen, device="cuda", dtype=torch.int64).to(torch.int32)
    # a sequence's row of the table ends with a number that is no page
    table = torch.full((case["B"], max(counts) + 1), -1, dtype=torch.int32)
    at = np.concatenate([[0], np.cumsum(counts)])
    order = order.cpu()
    for b, n in enumerate(counts):
        table[b, :n] = order[at[b]:at[b] + n]
    T = sum(new) + case["pad"]
    shape = (total, case["Hk"], case["page"], d)
    starts = np.concatenate([[0], np.cumsum(new)])
    ts.update(k_cache=_normal(gen, shape, case), v_cache=_normal(gen, shape, case), table=table.cuda(),
              lengths=torch.tensor([b + n for b, n in zip(before, new)], dtype=torch.int32, device="cuda"),
              starts=torch.tensor(starts, dtype=torch.int32, device="cuda"), q=_normal(gen, (T, case["Hq"], d), case))
    if kind == "append":
        ts.update(k=_normal(gen, (T, case["Hk"], d), case), v=_normal(gen, (T, case["Hk"], d), case))
    return ts


def prepare(case, seed):
    """Tensors, and what a program keeps beside them: the frequencies, output buffers, the attention's workspace."""
    st = _inputs(case, seed)
    st["case"] = case
    kind = case["kind"]
    if kind in ("norm", "append"):
        st["frequencies"] = torch.tensor(_frequencies(case), dtype=torch.float64, device="cuda")
        if own:
            from paper_2205_14135_amd.rotary import HeadNorm, Rotary
            st["rotary"] = Rotary(st["frequencies"], interleaved=case["interleaved"])
            st["norm"] = HeadNorm(st["wq"], st["wk"], eps=EPS)
    if kind in ("norm", "window") and case["train"]:
        for name in ("q", "k", "wq", "wk") if kind == "norm" else ("q", "k", "v"):
            st[name].requires_grad_(True)
    if kind in ("append", "step"):
        st["out"] = torch.zeros_like(st["q"])
        st["single"] = case["new"] == "single" and case["pad"] == 0
        st["ends"] = _sizes(case)      # what the program knows on the host, for the plain form's loop over sequences
    if kind == "step":
        st["lse"] = torch.zeros((case["Hq"], st["q"].shape[0]), dtype=torch.float32, device="cuda")
        if own:
            from paper_2205_14135_amd import binding
            st["workspace"] = binding.attn_paged_workspace(st["q"], st["k_cache"], case["B"])
    return st


# ---------------------------------------------------------------------------------------------
# The plain forms.

def _turn(x, positions, st, inverse=False):
    """x [..., tokens, d] in 32 bits, turned by its tokens' positions [tokens]; angles in 64 bits."""
    r = st["case"]["r"]
    angle = positions.to(torch.float64).unsqueeze(-1) * st["frequencies"]
    c, s = torch.cos(angle).float(), torch.sin(angle).float()
    if inverse:
        s = -s
    y = x.clone()
    if st["case"]["interleaved"]:
        a, b = x[..., 0:r:2], x[..., 1:r:2]
        y[..., 0:r:2], y[..., 1:r:2] = a * c - b * s, b * c + a * s
    else:
        a, b = x[..., :r // 2], x[..., r // 2:r]
        y[..., :r // 2], y[..., r // 2:r] = a * c - b * s, b * c + a * s
    return y


def _normed_and_turned(x, w, positions, st):
    x = x.float()
    return _turn(x * torch.rsqrt(x.square().mean(-1, keepdim=True) + EPS) * w.float(), positions, st)


def _norm_gradients(x, w, dy, positions, st):
    x = x.float()
    r = torch.rsqrt(x.square().mean(-1, keepdim=True) + EPS)
    g = _turn(dy.float(), positions, st, inverse=True)
    h = g * w.float()
    dx = r * (h - x * (r * r * (h * x).mean(-1, keepdim=True)))
    return dx, (g * x * r).sum((0, 1, 2))


def _plain_norm(st):
    with torch.no_grad():
        q, k = (_normed_and_turned(st[n], st["w" + n], st["positions"], st).to(st[n].dtype) for n in ("q", "k"))
        if not st["case"]["train"]:
            return q, k
        (dq, dwq), (dk, dwk) = (_norm_gradients(st[n], st["w" + n], st["d" + n], st["positions"], st) for n in ("q", "k"))
        return q, k, dq.to(q.dtype), dk.to(q.dtype), dwq.to(st["wq"].dtype), dwk.to(st["wk"].dtype)


def _plain_append(st):
    before, new = st["ends"]
    page = st["case"]["page"]
    positions = torch.cat([torch.arange(b, b + n, device="cuda") for b, n in zip(before, new)])
    seq = torch.repeat_interleave(torch.arange(len(new), device="cuda"), torch.tensor(new, device="cuda"))
    n = positions.numel()
    ids = st["table"][seq, positions // page].long()
    q, k = (_normed_and_turned(st[name][:n].transpose(0, 1), st["w" + name], positions, st).transpose(0, 1) for name in ("q", "k"))
    st["out"][:n] = q.to(st["q"].dtype)
    st["k_cache"][ids, :, positions % page] = k.to(st["q"].dtype)
    st["v_cache"][ids, :, positions % page] = st["v"][:n]
    return st["out"], st["k_cache"], st["v_cache"]


def _seen(key, pos, case):
    """Which keys [keys] the queries at positions [rows] see: [rows, keys]."""
    key, pos = key.unsqueeze(0), pos.unsqueeze(1)
    return (key <= pos) & ((key > pos - case["window"]) | (key < case["sinks"]))


def _plain_window(st):
    """Rows by the thousand, each with the keys that any of them sees."""
    case = st["case"]
    q, k, v = (st[n].detach() for n in ("q", "k", "v"))
    N, tau = case["N"], 1.0 / math.sqrt(case["d"])
    out = torch.empty(q.shape, dtype=torch.float32, device="cuda")
    lse = torch.empty(q.shape[:3], dtype=torch.float32, device="cuda")
    grads = [torch.zeros(q.shape, dtype=torch.float32, device="cuda") for _ in range(3)] if case["train"] else None
    lengths = st["key_lengths"].view(-1, 1, 1, 1) if case["padded"] else None
    for i0 in range(0, N, 1024):
        i1 = min(N, i0 + 1024)
        lo = max(0, i0 - case["window"] + 1)
        pos = torch.arange(i0, i1, device="cuda")
        key = torch.cat([torch.arange(min(case["sinks"], lo), device="cuda"), torch.arange(lo, i1, device="cuda")])
        hidden = ~_seen(key, pos, case)
        if lengths is not None:
            hidden = hidden | (key >= lengths) | (pos.unsqueeze(1) >= lengths)
        qi, kj, vj = q[:, :, i0:i1].float(), k[:, :, key].float(), v[:, :, key].float()
        s = torch.matmul(qi, kj.transpose(2, 3).contiguous()).mul_(tau).masked_fill_(hidden, -math.inf)
        top = s.amax(-1, keepdim=True).clamp_(min=-1e30)
        p = torch.exp(s.sub_(top))
        total = p.sum(-1, keepdim=True)
        lse[:, :, i0:i1] = (top + torch.log(total)).squeeze(-1)
        p = p / torch.where(total > 0, total, 1.0)
        out[:, :, i0:i1] = torch.matmul(p, vj)
        if grads is None:
            continue
        do = st["do"][:, :, i0:i1].float()
        dp = torch.matmul(do, vj.transpose(2, 3).contiguous())
        ds = p * (dp - (p * dp).sum(-1, keepdim=True)) * tau
        grads[0][:, :, i0:i1] = torch.matmul(ds, kj)
        grads[1].index_add_(2, key, torch.matmul(ds.transpose(2, 3).contiguous(), qi))
        grads[2].index_add_(2, key, torch.matmul(p.transpose(2, 3).contiguous(), do))
    if grads is None:
        return out.to(q.dtype), lse
    return (out.to(q.dtype), *(g.to(q.dtype) for g in grads))


def _plain_step(st):
    case = st["case"]
    before, new = st["ends"]
    Hk, G, d, page = case["Hk"], case["Hq"] // case["Hk"], case["d"], case["page"]
    at = 0
    for b in range(case["B"]):
        n, m = before[b] + new[b], new[b]
        lo = max(0, before[b] - case["window"] + 1)
        key = torch.cat([torch.arange(min(case["sinks"], lo), device="cuda"), torch.arange(lo, n, device="cuda")])
        ids = st["table"][b, key // page].long()
        k, v = (st[name][ids, :, key % page].transpose(0, 1).float() for name in ("k_cache", "v_cache"))      # [Hk, keys, d]
        q = st["q"][at:at + m].float().view(m, Hk, G, d).permute(1, 2, 0, 3).reshape(Hk, G * m, d)
        hidden = ~_seen(key, torch.arange(before[b], n, device="cuda"), case).repeat(G, 1)
        s = torch.matmul(q, k.transpose(1, 2).contiguous()).mul_(1.0 / math.sqrt(d)).masked_fill_(hidden, -math.inf)
        top = s.amax(-1, keepdim=True)
        p = torch.exp(s - top)
        total = p.sum(-1, keepdim=True)
        o = torch.matmul(p, v) / total
        st["out"][at:at + m] = o.view(Hk, G, m, d).permute(2, 0, 1, 3).reshape(m, Hk * G, d).to(st["q"].dtype)
        st["lse"][:, at:at + m] = (top + torch.log(total)).view(Hk * G, m)
        at += m
    return st["out"], st["lse"]


def run(st):
    case = st["case"]
    kind = case["kind"]
    if not own:
        return {"norm": _plain_norm, "append": _plain_append, "window": _plain_window, "step": _plain_step}[kind](st)
    from paper_2205_14135_amd import autograd, binding
    if kind == "norm":
        if not case["train"]:
            return binding.attn_norm_rotary(st["q"], st["k"], st["norm"], st["rotary"], positions=st["positions"])
        q, k = autograd.norm_rotary_embedding(st["q"], st["k"], st["norm"], st["rotary"], positions=st["positions"])
        return (q.detach(), k.detach(), *torch.autograd.grad((q, k), (st["q"], st["k"], st["wq"], st["wk"]), (st["dq"], st["dk"])))
    if kind == "window":
        tau = 1.0 / math.sqrt(case["d"])
        if not case["train"]:
            return binding.attn_window_fwd(st["q"], st["k"], st["v"], window=case["window"], sinks=case["sinks"], softmax_scale=tau, key_lengths=st.get("key_lengths"))
        out = autograd.flash_attention(st["q"], st["k"], st["v"], causal=True, window=case["window"], sinks=case["sinks"], key_lengths=st.get("key_lengths"))
        return (out.detach(), *torch.autograd.grad(out, (st["q"], st["k"], st["v"]), st["do"]))
    starts = None if st["single"] else st["starts"]
    if kind == "append":
        binding.attn_paged_append(st["k"], st["v"], st["k_cache"], st["v_cache"], st["table"], st["lengths"], starts, Q=st["q"], rotary=st["rotary"],
                                  norm=st["norm"], out=st["out"])
        return st["out"], st["k_cache"], st["v_cache"]
    return binding.attn_paged_fwd(st["q"], st["k_cache"], st["v_cache"], st["table"], st["lengths"], starts, softmax_scale=1.0 / math.sqrt(case["d"]),
                                  window=case["window"], sinks=case["sinks"], out=st["out"], lse=st["lse"], workspace=st["workspace"])


def _pairs(case, first, n):
    """Visible (query, key) pairs of the queries at positions first .. first + n - 1."""
    pos = np.arange(first, first + n, dtype=np.int64)
    lo = np.maximum(0, pos - case["window"] + 1)
    return int((pos - lo + 1 + np.minimum(lo, case["sinks"])).sum())


def work(case):
    """Every input that counts once, every output once; attention: two products over the visible (query, key) pairs, five more for the gradients; norm and rotation:
    four operations a column forward, and three for each that turns; three times that for the gradients."""
    d, kind = case["d"], case["kind"]
    heads = case["Hq"] + case["Hk"]
    if kind in ("norm", "append"):
        size = 4 if case["weights"] == "float32" else 2
    if kind == "norm":
        tokens = case["B"] * case["N"]
        train = case["train"]
        return {"bytes": tokens * (heads * d * 2 * (4 if train else 2) + 4) + 8 * (case["r"] // 2) + 2 * d * size * (2 if train else 1),
                "flops": tokens * heads * (4 * d + 3 * case["r"]) * (3 if train else 1)}
    if kind == "window":
        lengths = _true_lengths(case)
        rows = sum(lengths) * case["Hq"]
        pairs = sum(_pairs(case, 0, n) for n in lengths) * case["Hq"]
        return {"bytes": 2 * d * (4 * rows + 4 * case["B"] * case["N"] * case["Hq"]) if case["train"] else 2 * d * 4 * rows + 4 * rows,
                "flops": pairs * d * (14 if case["train"] else 4)}
    before, new = _sizes(case)
    table = 4 * sum(_pages_of(case)) + 8 * case["B"]
    T = sum(new)
    if kind == "append":
        return {"bytes": T * d * 4 * (case["Hq"] + 2 * case["Hk"]) + 2 * d * size + table, "flops": T * heads * (4 * d + 3 * case["r"])}
    held = sum(b + n - max(0, b - case["window"] + 1) + min(case["sinks"], max(0, b - case["window"] + 1)) for b, n in zip(before, new))
    pairs = sum(_pairs(case, b, n) for b, n in zip(before, new))
    return {"bytes": held * case["Hk"] * d * 4 + T * case["Hq"] * (4 * d + 4), "flops": 4 * pairs * case["Hq"] * d}


# ---------------------------------------------------------------------------------------------
# The same results in 64 bits, from the definitions.

def _exact_norm(x, w, angle, interleaved):
    """x [tokens, H, d]; angle [tokens, pairs].  The rotation as a product of complex numbers."""
    x = x.double()
    x = x / torch.sqrt((x * x).sum(-1, keepdim=True) / x.shape[-1] + EPS) * w
    r = 2 * angle.shape[-1]
    pairs = x[..., :r].unflatten(-1, (r // 2, 2)) if interleaved else x[..., :r].unflatten(-1, (2, r // 2)).transpose(-1, -2)
    z = torch.view_as_complex(pairs.contiguous()) * torch.polar(torch.ones_like(angle), angle).unsqueeze(-2)
    turned = torch.view_as_real(z)
    turned = turned.flatten(-2) if interleaved else turned.transpose(-1, -2).flatten(-2)
    return torch.cat([turned, x[..., r:]], dim=-1)


def _exact_attention(q, k, v, key, pos, case, length=None):
    """softmax(q k^T / sqrt(d)) v over the keys at positions `key` for one head, and its row statistic; rows without a key: zeros and -inf."""
    s = torch.mm(q, k.t()) / math.sqrt(case["d"])
    far = pos[:, None] - key[None, :]
    seen = (far >= 0) & ((far < case["window"]) | (key[None, :] < case["sinks"]))
    if length is not None:
        seen &= (key[None, :] < length) & (pos[:, None] < length)
    s = torch.where(seen, s, -math.inf)
    p = torch.nan_to_num(torch.softmax(s, -1), nan=0.0)
    return torch.mm(p, v), torch.logsumexp(s, -1), p


def exact(case, seed):
    kind, d = case["kind"], case["d"]
    t = _inputs(case, seed)
    if kind in ("norm", "append"):
        f = torch.tensor(_frequencies(case), device="cuda")
    if kind == "norm":
        angle = t["positions"].double().unsqueeze(-1) * f
        out, grads, dw = [], [], []
        for name in ("q", "k"):
            y = torch.empty(t[name].shape, dtype=torch.float64, device="cuda")
            g, w = torch.empty_like(y), t["w" + name].double().requires_grad_(case["train"])
            for b in range(case["B"]):
                x = t[name][b].transpose(0, 1).double().requires_grad_(case["train"])
                part = _exact_norm(x, w, angle, case["interleaved"])
                if case["train"]:     # the definition's gradient by 64-bit differentiation
                    part.backward(t["d" + name][b].transpose(0, 1).double())
                    g[b] = x.grad.transpose(0, 1)
                y[b] = part.detach().transpose(0, 1)
            out.append(y)
            grads.append(g)
            dw.append(w.grad)
        return (*out, *grads, *dw) if case["train"] else tuple(out)
    if kind == "window":
        N, w, sinks = case["N"], case["window"], case["sinks"]
        res = [torch.zeros(t["q"].shape, dtype=torch.float64, device="cuda") for _ in range(4)]
        lse = torch.zeros(t["q"].shape[:3], dtype=torch.float64, device="cuda")
        for b, length in enumerate(_true_lengths(case)):
            for h in range(case["Hq"]):
                q, k, v, do = (t[n][b, h].double() for n in ("q", "k", "v", "do"))
                for i0 in range(0, N, 2048):
                    i1 = min(N, i0 + 2048)
                    pos = torch.arange(i0, i1, device="cuda")
                    lo = max(0, i0 + 1 - w)
                    key = torch.arange(i1, device="cuda")
                    key = key[(key >= lo) | (key < sinks)]
                    o, l, p = _exact_attention(q[i0:i1], k[key], v[key], key, pos, case, length)
                    res[0][b, h, i0:i1], lse[b, h, i0:i1] = o, l
                    if case["train"]:
                        g = do[i0:i1]
                        ds = p * (torch.mm(g, v[key].t()) - (g * o).sum(-1, keepdim=True)) / math.sqrt(d)
                        res[1][b, h, i0:i1] = torch.mm(ds, k[key])
                        res[2][b, h, key] += torch.mm(ds.t(), q[i0:i1])
                        res[3][b, h, key] += torch.mm(p.t(), g)
        return tuple(res) if case["train"] else (res[0], lse)
    before, new = _sizes(case)
    page, G = case["page"], case["Hq"] // case["Hk"]
    out = torch.zeros(t["q"].shape, dtype=torch.float64, device="cuda")
    at = 0
    if kind == "append":
        caches = [t["k_cache"].double(), t["v_cache"].double()]
        for b in range(case["B"]):
            rows = slice(at, at + new[b])
            pos = torch.arange(before[b], before[b] + new[b], device="cuda")
            angle = pos.double().unsqueeze(-1) * f
            out[rows] = _exact_norm(t["q"][rows], t["wq"].double(), angle, case["interleaved"])
            slot = t["table"][b, (pos // page)].long() * page + pos % page
            for cache, rows_new in zip(caches, (_exact_norm(t["k"][rows], t["wk"].double(), angle, case["interleaved"]), t["v"][rows].double())):
                flat = cache.transpose(1, 2).reshape(-1, case["Hk"], d)
                flat[slot] = rows_new
                cache.copy_(flat.view(-1, page, case["Hk"], d).transpose(1, 2))
            at += new[b]
        return out, caches[0], caches[1]
    lse = torch.zeros((case["Hq"], t["q"].shape[0]), dtype=torch.float64, device="cuda")
    for b in range(case["B"]):
        n, m = before[b] + new[b], new[b]
        key = torch.arange(n, device="cuda")
        key = key[(key > before[b] - case["window"]) | (key < case["sinks"])]
        slot = t["table"][b, key // page].long() * (case["Hk"] * page) + key % page
        pos = torch.arange(before[b], n, device="cuda")
        for h in range(case["Hq"]):
            k, v = (t[name].view(-1, d)[slot + (h // G) * page].double() for name in ("k_cache", "v_cache"))
            out[at:at + m, h], lse[h, at:at + m], _ = _exact_attention(t["q"][at:at + m, h].double(), k, v, key, pos, case)
        at += m
    return out, lse
