"""Ragged batches over a paged cache, and the same attention in 64 bits on the CPU."""
import math

import torch

DTYPES = {"fp16": torch.float16, "bf16": torch.bfloat16}


class Batch:
    """`before` tokens held and `new` tokens of each sequence, in pages dealt out at random; everything of the cache that no sequence holds is NaN, and so are
    the rows of Q, K and V behind the last token."""

    def __init__(self, before, new, Hq, Hk, d, dtype, page, *, pad=0, seed=0, token_major=False, fused=False, extra_pages=3):
        gen = torch.Generator().manual_seed(seed)
        self.before, self.new, self.Hq, self.Hk, self.d, self.page = list(before), list(new), Hq, Hk, d, page
        self.B, self.tokens = len(new), sum(new)
        self.T = self.tokens + pad
        self.dtype = DTYPES[dtype]
        self.lengths = [max(b + n, 0) for b, n in zip(before, new)]
        counts = [-(-n // page) for n in self.lengths]
        self.pages = sum(counts) + extra_pages
        order = torch.randperm(self.pages, generator=gen).tolist()
        width = max(1, max(counts))
        self.table = torch.full((self.B, width), -7, dtype=torch.int32)
        at = 0
        for b, n in enumerate(counts):
            self.table[b, :n] = torch.tensor(order[at:at + n], dtype=torch.int32)
            at += n
        shape = (self.pages, page, Hk, d) if token_major else (self.pages, Hk, page, d)
        caches = []
        for _ in range(2):
            c = torch.randn(shape, generator=gen).to(self.dtype)
            c = c.transpose(1, 2) if token_major else c
            held = torch.zeros(self.pages, page, dtype=torch.bool)
            for b in range(self.B):
                for t in range(counts[b]):
                    held[self.table[b, t], :min(page, self.lengths[b] - t * page)] = True
            c.masked_fill_(~held.view(self.pages, 1, page, 1), math.nan)
            caches.append(c)
        self.kc, self.vc = caches
        heads = Hq + 2 * Hk
        if fused:   # views of one projection's output
            x = torch.randn(max(self.T, 1), heads, d, generator=gen).to(self.dtype)
            self.q, self.k, self.v = x[:, :Hq], x[:, Hq:Hq + Hk], x[:, Hq + Hk:]
        else:
            self.q, self.k, self.v = (torch.randn(max(self.T, 1), h, d, generator=gen).to(self.dtype) for h in (Hq, Hk, Hk))
        for x in (self.q, self.k, self.v):
            x[self.tokens:] = math.nan
        self.starts = torch.tensor([sum(new[:i]) for i in range(self.B + 1)], dtype=torch.int32)
        self.tau = 1.0 / math.sqrt(d)

    def gpu(self, single=False):
        """(q, k_cache, v_cache, table, lengths, starts) on the GPU, strides kept."""
        def move(x):
            base = torch.empty_strided(x.size(), x.stride(), dtype=x.dtype, device="cuda")
            return base.copy_(x)
        starts = None if single else self.starts.cuda()
        return (move(self.q), move(self.kc), move(self.vc), self.table.cuda(), torch.tensor(self.lengths, dtype=torch.int32).cuda(), starts)

    def rows(self, cache, b):
        """What sequence b holds of a cache, [length, Hk, d] in 64 bits; a number that is no page stands for zeros."""
        n = self.lengths[b]
        out = torch.zeros(n, self.Hk, self.d, dtype=torch.float64)
        for t in range(-(-n // self.page)):
            lo, hi = t * self.page, min(n, (t + 1) * self.page)
            number = int(self.table[b, t])
            if 0 <= number < self.pages:
                out[lo:hi] = cache[number, :, :hi - lo].transpose(0, 1).double()
        return out


def attention(batch, causal, tau=None):
    """(O [tokens, Hq, d], LSE [Hq, tokens], and the bounds of their errors) in 64 bits.

    u is half a step of the 16-bit type.  The kernel's weights are probabilities rounded to 16 bits (each off by u of itself) and O is divided by their own sum, so
    O is off by at most u (sum_j w_j |v_j| + |O|), and by u |O| for its own rounding.  A logit is a sum of d products in 32 bits, off by at most
    d 2^-24 tau sum |q k|, and what goes through the exponential and the moves of the reference adds a few steps of 2^-24 of the exponent: rho.  In fp16 a probability below
    2^-14 is off by up to 2^-25 whatever its size: n of them against a sum of at least 2^-8 (the reference lags by no more).  A row that sees no key is exact."""
    u = torch.finfo(batch.dtype).eps / 2
    tau = batch.tau if tau is None else tau
    O, L = torch.zeros(batch.tokens, batch.Hq, batch.d, dtype=torch.float64), torch.full((batch.Hq, batch.tokens), -math.inf, dtype=torch.float64)
    bO, bL = torch.zeros_like(O), torch.zeros_like(L)
    G = batch.Hq // batch.Hk
    for b in range(batch.B):
        m, n, at = batch.new[b], batch.lengths[b], int(batch.starts[b])
        if m == 0:
            continue
        k, v = batch.rows(batch.kc, b), batch.rows(batch.vc, b)
        last = torch.arange(n - m, n) if causal else torch.full((m,), n - 1)
        seen = torch.arange(n).unsqueeze(0) <= last.unsqueeze(1)
        some = seen.any(-1)
        for h in range(batch.Hq):
            q, kh, vh = batch.q[at:at + m, h].double(), k[:, h // G], v[:, h // G]
            s = tau * (q @ kh.t())
            size = tau * (q.abs() @ kh.abs().t())
            s = s.masked_fill(~seen, -math.inf)
            lse = torch.logsumexp(s, -1) if n else torch.full((m,), -math.inf, dtype=torch.float64)
            w = torch.exp(s - lse.unsqueeze(-1)).masked_fill(~seen, 0.0)
            o = w @ vh
            size = size.masked_fill(~seen, 0.0)
            top = size.amax(-1) if n else torch.zeros(m, dtype=torch.float64)
            rho = (batch.d + 32) * 2.0 ** -24 * (top + 8.0)
            spread = w @ vh.abs() + o.abs()
            bound = (u + 2 * rho).unsqueeze(-1) * spread + u * o.abs() + 2.0 ** -24
            if batch.dtype == torch.float16 and n:
                bound = bound + n * 2.0 ** -17 * 2.0 ** -8 * vh.abs().amax()
            O[at:at + m, h] = torch.where(some.unsqueeze(-1), o, torch.zeros_like(o))
            bO[at:at + m, h] = torch.where(some.unsqueeze(-1), bound, torch.zeros_like(bound))
            L[h, at:at + m] = torch.where(some, lse, torch.full_like(lse, -math.inf))
            bL[h, at:at + m] = rho + (n / 32 + 16) * 2.0 ** -24 + 2.0 ** -22 * lse.abs().clamp(max=1e9)
    return O, L, bO, bL


def assert_within(got, want, bound, what):
    got = got.detach().cpu().double()
    same = (got == want)   # infinities
    off = torch.where(same, torch.zeros_like(want), (got - want).abs())
    bad = ~(off <= bound)
    if bad.any():
        i = tuple(x[0].item() for x in bad.nonzero(as_tuple=True))
        raise AssertionError(f"{what}{list(i)}: {got[i].item()} for {want[i].item()}, bound {bound[i].item()}; {int(bad.sum())} of {bad.numel()} beyond")


def turned(x, positions, frequencies, interleaved, magnitude, inverse=False):
    """Rows x [tokens, heads, d] turned by their positions, in 64 bits, and the bound of a kernel's error before its last rounding: the angle is exact to 2^-22 radians,
    sine and cosine to 2^-23, three roundings of 2^-24 of the products."""
    r = 2 * frequencies.numel()
    x = x.double()
    angle = positions.double().unsqueeze(-1) * frequencies * (-1 if inverse else 1)
    c, s = (torch.cos(angle) * magnitude).unsqueeze(1), (torch.sin(angle) * magnitude).unsqueeze(1)
    a = torch.arange(0, r, 2) if interleaved else torch.arange(r // 2)
    b = a + 1 if interleaved else a + r // 2
    y, bound = x.clone(), torch.zeros_like(x)
    y[..., a], y[..., b] = x[..., a] * c - x[..., b] * s, x[..., b] * c + x[..., a] * s
    size = abs(magnitude) * (x[..., a].abs() + x[..., b].abs()) * 2.0 ** -21
    bound[..., a], bound[..., b] = size, size
    return y, bound


def rounding(want, dtype):
    """Half a step of the type at the value, relative, or half the smallest subnormal."""
    u = torch.finfo(dtype).eps / 2
    return u * want.abs() + (2.0 ** -25 if dtype == torch.float16 else 2.0 ** -134)
