"""Attention with a sliding window and sinks in 64 bits for one head, its gradients, and the bounds of a kernel's errors."""
import math

import torch


def visible(N, window, sinks, length=None, device="cuda"):
    """[N, N]: which keys a query sees."""
    i = torch.arange(N, device=device)
    far = i[:, None] - i[None, :]
    seen = (far >= 0) & ((far < window) | (i[None, :] < sinks))
    if length is not None:
        seen &= (i[None, :] < length) & (i[:, None] < length)
    return seen


class Head:
    """q, k, v, do [N, d] of a 16-bit type; keep: [N, N] of the dropout, or None, and the factor of what is kept.

    u is half a step of the type, rho what a probability exp(S - L) is off by, relative: a logit is a sum of d products in 32 bits, off by at most d 2^-24 tau sum |q k|, and what goes
    through the exponential, the row statistic and the moves of the reference adds a few steps of 2^-24 of the exponent.
    O: weights rounded to 16 bits (u each) and divided by their own sum: u (sum w |v| + |O|), and u |O| for its own rounding.  fp16 probabilities below 2^-14 are off by up to
    2^-25 whatever their size, against a sum of at least 2^-8 (the reference lags by no more).
    dV: (u + 2 rho) sum P |dO|, and half a step.  dS = P (dP - D): dP in 32 bits, D = dO . O with O as rounded, so off by sum |dO| (O's bound); dS is rounded once: e in all, and
    dQ, dK are off by tau sum e |k|, tau sum e |q|, and half a step.  Sums over n rows in 32 bits: n 2^-24 of the sum of the sizes.
    """

    def __init__(self, q, k, v, do, tau, window, sinks, length=None, keep=None, factor=1.0, o_rounded=True):
        self.dtype = q.dtype
        u = torch.finfo(q.dtype).eps / 2
        tiny = 2.0 ** -25 if q.dtype == torch.float16 else 0.0
        q, k, v, do = (x.double() for x in (q, k, v, do))
        N, d = q.shape
        seen = visible(N, window, sinks, length, q.device)
        some = seen.any(-1, keepdim=True)
        s = (tau * torch.mm(q, k.t())).masked_fill(~seen, -math.inf)
        size = (tau * torch.mm(q.abs(), k.abs().t())).masked_fill(~seen, 0.0).amax(-1, keepdim=True)
        rho = (d + 32) * 2.0 ** -24 * (size + 8.0)
        self.L = torch.logsumexp(s, -1)
        p = torch.where(some, torch.exp(s - torch.where(some, self.L[:, None], torch.zeros_like(size))), torch.zeros_like(s))
        n = seen.sum(-1, keepdim=True).double()
        self.bL = (rho + (n / 32 + 16) * 2.0 ** -24 + 2.0 ** -22 * torch.nan_to_num(self.L, neginf=0.0)[:, None].abs()).squeeze(-1)
        z = p if keep is None else p * keep * factor
        self.O = torch.mm(z, v)
        spread = torch.mm(z, v.abs())
        # (the kernel divides by the sum of all rounded weights, dropped ones among them: relative errors of the two are at most u each)
        b = (2 * u + 2 * rho) * spread + n * 2.0 ** -24 * spread
        if tiny:
            b = b + n * tiny * 2.0 ** 8 * factor * v.abs().amax()
        self.bO32 = torch.where(some, b + 2.0 ** -24, torch.zeros_like(b))
        self.bO = torch.where(some, self.bO32 + u * (self.O.abs() + self.bO32) + tiny, torch.zeros_like(b))
        # gradients
        dp = torch.mm(do, v.t())
        Z = None if keep is None else keep * factor
        dpz = dp if Z is None else dp * Z
        D = (do * self.O).sum(-1, keepdim=True)
        off_d = (do.abs() * (self.bO if o_rounded else self.bO32)).sum(-1, keepdim=True) + d * 2.0 ** -23 * (do.abs() * self.O.abs()).sum(-1, keepdim=True)
        ds = p * (dpz - D)
        off_dp = d * 2.0 ** -23 * torch.mm(do.abs(), v.abs().t()) * (1.0 if Z is None else Z)
        rho2 = 2 * rho + 2.0 ** -20
        e = p * (off_d + off_dp) * (1 + u) + (u + 2 * rho2) * ds.abs() + torch.where(seen, torch.full_like(p, tiny), torch.zeros_like(p))
        self.dQ, self.dK, self.dV = tau * torch.mm(ds, k), tau * torch.mm(ds.t(), q), torch.mm(z.t(), do)
        e = e + N * 2.0 ** -24 * ds.abs()
        bQ, bK = tau * torch.mm(e, k.abs()), tau * torch.mm(e.t(), q.abs())
        ev = (u + 2 * rho2 + N * 2.0 ** -24) * z + torch.where(seen, torch.full_like(p, tiny * factor), torch.zeros_like(p))
        bV = torch.mm(ev.t(), do.abs())
        self.bQ, self.bK, self.bV = (x + u * (g.abs() + x) + (tiny or 2.0 ** -134) for x, g in ((bQ, self.dQ), (bK, self.dK), (bV, self.dV)))
        self.some = some.squeeze(-1)


def assert_within(got, want, bound, what):
    got = got.detach().double()
    off = torch.where(got == want, torch.zeros_like(want), (got - want).abs())   # (infinities)
    bad = ~(off <= bound)
    if bad.any():
        i = tuple(x[0].item() for x in bad.nonzero(as_tuple=True))
        raise AssertionError(f"{what}{list(i)}: {got[i].item()} for {want[i].item()}, bound {bound[i].item()}; {int(bad.sum())} of {bad.numel()} beyond")


def relative(got, want):
    return float((got.double() - want).norm() / want.norm().clamp(min=1e-30))
