"""The norm of rows with the rotation, its gradients and the bounds of a kernel's errors, in 64 bits."""
import torch

from tests import paged_helpers as ph


def turn(x, positions, f, interleaved, magnitude, inverse=False):
    """x [tokens, heads, d] turned; f may be None."""
    if f is None:
        return x.clone(), torch.zeros_like(x)
    return ph.turned(x, positions, f, interleaved, magnitude, inverse)


def sizes(x, f, interleaved, magnitude):
    """What a turned column is made of: |x_a| + |x_b| times the factor where it turns."""
    y = x.abs().clone()
    if f is None:
        return y
    r = 2 * f.numel()
    a = torch.arange(0, r, 2) if interleaved else torch.arange(r // 2)
    b = a + 1 if interleaved else a + r // 2
    both = abs(magnitude) * (x[..., a].abs() + x[..., b].abs())
    y[..., a], y[..., b] = both, both
    return y


def forward(x, w, eps, positions, f, interleaved=False, magnitude=1.0):
    """(y, bound) of rows x [tokens, heads, d].  The sum of squares is one of d products in 32 bits by 16 and then by at most 8, with a product, a sum, a root and a quotient
    behind it, and two products: under 40 steps of 2^-24 of the normed value in all, and half a step of the type at the end."""
    x64, w64 = x.double(), w.double()
    normed = x64 * torch.rsqrt(x64.square().mean(-1, keepdim=True) + eps) * w64
    y, bound = turn(normed, positions, f, interleaved, magnitude)
    bound = bound + 40 * 2.0 ** -24 * sizes(normed, f, interleaved, magnitude)
    return y, bound + ph.rounding(y.abs() + bound, x.dtype)


def gradients(x, w, dy, eps, positions, f, interleaved=False, magnitude=1.0):
    """(dx, its bound, dw, its bound before it is rounded).  rho: the steps of r and of a sum over a row, relative to the sum of its terms' sizes; a term of dw is off by rho of
    itself, and a sum of R of them in 32 bits by at most R steps of 2^-24 of the sum of their sizes."""
    x64, w64 = x.double(), w.double()
    rho = 48 * 2.0 ** -24
    g, bg = turn(dy.double(), positions, f, interleaved, magnitude, inverse=True)
    bg = bg + 2.0 ** -23 * sizes(dy.double(), f, interleaved, magnitude)
    r = torch.rsqrt(x64.square().mean(-1, keepdim=True) + eps)
    h, bh = g * w64, (bg + 2.0 ** -23 * g.abs()) * w64.abs()
    dx = r * (h - x64 * r * r * (h * x64).mean(-1, keepdim=True))
    bound = r * (bh + 3 * rho * h.abs() + x64.abs() * r * r * ((bh + 5 * rho * h.abs()) * x64.abs()).mean(-1, keepdim=True))
    terms, off = g * x64 * r, (bg + 3 * rho * g.abs()) * x64.abs() * r
    rows = tuple(range(x.dim() - 1))
    count = x.numel() // x.shape[-1]
    dw, bw = terms.sum(rows), (off + count * 2.0 ** -24 * terms.abs()).sum(rows)
    return dx, bound + ph.rounding(dx.abs() + bound, x.dtype), dw, bw


def over_batch(fn, x, *args, positions, dy=None, **kw):
    """fn for every entry of [B,H,N,d] tensors; sums over entries where there are four results."""
    x = x.detach().cpu()
    out = []
    for b in range(x.shape[0]):
        pos = positions if positions.dim() == 1 else positions[b]
        more = () if dy is None else (dy[b].detach().cpu().transpose(0, 1),)
        out.append(fn(x[b].transpose(0, 1), args[0], *more, *args[1:], pos, **kw))
    stack = lambda i: torch.stack([o[i].transpose(0, 1) for o in out])  # noqa: E731
    if dy is None:
        return stack(0), stack(1)
    count = x.numel() // x.shape[-1]
    dw = sum(o[2] for o in out)
    # (the sum over entries goes on in 32 bits)
    return stack(0), stack(1), dw, sum(o[3] for o in out) + count * 2.0 ** -24 * sum(o[2].abs() for o in out) + 2.0 ** -22 * dw.abs()
