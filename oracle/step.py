"""What a decoder's step runs around its attention, in 64 bits, straight from the definitions: torch tensors of any type
in, float64 (or whole numbers) out.  Nothing here comes from the library."""
import math

import torch

MOST = {"i8": 127.0, "e4m3": 448.0}


def norm(x, weight, eps, offset=0.0, residual=None):
    """The sum s, the normed rows y (NaN where a row is no finite numbers) and the largest |y| of each."""
    s = x.double() if residual is None else x.double() + residual.double()
    w = weight.double() + offset
    y = s * w / torch.sqrt((s * s).mean(-1, keepdim=True) + eps)
    y = torch.where(torch.isfinite(y).all(-1, keepdim=True), y, torch.full_like(y, math.nan))
    return s, y, y.abs().amax(-1)


def norm_backward(total, weight, dy, eps, offset=0.0, dtotal=None):
    """dx, dweight, and of both the sums of magnitudes that their roundings are relative to."""
    s, d, w = total.double(), dy.double(), weight.double() + offset
    r = 1.0 / torch.sqrt((s * s).mean(-1, keepdim=True) + eps)
    u, g = s * r, d * w
    mean = (g * u).mean(-1, keepdim=True)
    last = torch.zeros_like(s) if dtotal is None else dtotal.double()
    # (each term of the mean has the weight's rounding, so that what it is off by goes by the terms' magnitudes)
    spread = (g * u).abs().mean(-1, keepdim=True)
    return r * (g - u * mean) + last, (d * u).sum(0), r * (g.abs() + u.abs() * spread) + last.abs(), (d * u).abs().sum(0)


def codes4(weights):
    """[n, k / 2] bytes -> [n, k] codes 0 .. 15."""
    w = weights.to(torch.int16)
    return torch.stack((w & 15, w >> 4), -1).flatten(-2)


def linear4(x, weights, scales, group, zeros=None, row_scales=None, bias=None):
    """The result, and sum |x| |c - z| |s|: what the sums' roundings are relative to."""
    n, k = weights.shape[0], 2 * weights.shape[1]
    c = codes4(weights).double().view(n, k // group, group)
    z = torch.full((n, k // group, 1), 8.0, dtype=torch.float64, device=weights.device) if zeros is None else zeros.double().unsqueeze(-1)
    s = scales.double().unsqueeze(-1)
    r = torch.ones(x.shape[0], 1, dtype=torch.float64, device=x.device) if row_scales is None else row_scales.double().unsqueeze(-1)
    b = torch.zeros(n, dtype=torch.float64, device=x.device) if bias is None else bias.double()
    y = torch.mm(x.double(), ((c - z) * s).view(n, k).t().contiguous()) * r + b
    size = torch.mm(x.double().abs(), ((c - z).abs() * s.abs()).view(n, k).t().contiguous()) * r.abs() + b.abs()
    return y, size


def verify(target, drafted, uniforms, draft=None, lengths=None):
    """tokens and accepted, sequence by sequence."""
    B, D = drafted.shape
    V = target.shape[2]
    tokens = torch.full((B, D + 1), -1, dtype=torch.int32)
    accepted = torch.zeros(B, dtype=torch.int32)
    drafted = drafted.cpu()
    u = uniforms.double().cpu()
    for b in range(B):
        n = D if lengths is None else min(max(int(lengths[b]), 0), D)
        a = 0
        while a < n:
            x = int(drafted[b, a])
            if not 0 <= x < V:
                break
            q = 1.0 if draft is None else float(draft[b, a, x].double())
            if not float(u[b, a]) * q < float(target[b, a, x].double()):
                break
            tokens[b, a] = x
            a += 1
        accepted[b] = a

        def clean(w):
            return torch.where((w > 0) & (w < math.inf), w, torch.zeros_like(w))
        p = target[b, a].double().cpu()
        w = clean(p)
        if a < n:
            if draft is not None:
                less = clean(p - draft[b, a].double().cpu())
            else:
                less = w.clone()
                if 0 <= int(drafted[b, a]) < V:
                    less[int(drafted[b, a])] = 0
            w = less if less.sum() > 0 else w
        upto = torch.cumsum(w, 0)
        over = torch.nonzero((upto > float(u[b, D]) * float(upto[-1])) & (w > 0)).flatten()
        some = torch.nonzero(w > 0).flatten()
        tokens[b, a] = int(over[0]) if len(over) else int(some[-1]) if len(some) else -1
    return tokens, accepted
