"""The operators around a decoder's attention in 64 bits, straight from their definitions: torch tensors of
any type in, float64 out.  Nothing here comes from the library."""
import math

import torch

MOST = {"i8": 127.0, "e4m3": 448.0}


def rotary(x, positions, frequencies, layout="half", magnitude=1.0, backward=False):
    """x [tokens, heads, D]: the first R = 2 len(frequencies) elements of a head turn, pair by pair."""
    y = x.double().clone()
    n = len(frequencies)
    angle = positions.double()[:, None] * torch.tensor([float(f) for f in frequencies], dtype=torch.float64, device=x.device)
    c, s = angle.cos()[:, None] * magnitude, angle.sin()[:, None] * magnitude
    s = -s if backward else s
    first, second = (slice(0, n), slice(n, 2 * n)) if layout == "half" else (slice(0, 2 * n, 2), slice(1, 2 * n, 2))
    a, b = x.double()[..., first], x.double()[..., second]
    y[..., first] = a * c - b * s
    y[..., second] = b * c + a * s
    return y


def encode(rows, storage):
    """Codes (as the storage's type) and scales of rows, with the roundings to 32 bits that the format names."""
    x = rows.float()
    a = x.abs().amax(-1)
    bad = ~torch.isfinite(a)
    # (quotients of two tensors: with a number torch multiplies by a reciprocal, which is rounded once more)
    most = torch.full_like(a, MOST[storage])
    up = torch.where(a < 2.0 ** -100, 2.0 ** 100, 1.0)
    inverse = torch.where((a > 0) & ~bad, most / (a * up), torch.zeros_like(a))
    y = torch.where(bad[..., None], torch.zeros_like(x), x * up[..., None] * inverse[..., None]).clamp(-MOST[storage], MOST[storage])
    codes = torch.round(y).to(torch.int8) if storage == "i8" else y.to(torch.float8_e4m3fn)
    return codes, torch.where(bad, torch.full_like(a, math.nan), a / most)


def stored_rows(pages, slots):
    """Values that the rows of the slots stand for: keys, values [n, kv_heads, D] in float64; None for a slot outside."""
    size = pages[0].shape[2]
    inside = (slots >= 0) & (slots < pages[0].shape[0] * size)
    at = torch.where(inside, slots, torch.zeros_like(slots))
    out = []
    for i in range(2):
        x = pages[i][at // size, :, at % size].double()
        if len(pages) == 4:
            x = x * pages[2 + i][at // size, :, at % size].double()[..., None]
        out.append(torch.where(inside[:, None, None], x, torch.zeros_like(x)))
    return out, inside


def _sequences(q, lengths, table, pages, prefix_table, prefix_length):
    """Sequence by sequence: its number, its query rows [heads, 1, D] and the keys and values they see [heads, tokens, D]."""
    size, count = pages[0].shape[2], pages[0].shape[0]
    group = q.shape[1] // pages[0].shape[1]

    def slots_of(row, n):
        t = torch.arange(n, device=q.device)
        page = row[t // size].long() if n else t
        page = torch.where((page >= 0) & (page < count), page, torch.full_like(page, -1))
        return torch.where(page >= 0, page * size + t % size, torch.full_like(page, -1))

    shared = slots_of(prefix_table, prefix_length) if prefix_length else None
    for b in range(q.shape[0]):
        n = max(0, min(int(lengths[b]), table.shape[1] * size))
        slots = slots_of(table[b], n)
        if shared is not None:
            slots = torch.cat((shared, slots))
        slots = slots[slots >= 0]
        if slots.numel() == 0:
            continue
        (k, v), _ = stored_rows(pages, slots)
        k, v = (x.repeat_interleave(group, 1).transpose(0, 1) for x in (k, v))
        yield b, q[b].double()[:, None, :], k, v


def attend(q, lengths, table, pages, scale, prefix_table=None, prefix_length=0):
    """Attention of one query token a sequence, [batch, heads, D]; also the largest |value|, the largest sum of |q k| and the
    largest sum of |k| that each result depends on (what a bound of the rounding errors is made of)."""
    batch, heads, D = q.shape
    out = torch.zeros((batch, heads, D), dtype=torch.float64, device=q.device)
    most = torch.zeros((batch, heads), dtype=torch.float64, device=q.device)
    sums, keys = (torch.zeros((batch, heads), dtype=torch.float64, device=q.device) for _ in range(2))
    for b, qb, k, v in _sequences(q, lengths, table, pages, prefix_table, prefix_length):
        products = (k * qb).sum(-1)
        out[b] = (torch.softmax(products * scale, -1)[..., None] * v).sum(1)
        most[b] = v.abs().amax((1, 2))
        sums[b] = (k * qb).abs().sum(-1).amax(-1)
        keys[b] = k.abs().sum(-1).amax(-1)
    return out, most, sums, keys


def attend_sizes(q, lengths, table, pages, scale, prefix_table=None, prefix_length=0):
    """What attend's results are the sums of: sum p |v| / sum p and sum |v|, [batch, heads, D], and the largest p |v| / sum p, the
    largest of all elements of a token's value, [batch, heads]."""
    share, whole = (torch.zeros(q.shape, dtype=torch.float64, device=q.device) for _ in range(2))
    heavy = torch.zeros(q.shape[:2], dtype=torch.float64, device=q.device)
    for b, qb, k, v in _sequences(q, lengths, table, pages, prefix_table, prefix_length):
        p = torch.softmax((k * qb).sum(-1) * scale, -1)
        share[b] = (p[..., None] * v.abs()).sum(1)
        whole[b] = v.abs().sum(1)
        heavy[b] = (p * v.abs().amax(-1)).amax(-1)
    return share, whole, heavy
