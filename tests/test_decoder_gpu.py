"""Rotary positions, the cache of keys and values, and attention over it on the GPU, against 64 bits
(oracle/decoder.py), at the sizes, strides and masks where they can go wrong."""
import math

import pytest
import torch

from oracle import decoder as plain

pytestmark = pytest.mark.gpu

TYPES = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
STORED = {"i8": torch.int8, "e4m3": torch.float8_e4m3fn}


@pytest.fixture(scope="module")
def ctx():
    from paper_2103_05288_amd import Context
    c = Context(0)
    yield c
    torch.cuda.synchronize()
    c.close()


def _half_step(dtype):
    return torch.finfo(dtype).eps / 2


def _generator(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return g


def _normal(shape, dtype, g, std=1.0):
    return torch.empty(shape, dtype=torch.float32, device="cuda").normal_(0.0, std, generator=g).to(dtype)


def _inside(got, want, bound, what):
    off = (got.double() - want).abs()
    bad = ~(off <= bound)
    assert not bad.any(), f"{what}: {int(bad.sum())} of {off.numel()} values outside the bound, worst {float((off - bound).max()):.3g} over it"


# ---- rotary positions ------------------------------------------------------------------------------


def _rotary_bound(x, positions, frequencies, layout, magnitude, dtype, want):
    """Sine and cosine: at most two units in the last place (2 * 2^-23 at most) and a reduced angle rounded to 32 bits
    (2^-26 quarter turns, 2^-25 in radians); two products and a sum, a half step each; the result's own half step."""
    n = len(frequencies)
    size = x.double().abs()
    both = size.clone()
    first, second = (slice(0, n), slice(n, 2 * n)) if layout == "half" else (slice(0, 2 * n, 2), slice(1, 2 * n, 2))
    both[..., first] = both[..., second] = size[..., first] + size[..., second]
    # (the angle itself, in 64 bits: the position times a rounded constant)
    angle = float(positions.abs().max() if positions.numel() else 0) * max(abs(float(f)) for f in frequencies) * 2.0 ** -51
    return _half_step(dtype) * want.abs() + both * abs(magnitude) * (2 * 2.0 ** -23 + 2.0 ** -25 + 4 * 2.0 ** -24 + angle) + torch.finfo(dtype).tiny * 2.0 ** -8


@pytest.mark.parametrize("dtype,D,R,layout,tokens,heads,far", [
    ("bf16", 128, 128, "half", 1, (32, 8), 4096),
    ("bf16", 128, 128, "interleaved", 777, (4, 1), 1 << 20),
    ("f16", 80, 32, "half", 130, (5, 5), 8192),
    ("f16", 80, 26, "interleaved", 33, (3, 1), 100),
    ("f32", 64, 64, "half", 4099, (2, 3), 1 << 20),
    ("f32", 256, 254, "interleaved", 9, (7, 1), 1 << 22),
    ("f32", 256, 2, "half", 17, (1, 1), 64),
    ("bf16", 2, 2, "interleaved", 65, (3, 2), 64),
    ("f16", 250, 250, "half", 3, (2, 2), 64),
])
@pytest.mark.parametrize("backward", [False, True])
def test_rotary_matches_64_bits(ctx, dtype, D, R, layout, tokens, heads, far, backward):
    from paper_2103_05288_amd import rotary_frequencies
    frequencies, magnitude = rotary_frequencies(R, scaling="by_parts", factor=8.0, original_length=2048)
    h = ctx.register_rotary(dtype, D, frequencies, layout=layout, magnitude=magnitude)
    g = _generator(tokens * D + R)
    t = TYPES[dtype]
    # rows of one product: other heads in between, so that strides are no sizes of the tensors
    rows = _normal((tokens, sum(heads) + 3, D), t, g)
    xs = [rows[:, 1:1 + heads[0]], rows[:, 2 + heads[0]:2 + heads[0] + heads[1]]]
    positions = torch.randint(0, far, (tokens,), generator=g, device="cuda", dtype=torch.int32)
    wide = torch.full((tokens, heads[1] + 1, D + 6), 7.0, dtype=t, device="cuda")
    ys = [torch.full((tokens, heads[0], D), math.nan, dtype=t, device="cuda"), wide[:, :heads[1], 3:3 + D]]
    h.launch(positions, xs, ys, backward=backward)
    for x, y in zip(xs, ys):
        want = plain.rotary(x, positions, frequencies, layout, magnitude, backward)
        _inside(y, want, _rotary_bound(x, positions, frequencies, layout, magnitude, t, want), "rotary")
        assert torch.equal(y[..., R:], x[..., R:])
    assert (wide[:, heads[1]:] == 7).all() and (wide[..., :3] == 7).all() and (wide[..., 3 + D:] == 7).all()
    # in place, and the same numbers of 64-bit positions
    held = [x.clone() for x in xs]
    h.launch(positions.long(), xs, xs, backward=backward)
    for x, y in zip(xs, ys):
        assert torch.equal(x, y)
    for i in (0, 1 + heads[0], 2 + sum(heads)):       # the heads between them are as they were
        assert torch.isfinite(rows[:, i]).all()
    del held


@pytest.mark.parametrize("dtype,D,R,layout", [("f32", 96, 64, "half"), ("bf16", 128, 128, "interleaved")])
def test_rotary_of_many_tokens(ctx, dtype, D, R, layout):
    """More than 64 MiB: the version past the caches."""
    from paper_2103_05288_amd import rotary_frequencies
    frequencies, magnitude = rotary_frequencies(R, scaling="linear", factor=2.0)
    h = ctx.register_rotary(dtype, D, frequencies, layout=layout, magnitude=magnitude)
    g = _generator(77)
    t = TYPES[dtype]
    rows = _normal((30011, 8, D), t, g)
    x = rows[:, 1:6]
    y = torch.empty((30011, 5, D), dtype=t, device="cuda")
    assert 2 * x.numel() * x.element_size() >= 64 << 20
    positions = torch.randint(0, 1 << 17, (30011,), generator=g, device="cuda")
    h.launch(positions, [x], [y])
    want = plain.rotary(x, positions, frequencies, layout, magnitude)
    _inside(y, want, _rotary_bound(x, positions, frequencies, layout, magnitude, t, want), "rotary")
    h.launch(positions, [x], [x])
    assert torch.equal(x, y)


def test_rotary_positions_below_zero_and_at_rest(ctx):
    from paper_2103_05288_amd import rotary_frequencies
    frequencies, magnitude = rotary_frequencies(64)
    h = ctx.register_rotary("f32", 64, frequencies)
    x = _normal((5, 2, 64), torch.float32, _generator(3))
    positions = torch.tensor([0, -1, -12345, 1 << 24, 7], device="cuda")
    y = torch.empty_like(x)
    h.launch(positions, [x], [y])
    want = plain.rotary(x, positions, frequencies)
    _inside(y, want, _rotary_bound(x, positions, frequencies, "half", 1.0, torch.float32, want), "rotary")
    assert torch.equal(y[0], x[0])
    # the same row for every head (a broadcast operand), nothing at all, and tensors without heads
    one = x[:, :1].expand(5, 2, 64)
    h.launch(positions, [one], [y])
    assert torch.equal(y[:, 0], y[:, 1])
    h.launch(positions[:0], [x[:0]], [y[:0]])
    h.launch(positions, [x[:, :0], x], [y[:, :0], y])


def test_rotary_gradient_is_the_transposed_map(ctx):
    """<dy, f(x)> = <df(dy), x> for a linear f, and f(x + h e) - f(x) = h times the gradient's column."""
    from paper_2103_05288_amd import rotary_frequencies
    for layout in ("half", "interleaved"):
        frequencies, magnitude = rotary_frequencies(32, scaling="by_parts", factor=4.0, original_length=100)
        h = ctx.register_rotary("f32", 48, frequencies, layout=layout, magnitude=magnitude)
        g = _generator(11)
        x, dy = _normal((6, 3, 48), torch.float32, g), _normal((6, 3, 48), torch.float32, g)
        positions = torch.randint(0, 3000, (6,), generator=g, device="cuda")
        y, dx = torch.empty_like(x), torch.empty_like(x)
        h.launch(positions, [x], [y])
        h.launch(positions, [dy], [dx], backward=True)
        lhs, rhs = (dy.double() * y.double()).sum(), (dx.double() * x.double()).sum()
        size = (dy.double().abs() * y.double().abs()).sum()
        assert abs(lhs - rhs) <= size * magnitude * 2 * 16 * 2.0 ** -24
        # differences: column (t=2, head 1, element 5) of the map, by a step of 1 from the zero vector
        e = torch.zeros_like(x)
        e[2, 1, 5] = 1.0
        h.launch(positions, [e], [y])
        back = torch.empty_like(x)
        for at in y.nonzero().tolist():
            one = torch.zeros_like(x)
            one[tuple(at)] = 1.0
            h.launch(positions, [one], [back], backward=True)
            assert abs(float(back[2, 1, 5]) - float(y[tuple(at)])) <= magnitude * 4 * 2.0 ** -24


# ---- store and load --------------------------------------------------------------------------------


def _cache(ctx, dtype, storage, D):
    return ctx.register_cache(dtype, D, storage=storage)


def _empty_pages(dtype, storage, pages, kv, size, D, fill):
    shape = (pages, kv, size, D)
    if storage not in STORED:
        return [torch.full(shape, fill, dtype=TYPES[dtype], device="cuda") for _ in range(2)]
    return [torch.full(shape, fill, dtype=torch.float32, device="cuda").to(STORED[storage]) for _ in range(2)] + \
           [torch.full(shape[:3], fill, dtype=torch.float32, device="cuda") for _ in range(2)]


def _bits(t):
    return t.contiguous().view(torch.uint8)


def _same(got, want, what):
    """Equal values; a NaN is as good as another."""
    differ = (got.float() != want.float()) & ~(torch.isnan(got.float()) & torch.isnan(want.float()))
    n = int(differ.sum())
    assert n == 0, f"{what}: {n} of {differ.numel()} differ, first at {differ.nonzero()[0].tolist()}: {got[differ][0].item()}, {want[differ][0].item()}"


@pytest.mark.parametrize("dtype,storage,D,kv,size,tokens", [
    ("bf16", "i8", 128, 8, 16, 1),
    ("bf16", "i8", 128, 3, 64, 401),
    ("bf16", "e4m3", 64, 2, 8, 77),
    ("f16", "e4m3", 80, 1, 128, 300),
    ("f16", "i8", 256, 2, 16, 33),
    ("f16", "i8", 16, 5, 8, 19),
    ("bf16", "bf16", 128, 2, 16, 50),
    ("f16", "f16", 48, 3, 8, 21),
])
def test_store_and_load(ctx, dtype, storage, D, kv, size, tokens):
    cache = _cache(ctx, dtype, storage, D)
    g = _generator(D * tokens + size)
    t = TYPES[dtype]
    pages = -(-tokens // size) + 4
    rows = _normal((tokens, 3 * kv, D), t, g, 3.0)
    k, v = rows[:, kv:2 * kv], rows[:, 2 * kv:]
    if tokens > 10:
        k[3] = 0.0                                             # a row of nothing
        v[4, :, 1] = math.inf
        k[5, 0, D - 1] = math.nan
        v[6] = v[6] * 1e-3 if dtype == "f16" else v[6] * 1e-30
        k[7, :, 0] = torch.finfo(t).max
        v[8] = torch.finfo(t).smallest_normal / 4              # below the normal numbers
    slots = torch.randperm(pages * size, generator=g, device="cuda")[:tokens]
    if tokens > 10:
        slots[0], slots[9], slots[10] = -1, pages * size, -(1 << 40)
    stored = _empty_pages(dtype, storage, pages, kv, size, D, 5.0)
    want = [p.clone() for p in stored]
    cache.store([k, v], slots, stored)
    live = (slots >= 0) & (slots < pages * size)
    at = slots[live]
    for i, x in enumerate((k[live], v[live])):
        if storage in STORED:
            codes, scales = plain.encode(x, storage)
            want[i].view(torch.uint8)[at // size, :, at % size] = _bits(codes)
            want[2 + i][at // size, :, at % size] = scales
        else:
            want[i][at // size, :, at % size] = x
    for i, (p, w) in enumerate(zip(stored, want)):             # every other place as it was
        _same(p, w, f"pages {i}")
    wide = torch.full((tokens, kv + 1, D + 8), 9.0, dtype=t, device="cuda")
    back = [torch.empty((tokens, kv, D), dtype=t, device="cuda"), wide[:, 1:, 5:5 + D]]
    cache.load(slots, stored, back)
    rows64, inside = plain.stored_rows(stored, slots)
    for i, (y, x, w) in enumerate(zip(back, (k, v), rows64)):
        assert (y[~inside] == 0).all()
        fine = torch.isfinite(w)
        assert torch.equal(torch.isnan(w), torch.isnan(y.double()))
        if storage in STORED:
            # (a product of two 32-bit numbers, rounded, then rounded to the type; overflow to infinity included)
            want_t = (stored[i].float()[at // size, :, at % size] * stored[2 + i][at // size, :, at % size][..., None]).to(t)
            _same(y[live], want_t, "rows read back")
            # back to what went in: half a step of the code, times the scale, and the roundings to 32 bits and to the type
            a = x.double().abs().amax(-1, keepdim=True)
            step = a / 127 / 2 if storage == "i8" else torch.maximum(x.double().abs() * 2.0 ** -4, a / 448 * 2.0 ** -10)
            bound = step * 1.001 + x.double().abs() * (4 * 2.0 ** -24 + _half_step(t)) + torch.finfo(t).tiny
            ok = ((w - x.double()).abs() <= bound) | ~fine | ~inside[:, None, None]
            assert ok.all()
        else:
            assert torch.equal(_bits(y[inside]), _bits(x[inside]))
    assert (wide[:, 0] == 9).all() and (wide[..., :5] == 9).all() and (wide[..., 5 + D:] == 9).all()
    cache.store([k[:0], v[:0]], slots[:0], stored)
    cache.load(slots[:0], stored, [back[0][:0], back[1][:0]])


@pytest.mark.parametrize("dtype,storage", [("bf16", "i8"), ("f16", "e4m3"), ("bf16", "bf16")])
def test_store_and_load_of_many_rows(ctx, dtype, storage):
    """More than 64 MiB: the versions past the caches."""
    cache = _cache(ctx, dtype, storage, 128)
    g = _generator(4)
    t = TYPES[dtype]
    tokens, kv, size = 20011, 6, 32
    rows = _normal((tokens, 2 * kv, 128), t, g, 2.0)
    k, v = rows[:, :kv], rows[:, kv:]
    pages = -(-tokens // size) + 1
    slots = torch.randperm(pages * size, generator=g, device="cuda")[:tokens]
    stored = _empty_pages(dtype, storage, pages, kv, size, 128, 0.0)
    cache.store([k, v], slots, stored)
    for i, x in enumerate((k, v)):
        if storage in STORED:
            codes, scales = plain.encode(x, storage)
            _same(stored[i][slots // size, :, slots % size], codes, "codes")
            _same(stored[2 + i][slots // size, :, slots % size], scales, "scales")
        else:
            _same(stored[i][slots // size, :, slots % size], x, "rows")
    back = [torch.empty((tokens, kv, 128), dtype=t, device="cuda") for _ in range(2)]
    cache.load(slots, stored, back)
    for i, y in enumerate(back):
        want = stored[i].float()[slots // size, :, slots % size]
        if storage in STORED:
            want = want * stored[2 + i][slots // size, :, slots % size][..., None]
        _same(y, want.to(t), "rows read back")


# ---- attention -------------------------------------------------------------------------------------


def _filled(dtype, storage, pages, kv, size, D, g, behind=None):
    """Pages of random rows."""
    x = [_normal((pages, kv, size, D), torch.float32, g) * _normal((D,), torch.float32, g).exp() for _ in range(2)]
    if storage not in STORED:
        return [y.to(TYPES[dtype]) for y in x]
    c = [plain.encode(y, storage) for y in x]
    return [c[0][0], c[1][0], c[0][1], c[1][1]]


def _poison(pages, dtype, storage, slots):
    """NaN, infinities and the lowest value into places that no token owns."""
    size = pages[0].shape[2]
    if slots.numel() == 0:
        return
    page, place = slots // size, slots % size
    values = torch.tensor([math.nan, math.inf, -math.inf, -3e38], device="cuda")[torch.arange(slots.numel(), device="cuda") % 4]
    if storage in STORED:
        pages[2][page, :, place] = values[:, None].expand(-1, pages[0].shape[1])
        pages[3][page, :, place] = values[:, None].expand(-1, pages[0].shape[1])
    else:
        x = values.to(TYPES[dtype])[:, None, None].expand(-1, pages[0].shape[1], pages[0].shape[3])
        pages[0][page, :, place] = x
        pages[1][page, :, place] = x


def _setup(dtype, storage, D, kv, group, size, lengths, prefix, g, spare=2):
    """A batch whose sequences own scattered pages; what is behind their last tokens is poisoned."""
    B = len(lengths)
    need = [-(-n // size) for n in lengths]
    np = -(-prefix // size)
    total = sum(need) + np + spare
    order = torch.randperm(total, generator=g, device="cuda").to(torch.int32)
    width = max(need + [1]) + 1
    table = torch.full((B, width), -1, dtype=torch.int32, device="cuda")
    at = np
    pages = _filled(dtype, storage, total, kv, size, D, g)
    free = []
    if prefix % size:
        free.append(int(order[np - 1]) * size + torch.arange(prefix % size, size, device="cuda"))
    for b, (n, m) in enumerate(zip(lengths, need)):
        table[b, :m] = order[at:at + m]
        at += m
        if n % size:
            free.append(int(table[b, m - 1]) * size + torch.arange(n % size, size, device="cuda"))
    _poison(pages, dtype, storage, torch.cat(free) if free else torch.zeros(0, dtype=torch.int64, device="cuda"))
    q = _normal((B, kv * group, D), TYPES[dtype], g, 1.5)
    return {"q": q, "lengths": torch.tensor(lengths, dtype=torch.int32, device="cuda"), "table": table, "pages": pages,
            "prefix_table": order[:np].contiguous(), "prefix": prefix}


def _attend_bound(dtype, storage, s, want, most, sums, keys, scale):
    """|out - exact| where every weight is off by at most w, relatively: 2 w max|v| and the result's own half step.
    A weight's parts: its score (D products, exact, summed in 32 bits, then two products), the power of two by the
    hardware (2^-22), its rounding -- to half precision with 8-bit storage, otherwise or for fp16 results to two
    numbers -- and sums over n tokens in 32 bits.  bf16 queries for 8-bit keys are half-precision numbers relative to the
    largest of them: of each, half of its smallest step 2^-24 may be lost, 2^-25 of the largest |q| (which has a factor of
    up to two in it) times the sum of |k|.  Half precision loses below 2^-25 of the largest product of a weight
    and a value's scale: n of those."""
    D = s["q"].shape[2]
    n = float(s["prefix"] + max(0, int(s["lengths"].max()) if s["lengths"].numel() else 0))
    one = 2.0 ** -11 if storage in STORED and dtype == "bf16" else 2.0 ** -16
    score = sums * scale * ((D + 4) * 2.0 ** -24)
    if storage in STORED and dtype == "bf16":
        score = score + scale * 2.0 ** -25 * float(s["q"].abs().max()) * keys
    w = one + score + 2.0 ** -22 + 4 * n * 2.0 ** -24
    return _half_step(TYPES[dtype]) * want.abs() + (2 * w * most)[..., None] * 1.01


def _run(cache, s, stream=None, out=None, workspace=None):
    B, H, D = s["q"].shape
    kv, size = s["pages"][0].shape[1], s["pages"][0].shape[2]
    if workspace is None:
        need = cache.workspace_bytes(B, H, kv, s["table"].shape[1] * size, s["prefix"], page_size=size)
        workspace = torch.empty(max(need, 16), dtype=torch.uint8, device="cuda").fill_(255)      # (as NaN)
    out = torch.full((B, H, D), math.nan, dtype=s["q"].dtype, device="cuda") if out is None else out
    more = {"prefix_table": s["prefix_table"], "prefix_length": s["prefix"]} if s["prefix"] else {}
    cache.attend(s["q"], s["lengths"], s["table"], s["pages"], out, workspace=workspace, stream=stream, **more)
    return out, workspace


def _check(cache, dtype, storage, s, scale, got=None):
    got = _run(cache, s)[0] if got is None else got
    want, *sizes = plain.attend(s["q"], s["lengths"], s["table"], s["pages"], scale, s["prefix_table"], s["prefix"])
    _inside(got, want, _attend_bound(dtype, storage, s, want, *sizes, scale), f"attention {dtype} {storage}")
    return got


LENGTHS = [0, 1, 7, 8, 9, 31, 32, 33, 127, 128, 129, 1000, 2, 0, 64]


@pytest.mark.parametrize("dtype,storage,D", [("bf16", "bf16", 128), ("bf16", "i8", 128), ("bf16", "e4m3", 64), ("f16", "f16", 80), ("f16", "i8", 96),
                                             ("f16", "e4m3", 256), ("bf16", "bf16", 256), ("bf16", "i8", 16), ("f16", "f16", 192), ("bf16", "e4m3", 32)])
@pytest.mark.parametrize("kv,group,size,prefix", [(2, 1, 8, 0), (1, 8, 16, 0), (2, 5, 64, 0), (1, 16, 8, 77), (2, 3, 128, 640), (1, 17, 16, 5), (1, 40, 32, 130)])
def test_attention_matches_64_bits(ctx, dtype, storage, D, kv, group, size, prefix):
    cache = _cache(ctx, dtype, storage, D)
    s = _setup(dtype, storage, D, kv, group, size, LENGTHS, prefix, _generator(D + 7 * group + prefix))
    got = _check(cache, dtype, storage, s, 1.0 / math.sqrt(D))
    if prefix == 0:
        assert (got[0] == 0).all() and (got[13] == 0).all()


@pytest.mark.parametrize("storage", ["bf16", "i8"])
def test_attention_of_one_long_sequence(ctx, storage):
    cache = _cache(ctx, "bf16", storage, 128)
    s = _setup("bf16", storage, 128, 2, 4, 16, [30011], 0, _generator(5))
    # scores that rise along the cache, so that the running maximum moves again and again
    q = s["q"]
    page = s["table"][0][: -(-30011 // 16)].long()
    ramp = torch.linspace(0.0, 6.0, page.numel(), device="cuda")[:, None]
    if storage == "i8":
        s["pages"][2][page] *= 0.05 + ramp[:, None] * 0.2
        s["pages"][3][page] *= 2.0 ** (ramp[:, None] * 4 - 12)
    else:
        s["pages"][0][page] = (s["pages"][0][page].float() * (0.05 + ramp[:, None, None] * 0.2)).to(torch.bfloat16)
    s["pages"] = [torch.nan_to_num(p, nan=0.0, posinf=0.0, neginf=0.0) if p.dtype is not torch.int8 else p for p in s["pages"]]
    _check(cache, "bf16", storage, s, 1.0 / math.sqrt(128))
    del q


@pytest.mark.parametrize("dtype,storage,D", [("bf16", "i8", 128), ("bf16", "e4m3", 64), ("f16", "i8", 64), ("bf16", "bf16", 128)])
@pytest.mark.parametrize("batch,group,prefix,longest", [(3, 4, 0, 300), (2, 4, 0, 3000), (600, 2, 0, 40), (5, 4, 200, 40), (40, 4, 1500, 40), (300, 4, 2500, 40)])
def test_queries_of_other_rows_change_nothing(ctx, dtype, storage, D, batch, group, prefix, longest):
    """Query rows that hold NaN, infinities, the largest and the smallest numbers (a padded batch's rows may hold anything) beside
    ordinary ones: the ordinary ones' results are as without them."""
    cache = _cache(ctx, dtype, storage, D)
    lengths = [int(x) for x in torch.randint(1, longest, (batch,), generator=torch.Generator().manual_seed(3))]
    s = _setup(dtype, storage, D, 2, group, 16, lengths, prefix, _generator(17 + batch))
    q, plain_rows = s["q"], s["q"].clone()
    most = torch.finfo(q.dtype).max
    odd = torch.zeros(q.shape[:2], dtype=torch.bool, device="cuda")
    # (heads 1 of every kv head: beside ordinary rows of their sequence; and whole sequences beside other sequences)
    for at, value in ((0, most), (1, math.nan)):
        q[at, 1::group] = value
        odd[at, 1::group] = True
    q[batch - 1] = math.inf
    odd[batch - 1] = True
    got = _run(cache, s)[0]
    s["q"] = plain_rows
    want, *sizes = plain.attend(s["q"], s["lengths"], s["table"], s["pages"], 1.0 / math.sqrt(D), s["prefix_table"], s["prefix"])
    bound = _attend_bound(dtype, storage, s, want, *sizes, 1.0 / math.sqrt(D))
    _inside(got[~odd], want[~odd], bound[~odd], f"attention {dtype} {storage} beside other rows")
    # rows far smaller than their neighbours: what they turn to still counts
    if dtype == "bf16":
        s["q"] = plain_rows.clone()
        s["q"][0, 1::group] *= 2.0 ** 60
        s["q"][1] *= 2.0 ** -40
        scale_up = ctx.register_cache(dtype, D, storage, softmax_scale=2.0 ** 40 / math.sqrt(D))
        got = _run(scale_up, s)[0]
        s["q"] = plain_rows
        _inside(got[1], want[1], bound[1], f"attention {dtype} {storage}, rows of 2^-100 of others")


def test_attention_shared_prefix_of_a_large_batch(ctx):
    cache = _cache(ctx, "bf16", "i8", 128)
    g = _generator(8)
    lengths = [int(x) for x in torch.randint(0, 60, (70,), generator=torch.Generator().manual_seed(1))]
    _check(cache, "bf16", "i8", _setup("bf16", "i8", 128, 2, 4, 16, lengths, 2500, g), 1.0 / math.sqrt(128))
    # every sequence with nothing of its own
    _check(cache, "bf16", "i8", _setup("bf16", "i8", 128, 1, 8, 16, [0] * 5, 33, g), 1.0 / math.sqrt(128))


@pytest.mark.parametrize("dtype,storage,D", [("bf16", "bf16", 128), ("bf16", "i8", 64), ("f16", "e4m3", 256), ("f16", "f16", 80)])
@pytest.mark.parametrize("batch,kv,group,size,prefix", [(5, 1, 8, 8, 0), (5, 2, 3, 8, 77), (3, 1, 17, 64, 512), (300, 1, 2, 16, 100), (420, 2, 1, 8, 0), (900, 2, 4, 32, 0),
                                                        (900, 2, 4, 32, 40), (900, 2, 4, 32, 2000), (420, 2, 4, 8, 4000)])
def test_attention_of_short_sequences(ctx, dtype, storage, D, batch, kv, group, size, prefix):
    """Sequences of one chunk each, by four wavefronts, two or one; prefixes that are gone through in line, and shared ones."""
    cache = _cache(ctx, dtype, storage, D)
    some = [0, 1, 8, 31, 33, 100, 128, 200, 250, 129]
    lengths = [some[(7 * i + i // 3) % len(some)] if i else 240 for i in range(batch)]
    _check(cache, dtype, storage, _setup(dtype, storage, D, kv, group, size, lengths, prefix, _generator(batch + D)), 1.0 / math.sqrt(D))


def test_attention_strides_scale_and_rows_behind_the_batch(ctx):
    cache = ctx.register_cache("f16", 64, softmax_scale=0.3)
    s = _setup("f16", "f16", 64, 2, 2, 8, [5, 40, 300], 0, _generator(2))
    wide = torch.full((5, 6, 80), 3.0, dtype=torch.float16, device="cuda")
    out = wide[:3, 1:5, 7:71]
    rows = _normal((3, 9, 64), torch.float16, _generator(4))
    s["q"] = rows[:, 2:6]
    _run(cache, s, out=out)
    _check(cache, "f16", "f16", s, 0.3, got=out)
    assert (wide[3:] == 3).all() and (wide[:, 0] == 3).all() and (wide[:, 5] == 3).all() and (wide[..., :7] == 3).all() and (wide[..., 71:] == 3).all()
    s["q"] = rows[:1, :1].expand(3, 4, 64)                     # one row for all heads of all sequences
    _check(cache, "f16", "f16", s, 0.3)


def test_attention_pages_that_are_none_and_lengths_out_of_range(ctx):
    for storage in ("bf16", "e4m3"):
        cache = _cache(ctx, "bf16", storage, 128)
        s = _setup("bf16", storage, 128, 2, 4, 8, [100, 64, 9, 40], 50, _generator(6))
        count = s["pages"][0].shape[0]
        for b, at, page in ((0, 0, -1), (0, 5, count), (1, 3, 2 ** 31 - 1), (1, 7, -2 ** 31), (2, 0, -7), (2, 1, count + 1)):
            s["table"][b, at] = page
        s["prefix_table"][2] = count
        s["lengths"][3] = 10 ** 9                              # longer than the table: what the table holds, -1 behind it left out
        tail = s["table"][3, 5:].clone()
        assert (tail == -1).all()
        _check(cache, "bf16", storage, s, 1.0 / math.sqrt(128))
        s["lengths"][3] = -5
        _check(cache, "bf16", storage, s, 1.0 / math.sqrt(128))
        s["prefix"] = 0
        _check(cache, "bf16", storage, s, 1.0 / math.sqrt(128))


def test_attention_of_what_is_not_finite(ctx):
    """A NaN among a sequence's own keys makes its result NaN; another sequence's is none the worse."""
    for storage in ("bf16", "i8"):
        cache = _cache(ctx, "bf16", storage, 128)
        s = _setup("bf16", storage, 128, 1, 4, 8, [1, 300, 300], 0, _generator(9))
        for b, t in ((0, 0), (1, 257)):
            page, place = int(s["table"][b, t // 8]), t % 8
            (s["pages"][2] if storage == "i8" else s["pages"][0])[page, :, place] = math.nan
        got = _run(cache, s)[0]
        assert torch.isnan(got[:2]).all() and torch.isfinite(got[2]).all()


def test_attention_of_zero_values_and_of_tiny_and_huge_scales(ctx):
    cache = _cache(ctx, "bf16", "i8", 64)
    s = _setup("bf16", "i8", 64, 1, 2, 8, [200, 200, 77], 0, _generator(12), spare=0)
    for i in range(4):
        s["pages"][i] = torch.nan_to_num(s["pages"][i], nan=0.0, posinf=0.0, neginf=0.0) if i > 1 else s["pages"][i]
    rows = s["table"][0][:25].long()
    s["pages"][3][rows] = 0.0                                  # values that are all nothing
    rows = s["table"][1][:25].long()
    s["pages"][3][rows] *= 1e-20
    rows = s["table"][2][:10].long()
    s["pages"][3][rows] *= 1e20
    got = _check(cache, "bf16", "i8", s, 0.125)
    assert (got[0] == 0).all() and (got[1] != 0).any()


def test_attention_past_32_bits(ctx):
    """Pages whose elements are past 2^31 from the first: 2.3 GB of codes."""
    pages, kv, size, D = 140001, 8, 16, 128
    cache = _cache(ctx, "bf16", "i8", D)
    k, v = (torch.empty((pages, kv, size, D), dtype=torch.int8, device="cuda") for _ in range(2))
    ks, vs = (torch.empty((pages, kv, size), dtype=torch.float32, device="cuda") for _ in range(2))
    g = _generator(1)
    rows = [_normal((40, kv, D), torch.bfloat16, g) for _ in range(2)]
    table = torch.tensor([[140000, 3, 139999], [139990, 0, 0]], dtype=torch.int32, device="cuda")
    t = torch.arange(40, device="cuda")
    slots = table[0].long()[t // size] * size + t % size
    cache.store(rows, slots, (k, v, ks, vs))
    slots1 = table[1].long()[t[:7] // size] * size + t[:7] % size
    cache.store([r[:7] for r in rows], slots1, (k, v, ks, vs))
    back = [torch.empty_like(r) for r in rows]
    cache.load(slots, (k, v, ks, vs), back)
    for a, b in zip(rows, back):
        a, b = a.double(), b.double()
        assert ((a - b).abs() <= a.abs().amax(-1, keepdim=True) / 254 * 1.001 + a.abs() * 2.0 ** -8).all()
    s = {"q": _normal((2, 16, D), torch.bfloat16, g), "lengths": torch.tensor([40, 7], dtype=torch.int32, device="cuda"), "table": table,
         "pages": [k, v, ks, vs], "prefix": 0, "prefix_table": None}
    got = _check(cache, "bf16", "i8", s, 1.0 / math.sqrt(D))
    # a table for all of it: the version that reads past the caches
    s["table"] = torch.nn.functional.pad(table, (0, 60000), value=-1).contiguous()
    again = _check(cache, "bf16", "i8", s, 1.0 / math.sqrt(D))
    assert (again.double() - got.double()).abs().max() <= got.double().abs().max() * 2 * _half_step(torch.bfloat16)


@pytest.mark.parametrize("dtype,storage,batch,size", [("bf16", "i8", 700, 64), ("f16", "e4m3", 500, 64), ("bf16", "bf16", 120, 16), ("bf16", "bf16", 300, 64)])
def test_attention_of_large_caches(ctx, dtype, storage, batch, size):
    """Caches of more than 128 MiB, of sequences long and short, and of so many short ones that one or two wavefronts have each."""
    cache = _cache(ctx, dtype, storage, 128)
    short = size == 64
    lengths = [(37 * i) % 500 + 12 if short else (911 * i) % 3000 + 1 for i in range(batch)]
    s = _setup(dtype, storage, 128, 4, 2, size, lengths, 0, _generator(batch))
    s["table"] = s["table"][:, :8 if short else None].contiguous()
    own = 2 * s["pages"][0].numel() * s["pages"][0].element_size()
    assert min(own, batch * s["table"].shape[1] * size * 4 * 2 * 128 * s["pages"][0].element_size()) >= 128 << 20
    _check(cache, dtype, storage, s, 1.0 / math.sqrt(128))


def test_attention_captured_and_replayed_on_another_stream(ctx):
    """One graph, its lengths and pages changed between replays, eager work in between; a second graph with its own workspace."""
    cache = _cache(ctx, "bf16", "i8", 128)
    g = _generator(21)
    sets = [_setup("bf16", "i8", 128, 2, 4, 16, lengths, 100, g, spare=0) for lengths in ([5, 200, 0, 64], [300, 1, 77, 300], [0, 0, 0, 0])]
    width = max(s["table"].shape[1] for s in sets)
    for s in sets:
        s["table"] = torch.nn.functional.pad(s["table"], (0, width - s["table"].shape[1]), value=-1).contiguous()
    total = max(s["pages"][0].shape[0] for s in sets)
    for s in sets:
        s["pages"] = [torch.cat((p, torch.zeros((total - p.shape[0],) + p.shape[1:], dtype=p.dtype, device="cuda"))) for p in s["pages"]]
    eager = [_run(cache, s)[0].clone() for s in sets]
    static = {k: ([p.clone() for p in v] if k == "pages" else v.clone() if torch.is_tensor(v) else v) for k, v in sets[0].items()}
    side = torch.cuda.Stream()
    graphs = []
    for _ in range(2):
        out, ws = _run(cache, static)
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=side):
            _run(cache, static, out=out, workspace=ws)
        graphs.append((graph, out, ws))
    for turn in range(6):
        s = sets[turn % 3]
        for k, v in s.items():
            if k == "pages":
                for a, b in zip(static["pages"], v):
                    a.copy_(b)
            elif torch.is_tensor(v):
                static[k].copy_(v)
        for _, out, ws in graphs:
            out.fill_(math.nan)
            ws.fill_(255)
        torch.cuda.synchronize()
        graphs[0][0].replay()
        with torch.cuda.stream(side):
            graphs[1][0].replay()
        torch.cuda.synchronize()
        for _, out, _ in graphs:
            assert torch.equal(out, eager[turn % 3])
    # the launch's own stream argument
    torch.cuda.synchronize()
    out, ws = _run(cache, sets[1], stream=side.cuda_stream)
    side.synchronize()
    torch.cuda.synchronize()
    assert torch.equal(out, eager[1])


def test_the_step_of_a_token(ctx):
    """Prompt rows rotated and stored, then a new token a sequence: rotated, stored, attended, against 64 bits all along."""
    from paper_2103_05288_amd import rotary_frequencies
    D, kv, group, size = 64, 2, 3, 16
    H = kv * group
    frequencies, _ = rotary_frequencies(D)
    rotary = ctx.register_rotary("f16", D, frequencies)
    cache = ctx.register_cache("f16", D)
    g = _generator(31)
    prefix, lengths = 20, [3, 17, 1]
    tokens = prefix + sum(lengths)
    qkv = _normal((tokens + 3, H + 2 * kv, D), torch.float16, g)
    positions, slots, table, page = list(range(prefix)), list(range(prefix)), [], 2
    for n in lengths:                                          # (the prefix owns pages 0 and 1)
        positions += range(prefix, prefix + n)
        slots += [page * size + i for i in range(n)]
        table.append([page, page + 1])
        page += 2
    new_positions = [prefix + n for n in lengths]
    new_slots = [t[n // size] * size + n % size for t, n in zip(table, lengths)]
    dev = dict(device="cuda")
    positions = torch.tensor(positions + new_positions, **dev)
    slots = torch.tensor(slots + new_slots, **dev)
    table = torch.tensor(table, dtype=torch.int32, **dev)
    raw = qkv.clone()
    pages = [torch.full((page + 1, kv, size, D), math.nan, dtype=torch.float16, **dev) for _ in range(2)]
    for part in (slice(0, tokens), slice(tokens, tokens + 3)):
        q, k, v = qkv[part, :H], qkv[part, H:H + kv], qkv[part, H + kv:]
        rotary.launch(positions[part], [q, k], [q, k])
        cache.store([k, v], slots[part], pages)
    lens = torch.tensor([n + 1 for n in lengths], dtype=torch.int32, **dev)
    out = torch.empty((3, H, D), dtype=torch.float16, **dev)
    ws = torch.empty(max(16, cache.workspace_bytes(3, H, kv, 2 * size, prefix)), dtype=torch.uint8, **dev)
    cache.attend(qkv[tokens:, :H], lens, table, pages, out, workspace=ws, prefix_table=torch.tensor([0, 1], dtype=torch.int32, **dev), prefix_length=prefix)
    q64 = plain.rotary(raw[:, :H], positions, frequencies)
    k64, v64 = plain.rotary(raw[:, H:H + kv], positions, frequencies), raw[:, H + kv:].double()
    at = prefix
    for b, n in enumerate(lengths):
        own = list(range(prefix)) + list(range(at, at + n)) + [tokens + b]
        at += n
        k, v = (x[own].repeat_interleave(group, 1).transpose(0, 1) for x in (k64, v64))
        q = q64[tokens + b][:, None]
        scores = (q * k).sum(-1) / math.sqrt(D)
        want = (torch.softmax(scores, -1)[..., None] * v).sum(1)
        # q and k were rounded to fp16 (half a step each, relatively) before their product: that much of sum |q k|
        slack = (q.abs() * k.abs()).sum(-1).amax() / math.sqrt(D) * (2 * 2.0 ** -11 + 2.0 ** -20) + 2.0 ** -16
        bound = _half_step(torch.float16) * want.abs() + 2 * slack * 1.01 * v.abs().amax()
        _inside(out[b], want, bound, f"sequence {b}")


# ---- weights, values and rows of every size --------------------------------------------------------


def _shaped(dtype, storage, D, kv, group, size, lengths, prefix, kind, gap, g):
    """A batch whose scores and values are set: every token's first key element times 16 is its score beside a small random
    one.  "sink": two tokens of every sequence and of the prefix score `gap` nats above the others and have no value, or
    2^-12 of one.  "loud": two score 50 nats below and have values 2^25 times the others' (2^15 in fp16).  "spread":
    scores spread over `gap` nats.  "huge": every row's largest value is the type's."""
    s = _setup(dtype, storage, D, kv, group, size, lengths, prefix, g)
    count = s["pages"][0].shape[0]
    k, v = (_normal((count, kv, size, D), torch.float32, g, 0.5) for _ in range(2))
    up = math.sqrt(D) / 16
    k[..., 0] = 0.0
    if kind == "spread":
        k[..., 0] = torch.rand((count, kv, size), generator=g, device="cuda") * (-gap * up)
    if kind == "huge":
        v = v / v.abs().amax(-1, keepdim=True) * torch.finfo(TYPES[dtype]).max
    if dtype == "f16" and kind != "huge":
        v *= 2.0 ** (-4 if kind == "loud" else 10)             # (results that are normal numbers)
    rows = [(s["table"][b].tolist(), n) for b, n in enumerate(lengths)] + [(s["prefix_table"].tolist(), prefix)]
    for row, n in rows:
        for i, t in enumerate((5, n // 2 + 3)):
            if t >= n or n < 8:
                continue
            page, place = row[t // size], t % size
            if kind == "sink":
                k[page, :, place, 0] = gap * up
                v[page, :, place] *= i * 2.0 ** -12
            elif kind == "loud":
                k[page, :, place, 0] = -50 * up
                v[page, :, place] *= 2.0 ** (25 if dtype == "bf16" else 15)
    if storage in STORED:
        c = [plain.encode(x.to(TYPES[dtype]), storage) for x in (k, v)]
        s["pages"] = [c[0][0], c[1][0], c[0][1], c[1][1]]
    else:
        s["pages"] = [x.to(TYPES[dtype]) for x in (k, v)]
    s["q"][..., 0] = 16.0
    return s


def _own_sum_bound(dtype, storage, s, scale):
    """The result's own half step, and twice the relative error of a weight times sum p |v| / sum p: of the very products that
    the result is the sum of, so that nothing may be lost beside a larger score or value of another token.  A weight's
    error: its rounding (to half precision 2^-11; as two half-precision or bf16 numbers 2^-16), its score's, the
    hardware's power of two 2^-22; sums of n terms in 32 bits, n 2^-24 each of numerator and denominator.  Half precision
    ends at 2^-25: 2^-34 of the largest product of a weight and a value over 8-bit rows, n times, and of fp16 values 2^-35 of
    the largest probability times each of them."""
    a = (s["q"], s["lengths"], s["table"], s["pages"], scale, s["prefix_table"], s["prefix"])
    want, most, sums, keys = plain.attend(*a)
    share, whole, heavy = plain.attend_sizes(*a)
    D = s["q"].shape[2]
    n = float(s["prefix"] + max(0, int(s["lengths"].max())))
    one = 2.0 ** -11 if storage in STORED and dtype == "bf16" else 2.0 ** -16
    score = sums * scale * ((D + 4) * 2.0 ** -24)
    if storage in STORED and dtype == "bf16":
        score = score + scale * 2.0 ** -25 * float(s["q"].abs().max()) * keys
    w = one + score + 2.0 ** -22 + n * 2.0 ** -24
    end = n * 2.0 ** -34 * heavy[..., None] if storage in STORED else 2.0 ** -35 * whole if dtype == "f16" else 0.0
    return want, _half_step(TYPES[dtype]) * want.abs() + (2 * w)[..., None] * 1.01 * share + end + torch.finfo(TYPES[dtype]).smallest_normal * _half_step(TYPES[dtype])


# sequences of their own, long and short; a prefix in the sequences' own launch, in line, and in a launch of its own
SHAPES = [(2, 2, 16, [1500, 33, 300, 7], 0), (2, 4, 16, [40, 9, 1], 700), (1, 3, 8, [100, 31], 150), (8, 16, 16, [(11 * i) % 40 for i in range(40)], 2600)]
KINDS = [("bf16", "i8", 128), ("bf16", "e4m3", 64), ("f16", "i8", 64), ("f16", "f16", 80), ("bf16", "bf16", 128), ("f16", "e4m3", 256)]


@pytest.mark.parametrize("dtype,storage,D", KINDS)
def test_attention_of_the_largest_values(ctx, dtype, storage, D):
    """Rows whose largest value is the type's: no sum on the way to a finite result overflows."""
    cache = _cache(ctx, dtype, storage, D)
    for kv, group, size, lengths, prefix in SHAPES + [(1, 2, 8, [1, 2], 0)]:
        s = _shaped(dtype, storage, D, kv, group, size, lengths, prefix, "huge", 0, _generator(41 + prefix))
        want, bound = _own_sum_bound(dtype, storage, s, 1.0 / math.sqrt(D))
        # (no token's value may round up past the type)
        assert float(want.abs().max()) < torch.finfo(TYPES[dtype]).max * 1.001
        fine = want.abs() + bound < torch.finfo(TYPES[dtype]).max
        got = _run(cache, s)[0]
        _inside(got[fine], want[fine], bound[fine], f"largest values, {len(lengths)} sequences behind {prefix}")


@pytest.mark.parametrize("dtype,storage,D", KINDS)
@pytest.mark.parametrize("kind,gap", [("sink", 12), ("sink", 17), ("sink", 40), ("loud", 0), ("spread", 60)])
def test_attention_beside_larger_scores_and_values(ctx, dtype, storage, D, kind, gap):
    cache = _cache(ctx, dtype, storage, D)
    for kv, group, size, lengths, prefix in SHAPES:
        s = _shaped(dtype, storage, D, kv, group, size, lengths, prefix, kind, gap, _generator(51 + prefix))
        want, bound = _own_sum_bound(dtype, storage, s, 1.0 / math.sqrt(D))
        _inside(_run(cache, s)[0], want, bound, f"{kind} {gap}, {len(lengths)} sequences behind {prefix}")


@pytest.mark.parametrize("storage,D", [("i8", 128), ("e4m3", 64)])
def test_store_of_rows_near_the_smallest_numbers(ctx, storage, D):
    """Rows of bf16 down to its last numbers, large and small elements and zeros among them, against codes in 64 bits."""
    cache = _cache(ctx, "bf16", storage, D)
    g = _generator(61)
    a = torch.tensor([2.0 ** -e for e in (90, 99, 100, 101, 110, 119, 120, 121, 125, 126, 127, 130, 133)] + [3.7e-37, 1.3e-36, 1e-38], device="cuda")
    x = torch.rand((a.numel(), 2, D), generator=g, device="cuda").mul_(2).sub_(1) * a[:, None, None]
    x[..., 3] = 0.0
    x[..., 5] = a[:, None]
    x[:, 1, 6] = -a / 2
    k = x.bfloat16()
    v = k.flip(0).contiguous()
    n, size = k.shape[0], 8
    pages = _empty_pages("bf16", storage, 3, 2, size, D, 1.0)
    slots = torch.randperm(3 * size, generator=g, device="cuda")[:n]
    cache.store([k, v], slots, pages)
    back = [torch.empty_like(k) for _ in range(2)]
    cache.load(slots, pages, back)
    most = 127.0 if storage == "i8" else 448.0
    for i, rows in enumerate((k, v)):
        codes = pages[i][slots // size, :, slots % size].double()
        scales = pages[2 + i][slots // size, :, slots % size]
        large = rows.double().abs().amax(-1)
        assert torch.equal(scales, (large / most).float())
        exact = rows.double() * most / large[..., None]
        # (half a step of the code; Q / a and its product with the element are rounded to 32 bits)
        step = torch.full_like(exact, 0.5) if storage == "i8" else torch.maximum(exact.abs() * 2.0 ** -4, torch.tensor(2.0 ** -10, dtype=torch.float64, device="cuda"))
        assert ((codes - exact).abs() <= step + exact.abs() * 2.0 ** -22).all()
        assert (codes[rows == 0] == 0).all() and (back[i][rows == 0] == 0).all()


# ---- calls of more threads than a launch has -------------------------------------------------------


def test_rotary_of_more_tokens_than_a_launch_has_blocks(ctx):
    """2^24 tokens and more: a block each, of which one launch has less than 2^24."""
    h = ctx.register_rotary("bf16", 2, [1.0], layout="interleaved")
    tokens = (1 << 24) + 5
    g = _generator(81)
    x = _normal((tokens, 1, 2), torch.bfloat16, g)
    positions = torch.randint(0, 1000, (tokens,), generator=g, device="cuda", dtype=torch.int32)
    y = torch.zeros_like(x)
    before = ctx.stats()
    h.launch(positions, [x], [y])
    after = ctx.stats()
    assert after["launch_calls"] == before["launch_calls"] + 1 and after["device_launches"] > before["device_launches"] + 1
    want = plain.rotary(x, positions, [1.0], "interleaved")
    _inside(y, want, _rotary_bound(x, positions, [1.0], "interleaved", 1.0, torch.bfloat16, want), "rotary")


def test_store_of_more_rows_than_a_launch_has_threads(ctx):
    """2^32 threads and more (of rows that all heads share, nearly all of them padding): the tokens at both sides of a launch's end."""
    cache = _cache(ctx, "bf16", "i8", 16)
    tokens, kv = 32767 + 9, 65536
    rows = [_normal((tokens, 1, 16), torch.bfloat16, _generator(82 + i)) for i in range(2)]
    pages = _empty_pages("bf16", "i8", 1, kv, 8, 16, 1.0)
    at = torch.tensor([0, 32766, 32767, tokens - 1], device="cuda")
    slots = torch.full((tokens,), -1, dtype=torch.int64, device="cuda")
    slots[at] = torch.tensor([4, 0, 7, 2], device="cuda")
    cache.store([r.expand(tokens, kv, 16) for r in rows], slots, pages)
    for i, r in enumerate(rows):
        codes, scales = plain.encode(r[at, 0], "i8")
        want, want_scales = torch.ones((8, 16), dtype=torch.int8, device="cuda"), torch.ones(8, device="cuda")
        want[slots[at]], want_scales[slots[at]] = codes, scales
        assert (pages[i][0] == want).all() and (pages[2 + i][0] == want_scales).all()


@pytest.mark.parametrize("dtype,storage,D,batch,longest,prefix", [("bf16", "bf16", 256, 300, 512, 0), ("bf16", "i8", 128, 66, 600, 2500), ("bf16", "bf16", 256, 40, 400, 700)])
def test_attention_with_the_workspace_of_a_larger_call(ctx, dtype, storage, D, batch, longest, prefix):
    """One workspace for the largest batch, prefix and table, and nothing written behind it."""
    cache = _cache(ctx, dtype, storage, D)
    need = max(16, cache.workspace_bytes(batch, 16, 4, longest, prefix))
    held = torch.full((need + 4096,), 7, dtype=torch.uint8, device="cuda")
    for b, p in ((batch, prefix), (batch - 1, prefix), (33, prefix), (32, prefix // 2), (4, prefix), (1, 600 if prefix else 0)):
        lengths = [(13 * i) % min(40, longest) for i in range(b - 1)] + [longest - 20]
        s = _setup(dtype, storage, D, 4, 4, 8, lengths, p, _generator(b + D))
        s["table"] = s["table"][:, :-1].contiguous()
        got = _run(cache, s, workspace=held[:need])[0]
        _check(cache, dtype, storage, s, 1.0 / math.sqrt(D), got=got)
        assert (held[need:] == 7).all()


@pytest.mark.parametrize("storage,D", [("i8", 128), ("e4m3", 64)])
@pytest.mark.parametrize("batch,prefix,longest", [(3, 0, 300), (600, 0, 40), (40, 1500, 40), (300, 2500, 40), (300, 0, 3000)])
def test_queries_of_the_largest_rows_beside_large_keys(ctx, storage, D, batch, prefix, longest):
    """Rows as large as the type has beside ordinary ones whose scores come of small queries and large keys, or the other way:
    the powers of two that they are brought to are taken back row by row."""
    cache = _cache(ctx, "bf16", storage, D)
    lengths = [int(x) for x in torch.randint(1, longest, (batch,), generator=torch.Generator().manual_seed(4))]
    for up in (2.0 ** 20, 2.0 ** 90, 2.0 ** -60):
        s = _setup("bf16", storage, D, 2, 4, 16, lengths, prefix, _generator(71 + batch))
        s["pages"][2] *= up
        s["q"] /= up
        want, *sizes = plain.attend(s["q"], s["lengths"], s["table"], s["pages"], 1.0 / math.sqrt(D), s["prefix_table"], s["prefix"])
        bound = _attend_bound("bf16", storage, s, want, *sizes, 1.0 / math.sqrt(D))
        odd = torch.zeros(s["q"].shape[:2], dtype=torch.bool, device="cuda")
        odd[0, 1::4] = odd[batch - 1] = True
        s["q"][odd] = torch.finfo(torch.bfloat16).max
        got = _run(cache, s)[0]
        _inside(got[~odd], want[~odd], bound[~odd], f"queries of 2^{-math.log2(up):.0f} beside the largest")
        if up < 1.0:                                               # (their own scores are numbers of 32 bits here)
            assert torch.isfinite(got).all()


# ---- more of what the documents allow --------------------------------------------------------------


def test_rotary_in_place_leaves_the_heads_between(ctx):
    """In place, queries and keys of one product's rows: the values and whatever else lies between them keep their bits."""
    from paper_2103_05288_amd import rotary_frequencies
    for dtype, D, R, layout in (("bf16", 128, 128, "half"), ("f16", 80, 26, "interleaved"), ("f32", 64, 64, "half")):
        frequencies, _ = rotary_frequencies(R)
        h = ctx.register_rotary(dtype, D, frequencies, layout=layout)
        rows = _normal((131, 9, D), TYPES[dtype], _generator(91))
        before = rows.clone()
        positions = torch.arange(131, device="cuda") * 7
        h.launch(positions, [rows[:, 1:4], rows[:, 5:7]], [rows[:, 1:4], rows[:, 5:7]])
        for i in (0, 4, 7, 8):
            assert torch.equal(_bits(rows[:, i]), _bits(before[:, i]))
        for part in (slice(1, 4), slice(5, 7)):
            want = plain.rotary(before[:, part], positions, frequencies, layout)
            _inside(rows[:, part], want, _rotary_bound(before[:, part], positions, frequencies, layout, 1.0, TYPES[dtype], want), "rotary")


def test_attention_of_stretches_of_more_pages_than_a_block_keeps(ctx):
    """1024 pages are staged at a time: so many kv heads that a block has whole sequences of more, a prefix whose chunks end there,
    and pages that are none behind that."""
    cache = _cache(ctx, "bf16", "i8", 16)
    kv, size = 1024, 8
    g = _generator(95)
    for lengths, prefix in (([9001, 300, 8193], 0), ([17, 40], 9003)):
        s = _setup("bf16", "i8", 16, kv, 1, size, lengths, prefix, g)
        where = s["prefix_table"] if prefix else s["table"][0]
        where[[3, 1023, 1024, 1100]] = torch.tensor([-1, 10 ** 9, -7, s["pages"][0].shape[0]], dtype=torch.int32, device="cuda")
        s["pages"][2] = torch.nan_to_num(s["pages"][2], nan=0.0, posinf=0.0, neginf=0.0)
        _check(cache, "bf16", "i8", s, 0.25)
        del s


def test_the_step_of_a_token_captured(ctx):
    """Rotation in place, store, attention behind a shared prefix and load in one graph; its inputs, slots, lengths and positions
    change between the replays, with eager work in between, and every replay gives what eager calls give."""
    from paper_2103_05288_amd import rotary_frequencies
    D, kv, group, size, prefix, batch = 64, 2, 3, 16, 40, 5
    H = kv * group
    rotary = ctx.register_rotary("bf16", D, rotary_frequencies(D)[0])
    cache = _cache(ctx, "bf16", "e4m3", D)
    g = _generator(97)
    shape = (3 + 3 * batch, kv, size, D)
    table = torch.arange(3, 3 + 3 * batch, device="cuda", dtype=torch.int32).view(batch, 3)
    prefix_table = torch.arange(3, device="cuda", dtype=torch.int32)
    filled = _filled("bf16", "e4m3", shape[0], kv, size, D, g)
    ws = torch.empty(max(16, cache.workspace_bytes(batch, H, kv, 3 * size, prefix)), dtype=torch.uint8, device="cuda")

    def inputs(turn):
        n = torch.tensor([(5 * turn + 11 * b) % 47 for b in range(batch)], device="cuda")
        page = table.long()[torch.arange(batch, device="cuda"), n // size]
        return {"qkv": _normal((batch, H + 2 * kv, D), torch.bfloat16, _generator(200 + turn)), "positions": n + prefix, "slots": page * size + n % size,
                "lengths": (n + 1).int()}

    def step(x, pages, out, back):
        q, k, v = x["qkv"][:, :H], x["qkv"][:, H:H + kv], x["qkv"][:, H + kv:]
        rotary.launch(x["positions"], [q, k], [q, k])
        cache.store([k, v], x["slots"], pages)
        cache.attend(q, x["lengths"], table, pages, out, workspace=ws, prefix_table=prefix_table, prefix_length=prefix)
        cache.load(x["slots"], pages, back)

    static, pages = inputs(0), [p.clone() for p in filled]
    out = torch.empty((batch, H, D), dtype=torch.bfloat16, device="cuda")
    back = [torch.empty((batch, kv, D), dtype=torch.bfloat16, device="cuda") for _ in range(2)]
    step(static, pages, out, back)                             # (nothing is compiled or looked up within the capture)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step(static, pages, out, back)
    for turn in range(5):
        x = inputs(turn)
        eager_pages, eager_out, eager_back = [p.clone() for p in filled], torch.empty_like(out), [torch.empty_like(b) for b in back]
        for name, t in x.items():
            static[name].copy_(t)
        for a, b in zip(pages, filled):
            a.copy_(b)
        out.fill_(math.nan)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        step(x, eager_pages, eager_out, eager_back)
        torch.cuda.synchronize()
        assert torch.equal(out, eager_out) and torch.equal(static["qkv"], x["qkv"])
        for a, b in zip(pages + back, eager_pages + eager_back):
            assert torch.equal(_bits(a), _bits(b))
        want, *sizes = plain.attend(x["qkv"][:, :H], x["lengths"], table, eager_pages, 0.125, prefix_table, prefix)
        s = {"q": x["qkv"][:, :H], "prefix": prefix, "lengths": x["lengths"]}
        _inside(out, want, _attend_bound("bf16", "e4m3", s, want, *sizes, 0.125), f"replay {turn}")


def test_attention_with_the_largest_softmax_scales(ctx):
    """Queries and keys so small that their scores are ordinary ones again."""
    for dtype, storage, D, scale in (("bf16", "i8", 64, 2.0 ** 119), ("bf16", "e4m3", 64, 2.0 ** 120), ("f16", "i8", 64, 2.0 ** 40), ("bf16", "bf16", 64, -(2.0 ** 100))):
        cache = ctx.register_cache(dtype, D, storage, softmax_scale=scale / math.sqrt(D))
        s = _setup(dtype, storage, D, 2, 4, 16, [200, 33, 1, 90], 150, _generator(99))
        if storage in STORED:
            s["pages"][2] /= abs(scale)
        else:
            s["pages"][0] = (s["pages"][0].float() / abs(scale)).to(TYPES[dtype])
        want, *sizes = plain.attend(s["q"], s["lengths"], s["table"], s["pages"], scale / math.sqrt(D), s["prefix_table"], s["prefix"])
        _inside(_run(cache, s)[0], want, _attend_bound(dtype, storage, s, want, *sizes, abs(scale) / math.sqrt(D)), f"softmax scale {scale:g}")


@pytest.mark.parametrize("dtype,storage,D", [("f16", "i8", 64), ("f16", "e4m3", 256), ("f16", "f16", 80), ("bf16", "bf16", 128)])
def test_attention_weights_of_two_numbers(ctx, dtype, storage, D):
    """A hundred thousand weights, of which a few are close to half way between two 16-bit numbers: the second number is what is
    left of the first, of every one."""
    cache = _cache(ctx, dtype, storage, D)
    s = _shaped(dtype, storage, D, 8, 16, 8, [2 + i % 3 for i in range(260)], 0, "plain", 0, _generator(103))
    want, bound = _own_sum_bound(dtype, storage, s, 1.0 / math.sqrt(D))
    _inside(_run(cache, s)[0], want, bound, "weights")
