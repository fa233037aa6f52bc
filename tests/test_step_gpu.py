"""The norm into 8-bit rows and its gradient, products with 4-bit weights and the check of drafted tokens on the GPU,
against 64 bits (oracle/step.py), at the sizes, strides and values where they can go wrong."""
import math

import pytest
import torch

from oracle import step as plain

pytestmark = pytest.mark.gpu

TYPES = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
STORED = {"i8": torch.int8, "e4m3": torch.float8_e4m3fn}
EPS = 1e-5
UNIT = 2.0 ** -24          # half a step of 32 bits


@pytest.fixture(scope="module")
def ctx():
    from paper_2103_05288_amd import Context
    c = Context(0)
    yield c
    torch.cuda.synchronize()
    c.close()


def _half_step(dtype):
    return torch.finfo(dtype).eps / 2


def _least(dtype):
    """Half a step of the smallest numbers."""
    return torch.finfo(dtype).tiny * torch.finfo(dtype).eps / 2


def _generator(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return g


def _normal(shape, dtype, g, std=1.0):
    return torch.empty(shape, dtype=torch.float32, device="cuda").normal_(0.0, std, generator=g).to(dtype)


def _channels(shape, dtype, g):
    size = torch.empty(shape[-1], dtype=torch.float32, device="cuda").normal_(0.0, 0.5, generator=g).exp_()
    size[::97] *= 12
    return (torch.empty(shape, dtype=torch.float32, device="cuda").normal_(0.0, 1.0, generator=g) * size).to(dtype)


def _inside(got, want, bound, what):
    off = (got.double() - want).abs()
    bad = ~(off <= bound)
    assert not bad.any(), f"{what}: {int(bad.sum())} of {off.numel()} values outside the bound, worst {float((off - bound).max()):.3g} over it"


def _apart(rows, width, dtype, fill=0):
    """[rows, width] inside a wider tensor (all of `fill`): the view and the whole."""
    size = torch.empty((), dtype=dtype).element_size()
    whole = torch.full((rows, (width + 5) * size), fill, dtype=torch.uint8, device="cuda").view(dtype)
    return whole[:, 2:2 + width], whole


# ---- the norm --------------------------------------------------------------------------------------


def _check_codes(codes, scales, y, largest, storage, what):
    """Scale: s and weight + offset a half step of 32 bits each, their product, the quotient's and the result's own (and the
    64-bit sums): 6.  Code: the same, the quotient Q / a and the product with it, 8, and its own half step."""
    most = plain.MOST[storage]
    bad = torch.isnan(largest)
    assert torch.equal(torch.isnan(scales), bad), what
    assert (codes[bad].float() == 0).all(), what
    fine = ~bad
    _inside(scales[fine], largest[fine] / most, 6 * UNIT * largest[fine] / most + 2.0 ** -149, what + " scales")
    zero = fine & (largest == 0)
    assert (codes[zero].float() == 0).all() and (scales[zero] == 0).all()
    some = fine & (largest > 0)
    # (what the code stands for, in units of the row's largest)
    want = y[some] / largest[some].unsqueeze(-1) * most
    got = codes[some].double()
    half = torch.full_like(want, 0.5) if storage == "i8" else torch.maximum(want.abs() * 2.0 ** -4, torch.full_like(want, 2.0 ** -10))
    _inside(got, want, half + 8 * UNIT * want.abs() + 2.0 ** -120, what + " codes")


def _norm(ctx, dtype, storage, rows, width, offset, residual, seed, strided=True, x=None, weight=None, eps=EPS):
    h = ctx.register_norm(dtype, storage, eps=eps, offset=offset)
    g = _generator(seed)
    t = TYPES[dtype]
    x = _channels((rows, width), t, g) if x is None else x
    weight = (1 - offset + _normal((width,), torch.float32, g, 0.2)).to(t) if weight is None else weight
    if strided:
        a, _ = _apart(rows, width, t, 255)
        a.copy_(x)
        x = a
    codes, whole = _apart(rows, width, STORED[storage], 7) if strided else (torch.empty((rows, width), dtype=STORED[storage], device="cuda"), None)
    scales = torch.full((rows,), -5.0, device="cuda")
    more, total_whole = {}, None
    if residual is not None:
        total, total_whole = _apart(rows, width, t, 7) if strided else (torch.empty((rows, width), dtype=t, device="cuda"), None)
        more = {"residual": residual, "total": total}
    h.launch(x, weight, codes, scales, **more)
    s, y, largest = plain.norm(x, weight, eps, offset, residual)
    if residual is not None:
        assert torch.equal(more["total"], (x.float() + residual.float()).to(t))
    _check_codes(codes, scales, y, largest, storage, f"{dtype} {storage} {rows} x {width}")
    for w, dt in ((whole, STORED[storage]), (total_whole, t)):
        if w is not None:
            size = torch.empty((), dtype=dt).element_size()
            b = w.view(torch.uint8)
            assert (b[:, :2 * size] == 7).all() and (b[:, (2 + width) * size:] == 7).all(), "written outside the rows"
    return codes, scales, more.get("total")


@pytest.mark.parametrize("dtype,storage", [("bf16", "i8"), ("bf16", "e4m3"), ("f16", "e4m3"), ("f32", "i8")])
@pytest.mark.parametrize("rows,width", [(1, 1), (1, 4096), (3, 7), (5, 8), (33, 63), (17, 64), (130, 65), (9, 513), (300, 1001), (2, 1280), (7, 2049), (600, 4100), (3, 8192),
                                        (300, 12288), (2, 16384)])
def test_norm_matches_64_bits(ctx, dtype, storage, rows, width):
    g = _generator(rows * width)
    residual = _channels((rows, width), TYPES[dtype], g)
    _norm(ctx, dtype, storage, rows, width, 0.0, residual, rows + width)
    _norm(ctx, dtype, storage, rows, width, 1.0, None, rows + width + 1, strided=False)


@pytest.mark.parametrize("dtype,storage,rows,width", [("bf16", "i8", 5, 32768), ("f16", "e4m3", 400, 32761), ("f32", "i8", 300, 16383)])
def test_norm_of_the_widest_rows(ctx, dtype, storage, rows, width):
    residual = _channels((rows, width), TYPES[dtype], _generator(3))
    _norm(ctx, dtype, storage, rows, width, 0.0, residual, 4)


@pytest.mark.parametrize("dtype,storage,rows,width", [("bf16", "e4m3", 4099, 4096), ("f32", "i8", 10007, 1003)])
def test_norm_past_the_caches(ctx, dtype, storage, rows, width):
    """More than 64 MiB: the version that goes past them."""
    residual = _channels((rows, width), TYPES[dtype], _generator(5))
    _norm(ctx, dtype, storage, rows, width, 1.0, residual, 6)


@pytest.mark.parametrize("dtype,storage", [("bf16", "i8"), ("f32", "i8"), ("f16", "e4m3")])
def test_norm_in_place(ctx, dtype, storage):
    h = ctx.register_norm(dtype, storage, eps=EPS)
    g = _generator(8)
    t = TYPES[dtype]
    for rows, width in ((1, 640), (70, 1000), (5, 9000)):
        x, residual, weight = _channels((rows, width), t, g), _channels((rows, width), t, g), _normal((width,), t, g)
        want = [torch.empty((rows, width), dtype=STORED[storage], device="cuda"), torch.empty(rows, device="cuda"), torch.empty_like(x)]
        h.launch(x, weight, want[0], want[1], residual=residual, total=want[2])
        for into in (0, 1):
            a, b = x.clone(), residual.clone()
            codes, scales = torch.empty_like(want[0]), torch.empty_like(want[1])
            h.launch(a, weight, codes, scales, residual=b, total=(a, b)[into])
            assert torch.equal((a, b)[into], want[2]) and torch.equal(codes.view(torch.uint8), want[0].view(torch.uint8)) and torch.equal(scales, want[1])
            assert torch.equal((b, a)[into], (residual, x)[into])


@pytest.mark.parametrize("dtype,storage", [("bf16", "i8"), ("bf16", "e4m3"), ("f32", "i8"), ("f16", "e4m3")])
def test_norm_of_rows_at_the_ends_of_their_type(ctx, dtype, storage):
    """Zeros, the smallest and the largest numbers, infinities and NaN, each beside ordinary rows (which stay what they are)."""
    t = TYPES[dtype]
    g = _generator(9)
    for width in (40, 700, 5000):
        x = _channels((16, width), t, g)
        weight = (1 + _normal((width,), torch.float32, g, 0.2)).to(t)
        big, small = torch.finfo(t).max, torch.finfo(t).tiny
        x[1] = 0
        x[3] = (torch.sign(x[3].float()) * big).to(t)
        x[4] = big * 0.25
        x[5] = small
        x[6] = 0
        x[6, width // 2] = small * 0.5
        x[8, width - 1] = math.inf
        x[9, 3] = -math.inf
        x[10, width // 3] = math.nan
        x[12] = (x[12].float() * small).to(t)
        x[13, 0] = big
        codes, scales, _ = _norm(ctx, dtype, storage, 16, width, 0.0, None, 10, x=x, weight=weight)
        only = [0, 2, 7, 11, 14, 15]
        again, those, _ = _norm(ctx, dtype, storage, 6, width, 0.0, None, 10, x=x[only].contiguous(), weight=weight)
        assert torch.equal(codes[only].view(torch.uint8), again.contiguous().view(torch.uint8)) and torch.equal(scales[only], those)
        if dtype != "f16":      # (products that pass 32 bits, and that fall below them)
            for w in (2.0 ** 90, 2.0 ** -100):
                _norm(ctx, dtype, storage, 16, width, 0.0, None, 11, x=x, weight=(weight.float() * w).to(t))
        weight[5] = math.nan
        _norm(ctx, dtype, storage, 3, width, 0.0, None, 12, x=x[:3].contiguous(), weight=weight)


def test_norm_of_nothing(ctx):
    h = ctx.register_norm("bf16", "i8")
    x = torch.empty((0, 64), dtype=torch.bfloat16, device="cuda")
    h.launch(x, torch.ones(64, dtype=torch.bfloat16, device="cuda"), torch.empty((0, 64), dtype=torch.int8, device="cuda"), torch.empty(0, device="cuda"))
    dw = torch.full((64,), 3.0, device="cuda")
    h.backward(x, torch.ones(64, dtype=torch.bfloat16, device="cuda"), x, x, dw)
    assert (dw == 0).all()


# ---- its gradient ----------------------------------------------------------------------------------


def _backward(ctx, dtype, rows, width, offset, with_total, seed, strided=True, into=None, total=None, dy=None, weight=None):
    h = ctx.register_norm(dtype, "e4m3" if dtype == "f16" else "i8", eps=EPS, offset=offset)
    g = _generator(seed)
    t = TYPES[dtype]
    total = _channels((rows, width), t, g) if total is None else total
    dy = _normal((rows, width), t, g, 0.1) if dy is None else dy
    dtotal = _normal((rows, width), t, g, 0.1) if with_total else None
    weight = (1 - offset + _normal((width,), torch.float32, g, 0.2)).to(t) if weight is None else weight
    want, dweight, size, dsize = plain.norm_backward(total, weight, dy, EPS, offset, dtotal)
    dx, whole = _apart(rows, width, t, 7) if strided else (torch.empty((rows, width), dtype=t, device="cuda"), None)
    if into is not None:
        dx = (total, dy, dtotal)[into]
    dw = torch.full((width,), 9.0, device="cuda")
    ws = torch.full((max(16, h.workspace_bytes(rows, width)),), 255, dtype=torch.uint8, device="cuda")
    h.backward(total, weight, dy, dx, dw, dtotal=dtotal, workspace=ws)
    # dx: u = h r two roundings and r's own, g = dy w two, k one and of its terms w's (relative to the mean of |g u|), u k five in all,
    # g - u k six, times r eight, plus dtotal nine; and the result's own
    _inside(dx, want, _half_step(t) * want.abs() + 9 * UNIT * size + _least(t) + 2.0 ** -149, f"dx {dtype} {rows} x {width}")
    # dweight: three roundings of a term, and one for each sum that it goes through: the rows of a thread, then the parts
    parts = ws.numel() // (4 * width)
    steps = -(-rows // max(1, min(parts, rows))) + parts + 4
    _inside(dw, dweight, (3 + min(steps, rows + 8)) * UNIT * dsize + 2.0 ** -149, f"dweight {dtype} {rows} x {width}")
    if whole is not None and into is None:
        size = torch.empty((), dtype=t).element_size()
        assert (whole.view(torch.uint8)[:, :2 * size] == 7).all() and (whole.view(torch.uint8)[:, (2 + width) * size:] == 7).all()
    return dx, dw


@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("rows,width", [(1, 1), (1, 4096), (3, 7), (5, 8), (65, 63), (17, 64), (1300, 65), (9, 513), (700, 1001), (2, 1280), (7, 2049), (1100, 4100), (3, 8192), (600, 12288),
                                        (2, 16384)])
def test_norm_backward_matches_64_bits(ctx, dtype, rows, width):
    _backward(ctx, dtype, rows, width, 0.0, True, rows + width)
    _backward(ctx, dtype, rows, width, 1.0, False, rows + width + 1, strided=False)


@pytest.mark.parametrize("dtype,rows,width", [("bf16", 5, 32768), ("f32", 300, 16383), ("bf16", 6001, 2048), ("f32", 9001, 640)])
def test_norm_backward_of_wide_and_of_many_rows(ctx, dtype, rows, width):
    _backward(ctx, dtype, rows, width, 0.0, True, 21)


@pytest.mark.parametrize("into", [0, 1, 2])
def test_norm_backward_in_place(ctx, into):
    _backward(ctx, "bf16", 300, 1000, 0.0, True, 22, into=into)
    _backward(ctx, "f32", 3, 9000, 1.0, True, 23, into=into)


def test_norm_backward_of_the_largest_and_smallest_rows(ctx):
    for dtype in ("f32", "bf16"):
        t = TYPES[dtype]
        g = _generator(24)
        total = _channels((8, 600), t, g)
        total[0] = (total[0].float() * 2.0 ** 115).to(t)
        total[1] = torch.finfo(t).max
        total[2] = 0
        total[3] = (total[3].float() * 2.0 ** -120).to(t)
        total[5] = (torch.sign(total[5].float()) * 2.0 ** 64).to(t)
        _backward(ctx, dtype, 8, 600, 0.0, True, 25, total=total)


def test_norm_backward_against_differences(ctx):
    """The step of the unrounded norm along a direction, in 64 bits, and what the gradient says of it."""
    g = _generator(26)
    rows, width, offset = 7, 130, 1.0
    h = ctx.register_norm("f32", "i8", eps=EPS, offset=offset)
    x, weight, dy, dtotal = (_normal(s, torch.float32, g) for s in ((rows, width), (width,), (rows, width), (rows, width)))
    dx, dw = torch.empty_like(x), torch.empty_like(weight)
    h.backward(x, weight, dy, dx, dw, dtotal=dtotal, workspace=torch.empty(h.workspace_bytes(rows, width), dtype=torch.uint8, device="cuda"))

    def loss(x, w):
        return ((plain.norm(x, w, EPS, offset)[1] * dy.double()).sum() + (x * dtotal.double()).sum()).item()
    for k in range(8):
        a, b = (_normal(s, torch.float32, g).double() for s in ((rows, width), (width,)))
        step = 1e-5
        slope = (loss(x.double() + step * a, weight.double() + step * b) - loss(x.double() - step * a, weight.double() - step * b)) / (2 * step)
        said = (dx.double() * a).sum() + (dw.double() * b).sum()
        size = (dx.double() * a).abs().sum() + (dw.double() * b).abs().sum()
        # (32-bit gradients: 16 half steps of each; the differences' own error, step^2 times the third derivative: below 1e-8 of the size)
        assert abs(slope - said.item()) < (16 * UNIT + 1e-7) * size.item()


def test_norm_backward_gives_the_same_sums_again(ctx):
    a = _backward(ctx, "bf16", 3000, 700, 0.0, True, 27)
    b = _backward(ctx, "bf16", 3000, 700, 0.0, True, 27)
    assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1])


# ---- products with 4-bit weights -------------------------------------------------------------------


def _linear_inputs(dtype, rows, group, zeros, bias, M, N, K, seed):
    g = _generator(seed)
    t = TYPES[dtype]
    weights = torch.randint(0, 256, (N, K // 2), generator=g, device="cuda", dtype=torch.uint8)
    scales = (torch.empty((N, K // group), device="cuda").normal_(0.0, 0.4, generator=g).exp_() * (0.4 / math.sqrt(K))).to(t)
    more = {}
    if zeros:
        more["zeros"] = torch.randint(0, 16, (N, K // group), generator=g, device="cuda", dtype=torch.uint8)
    if bias:
        more["bias"] = _normal((N,), t, g)
    x = _channels((M, K), torch.float32, g)
    if rows == "same":
        x = x.to(t)
    else:
        a = x.abs().amax(-1)
        y = x * (plain.MOST[rows] / a)[:, None]
        x = (y.round() if rows == "i8" else y.clamp(-448, 448)).to(STORED[rows])
        more["row_scales"] = a / plain.MOST[rows]
    return x, weights, scales, more


def _linear_check(out, x, weights, scales, group, more, what):
    """Sums of 32 bits: a group's elements, each step off by at most a step (2^-23) of what was summed so far with the
    codes' 128; of the groups' results two roundings and one for each sum; the result's own half step."""
    K = x.shape[1]
    want, size = plain.linear4(x, weights, scales, group, more.get("zeros"), more.get("row_scales"), more.get("bias"))
    t = out.dtype
    steps = 2 * (group + 8) + K // group + 24
    want_t = want.clamp(-torch.finfo(t).max, torch.finfo(t).max)
    _inside(out, want_t, _half_step(t) * want.abs() + steps * UNIT * size + _least(t), what)
    # (those are bounds of the worst case: over all values the roundings are one of the result's type)
    if want.numel() > 200:
        off = (out.double() - want_t).norm() / want_t.norm()
        assert off < 1.05 * _half_step(t), f"{what}: {float(off):.3g} off in all"


def _linear(ctx, dtype, rows, group, zeros, bias, M, N, K, seed, strided=True):
    h = ctx.register_linear4(dtype, group=group, rows=None if rows == "same" else rows, zeros=zeros)
    x, weights, scales, more = _linear_inputs(dtype, rows, group, zeros, bias, M, N, K, seed)
    if strided:
        a, _ = _apart(M, K, x.dtype, 127)
        a.copy_(x)
        x = a
    out, whole = _apart(M, N, TYPES[dtype], 7) if strided else (torch.empty((M, N), dtype=TYPES[dtype], device="cuda"), None)
    h.launch(x, weights, scales, out, **more)
    _linear_check(out, x, weights, scales, group, more, f"{dtype} {rows} {group} {M} x {N} x {K}")
    if whole is not None:
        b = whole.view(torch.uint8)
        assert (b[:, :4] == 7).all() and (b[:, (2 + N) * 2:] == 7).all(), "written outside the rows"
    return out


@pytest.mark.parametrize("dtype,rows,group,zeros", [("bf16", "same", 128, False), ("bf16", "same", 64, True), ("f16", "same", 32, True), ("f16", "same", 64, False),
                                                    ("bf16", "i8", 128, False), ("f16", "i8", 64, True), ("bf16", "i8", 32, True), ("bf16", "e4m3", 128, True), ("f16", "e4m3", 32, False)])
def test_linear_matches_64_bits(ctx, dtype, rows, group, zeros):
    # (each kernel: of 1, 2 .. 4, 5 .. 16, 17 .. 32 and more rows, of few and many columns; ends of rows that are no whole run, chunk or block)
    for i, (M, N, blocks) in enumerate([(1, 16, 1), (1, 1, 3), (2, 33, 9), (16, 64, 8), (17, 100, 17), (5, 1003, 33), (32, 17, 64), (33, 48, 5), (64, 131, 31), (65, 20, 2), (150, 40, 40),
                                        (1, 70, 4), (3, 4200, 40), (4, 40, 64), (1, 20001, 18), (2, 17000, 16), (12, 9000, 12), (9, 16500, 37), (30, 16401, 21), (50, 16390, 35), (130, 16450, 9)]):
        _linear(ctx, dtype, rows, group, zeros, bool(i % 2), M, N, blocks * group, 100 + i, strided=bool((i // 2) % 2))


@pytest.mark.parametrize("dtype,rows,group,M,N,K", [("bf16", "same", 64, 1, 4096, 4096), ("f16", "same", 32, 1, 1000, 16384), ("bf16", "i8", 32, 16, 3001, 4096), ("bf16", "same", 64, 61, 2048, 8192),
                                                    ("bf16", "same", 64, 5, 40000, 2048), ("bf16", "e4m3", 128, 8, 20011, 1024), ("f16", "same", 32, 3, 16, 65536), ("f16", "i8", 64, 300, 512, 2048)])
def test_linear_of_larger_sizes(ctx, dtype, rows, group, M, N, K):
    _linear(ctx, dtype, rows, group, True, True, M, N, K, 7)


@pytest.mark.parametrize("dtype,rows,group,zeros", [("bf16", "same", 64, True), ("f16", "same", 32, False), ("f16", "i8", 32, True), ("bf16", "i8", 128, False), ("bf16", "e4m3", 64, True)])
def test_linear_of_blocks_of_every_shape(ctx, dtype, rows, group, zeros):
    # (rows of x and columns by which 2 x 4, 4 x 2 and 4 x 4 tiles make a block, ragged ends of both; rows of weights of short and of long k)
    for i, (M, N, K) in enumerate([(31, 9001, 9 * group), (40, 4111, 11 * group), (64, 8190, 4096), (33, 4100, 4096 + group), (61, 8191, 4096 + 3 * group), (90, 4095, 7 * group),
                                   (49, 12301, 5 * group), (64, 16384, 3 * group), (129, 5003, 1024 + group), (270, 2010, group), (9, 1003, 4096 + group), (16, 2049, 1024 + 5 * group),
                                   (6, 4081, 4096 + 3 * group), (5, 4113, 1024 + group), (13, 8191, 2048 + 7 * group), (7, 8205, 9 * group), (16, 16383, 17 * group), (3, 16401, 1024 + 7 * group),
                                   (16, 16500, 2048 + 9 * group), (20, 1001, 13 * group), (40, 1999, 21 * group), (18, 16500, 5 * group), (8, 16999, 1024)]):
        _linear(ctx, dtype, rows, group, zeros, bool(i % 2), M, N, K, 200 + i, strided=bool((i // 2) % 2))


# ---- drafted tokens --------------------------------------------------------------------------------


def _verify_inputs(dtype, B, D, V, seed, near=0.8):
    g = _generator(seed)
    t = TYPES[dtype]
    logits = _normal((B, D + 1, V), torch.float32, g, 2.0)
    close = logits[:, :D] + _normal((B, D, V), torch.float32, g, near)
    target, draft = torch.softmax(logits, -1).to(t), torch.softmax(close, -1).to(t)
    drafted = (close - torch.empty_like(close).exponential_(generator=g).log_()).argmax(-1).to(torch.int32) if D else torch.empty((B, 0), dtype=torch.int32, device="cuda")
    uniforms = torch.empty((B, D + 1), device="cuda").uniform_(0.0, 1.0, generator=g).clamp_(max=1 - 2.0 ** -24)
    return target, drafted, uniforms, draft


def _verify(ctx, dtype, target, drafted, uniforms, draft=None, lengths=None):
    h = ctx.register_verify(dtype)
    B, D = drafted.shape
    tokens = torch.full((B, D + 1), -9, dtype=torch.int32, device="cuda")
    accepted = torch.full((B,), -9, dtype=torch.int32, device="cuda")
    ws = torch.full((max(16, h.workspace_bytes(B, target.shape[2])),), 255, dtype=torch.uint8, device="cuda")
    h.launch(target, drafted, uniforms, tokens, accepted, draft=draft, lengths=lengths, workspace=ws)
    want, kept = plain.verify(target, drafted, uniforms, draft, lengths)
    assert torch.equal(accepted.cpu(), kept), (accepted.cpu(), kept)
    assert torch.equal(tokens.cpu(), want), (tokens.cpu(), want)
    return tokens, accepted


@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("B,D,V", [(1, 4, 32000), (3, 1, 1), (5, 3, 7), (40, 8, 1003), (9, 12, 4096), (7, 5, 4097), (16, 0, 5000), (2, 70, 513), (3, 130, 40), (3, 2, 200001)])
def test_verify_matches_64_bits(ctx, dtype, B, D, V):
    target, drafted, uniforms, draft = _verify_inputs(dtype, B, D, V, B + D + V)
    lengths = torch.randint(-1, D + 3, (B,), generator=_generator(1), device="cuda", dtype=torch.int32)
    _verify(ctx, dtype, target, drafted, uniforms, draft)
    _verify(ctx, dtype, target, drafted, uniforms, draft, lengths)
    _verify(ctx, dtype, target, drafted, uniforms)
    _verify(ctx, dtype, target, drafted, uniforms, None, lengths)


def test_verify_strides(ctx):
    """Rows of a larger tensor, sequences innermost in one and padded vocabularies in the other."""
    target, drafted, uniforms, draft = _verify_inputs("f32", 6, 4, 5000, 31)
    want = _verify(ctx, "f32", target, drafted, uniforms, draft)
    wide = torch.full((5, 6, 5017), math.nan, device="cuda")
    wide[:, :, 3:5003] = target.transpose(0, 1)
    long = torch.full((6, 9, 5001), math.nan, device="cuda")
    long[:, 2:6, 1:] = draft
    got = _verify(ctx, "f32", wide.transpose(0, 1)[:, :, 3:5003], drafted, uniforms, long[:, 2:6, 1:])
    assert torch.equal(got[0], want[0])


def test_verify_at_the_borders(ctx):
    """Uniforms of 0 and just below 1, equal and disjoint distributions, tokens without probability and outside the vocabulary,
    rows without anything, infinities, NaN and negative numbers."""
    B, D, V = 14, 3, 9000
    target, drafted, uniforms, draft = _verify_inputs("f32", B, D, V, 33)
    uniforms[0] = 0
    uniforms[1] = 1 - 2.0 ** -24
    draft[2] = target[2, :D]                              # all kept but for the uniforms' strictness; nothing left over
    uniforms[2, 0] = 1.0                                  # (not kept: u q < p fails, and the rest is empty: the target's row)
    target[3, :, : V // 2] = 0
    draft[3, :, V // 2:] = 0
    drafted[3] = 5                                        # the target has nothing there
    drafted[4, 0], drafted[5, 1], drafted[6, 0] = -1, V, 2 ** 31 - 1
    target[7] = 0
    draft[7] = 0
    target[8, :, 17] = math.nan
    target[8, :, 18] = math.inf
    target[8, :, 19] = -3.0
    drafted[8] = 17
    target[9] = 0
    target[9, :, V - 1] = 1.0
    target[10] = 0
    target[10, :, 0] = 2.0 ** -126                        # (sums of a few of the smallest numbers)
    target[10, :, 4500] = 2.0 ** -126
    draft[11] = math.nan
    uniforms[12, :D] = math.nan
    target[13], draft[13] = 1.0 / V, 0.0                  # a draft that says that its token could not come: kept
    _verify(ctx, "f32", target, drafted, uniforms, draft)
    _verify(ctx, "f32", target, drafted, uniforms)


def test_verify_follows_the_target(ctx):
    """Many sequences of one place: the tokens that come out have the target's frequencies, whatever the draft's."""
    V, B = 6, 20000
    g = _generator(35)
    p, q = torch.softmax(_normal((V,), torch.float32, g), 0), torch.softmax(_normal((V,), torch.float32, g), 0)
    drafted = torch.multinomial(q, B, replacement=True, generator=g).to(torch.int32)[:, None]
    uniforms = torch.empty((B, 2), device="cuda").uniform_(0, 1, generator=g).clamp_(max=1 - 2.0 ** -24)
    h = ctx.register_verify("f32")
    tokens, accepted = torch.empty((B, 2), dtype=torch.int32, device="cuda"), torch.empty(B, dtype=torch.int32, device="cuda")
    h.launch(p.expand(B, 2, V), drafted, uniforms, tokens, accepted, draft=q.expand(B, 1, V), workspace=torch.empty(h.workspace_bytes(B, V), dtype=torch.uint8, device="cuda"))
    share = torch.bincount(tokens[:, 0].long(), minlength=V).double() / B
    assert ((share - p.double()).abs() < 5 * (p.double() * (1 - p.double()) / B).sqrt()).all()
    assert (accepted.double().mean() - torch.minimum(p, q).double().sum()).abs() < 5 * 0.5 / math.sqrt(B)


def test_verify_of_more_chunks_than_lanes(ctx):
    """Vocabularies of more than 64 chunks of 4096: a lane has several, and the goal falls into one of them."""
    for V, drafts in ((300001, 2), (1200000, 1)):
        target, drafted, uniforms, draft = _verify_inputs("f32", 3, drafts, V, V)
        uniforms[1, -1] = 1 - 2.0 ** -24
        _verify(ctx, "f32", target, drafted, uniforms, draft)
        target[2] = 0
        target[2, :, V - 1] = 0.5
        _verify(ctx, "f32", target, drafted, uniforms)


# ---- products at the ends of their types -----------------------------------------------------------


@pytest.mark.parametrize("M,N", [(1, 40), (3, 40), (12, 40), (24, 40), (50, 40), (12, 16500), (60, 16500)])
def test_linear_of_the_largest_rows_and_scales(ctx, M, N):
    """Sums that pass 32 bits on the way to a result that does not, beside ordinary rows."""
    K, group = 512, 128
    h = ctx.register_linear4("bf16", group=group)
    x, weights, scales, _ = _linear_inputs("bf16", "same", group, False, False, M, N, K, 61)
    big = torch.finfo(torch.bfloat16).max
    x[M - 1] = (torch.sign(x[M - 1].float()) * big).to(torch.bfloat16)
    scales *= 2.0 ** -10
    scales[5] = (scales[5].float() * 2.0 ** 120).to(torch.bfloat16)      # (a column of scales that make large rows infinite)
    out = torch.empty((M, N), dtype=torch.bfloat16, device="cuda")
    h.launch(x, weights, scales, out)
    want, size = plain.linear4(x, weights, scales, group)
    finite = want.abs() < 0.99 * big
    assert bool(finite[M - 1].float().mean() > 0.9) and torch.equal(torch.isfinite(out[:, :5]), finite[:, :5])
    # (as _linear_check; the second time around every term is the same number times a power of two)
    steps = 2 * (group + 8) + K // group + 24
    bound = _half_step(torch.bfloat16) * want.abs() + steps * UNIT * size + _least(torch.bfloat16)
    _inside(out[finite], want[finite], bound[finite], "largest rows")
    # i8 rows whose scales take the weights' back
    h = ctx.register_linear4("bf16", group=group, rows="i8")
    x, weights, scales, more = _linear_inputs("bf16", "i8", group, False, False, M, N, K, 62)
    scales = (scales.float() * 2.0 ** 122).to(torch.bfloat16)
    more["row_scales"] = torch.full((M,), 2.0 ** -60, device="cuda")
    more["row_scales"][0] = 2.0 ** -100
    h.launch(x, weights, scales, out, **more)
    want, size = plain.linear4(x, weights, scales, group, row_scales=more["row_scales"])
    assert torch.isfinite(out).all()
    _inside(out, want, _half_step(torch.bfloat16) * want.abs() + steps * UNIT * size + _least(torch.bfloat16), "largest scales")


@pytest.mark.parametrize("rows", ["same", "i8", "e4m3"])
@pytest.mark.parametrize("M,N", [(2, 70), (9, 70), (20, 70), (40, 70)])
def test_linear_rows_do_not_see_each_other(ctx, rows, M, N):
    dtype, group, zeros = {"same": ("bf16", 64, True), "i8": ("f16", 64, True), "e4m3": ("bf16", 128, True)}[rows]
    K = 9 * group
    h = ctx.register_linear4(dtype, group=group, rows=None if rows == "same" else rows, zeros=zeros)
    x, weights, scales, more = _linear_inputs(dtype, rows, group, zeros, True, M, N, K, 63)
    want = torch.empty((M, N), dtype=TYPES[dtype], device="cuda")
    h.launch(x, weights, scales, want, **more)
    other = x.clone()
    if rows == "same":
        other[M - 1, 3] = math.inf
        other[M - 1, 70] = -math.inf
        other[M // 2, 9] = math.nan
    elif rows == "e4m3":
        other[M - 1, 3] = math.nan
    else:
        other[M - 1] = 127
    if rows != "same":
        more["row_scales"] = more["row_scales"].clone()
        more["row_scales"][M // 2] = math.nan
    got = torch.empty_like(want)
    h.launch(other, weights, scales, got, **more)
    kept = [m for m in range(M) if m not in (M - 1, M // 2)]
    assert torch.equal(got[kept], want[kept]) and not torch.isfinite(got[M // 2]).any()
    assert rows == "i8" or not torch.isfinite(got[M - 1]).any()


@pytest.mark.parametrize("M,N", [(20, 8209), (40, 4099), (40, 8200), (12, 4100), (12, 8200)])
def test_linear_of_the_largest_rows_by_columns(ctx, M, N):
    test_linear_of_the_largest_rows_and_scales(ctx, M, N)
    test_linear_rows_do_not_see_each_other(ctx, "same", M, N)
    test_linear_rows_do_not_see_each_other(ctx, "i8", M, N)


def test_past_32_bits(ctx):
    """Weights, rows and probabilities that lie further apart than 32 bits count bytes or elements."""
    g = _generator(64)
    # weights of more than 2^32 bytes
    N, K, group = 330003, 32768, 128
    h = ctx.register_linear4("bf16", group=group)
    weights = torch.randint(0, 256, (N, K // 2), generator=g, device="cuda", dtype=torch.uint8)
    scales = torch.empty((N, K // group), dtype=torch.bfloat16, device="cuda").uniform_(0.001, 0.002, generator=g)
    for M in (1, 12, 40):
        x = _channels((M, K), torch.bfloat16, g)
        out = torch.empty((M, N), dtype=torch.bfloat16, device="cuda")
        h.launch(x, weights, scales, out)
        for part in (slice(0, 40), slice(N // 2, N // 2 + 40), slice(N - 40, N)):
            _linear_check(out[:, part], x, weights[part], scales[part], group, {}, f"{M} rows, columns {part}")
    del weights, scales, out
    # rows 2^31 elements apart
    whole = torch.zeros(2 ** 32 + 2 ** 31 + 2 ** 14, dtype=torch.bfloat16, device="cuda")
    x = whole.as_strided((3, 1000), (2 ** 31, 1))
    x.copy_(_channels((3, 1000), torch.bfloat16, g))
    codes, scales, _ = _norm(ctx, "bf16", "i8", 3, 1000, 0.0, None, 65, strided=False, x=x)
    h = ctx.register_norm("bf16", "i8", eps=EPS)
    dw, dx = torch.empty(1000, device="cuda"), torch.empty((3, 1000), dtype=torch.bfloat16, device="cuda")
    dense, weight = x.contiguous(), _normal((1000,), torch.bfloat16, g)
    ws = torch.empty(h.workspace_bytes(3, 1000), dtype=torch.uint8, device="cuda")
    h.backward(dense, weight, dense, dx, dw, workspace=ws)
    into = whole.as_strided((3, 1000), (2 ** 31, 1), 2000)
    also = torch.empty_like(dw)
    h.backward(x, weight, x, into, also, workspace=ws)
    assert torch.equal(into, dx) and torch.equal(also, dw)
    # places and sequences as far apart
    target, drafted, uniforms, _ = _verify_inputs("bf16", 2, 1, 5000, 66)
    far = whole.as_strided((2, 2, 5000), (2 ** 32, 2 ** 31, 1), 4000)
    far.copy_(target)
    _verify(ctx, "bf16", far, drafted, uniforms)


# ---- streams, graphs, a step of all of them --------------------------------------------------------


def test_calls_on_other_streams(ctx):
    """Torch's current stream and the launch's own; two streams at once, each with a workspace of its own."""
    g = _generator(67)
    t = torch.bfloat16
    norm, verify, linear = ctx.register_norm("bf16", "i8", eps=EPS), ctx.register_verify("f32"), ctx.register_linear4("bf16", rows="i8")
    total, dy, weight = _channels((2000, 1024), t, g), _normal((2000, 1024), t, g), _normal((1024,), t, g)
    target, drafted, uniforms, draft = _verify_inputs("f32", 20, 3, 50000, 68)
    _, weights, scales, _ = _linear_inputs("bf16", "i8", 128, False, False, 4, 500, 1024, 69)

    def run(stream=None):
        dx, dw = torch.empty_like(total), torch.empty(1024, device="cuda")
        codes, row_scales = torch.empty((4, 1024), dtype=torch.int8, device="cuda"), torch.empty(4, device="cuda")
        out = torch.empty((4, 500), dtype=t, device="cuda")
        tokens, accepted = torch.empty((20, 4), dtype=torch.int32, device="cuda"), torch.empty(20, dtype=torch.int32, device="cuda")
        ws = [torch.empty(n, dtype=torch.uint8, device="cuda") for n in (norm.workspace_bytes(2000, 1024), verify.workspace_bytes(20, 50000))]
        norm.backward(total, weight, dy, dx, dw, workspace=ws[0], stream=stream)
        verify.launch(target, drafted, uniforms, tokens, accepted, draft=draft, workspace=ws[1], stream=stream)
        norm.launch(total[:4], weight, codes, row_scales, stream=stream)
        linear.launch(codes, weights, scales, out, row_scales=row_scales, stream=stream)
        return [dx, dw, tokens, accepted, codes, row_scales, out], ws
    want, _ = run()
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(2)]
    kept = []
    for turn in range(4):
        with torch.cuda.stream(streams[turn % 2]):
            kept.append(run())
    torch.cuda.synchronize()
    kept.append(run(stream=streams[0].cuda_stream))
    torch.cuda.synchronize()
    for got, _ in kept:
        assert all(torch.equal(a, b) for a, b in zip(got, want))


def test_a_gradient_captured_while_eager_ones_live(ctx):
    """Forward and backward in a graph, replayed with other rows between eager calls of the same tensors."""
    g = _generator(70)
    rows, width = 700, 1000
    h = ctx.register_norm("f32", "i8", eps=EPS)
    sets = [[_normal(s, torch.float32, _generator(71 + i)) for s in ((rows, width), (rows, width), (width,), (rows, width), (rows, width))] for i in range(3)]
    need = h.workspace_bytes(rows, width)

    def run(x, residual, weight, dy, dtotal, outs, ws):
        total, codes, scales, dx, dw = outs
        h.launch(x, weight, codes, scales, residual=residual, total=total)
        h.backward(total, weight, dy, dx, dw, dtotal=dtotal, workspace=ws)

    def outputs():
        return [torch.empty((rows, width), device="cuda"), torch.empty((rows, width), dtype=torch.int8, device="cuda"), torch.empty(rows, device="cuda"),
                torch.empty((rows, width), device="cuda"), torch.empty(width, device="cuda")]
    static, outs, ws = [t.clone() for t in sets[0]], outputs(), torch.empty(need, dtype=torch.uint8, device="cuda")
    run(*static, outs, ws)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        run(*static, outs, ws)
    for turn in range(5):
        s = sets[turn % 3]
        for a, b in zip(static, s):
            a.copy_(b)
        ws.fill_(255)
        eager, own = outputs(), torch.empty(need, dtype=torch.uint8, device="cuda")
        run(*s, eager, own)
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(outs, eager))
        assert torch.equal(eager[0], s[0] + s[1])
    del g


def _softmax_pattern(ctx):
    from workloads import PatternBuilder
    pb = PatternBuilder("softmax_f32")
    T, V = pb.dims(2)
    x = pb.cast(pb.param("bf16", [T, V]), "f32")
    e = pb.op("exp", pb.op("sub", x, pb.broadcast(pb.reduce("max", x, 1), [T, V], [0])))
    pb.output(pb.op("div", e, pb.broadcast(pb.reduce("sum", e, 1), [T, V], [0])))
    return ctx.register(pb.build())


def test_a_step_with_drafted_tokens(ctx):
    """What a decoder's step is: norm into 8-bit rows, their product with 4-bit weights, rotation, store, attention, the product back, the
    next norm with the residual, logits, softmax and the check of the drafted tokens; each against 64 bits of what it was given.
    Captured, and replayed with other rows, tokens and uniforms: the same as eager calls."""
    from oracle import decoder
    from paper_2103_05288_amd import rotary_frequencies
    t = torch.bfloat16
    B, D, width, heads, kv, dim, size, V = 3, 2, 512, 4, 2, 64, 16, 3001
    M = B * (D + 1)                                            # (a drafted token is a row of the batch: its sequence's pages, one token longer)
    norm, rotary, cache = ctx.register_norm("bf16", "i8", eps=EPS), ctx.register_rotary("bf16", dim, rotary_frequencies(dim)[0]), ctx.register_cache("bf16", dim, "i8")
    from_norm, plainly, verify, softmax = ctx.register_linear4("bf16", rows="i8"), ctx.register_linear4("bf16", group=64, zeros=True), ctx.register_verify("f32"), _softmax_pattern(ctx)
    g = _generator(81)
    qkv_rows = (heads + 2 * kv) * dim
    weights = [_linear_inputs("bf16", "i8", 128, False, False, 1, qkv_rows, width, 82), _linear_inputs("bf16", "same", 64, True, True, 1, width, heads * dim, 83),
               _linear_inputs("bf16", "i8", 128, False, False, 1, V, width, 84)]
    gains = [(1 + _normal((width,), torch.float32, g, 0.1)).to(t) for _ in range(2)]
    lengths = torch.tensor([5, 20, 31], device="cuda")
    table = torch.arange(3 * 3, device="cuda", dtype=torch.int32).view(3, 3).repeat_interleave(D + 1, 0).contiguous()
    filled = [torch.randint(-127, 128, (9, kv, size, dim), generator=g, device="cuda", dtype=torch.int8) for _ in range(2)]
    filled += [torch.full((9, kv, size), 0.01, device="cuda") for _ in range(2)]
    at = (lengths[:, None] + torch.arange(D + 1, device="cuda")).flatten()
    slots = table.long()[torch.arange(M, device="cuda"), at // size] * size + at % size
    seen = (at + 1).int()
    sizes = [norm.workspace_bytes(1, 1), cache.workspace_bytes(M, heads, kv, 3 * size), verify.workspace_bytes(B, V)]

    def inputs(turn):
        k = _generator(90 + turn)
        return {"x": _channels((M, width), t, k), "residual": _channels((M, width), t, k), "drafted": torch.randint(0, V, (B, D), generator=k, device="cuda", dtype=torch.int32),
                "uniforms": torch.empty((B, D + 1), device="cuda").uniform_(0, 1, generator=k).clamp_(max=1 - 2.0 ** -24) * 0.01}

    def buffers():
        e = lambda *s, dtype=t: torch.empty(s, dtype=dtype, device="cuda")  # noqa: E731
        return {"pages": [p.clone() for p in filled], "total": e(M, width), "codes": e(M, width, dtype=torch.int8), "scales": e(M, dtype=torch.float32), "qkv": e(M, qkv_rows),
                "attended": e(M, heads, dim), "back": e(M, width), "total2": e(M, width), "codes2": e(M, width, dtype=torch.int8), "scales2": e(M, dtype=torch.float32),
                "logits": e(M, V), "p": e(M, V, dtype=torch.float32), "tokens": e(B, D + 1, dtype=torch.int32), "accepted": e(B, dtype=torch.int32),
                "ws": [torch.empty(max(16, n), dtype=torch.uint8, device="cuda") for n in sizes]}

    def step(i, o):
        norm.launch(i["x"], gains[0], o["codes"], o["scales"], residual=i["residual"], total=o["total"])
        from_norm.launch(o["codes"], weights[0][1], weights[0][2], o["qkv"], row_scales=o["scales"])
        rows = o["qkv"].view(M, heads + 2 * kv, dim)
        q, k, v = rows[:, :heads], rows[:, heads:heads + kv], rows[:, heads + kv:]
        rotary.launch(at, [q, k], [q, k])
        cache.store([k, v], slots, o["pages"])
        cache.attend(q, seen, table, o["pages"], o["attended"], workspace=o["ws"][1])
        plainly.launch(o["attended"].view(M, heads * dim), weights[1][1], weights[1][2], o["back"], **weights[1][3])
        norm.launch(o["back"], gains[1], o["codes2"], o["scales2"], residual=o["total"], total=o["total2"])
        from_norm.launch(o["codes2"], weights[2][1], weights[2][2], o["logits"], row_scales=o["scales2"])
        softmax.launch([M, V], [o["logits"]], [o["p"]])
        verify.launch(o["p"].view(B, D + 1, V), i["drafted"], i["uniforms"], o["tokens"], o["accepted"], workspace=o["ws"][2])

    static, outs = inputs(0), buffers()
    step(static, outs)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step(static, outs)
    for turn in range(4):
        i, o = inputs(turn), buffers()
        step(i, o)
        for k, x in i.items():
            static[k].copy_(x)
        for a, b in zip(outs["pages"], filled):
            a.copy_(b)
        graph.replay()
        torch.cuda.synchronize()
        for k in o:
            for a, b in zip(*([o[k], outs[k]] if isinstance(o[k], list) else [[o[k]], [outs[k]]])):
                assert k == "ws" or torch.equal(a, b), (turn, k)
        for x, gain, codes, scales, residual, total in ((i["x"], gains[0], o["codes"], o["scales"], i["residual"], o["total"]), (o["back"], gains[1], o["codes2"], o["scales2"], o["total"], o["total2"])):
            _, y, largest = plain.norm(x, gain, EPS, 0.0, residual)
            _check_codes(codes, scales, y, largest, "i8", "step")
            assert torch.equal(total, (x.float() + residual.float()).to(t))
        fresh = torch.empty_like(o["qkv"])
        from_norm.launch(o["codes"], weights[0][1], weights[0][2], fresh, row_scales=o["scales"])      # (the first was turned in place)
        _linear_check(fresh, o["codes"], weights[0][1], weights[0][2], 128, {"row_scales": o["scales"]}, "qkv")
        want = decoder.attend(o["qkv"].view(M, heads + 2 * kv, dim)[:, :heads], seen, table, o["pages"], 0.125)[0]
        assert (o["attended"].double() - want).abs().max() < 2.0 ** -7 * want.abs().max()
        _linear_check(o["back"], o["attended"].view(M, heads * dim), weights[1][1], weights[1][2], 64, weights[1][3], "back")
        _linear_check(o["logits"], o["codes2"], weights[2][1], weights[2][2], 128, {"row_scales": o["scales2"]}, "logits")
        # (the softmax in 32 bits: exp of a difference of logits, both roundings of it, the sum and the quotient)
        p = torch.softmax(o["logits"].double(), -1)
        _inside(o["p"], p, p * (1e-5 + 2 * UNIT * o["logits"].double().abs().amax()) + 2.0 ** -126, "softmax")
        tokens, kept = plain.verify(o["p"].view(B, D + 1, V), i["drafted"], i["uniforms"])
        assert torch.equal(o["tokens"].cpu(), tokens) and torch.equal(o["accepted"].cpu(), kept)


# ---- products whose largest channels have no weight ------------------------------------------------


def _heavy_inputs(dtype, rows, group, zeros, M, N, K, seed):
    """Ordinary rows with a few channels that are 2^13 .. 2^22 times as large, at which every code is its zero point."""
    x, weights, scales, more = _linear_inputs(dtype, rows, group, zeros, False, M, N, K, seed)
    g = _generator(seed + 1)
    if zeros:                                                  # (any byte is a zero point; only one of 0 .. 15 is a code too)
        more["zeros"] = torch.randint(0, 256, more["zeros"].shape, generator=g, device="cuda", dtype=torch.uint8)
    z = more["zeros"] if zeros else torch.full((N, K // group), 8, dtype=torch.uint8, device="cuda")
    at = torch.arange(3, K, 41, device="cuda")
    of = at // group
    if zeros:
        z[:, of] = z[:, of] % 16
    codes = plain.codes4(weights).to(torch.uint8)
    codes[:, at] = z[:, of]
    weights = codes[:, 0::2] | codes[:, 1::2] << 4
    std, most = {"same": (1.0, 2.0 ** 22) if dtype == "bf16" else (2.0 ** -6, 6e4), "i8": (2.0, 127.0), "e4m3": (2.0 ** -4, 448.0)}[rows]
    x = torch.empty((M, K), device="cuda").normal_(0.0, std, generator=g)
    x[:, at] = most * torch.where(torch.rand((M, len(at)), generator=g, device="cuda") < 0.5, -1.0, 1.0) * (1 - 0.5 * torch.rand((M, len(at)), generator=g, device="cuda"))
    x = (x.round() if rows == "i8" else x).to(TYPES[dtype] if rows == "same" else STORED[rows])
    if rows != "same":
        more["row_scales"] = torch.full((M,), 0.01, device="cuda")
    return x, weights.contiguous(), scales, more


@pytest.mark.parametrize("dtype,rows,group,zeros", [("bf16", "same", 128, False), ("bf16", "same", 64, True), ("bf16", "same", 32, True), ("bf16", "same", 32, False),
                                                    ("f16", "same", 128, True), ("f16", "same", 64, False), ("f16", "same", 32, True), ("f16", "e4m3", 64, True),
                                                    ("bf16", "e4m3", 32, False), ("bf16", "i8", 128, True), ("f16", "i8", 32, False)])
def test_linear_of_large_channels_without_weight(ctx, dtype, rows, group, zeros):
    """A channel whose code is the zero point adds nothing, however large it is: rounded to nothing but what 32 bits leave of the others'
    sum.  Through each kernel."""
    h = ctx.register_linear4(dtype, group=group, rows=None if rows == "same" else rows, zeros=zeros)
    for i, (M, N, K) in enumerate([(1, 40, 512), (1, 64, 4096), (1, 5000, 2048 + group), (1, 17001, 2048), (3, 40, 512), (3, 300, 2048 + 3 * group), (12, 40, 512), (12, 17000, 512), (12, 64, 4096),
                                   (12, 5000, 2048), (12, 9000, 2048 + group), (3, 17000, 2048), (24, 64, 2048), (24, 5000, 2048), (24, 9000, 2048 + group), (24, 17000, 1024),
                                   (50, 64, 2048), (50, 3000, 2048 + group), (61, 6000, 2048), (50, 9000, 1024 + group), (64, 17000, 1024)]):
        x, weights, scales, more = _heavy_inputs(dtype, rows, group, zeros, M, N, K, 300 + i)
        out = torch.empty((M, N), dtype=TYPES[dtype], device="cuda")
        h.launch(x, weights, scales, out, **more)
        _linear_check(out, x, weights, scales, group, more, f"{dtype} {rows} {group} {M} x {N} x {K}")


# ---- in place, where an access reaches over a wavefront's own elements -----------------------------


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_in_place_at_ragged_ends(ctx, dtype):
    """The last access of a ragged row starts among its neighbour's elements, which may be another wavefront's, written by then."""
    t, g = TYPES[dtype], _generator(401)
    v = 8 if dtype == "bf16" else 4
    h = ctx.register_norm(dtype, "i8", eps=EPS)
    for rows, accesses in ((3, 65), (700, 129), (900, 257), (3, 513), (700, 1025), (600, 2049), (5, 2049), (300, 2500)):
        for over in (1, v - 1):
            width = (accesses - 1) * v + over
            x, residual, dy, dtotal = (_channels((rows, width), t, g) for _ in range(4))
            weight = _normal((width,), t, g)

            def forward(x, residual, total):
                codes, scales = torch.empty((rows, width), dtype=torch.int8, device="cuda"), torch.empty(rows, device="cuda")
                h.launch(x, weight, codes, scales, residual=residual, total=total)
                return total, codes, scales
            want = forward(x, residual, torch.empty_like(x))
            for into in (0, 1):
                a = [x.clone(), residual.clone()]
                assert all(torch.equal(p, q) for p, q in zip(forward(*a, a[into]), want)), (rows, width, into)
            twice = forward(x, x, torch.empty_like(x))
            a = x.clone()
            assert all(torch.equal(p, q) for p, q in zip(forward(a, a, a), twice)), (rows, width)

            def backward(total, dy, dtotal, dx):
                dw, ws = torch.empty(width, device="cuda"), torch.empty(h.workspace_bytes(rows, width), dtype=torch.uint8, device="cuda")
                h.backward(total, weight, dy, dx, dw, dtotal=dtotal, workspace=ws)
                return dx, dw
            want = backward(x, dy, dtotal, torch.empty_like(x))
            for into in (0, 1, 2):
                a = [x.clone(), dy.clone(), dtotal.clone()]
                assert all(torch.equal(p, q) for p, q in zip(backward(*a, a[into]), want)), (rows, width, into)
