"""Rotary positions, the cache and attention over it without a GPU: what is refused, the plans' sizes, the device
header's index arithmetic built for the CPU, the frequencies, and that every combination compiles."""
import ctypes as C
import math
import os
import random
import re

import pytest
import torch

import paper_2103_05288_amd as pkg
from oracle import decoder as plain
from paper_2103_05288_amd import binding
from tests.util import host_build


@pytest.fixture(scope="module")
def ctx():
    c = pkg.Context(-1)
    yield c
    c.close()


def _refused(status, words, call):
    with pytest.raises(pkg.DiscError) as e:
        call()
    assert e.value.status == status and words in e.value.message, (e.value.status, e.value.message)


HOST_ONLY = "host-only context cannot launch"


# ---- registration ----------------------------------------------------------------------------------


def test_registrations_compile_once(ctx):
    f, _ = pkg.rotary_frequencies(64)
    before = ctx.stats()["compile_events"]
    a = ctx.register_rotary("bf16", 64, f)
    b = ctx.register_rotary("bf16", 64, list(f))
    c = ctx.register_rotary("bf16", 64, f, layout="interleaved")
    d = ctx.register_cache("bf16", 64, "i8")
    e = ctx.register_cache("bf16", 64, "i8", softmax_scale=0.125)      # what the head size gives by itself
    assert a.id == b.id and a.id != c.id and d.id == e.id and d.id not in (a.id, c.id)
    assert ctx.stats()["compile_events"] == before + 3


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("layout", ["half", "interleaved"])
@pytest.mark.parametrize("D,R", [(2, 2), (80, 26), (255, 2), (256, 254), (99, 50)])
def test_rotary_compiles(ctx, dtype, layout, D, R):
    ctx.register_rotary(dtype, D, pkg.rotary_frequencies(R)[0], layout=layout)


@pytest.mark.parametrize("dtype,storage", [("bf16", None), ("f16", "i8"), ("bf16", "e4m3")])
@pytest.mark.parametrize("D", [16, 112, 256])
def test_cache_compiles(ctx, dtype, storage, D):
    ctx.register_cache(dtype, D, storage)


def test_registrations_that_are_refused(ctx):
    f, _ = pkg.rotary_frequencies(64)
    _refused("INVALID_ARG", "no such type", lambda: ctx.register_rotary("i8", 64, f))
    _refused("INVALID_ARG", "no such type", lambda: ctx.register_rotary("f32", 64, f, layout="thirds"))
    _refused("INVALID_ARG", "f32, f16 or bf16", lambda: ctx.register_rotary("i32", 64, f))
    _refused("SHAPE", "rotary_dim", lambda: ctx.register_rotary("f32", 62, f))
    _refused("SHAPE", "rotary_dim", lambda: ctx.register_rotary("f32", 64, []))
    _refused("SHAPE", "head_dim", lambda: ctx.register_rotary("f32", 257, f))
    _refused("INVALID_ARG", "frequency", lambda: ctx.register_rotary("f32", 64, [math.nan] * 32))
    _refused("INVALID_ARG", "frequency", lambda: ctx.register_rotary("f32", 64, [4.0] * 32))
    _refused("INVALID_ARG", "magnitude", lambda: ctx.register_rotary("f32", 64, f, magnitude=math.inf))
    _refused("INVALID_ARG", "no such type", lambda: ctx.register_cache("bf16", 64, "f16"))
    _refused("INVALID_ARG", "f16 or bf16", lambda: ctx.register_cache("f32", 64))
    for D in (0, 8, 72, 272):
        _refused("SHAPE", "head_dim", lambda: ctx.register_cache("bf16", D, "i8"))
    _refused("INVALID_ARG", "softmax", lambda: ctx.register_cache("bf16", 64, softmax_scale=0))
    _refused("INVALID_ARG", "softmax", lambda: ctx.register_cache("bf16", 64, softmax_scale=math.nan))
    # finite in 64 bits, not in the 32 that the kernels have
    _refused("INVALID_ARG", "softmax", lambda: ctx.register_cache("bf16", 64, softmax_scale=3e38))
    _refused("INVALID_ARG", "magnitude", lambda: ctx.register_rotary("f32", 64, f, magnitude=1e39))
    lib, out = ctx.lib, C.c_int32(5)
    assert lib.disc_register_cache(ctx.h, None, C.byref(out)) == -1 and lib.disc_register_rotary(ctx.h, None, C.byref(out)) == -1
    assert lib.disc_register_cache(None, None, C.byref(out)) == -1 and out.value == 5
    desc = binding.disc_cache_desc(2, 3, 64, 0.0)
    assert lib.disc_register_cache(ctx.h, C.byref(desc), C.byref(out)) == -1


def test_softmax_scales_at_the_end_of_32_bits(ctx):
    """... where i8's codes take 2^9 of them from fp16 queries."""
    ctx.register_cache("f16", 64, "i8", softmax_scale=4e35)
    _refused("INVALID_ARG", "softmax", lambda: ctx.register_cache("f16", 64, "i8", softmax_scale=5e35))
    _refused("INVALID_ARG", "softmax", lambda: ctx.register_cache("f16", 64, "i8", softmax_scale=-5e35))
    ctx.register_cache("bf16", 64, "i8", softmax_scale=5e35)
    ctx.register_cache("f16", 64, softmax_scale=2e38)


def test_frequencies():
    f, m = pkg.rotary_frequencies(8, base=10000.0)
    assert m == 1.0 and f == [10000.0 ** (-j / 4) for j in range(4)]
    g, m = pkg.rotary_frequencies(8, scaling="linear", factor=4.0)
    assert m == 1.0 and g == [x / 4 for x in f]
    g, m = pkg.rotary_frequencies(8, scaling="base", factor=4.0)
    assert m == 1.0 and g[0] == 1.0 and g[3] == pytest.approx(f[3] / 4, rel=1e-12)         # the slowest pair: stretched by the factor
    g, m = pkg.rotary_frequencies(64, scaling="by_parts", factor=16.0, original_length=4096)
    f, _ = pkg.rotary_frequencies(64)
    assert m == pytest.approx(0.1 * math.log(16.0) + 1.0)
    for x, y in zip(f, g):
        turns = 4096 * x / (2 * math.pi)
        assert y == x if turns >= 32 else y == pytest.approx(x / 16) if turns <= 1 else x / 16 < y < x
    for bad in (dict(rotary_dim=7), dict(rotary_dim=0), dict(rotary_dim=8, base=-1.0), dict(rotary_dim=8, scaling="cubic"),
                dict(rotary_dim=8, scaling="linear", factor=0.5), dict(rotary_dim=8, scaling="by_parts", factor=2.0), dict(rotary_dim=2, scaling="base", factor=2.0)):
        with pytest.raises(pkg.DiscError):
            pkg.rotary_frequencies(**bad)


# ---- calls -----------------------------------------------------------------------------------------
# (a host-only context goes through every check of a launch and then says that it cannot launch)


@pytest.fixture(params=["quick", "slow"])
def path(request, monkeypatch):
    """With the checks and the marshalling of a call that fits in C, and without."""
    if request.param == "slow":
        monkeypatch.setattr(binding, "_pylaunch", binding._CtypesLaunch)
    return request.param


def test_rotary_calls(ctx, path):
    h = ctx.register_rotary("f32", 8, pkg.rotary_frequencies(8)[0])
    x, y = torch.zeros(5, 3, 8), torch.zeros(5, 3, 8)
    p = torch.arange(5)
    ok = lambda *a, **k: _refused("INVALID_ARG", HOST_ONLY, lambda: h.launch(*a, **k))  # noqa: E731
    no = lambda words, *a, **k: _refused(k.pop("status", "INVALID_ARG"), words, lambda: h.launch(*a, **k))  # noqa: E731
    ok(p, [x], [y])
    ok(p.int(), [x, y], (y, x), backward=True)
    ok(p, [x, x, x, x], [y, y, y, y])
    ok(p, [x], [x])                                                          # in place
    ok(p, [x[:, :1].expand(5, 3, 8)], [y])                                   # a broadcast operand
    ok(p[:0], [x[:0]], [y[:0]])
    ok(p, [x[:, :0]], [y[:, :0]])
    wide = torch.zeros(5, 9, 12)
    ok(p, [wide[:, 1:4, 2:10]], [wide[:, 5:8, 2:10]])
    ok(p, [x.transpose(0, 1).contiguous().transpose(0, 1)], [y])             # heads outermost
    no("positions", p.float(), [x], [y])
    no("positions", p[None], [x], [y])
    no("positions", torch.arange(10)[::2], [x], [y])
    no("1 .. 4", p, [], [])
    no("1 .. 4", p, [x] * 5, [y] * 5)
    no("2 inputs and 1", p, [x, x], [y])
    no("registered for", p, [x.half()], [y])
    no("heads of 4", p, [x[..., :4]], [y[..., :4]])
    no("axes", p, [x[0]], [y[0]])
    no("next to each other", p, [torch.zeros(5, 3, 16)[..., ::2]], [y])
    no("rows at 5 positions", p, [x[:4]], [y[:4]])
    no("rows at 5 positions", p, [x[:, :2]], [y])
    no("overlap", p, [x], [y[:, :1].expand(5, 3, 8)], status="SHAPE")
    no("overlap", p, [x], [torch.zeros(100).as_strided((5, 3, 8), (8, 8, 1))], status="SHAPE")
    no("same strides", p, [wide.view(-1).as_strided((5, 3, 8), (24, 8, 1))], [wide.view(-1).as_strided((5, 3, 8), (32, 8, 1))])
    dims = [5, 8, 0, 3, 24, 8, 24, 8]

    def raw(words, status, d=dims, ins=(p, x), outs=(y,)):
        _refused(status, words, lambda: h._call(h._fn, d, list(ins), list(outs), None, 0))
    raw(HOST_ONLY, "INVALID_ARG")
    raw("4 or 8 bytes", "INVALID_ARG", [5, 2] + dims[2:])
    raw("tokens", "SHAPE", [-1] + dims[1:])
    raw("tokens", "SHAPE", [1 << 31] + dims[1:])
    raw("heads", "SHAPE", dims[:3] + [-1] + dims[4:])
    raw("negative", "SHAPE", dims[:4] + [-24] + dims[5:])
    raw("overflows", "SHAPE", dims[:4] + [1 << 60] + dims[5:])
    raw("null", "INVALID_ARG", ins=(0, x))
    raw("null", "INVALID_ARG", ins=(p, 0))
    raw("null", "INVALID_ARG", outs=(0,))
    raw("aligned", "INVALID_ARG", ins=(p, x.data_ptr() + 2))
    raw("aligned", "INVALID_ARG", ins=(p.data_ptr() + 4, x))
    raw("dims", "INVALID_ARG", dims[:-1])
    other = ctx.register_cache("bf16", 16)
    _refused("INVALID_ARG", "bad rotary id", lambda: other._call(h._fn, dims, [p, x], [y], None, 0))


def _pages(kv=2, size=8, D=16, pages=4, stored=torch.int8):
    out = [torch.zeros(pages, kv, size, D, dtype=stored) for _ in range(2)]
    return out + [torch.zeros(pages, kv, size) for _ in range(2)] if stored in (torch.int8, torch.float8_e4m3fn) else out


def test_store_and_load_calls(ctx, path):
    h = ctx.register_cache("bf16", 16, "i8")
    pages, slots = _pages(), torch.arange(5)
    k, v = (torch.zeros(5, 2, 16, dtype=torch.bfloat16) for _ in range(2))
    for name, call in (("store", lambda s=slots, r=(k, v), p=pages: h.store(list(r), s, p)), ("load", lambda s=slots, r=(k, v), p=pages: h.load(s, p, list(r)))):
        _refused("INVALID_ARG", HOST_ONLY, call)
        _refused("INVALID_ARG", HOST_ONLY, lambda: call(p=tuple(pages)))
        _refused("INVALID_ARG", HOST_ONLY, lambda: call(slots[:0], (k[:0], v[:0])))
        _refused("INVALID_ARG", "slots", lambda: call(slots.int()))
        _refused("INVALID_ARG", "slots", lambda: call(slots[:4]))
        _refused("INVALID_ARG", "keys of 5 x 2", lambda: call(r=(k, v[:4])))
        _refused("INVALID_ARG", "pages of 3 heads", lambda: call(p=_pages(kv=3)))
        _refused("INVALID_ARG", "pages is (k_pages", lambda: call(p=pages[:2]))
        _refused("INVALID_ARG", "k_pages", lambda: call(p=_pages(D=32)))
        _refused("INVALID_ARG", "k_pages", lambda: call(p=[p.view(torch.uint8) if p.dim() == 4 else p for p in pages]))
        _refused("INVALID_ARG", "k_scales", lambda: call(p=pages[:2] + [pages[2].double(), pages[3]]))
        _refused("INVALID_ARG", "v_pages", lambda: call(p=[pages[0], _pages(pages=8)[1][::2]] + pages[2:]))
        _refused("INVALID_ARG", "keys is", lambda: call(r=(k.half(), v)))
        _refused("SHAPE", "page_size", lambda: call(p=_pages(size=12)))
        _refused("SHAPE", "page_size", lambda: call(p=_pages(size=4)))
        _refused("SHAPE", "pages is 1", lambda: call(p=_pages(pages=0)))
    _refused("SHAPE", "overlap", lambda: h.load(slots, pages, [k[:, :1].expand(5, 2, 16), v]))
    _refused("INVALID_ARG", HOST_ONLY, lambda: h.store([k[:, :1].expand(5, 2, 16), v], slots, pages))
    same = ctx.register_cache("bf16", 16)
    _refused("INVALID_ARG", HOST_ONLY, lambda: same.store([k, v], slots, _pages(stored=torch.bfloat16)))
    _refused("INVALID_ARG", "pages is (k_pages, v_pages)", lambda: same.store([k, v], slots, pages))
    dims = [5, 2, 4, 8, 32, 16, 32, 16]

    def raw(words, status, d=dims, ins=(slots, k, v), outs=tuple(pages)):
        _refused(status, words, lambda: h._call(h._store, d, list(ins), list(outs), None, 0))
    raw(HOST_ONLY, "INVALID_ARG")
    raw("tokens", "SHAPE", [1 << 31] + dims[1:])
    raw("kv_heads", "SHAPE", [5, 0] + dims[2:])
    raw("larger than any memory", "SHAPE", [5, 65536, (1 << 31) - 1, 65536] + dims[4:])
    raw("negative", "SHAPE", dims[:6] + [-1, 16])
    raw("16-byte", "INVALID_ARG", outs=(pages[0].data_ptr() + 8, *pages[1:]))
    raw("8-byte", "INVALID_ARG", ins=(slots.data_ptr() + 4, k, v))
    raw("null", "INVALID_ARG", ins=(slots, 0, v))
    raw("8 dims", "INVALID_ARG", outs=tuple(pages[:2]))


def test_attention_calls(ctx, path):
    h = ctx.register_cache("bf16", 16, "i8")
    pages = _pages()
    q, out = (torch.zeros(3, 4, 16, dtype=torch.bfloat16) for _ in range(2))
    lengths, table, prefix = torch.zeros(3, dtype=torch.int32), torch.zeros(3, 200, dtype=torch.int32), torch.zeros(3, dtype=torch.int32)
    need = h.workspace_bytes(3, 4, 2, 1600, 24)
    ws = torch.zeros(need, dtype=torch.uint8)
    good = dict(q=q, lengths=lengths, table=table, pages=pages, out=out, workspace=ws)

    def call(**k):
        a = {**good, **k}
        h.attend(a.pop("q"), a.pop("lengths"), a.pop("table"), a.pop("pages"), a.pop("out"), **a)
    _refused("INVALID_ARG", HOST_ONLY, call)
    _refused("INVALID_ARG", HOST_ONLY, lambda: call(prefix_table=prefix, prefix_length=24))
    _refused("INVALID_ARG", HOST_ONLY, lambda: call(table=table[:, :0].contiguous()))
    _refused("INVALID_ARG", HOST_ONLY, lambda: call(q=q[:0], out=out[:0], lengths=lengths[:0], table=table[:0], workspace=None))
    _refused("INVALID_ARG", HOST_ONLY, lambda: call(table=table[:, :8].contiguous(), workspace=None))        # nothing to join
    _refused("INVALID_ARG", HOST_ONLY, lambda: call(q=q[:1, :1].expand(3, 4, 16)))
    _refused("WORKSPACE", "missing or too small", lambda: call(workspace=None))
    _refused("WORKSPACE", "missing or too small", lambda: call(workspace=ws[:64]))
    _refused("INVALID_ARG", "16-byte", lambda: call(workspace=torch.zeros(need + 64, dtype=torch.uint8)[8:]))
    _refused("INVALID_ARG", "lengths", lambda: call(lengths=lengths.long()))
    _refused("INVALID_ARG", "lengths", lambda: call(lengths=lengths[:2]))
    _refused("INVALID_ARG", "table", lambda: call(table=table.long()))
    _refused("INVALID_ARG", "table", lambda: call(table=table[:2]))
    _refused("INVALID_ARG", "table", lambda: call(table=table[0]))
    _refused("INVALID_ARG", "table", lambda: call(table=table.t().contiguous().t()))
    _refused("INVALID_ARG", "q of 3 x 4 and out of 3 x 2", lambda: call(out=out[:, :2]))
    _refused("INVALID_ARG", "q is", lambda: call(q=q.half()))
    _refused("SHAPE", "multiple of kv_heads", lambda: call(q=q[:, :3], out=out[:, :3]))
    _refused("SHAPE", "multiple of kv_heads", lambda: call(q=q[:, :1], out=out[:, :1]))
    _refused("SHAPE", "overlap", lambda: call(out=out[:, :1].expand(3, 4, 16)))
    _refused("SHAPE", "shorter than the prefix", lambda: call(prefix_table=prefix, prefix_length=25))
    _refused("SHAPE", "prefix_length", lambda: call(prefix_table=prefix, prefix_length=-1))
    _refused("INVALID_ARG", "prefix has a table", lambda: call(prefix_length=5))
    _refused("INVALID_ARG", "prefix_table", lambda: call(prefix_table=prefix.long(), prefix_length=5))
    dims = [3, 4, 2, 4, 8, 200, 0, 0, 64, 16, 64, 16]
    ins = [q, lengths, table, *pages]

    def raw(words, status, d=dims, i=ins, o=(out,)):
        _refused(status, words, lambda: h._call(h._attend, d, list(i), list(o), ws, 0))
    raw(HOST_ONLY, "INVALID_ARG")
    raw("12 dims", "INVALID_ARG", dims[:-1])
    raw("batch", "SHAPE", [-1] + dims[1:])
    raw("batch", "SHAPE", [(1 << 20) + 1] + dims[1:])
    raw("table_width", "SHAPE", dims[:5] + [1 << 28] + dims[6:])
    raw("table_width", "SHAPE", dims[:5] + [-1] + dims[6:])
    raw("32 bits", "SHAPE", dims[:3] + [1 << 28] + dims[4:])
    raw("negative", "SHAPE", dims[:8] + [-64] + dims[9:])
    raw("too many rows", "SHAPE", [1 << 20, 1 << 12, 2] + dims[3:])
    raw("prefix its table", "INVALID_ARG", dims[:6] + [8, 1] + dims[8:])
    raw("null", "INVALID_ARG", i=[0] + ins[1:])
    raw("null", "INVALID_ARG", o=(0,))
    raw("4-byte", "INVALID_ARG", i=[q, lengths.data_ptr() + 2] + ins[2:])
    raw("16-byte", "INVALID_ARG", i=ins[:4] + [pages[1].data_ptr() + 4] + ins[5:])


def test_a_workspace_that_is_not_dense_is_refused(ctx, path):
    """Its elements are fewer bytes than it says (expanded), or not all its own (every other one)."""
    h = ctx.register_cache("bf16", 16, "i8")
    q, out = (torch.zeros(3, 4, 16, dtype=torch.bfloat16) for _ in range(2))
    need = h.workspace_bytes(3, 4, 2, 1600)
    call = lambda ws: h.attend(q, torch.zeros(3, dtype=torch.int32), torch.zeros(3, 200, dtype=torch.int32), _pages(), out, workspace=ws)  # noqa: E731
    _refused("INVALID_ARG", HOST_ONLY, lambda: call(torch.zeros(need, dtype=torch.uint8)))
    _refused("INVALID_ARG", HOST_ONLY, lambda: call(torch.zeros(need // 8, 2)))
    for ws in (torch.zeros(1).expand(need), torch.zeros(2 * need, dtype=torch.uint8)[::2], torch.zeros(64, 1).expand(64, need // 4), torch.zeros(64, need).t()):
        _refused("INVALID_ARG", "dense", lambda: call(ws))


def test_attention_of_more_threads_than_a_launch_has(ctx):
    """Less than 2^32 threads a launch: 2^24 blocks of 256, 2^23 of the prefix's 512, are refused before anything is enqueued."""
    h = ctx.register_cache("bf16", 16, "i8")
    many = 1 << 20
    ok = lambda *a, **k: h.workspace_bytes(*a, **k) >= 0  # noqa: E731
    no = lambda *a, **k: _refused("SHAPE", "too many rows", lambda: h.workspace_bytes(*a, **k))  # noqa: E731
    assert ok(many, 63, 63, 8) and ok(many, 32, 32, 8) and ok(many, 60, 1, 1000)
    no(many, 64, 64, 8)                                        # one wavefront a (sequence, kv head), four a block
    no(many, 64, 1, 1000)                                      # a wavefront a row that is joined
    no(many, 1 << 7, 1 << 7, 8, 1 << 20)                       # the prefix's rows
    dims = [many, 64, 64, 1, 8, 1, 0, 0, 1024, 16, 1024, 16]
    x = torch.zeros(16, dtype=torch.uint8)
    _refused("SHAPE", "too many rows", lambda: h._call(h._attend, dims, [x] * 7, [x], None, 0))


def test_a_context_of_another_kind_of_operator_and_unknown_ids(ctx):
    lib = ctx.lib
    f = pkg.rotary_frequencies(8)[0]
    rotary = ctx.register_rotary("f32", 8, f)
    out = C.c_size_t(7)
    d = (C.c_int64 * 12)(*[1, 1, 1, 1, 8, 1, 0, 0, 16, 16, 16, 16])
    for bad in (-1, 10 ** 6, rotary.id):
        assert lib.disc_cache_workspace_bytes(ctx.h, bad, d, 12, C.byref(out)) == -1
        assert lib.disc_cache_attend(ctx.h, bad, d, 12, None, 0, None, 0, None, 0, None) == -1
        assert lib.disc_cache_store(ctx.h, bad, d, 8, None, 0, None, 0, None, 0, None) == -1
    assert out.value == 7
    assert lib.disc_rotary(None, 0, d, 3, None, 0, None, 0, None, 0, None) == -1
    cache = ctx.register_cache("bf16", 16)
    assert lib.disc_cache_attend(ctx.h, cache.id, None, 12, None, 0, None, 0, None, 0, None) == -1
    assert lib.disc_cache_workspace_bytes(ctx.h, cache.id, None, 12, C.byref(out)) == -1


def test_tensors_on_another_device_are_refused():
    """A context of a GPU refuses tensors of the host (and of any other device): checked before anything is launched."""
    h = object.__new__(pkg.CacheHandle)
    h._device, h._dtype, h.head_dim = 0, torch.bfloat16, 16
    _refused("INVALID_ARG", "is on cpu", lambda: h._rows(torch.zeros(1, 1, 16, dtype=torch.bfloat16), "keys"))
    _refused("INVALID_ARG", "is on cpu", lambda: h._plain(torch.zeros(1, dtype=torch.int64), "slots", (torch.int64,), (1,)))


def test_workspace_covers_smaller_calls(ctx):
    """What was asked for at a size serves every page size, and the bytes are what the chunks take."""
    for storage, D in (("i8", 128), (None, 256)):
        h = ctx.register_cache("bf16", D, storage)
        for B, q, kv in ((1, 8, 8), (7, 32, 8), (64, 64, 8), (300, 4, 1)):
            for longest, prefix in ((0, 0), (100, 0), (513, 0), (100000, 0), (64, 512), (513, 513), (300, 70000), (100000, 40)):
                most = h.workspace_bytes(B, q, kv, longest, prefix)
                for size in (16, 128, 4096):
                    assert h.workspace_bytes(B, q, kv, longest // size * size, prefix, page_size=size) <= most
                assert most % (4 * D + 8) == 0
        assert h.workspace_bytes(0, 8, 8, 1000) == 0
        assert h.workspace_bytes(300, 32, 8, 512) == 0                       # one chunk each, written where it belongs


def test_workspace_covers_smaller_batches_prefixes_and_tables(ctx, path):
    """What was asked for at the largest batch, prefix and table serves every smaller one: by its size, and in the call."""
    rng = random.Random(11)
    for storage, D, q, kv in (("i8", 128, 64, 8), ("bf16", 128, 32, 8), ("bf16", 256, 8, 8), ("e4m3", 64, 40, 1), ("bf16", 192, 4, 2)):
        h = ctx.register_cache("bf16", D, storage)
        pages = _pages(kv=kv, D=D, stored={"i8": torch.int8, "e4m3": torch.float8_e4m3fn, "bf16": torch.bfloat16}[storage])
        for B, longest, prefix in ((128, 8192, 16384), (64, 512, 0), (40, 512, 3000), (33, 300, 8320), (700, 40, 700), (1500, 8, 100000), (128, 8192, 8192)):
            most = h.workspace_bytes(B, q, kv, longest, prefix)
            ws = torch.empty(most, dtype=torch.uint8)
            smaller = [(b, longest, prefix) for b in {1, B // 2, B - 1, 32, 33, 64, 65} if b <= B] + [(B, longest, p) for p in (prefix // 2, prefix - 1, 513, 128, 0) if 0 <= p <= prefix]
            smaller += [(rng.randint(1, B), rng.randint(0, longest), rng.randint(0, prefix)) for _ in range(40)] + [(B, n, prefix) for n in (0, 8, 256, 512) if n <= longest]
            for b, n, p in smaller:
                width = n // 8
                if storage != "bf16" or D <= 128 or n <= 256 or longest > 512:      # (one that fewer sequences take is left, see below)
                    assert h.workspace_bytes(b, q, kv, width * 8, p) <= most, (storage, D, B, longest, prefix, b, n, p)
                x = torch.zeros(1, 1, D, dtype=torch.bfloat16).expand(b, q, D)
                out = torch.empty(b, q, D, dtype=torch.bfloat16)
                table = torch.zeros(b, width, dtype=torch.int32)
                more = {"prefix_table": torch.zeros(-(-p // 8), dtype=torch.int32), "prefix_length": p} if p else {}
                _refused("INVALID_ARG", HOST_ONLY, lambda: h.attend(x, torch.zeros(b, dtype=torch.int32), table, pages, out, workspace=ws if most else None, **more))
    # 16-bit rows above 128: a few sequences of up to 512 tokens are cut where there is workspace for it, and one chunk each without
    h = ctx.register_cache("bf16", 256)
    assert h.workspace_bytes(300, 32, 8, 512) == 0 and h.workspace_bytes(4, 32, 8, 512) > 0


# ---- the device header on the CPU ------------------------------------------------------------------


def _header():
    with open(os.path.join(os.path.dirname(pkg.__file__), "csrc", "decoder_device.h")) as f:
        return f.read()


def test_page_rows(tmp_path):
    """Row of a slot: inside the pages for every slot inside, each its own, past 2^31 and 2^32."""
    body = re.search(r"^DISC_DEV i64 page_row\(.*?^}$", _header(), re.M | re.S)[0]
    lib = host_build(body + '\nextern "C" i64 row(i64 s, int h, int n, int shift) { return page_row(s, h, n, shift); }\n', tmp_path / "rows")
    lib.row.restype = C.c_longlong
    row = lambda s, h, n, shift: lib.row(C.c_longlong(s), h, n, shift)  # noqa: E731
    for pages, heads, shift in ((3, 2, 3), (5, 1, 4), (2, 7, 6)):
        seen = {row(s, h, heads, shift) for s in range(pages << shift) for h in range(heads)}
        assert seen == set(range((pages << shift) * heads))
    rng = random.Random(2)
    for _ in range(2000):
        shift, heads = rng.randint(3, 16), rng.randint(1, 128)
        slot, h = rng.randrange(1 << 40), rng.randrange(heads)
        assert row(slot, h, heads, shift) == (((slot >> shift) * heads + h) << shift) + slot % (1 << shift)


SHARES = """
static inline int __ffsll(unsigned long long x) { return __builtin_ffsll((long long)x); }
%s
extern "C" void cut(u64 total, u32 target, u64* first) {
  Shares S;
  S.each = total / target;
  S.more = (u32)(total - S.each * target);
  for (u32 j = 0; j <= target; ++j) first[j] = S.first(j);
}
extern "C" u32 block(u64 total, u32 target, u64 unit) {
  Shares S;
  S.each = total / target;
  S.more = (u32)(total - S.each * target);
  return S.block_of(unit);
}
"""


def test_shares_of_the_blocks(tmp_path):
    """The blocks' shares follow each other, differ by one unit at most and cover everything; block_of() is their inverse."""
    text = re.search(r"^struct Shares \{.*?^\};$", _header(), re.M | re.S)[0].replace("DISC_DEV ", "inline ").replace("static inline", "static")
    lib = host_build(SHARES % text, tmp_path / "shares")
    lib.block.restype = C.c_uint
    rng = random.Random(3)
    for total, target in [(0, 5), (1, 5), (5, 5), (4, 768), (768, 768), (769, 768), (10 ** 6, 96), (2 ** 33 + 7, 3), (2 ** 43, 768)] + \
            [(rng.randrange(5000), rng.randint(1, 800)) for _ in range(60)]:
        first = (C.c_ulonglong * (target + 1))()
        lib.cut(C.c_ulonglong(total), target, first)
        sizes = [first[j + 1] - first[j] for j in range(target)]
        assert first[0] == 0 and first[target] == total and max(sizes) - min(sizes) <= 1
        for unit in {0, 1, total // 2, total - 1} | {rng.randrange(total) for _ in range(30)} if total > 1 else set(range(total)):
            j = lib.block(C.c_ulonglong(total), target, C.c_ulonglong(unit))
            assert first[j] <= unit < first[j + 1]


ROWS = """
typedef int i32;
static inline int min(int a, int b) { return a < b ? a : b; }
struct AttendArgs { int shift, kv_heads, pages; };
%s
extern "C" long long outside(int shift, int kv, int pages, const int* table, int width, int begin, int end, int h, u32* rows) {
  AttendArgs A = {shift, kv, pages};
  stage_pages(A, table, width, begin, end, h, rows, 0, 1);
  const int base = begin >> shift, last = (end - 1) & ~7;
  const long long all = (long long)pages * kv << shift;
  long long bad = 0;
  // every place that a step of the kernel reads: its keys, its values, its scales, one step behind the end too
  for (int t0 = begin; t0 < end + 64; t0 += 32) {
    bool there;
    for (int m = 0; m < 16; ++m)
      for (int mt = 0; mt < 2; ++mt) {
        const u32 r = row_of(A, rows, base, min(t0 + (m >> 2) * 8, last), there) + mt * 4 + (m & 3);
        bad += r >= all;
      }
    for (int g = 0; g < 4; ++g)
      for (int j = 0; j < 8; ++j) bad += row_of(A, rows, base, min(t0 + g * 8, last), there) + j >= all;
    for (int l = 0; l < 32; ++l) {
      const u32 r = row_of(A, rows, base, min(t0 + l, last + 7), there);
      bad += r >= all;
      const int t = t0 + l;
      if (t < end) {                      // a token that is there: its own place, of this head
        const int p = table[t >> shift];
        const bool page = (t >> shift) < width && p >= 0 && p < pages;
        bad += page != there || (page && r != ((u32)p * kv + h << shift) + (t & ((1 << shift) - 1)));
      }
    }
  }
  return bad;
}
"""


def test_rows_that_attention_reads(tmp_path):
    """Bad pages, pages that end inside a step, steps behind the end: no row outside the pages is ever formed, and a token's
    row is its own."""
    text = _header()
    body = re.search(r"^constexpr u32 kNoPage.*?^}$", text, re.M | re.S)[0] + "\n" + re.search(r"^DISC_DEV void stage_pages\(.*?^}$", text, re.M | re.S)[0]
    lib = host_build(ROWS % body, tmp_path / "pages")
    lib.outside.restype = C.c_longlong
    rng = random.Random(5)
    for _ in range(400):
        shift, kv, pages = rng.randint(3, 8), rng.randint(1, 5), rng.randint(1, 9)
        width = rng.randint(1, 12)
        table = (C.c_int * width)(*[rng.choice([rng.randrange(pages), rng.randrange(pages), -1, pages, -2 ** 31, 2 ** 31 - 1]) for _ in range(width)])
        most = width << shift
        begin = rng.randrange(0, most, 8) // 128 * 128
        end = rng.randint(begin + 1, most) if begin + 1 <= most else most
        if end <= begin:
            continue
        rows = (C.c_uint * (width + 2))()
        assert lib.outside(shift, kv, pages, table, width, begin, end, rng.randrange(kv), rows) == 0


# ---- the oracle ------------------------------------------------------------------------------------


def test_oracle_of_rotary():
    """Norms stay, positions add up, the gradient is the transposed map."""
    f = pkg.rotary_frequencies(6)[0]
    g = torch.Generator().manual_seed(1)
    for layout in ("half", "interleaved"):
        x = torch.randn(4, 2, 10, generator=g, dtype=torch.float64)
        p = torch.tensor([0, 3, 50, 1000])
        y = plain.rotary(x, p, f, layout)
        assert torch.equal(y[0], x[0]) and torch.equal(y[..., 6:], x[..., 6:])
        assert torch.allclose(y.norm(dim=-1), x.norm(dim=-1), rtol=1e-13, atol=0)
        assert torch.allclose(plain.rotary(y, p, f, layout), plain.rotary(x, 2 * p, f, layout), rtol=0, atol=1e-12)
        assert torch.allclose(plain.rotary(y, p, f, layout, backward=True), x, rtol=0, atol=1e-12)
        xg = x.clone().requires_grad_()
        angle = p.double()[:, None] * torch.tensor(f, dtype=torch.float64)
        c, s = angle.cos()[:, None], angle.sin()[:, None]
        a, b = (xg[..., :3], xg[..., 3:6]) if layout == "half" else (xg[..., 0:6:2], xg[..., 1:6:2])
        ya, yb = a * c - b * s, b * c + a * s
        dy = torch.randn(4, 2, 10, generator=g, dtype=torch.float64)
        da, db = (dy[..., :3], dy[..., 3:6]) if layout == "half" else (dy[..., 0:6:2], dy[..., 1:6:2])
        ((ya * da).sum() + (yb * db).sum() + (xg[..., 6:] * dy[..., 6:]).sum()).backward()
        assert torch.allclose(plain.rotary(dy, p, f, layout, backward=True), xg.grad, rtol=0, atol=1e-12)


def test_oracle_of_attention():
    """One token gives its value, equal keys the mean, a shared prefix the same as the prefix in every sequence's own pages."""
    g = torch.Generator().manual_seed(2)
    k, v = (torch.randn(6, 1, 8, 16, generator=g, dtype=torch.float64) for _ in range(2))
    q = torch.randn(2, 2, 16, generator=g, dtype=torch.float64)
    table = torch.tensor([[1, 2, 3], [4, 5, 0]], dtype=torch.int32)
    out = plain.attend(q, torch.tensor([1, 0]), table, [k, v], 0.25)[0]
    assert torch.allclose(out[0], v[1, 0, 0].expand(2, 16), rtol=1e-14, atol=0) and (out[1] == 0).all()
    same = plain.attend(q, torch.tensor([20, 24]), table, [torch.ones_like(k), v], 0.25)[0]
    assert torch.allclose(same[0, 0], torch.cat((v[1, 0], v[2, 0], v[3, 0, :4])).mean(0), rtol=1e-12, atol=1e-14)
    shared = plain.attend(q, torch.tensor([5, 3]), table[:, 1:], [k, v], 0.25, torch.tensor([0], dtype=torch.int32), 8)[0]
    mine = torch.tensor([[0, 2], [0, 5]], dtype=torch.int32)
    own = plain.attend(q, torch.tensor([13, 11]), mine, [k, v], 0.25)[0]
    assert torch.allclose(shared, own, rtol=1e-12, atol=1e-14)


def test_oracle_of_codes():
    x = torch.tensor([[0.0, 0.0], [1.0, -2.0], [math.inf, 1.0], [math.nan, 1.0]])
    codes, scales = plain.encode(x, "i8")
    assert codes.tolist() == [[0, 0], [64, -127], [0, 0], [0, 0]] and scales[0] == 0 and torch.isnan(scales[2:]).all()
    codes, scales = plain.encode(x[:2], "e4m3")
    assert codes.float().tolist() == [[0, 0], [224, -448]]
