"""The norm, products with 4-bit weights and the check of drafted tokens without a GPU: what is refused, workspaces, registrations, where
the device code finds its elements, and the oracle."""
import ctypes as C
import math
import os
import re
from fractions import Fraction

import pytest
import torch

import paper_2103_05288_amd as pkg
from oracle import step as plain
from paper_2103_05288_amd import binding
from tests.util import host_build

HOST_ONLY = "host-only context cannot launch"


@pytest.fixture(scope="module")
def ctx():
    c = pkg.Context(-1)
    yield c
    c.close()


@pytest.fixture(params=["quick", "slow"])
def path(request, monkeypatch):
    """With the checks and the marshalling of a call that fits in C, and without."""
    if request.param == "slow":
        monkeypatch.setattr(binding, "_pylaunch", binding._CtypesLaunch)
    return request.param


def _refused(status, words, call):
    with pytest.raises(pkg.DiscError) as e:
        call()
    assert e.value.status == status and words in e.value.message, (e.value.status, e.value.message)


def test_registrations_compile_once(ctx):
    before = ctx.stats()["compile_events"]
    a = ctx.register_norm("bf16", "i8", eps=1e-5)
    b = ctx.register_norm("bf16", "i8", eps=1e-5, offset=0.0)
    c = ctx.register_norm("bf16", "i8", eps=1e-6)              # (another operator of the same code)
    d = ctx.register_norm("bf16", "i8", eps=1e-5, offset=1.0)
    assert a.id == b.id and len({a.id, c.id, d.id}) == 3 and ctx.stats()["compile_events"] == before + 1
    e, f, g = ctx.register_linear4("bf16"), ctx.register_linear4("bf16", group=128, rows="bf16", zeros=False), ctx.register_linear4("bf16", zeros=True)
    assert e.id == f.id != g.id
    assert ctx.register_verify("f32").id == ctx.register_verify("f32").id


@pytest.mark.parametrize("dtype,rows,group,zeros", [("f16", None, 128, True), ("bf16", "e4m3", 64, True), ("f16", "i8", 32, False)])
def test_linear_compiles(ctx, dtype, rows, group, zeros):
    ctx.register_linear4(dtype, group, rows, zeros)


def test_norm_and_verify_compile(ctx):
    ctx.register_norm("f32", "e4m3")
    ctx.register_norm("f16", "i8")
    ctx.register_verify("bf16")


def test_registrations_that_are_refused(ctx):
    _refused("INVALID_ARG", "no such type", lambda: ctx.register_norm("f64", "i8"))
    _refused("INVALID_ARG", "no such type", lambda: ctx.register_norm("bf16", "i4"))
    _refused("INVALID_ARG", "f32, f16 or bf16", lambda: ctx.register_norm("i32", "i8"))
    for eps in (0.0, -1e-5, math.nan, math.inf, 1e-60, 1e39):
        _refused("INVALID_ARG", "eps", lambda: ctx.register_norm("bf16", "i8", eps=eps))
    _refused("INVALID_ARG", "weight_offset", lambda: ctx.register_norm("bf16", "i8", offset=math.inf))
    _refused("INVALID_ARG", "f16 or bf16", lambda: ctx.register_linear4("f32"))
    _refused("INVALID_ARG", "no such type", lambda: ctx.register_linear4("bf16", rows="f16"))
    for group in (0, 16, 96, 256, -32):
        _refused("SHAPE", "group", lambda: ctx.register_linear4("bf16", group=group))
    _refused("INVALID_ARG", "f32, f16 or bf16", lambda: ctx.register_verify("i64"))
    _refused("INVALID_ARG", "no such type", lambda: ctx.register_verify("e4m3"))
    lib, out = ctx.lib, C.c_int32(5)
    for register in (lib.disc_register_norm, lib.disc_register_linear4, lib.disc_register_verify):
        assert register(ctx.h, None, C.byref(out)) == -1 and register(None, None, C.byref(out)) == -1
    assert lib.disc_register_norm(ctx.h, C.byref(binding.disc_norm_desc(2, 0, 1e-5, 0.0)), C.byref(out)) == -1
    assert lib.disc_register_linear4(ctx.h, C.byref(binding.disc_linear4_desc(2, 3, 64, 0)), C.byref(out)) == -1 and out.value == 5


def test_norm_calls(ctx, path):
    h = ctx.register_norm("bf16", "i8", eps=1e-5)
    t = torch.bfloat16
    good = dict(x=torch.zeros(5, 24, dtype=t), weight=torch.zeros(24, dtype=t), codes=torch.zeros(5, 24, dtype=torch.int8), scales=torch.zeros(5))
    more = dict(residual=torch.zeros(5, 24, dtype=t), total=torch.zeros(5, 24, dtype=t))

    def call(**k):
        a = {**good, **k}
        h.launch(a.pop("x"), a.pop("weight"), a.pop("codes"), a.pop("scales"), **a)
    no = lambda words, status="INVALID_ARG", **k: _refused(status, words, lambda: call(**k))  # noqa: E731
    no(HOST_ONLY)
    no(HOST_ONLY, **more)
    no(HOST_ONLY, residual=more["residual"], total=more["residual"])
    no(HOST_ONLY, x=more["total"], **more)
    no(HOST_ONLY, x=good["x"][:1].expand(5, 24))
    no(HOST_ONLY, x=torch.zeros(5, 40, dtype=t)[:, 3:27], codes=torch.zeros(5, 33, dtype=torch.int8)[:, 1:25])
    no(HOST_ONLY, **{k: v[:0] if k != "weight" else v for k, v in good.items()})
    no("x is", x=good["x"].half())
    no("x has 1 axes", x=good["x"][0])
    no("next to each other", x=torch.zeros(24, 5, dtype=t).t())
    no("weight", weight=torch.zeros(25, dtype=t))
    no("weight", weight=torch.zeros(24))
    no("weight", weight=torch.zeros(48, dtype=t)[::2])
    no("codes is", codes=torch.zeros(5, 24, dtype=torch.uint8))
    no("codes is 4 x 24", codes=good["codes"][:4])
    no("scales", scales=torch.zeros(5, dtype=torch.float64))
    no("scales", scales=torch.zeros(5, 1))
    no("residual goes with", residual=more["residual"])
    no("residual goes with", total=more["total"])
    no("total is 5 x 23", residual=more["residual"], total=torch.zeros(5, 23, dtype=t))
    no("overlap", "SHAPE", codes=good["codes"][:1].expand(5, 24))
    no("overlap", "SHAPE", residual=more["residual"], total=torch.zeros(200, dtype=t).as_strided((5, 24), (23, 1)))
    wide = torch.zeros(5, 48, dtype=t)
    no("same strides", residual=wide.view(-1).as_strided((5, 24), (24, 1)), total=wide[:, :24])
    no("width", "SHAPE", x=torch.zeros(5, 0, dtype=t), weight=torch.zeros(0, dtype=t), codes=torch.zeros(5, 0, dtype=torch.int8))
    no("width", "SHAPE", x=torch.zeros(1, 32769, dtype=t), weight=torch.zeros(32769, dtype=t), codes=torch.zeros(1, 32769, dtype=torch.int8), scales=torch.zeros(1))
    f32 = ctx.register_norm("f32", "i8", eps=1e-5)
    wide = [torch.zeros(1, 16385), torch.zeros(16385), torch.zeros(1, 16385, dtype=torch.int8), torch.zeros(1)]
    _refused("SHAPE", "width", lambda: f32.launch(*wide))
    dims, ins, outs = [5, 24, 24, 0, 0, 24], [good["x"], good["weight"]], [good["codes"], good["scales"]]

    def raw(words, status, d=dims, i=ins, o=outs):
        _refused(status, words, lambda: h._call(h._fn, d, list(i), list(o), None, 0))
    raw(HOST_ONLY, "INVALID_ARG")
    raw("6 dims", "INVALID_ARG", dims[:-1])
    raw("6 dims", "INVALID_ARG", i=ins + [good["x"]])
    raw("rows", "SHAPE", [-1] + dims[1:])
    raw("rows", "SHAPE", [1 << 31] + dims[1:])
    raw("negative", "SHAPE", dims[:2] + [-24] + dims[3:])
    raw("overflows", "SHAPE", dims[:2] + [1 << 59] + dims[3:])
    raw("null", "INVALID_ARG", i=[0, good["weight"]])
    raw("null", "INVALID_ARG", o=[good["codes"], 0])
    raw("aligned", "INVALID_ARG", i=[good["x"].data_ptr() + 1, good["weight"]])
    raw("aligned", "INVALID_ARG", o=[good["codes"], good["scales"].data_ptr() + 2])
    other = ctx.register_verify("f32")
    _refused("INVALID_ARG", "bad norm id", lambda: other._call(h._fn, dims, ins, outs, None, 0))


def test_norm_backward_calls(ctx, path):
    h = ctx.register_norm("bf16", "i8", eps=1e-5)
    t = torch.bfloat16
    need = h.workspace_bytes(5, 24)
    rows = lambda: torch.zeros(5, 24, dtype=t)  # noqa: E731
    good = dict(total=rows(), weight=torch.zeros(24, dtype=t), dy=rows(), dx=rows(), dweight=torch.zeros(24), workspace=torch.zeros(need, dtype=torch.uint8))

    def call(**k):
        a = {**good, **k}
        h.backward(a.pop("total"), a.pop("weight"), a.pop("dy"), a.pop("dx"), a.pop("dweight"), **a)
    no = lambda words, status="INVALID_ARG", **k: _refused(status, words, lambda: call(**k))  # noqa: E731
    no(HOST_ONLY)
    no(HOST_ONLY, dtotal=rows())
    for into in ("total", "dy"):
        no(HOST_ONLY, dx=good[into])
    no(HOST_ONLY, total=rows()[:0], dy=rows()[:0], dx=rows()[:0], workspace=None)
    no("missing or too small", "WORKSPACE", workspace=None)
    no("missing or too small", "WORKSPACE", workspace=good["workspace"][:need - 1])
    no("16-byte", workspace=torch.zeros(need + 64, dtype=torch.uint8)[8:])
    no("dense", workspace=torch.zeros(2 * need, dtype=torch.uint8)[::2])
    no("dense", workspace=torch.zeros(1, dtype=torch.uint8).expand(need))
    no("dweight", dweight=torch.zeros(24, dtype=t))
    no("dweight", dweight=torch.zeros(23))
    no("dy is 4 x 24", dy=rows()[:4])
    no("dtotal is", dtotal=torch.zeros(5, 24))
    no("overlap", "SHAPE", dx=rows()[:1].expand(5, 24))
    wide = torch.zeros(5, 48, dtype=t)
    no("same strides", dtotal=wide.view(-1).as_strided((5, 24), (24, 1)), dx=wide[:, :24])
    out = C.c_size_t(7)
    d = (C.c_int64 * 6)(5, 24, 0, 0, 0, 0)
    assert ctx.lib.disc_norm_workspace_bytes(ctx.h, -1, d, 6, C.byref(out)) == -1 and ctx.lib.disc_norm_workspace_bytes(ctx.h, h.id, d, 5, C.byref(out)) == -1
    assert ctx.lib.disc_norm_workspace_bytes(ctx.h, h.id, None, 6, C.byref(out)) == -1 and out.value == 7
    for width in (1, 7, 64, 65, 700, 2048, 5000, 9000, 30000):
        most = h.workspace_bytes(5000, width)
        assert most % (4 * width) == 0 and h.workspace_bytes(0, width) == 0
        for fewer in (1, 2, 3, 40, 41, 255, 256, 257, 511, 513, 700, 767, 769, 1000, 1025, 2047, 4999):
            assert 0 < h.workspace_bytes(fewer, width) <= most
            x = torch.zeros(1, width, dtype=t).expand(fewer, width)
            dx = torch.empty(fewer, width, dtype=t)
            ws = torch.empty(most, dtype=torch.uint8)
            _refused("INVALID_ARG", HOST_ONLY, lambda: h.backward(x, torch.zeros(width, dtype=t), x, dx, torch.zeros(width), workspace=ws))


def test_linear_calls(ctx, path):
    h = ctx.register_linear4("bf16", group=32)
    z = ctx.register_linear4("bf16", group=32, rows="i8", zeros=True)
    t = torch.bfloat16
    good = dict(x=torch.zeros(5, 96, dtype=t), weights=torch.zeros(7, 48, dtype=torch.uint8), scales=torch.zeros(7, 3, dtype=t), out=torch.zeros(5, 7, dtype=t))
    full = dict(good, x=torch.zeros(5, 96, dtype=torch.int8), row_scales=torch.zeros(5), zeros=torch.zeros(7, 3, dtype=torch.uint8))

    def call(h, a):
        a = dict(a)
        h.launch(a.pop("x"), a.pop("weights"), a.pop("scales"), a.pop("out"), **a)
    no = lambda words, status="INVALID_ARG", **k: _refused(status, words, lambda: call(h, {**good, **k}))  # noqa: E731
    non = lambda words, status="INVALID_ARG", **k: _refused(status, words, lambda: call(z, {**full, **k}))  # noqa: E731
    no(HOST_ONLY)
    no(HOST_ONLY, bias=torch.zeros(7, dtype=t))
    no(HOST_ONLY, x=good["x"][:0], out=good["out"][:0])
    no(HOST_ONLY, x=torch.zeros(5, 100, dtype=t)[:, 1:97], out=torch.zeros(5, 9, dtype=t)[:, 1:8])
    non(HOST_ONLY)
    non(HOST_ONLY, bias=torch.zeros(7, dtype=t))
    no("x is", x=good["x"].half())
    no("multiple of the group", x=torch.zeros(5, 80, dtype=t))
    no("weights is", weights=torch.zeros(7, 48, dtype=torch.int8))
    no("weights is", weights=torch.zeros(7, 40, dtype=torch.uint8))
    no("weights is", weights=torch.zeros(48, 7, dtype=torch.uint8).t())
    no("weights has", weights=torch.zeros(7 * 48, dtype=torch.uint8))
    no("scales is", scales=torch.zeros(7, 3))
    no("scales is", scales=torch.zeros(7, 4, dtype=t))
    no("out is 5 x 8", out=torch.zeros(5, 8, dtype=t))
    no("no row_scales", row_scales=torch.zeros(5))
    no("without zero points", zeros=full["zeros"])
    no("bias", bias=torch.zeros(7))
    no("overlap", "SHAPE", out=good["out"][:1].expand(5, 7))
    no("16-byte", weights=torch.zeros(7 * 48 + 8, dtype=torch.uint8)[8:].view(7, 48))
    no("k is a multiple", "SHAPE", x=torch.zeros(5, 0, dtype=t), weights=torch.zeros(7, 0, dtype=torch.uint8), scales=torch.zeros(7, 0, dtype=t))
    no("n is 1", "SHAPE", weights=torch.zeros(0, 48, dtype=torch.uint8), scales=torch.zeros(0, 3, dtype=t), out=torch.zeros(5, 0, dtype=t))
    non("come with row_scales", row_scales=None)
    non("row_scales", row_scales=torch.zeros(4))
    non("with zero points", zeros=None)
    non("zeros is", zeros=torch.zeros(7, 3, dtype=torch.int8))
    non("x is", x=good["x"])
    dims, ins = [5, 7, 96, 96, 7], [good["x"], good["weights"], good["scales"]]

    def raw(words, status, d=dims, i=ins, o=(good["out"],)):
        _refused(status, words, lambda: h._call(h._fn, d, list(i), list(o), None, 0))
    raw(HOST_ONLY, "INVALID_ARG")
    raw("5 dims", "INVALID_ARG", dims[:-1])
    raw("5 dims", "INVALID_ARG", i=ins[:2])
    raw("rows", "SHAPE", [-1] + dims[1:])
    raw("rows", "SHAPE", [(1 << 20) + 1] + dims[1:])
    raw("n is", "SHAPE", [5, (1 << 26) + 1] + dims[2:])
    raw("k is", "SHAPE", [5, 7, (1 << 24) + 32] + dims[3:])
    raw("k is", "SHAPE", [5, 7, 97] + dims[3:])
    raw("negative", "SHAPE", [5, 7, 96, -96, 7])
    raw("null", "INVALID_ARG", i=[good["x"], 0, good["scales"]])
    raw("null", "INVALID_ARG", i=ins + [0])
    raw("aligned to its", "INVALID_ARG", i=[good["x"].data_ptr() + 1] + ins[1:])
    other = ctx.register_norm("bf16", "i8", eps=1e-5)
    _refused("INVALID_ARG", "bad product id", lambda: other._call(h._fn, dims, ins, [good["out"]], None, 0))


def test_verify_calls(ctx, path):
    h = ctx.register_verify("f32")
    need = h.workspace_bytes(3, 50)
    i32 = torch.int32
    good = dict(target=torch.zeros(3, 3, 50), drafted=torch.zeros(3, 2, dtype=i32), uniforms=torch.zeros(3, 3), tokens=torch.zeros(3, 3, dtype=i32),
                accepted=torch.zeros(3, dtype=i32), workspace=torch.zeros(need, dtype=torch.uint8))

    def call(**k):
        a = {**good, **k}
        h.launch(a.pop("target"), a.pop("drafted"), a.pop("uniforms"), a.pop("tokens"), a.pop("accepted"), **a)
    no = lambda words, status="INVALID_ARG", **k: _refused(status, words, lambda: call(**k))  # noqa: E731
    draft, lengths = torch.zeros(3, 2, 50), torch.zeros(3, dtype=i32)
    no(HOST_ONLY)
    no(HOST_ONLY, draft=draft)
    no(HOST_ONLY, lengths=lengths)
    no(HOST_ONLY, draft=draft, lengths=lengths)
    no(HOST_ONLY, draft=draft[:1].expand(3, 2, 50))
    no(HOST_ONLY, target=torch.zeros(3, 1, 50), drafted=good["drafted"][:, :0].contiguous(), uniforms=torch.zeros(3, 1), tokens=torch.zeros(3, 1, dtype=i32))
    no(HOST_ONLY, target=good["target"].transpose(0, 1).contiguous().transpose(0, 1))
    no(HOST_ONLY, **{k: v[:0] for k, v in good.items()})
    no("missing or too small", "WORKSPACE", workspace=None)
    no("missing or too small", "WORKSPACE", workspace=good["workspace"][:need - 1])
    no("16-byte", workspace=torch.zeros(need + 16, dtype=torch.uint8)[4:])
    no("dense", workspace=torch.zeros(2 * need, dtype=torch.uint8)[::2])
    no("target is", target=good["target"].half())
    no("target has", target=good["target"][0])
    no("next to each other", target=torch.zeros(3, 50, 3).transpose(1, 2))
    no("place behind", target=torch.zeros(3, 0, 50))
    no("drafted", drafted=good["drafted"].long())
    no("drafted", drafted=torch.zeros(3, 3, dtype=i32))
    no("uniforms", uniforms=torch.zeros(3, 2))
    no("uniforms", uniforms=torch.zeros(3, 3, dtype=torch.float64))
    no("tokens", tokens=torch.zeros(3, 2, dtype=i32))
    no("accepted", accepted=torch.zeros(4, dtype=i32))
    no("draft is", draft=torch.zeros(3, 2, 49))
    no("draft is", draft=torch.zeros(3, 2, 50, dtype=torch.float16))
    no("lengths", lengths=lengths.long())
    no("vocabulary", "SHAPE", target=torch.zeros(3, 3, 0))
    dims = [3, 2, 50, 150, 50, 0, 0, 0, 0]
    ins, outs = [good["target"], good["drafted"], good["uniforms"]], [good["tokens"], good["accepted"]]

    def raw(words, status, d=dims, i=ins, o=outs):
        _refused(status, words, lambda: h._call(h._fn, d, list(i), list(o), good["workspace"], 0))
    raw(HOST_ONLY, "INVALID_ARG")
    raw("9 dims", "INVALID_ARG", dims[:-1])
    raw("probabilities", "INVALID_ARG", dims[:7] + [1, 0])
    raw("batch", "SHAPE", [-1] + dims[1:])
    raw("batch", "SHAPE", [(1 << 20) + 1] + dims[1:])
    raw("drafts", "SHAPE", [3, 4097] + dims[2:])
    raw("drafts", "SHAPE", [3, -1] + dims[2:])
    raw("vocabulary", "SHAPE", [3, 2, (1 << 30) + 1] + dims[3:])
    raw("too many rows", "SHAPE", [1 << 20, 2, 1 << 20] + dims[3:])
    raw("negative", "SHAPE", dims[:3] + [-1] + dims[4:])
    raw("null", "INVALID_ARG", i=[0] + ins[1:])
    raw("null", "INVALID_ARG", i=[ins[0], 0, ins[2]])
    raw("aligned", "INVALID_ARG", i=[ins[0].data_ptr() + 2] + ins[1:])
    other = ctx.register_norm("bf16", "i8", eps=1e-5)
    _refused("INVALID_ARG", "bad verification id", lambda: other._call(h._fn, dims, ins, outs, None, 0))
    for B, V in ((1, 1), (64, 131072), (7, 4097)):
        assert h.workspace_bytes(B, V) == 16 * B * -(-V // 4096) >= max(h.workspace_bytes(B - 1, V), h.workspace_bytes(B, max(1, V - 4000)))


def test_tensors_on_another_device_are_refused():
    """A context of a GPU refuses tensors of the host: checked before anything is launched."""
    pkg.decoder._types()
    h = object.__new__(pkg.NormHandle)
    h._device, h._dtype = 0, torch.bfloat16
    _refused("INVALID_ARG", "is on cpu", lambda: h._rows(torch.zeros(1, 16, dtype=torch.bfloat16), "x", torch.bfloat16))
    _refused("INVALID_ARG", "is on cpu", lambda: h._dense(torch.zeros(1), "scales", torch.float32, (1,)))
    _refused("INVALID_ARG", "is on cpu", lambda: h._scratch(torch.zeros(1)))


# ---- the device header on the CPU ------------------------------------------------------------------


def _header():
    with open(os.path.join(os.path.dirname(pkg.__file__), "csrc", "step_device.h")) as f:
        return f.read()


@pytest.mark.parametrize("group", [32, 64, 128])
def test_places_of_codes(tmp_path, group):
    """After the lanes' exchange, the four lanes of a product have elements of one group, every element of a block comes once, and a lane's
    dword is the one that the exchange brings it: what place() says."""
    body = re.search(r"^DISC_DEV int place\(.*?^}$", _header(), re.M | re.S)[0]
    lib = host_build("constexpr int kG = %d;\n%s\nextern \"C\" int at(int j, int q) { return place(j, q); }\n" % (group, body), tmp_path / f"place{group}")
    at = [[lib.at(j, q) for q in range(4)] for j in range(4)]
    assert sorted(x + e for row in at for x in row for e in range(8)) == list(range(128))
    for j in range(4):
        assert {x // group for x in at[j]} == {j * 128 // (4 * group)}
    # dword j of lane row q holds codes q * 32 + j * 8 ..; halves swapped (0, 2), (1, 3), then rows of 16 (0, 1), (2, 3)
    d = [[q * 32 + j * 8 for q in range(4)] for j in range(4)]

    def swap(a, b, first, second):
        for p, q in zip(first, second):                     # (the odd rows of one and the even rows of the other)
            d[a][p], d[b][q] = d[b][q], d[a][p]
    if group <= 64:
        swap(0, 2, (2, 3), (0, 1))
        swap(1, 3, (2, 3), (0, 1))
        d = [d[0], d[1], d[2], d[3]]
    if group == 32:
        swap(0, 1, (1, 3), (0, 2))
        swap(2, 3, (1, 3), (0, 2))
    assert d == at


# ---- the oracle ------------------------------------------------------------------------------------


def test_oracle_of_the_norm():
    g = torch.Generator().manual_seed(1)
    x, r, w, dy, dt = (torch.randn(s, generator=g, dtype=torch.float64) for s in ((4, 9), (4, 9), (9,), (4, 9), (4, 9)))
    s, y, largest = plain.norm(x, w, 1e-3, 1.0, r)
    assert torch.equal(s, x + r) and torch.equal(largest, y.abs().amax(-1))
    assert torch.allclose((y / (w + 1)).square().mean(-1), s.square().mean(-1) / (s.square().mean(-1) + 1e-3), rtol=1e-12, atol=0)
    a, b, c = (t.clone().requires_grad_() for t in (x, r, w))
    total = a + b
    (total * torch.rsqrt(total.square().mean(-1, keepdim=True) + 1e-3) * (c + 1) * dy).sum().add((total * dt).sum()).backward()
    dx, dw, *_ = plain.norm_backward(s, w, dy, 1e-3, 1.0, dt)
    assert torch.allclose(a.grad, dx, rtol=1e-11, atol=1e-12) and torch.allclose(b.grad, dx, rtol=1e-11, atol=1e-12) and torch.allclose(c.grad, dw, rtol=1e-11, atol=1e-12)
    x[1, 2], x[3, 0] = math.inf, math.nan
    assert torch.isnan(plain.norm(x, w, 1e-3)[1]).all(-1).tolist() == [False, True, False, True]


def test_oracle_of_the_product():
    weights = torch.tensor([[0x21, 0xf8] + [0x88] * 14], dtype=torch.uint8)
    assert plain.codes4(weights)[0, :4].tolist() == [1, 2, 8, 15]
    x = torch.zeros(1, 32)
    x[0, :4] = torch.tensor([1.0, 10.0, 100.0, 1000.0])
    y, _ = plain.linear4(x, weights, torch.tensor([[0.5]]), 32)
    assert y.item() == 0.5 * (-7 - 60 + 0 + 7000)
    y, _ = plain.linear4(x, weights, torch.tensor([[0.5]]), 32, zeros=torch.tensor([[1]], dtype=torch.uint8), row_scales=torch.tensor([2.0]), bias=torch.tensor([3.0]))
    assert y.item() == 0 + 10 + 700 + 14000 + 3


def test_oracle_of_the_verification():
    """Against exact fractions: the tokens of every uniform on a grid, and that they come with the target's probabilities."""
    p, q = [Fraction(1, 2), Fraction(1, 8), Fraction(3, 8)], [Fraction(1, 8), Fraction(5, 8), Fraction(1, 4)]
    n = 64
    share = [Fraction(0)] * 3
    for x in range(3):
        for u in range(n):
            for v in range(n):
                kept = Fraction(u, n) * q[x] < p[x]
                less = [max(a - b, 0) for a, b in zip(p, q)]
                token, upto = x, Fraction(0)
                if not kept:
                    for token in range(3):
                        upto += less[token]
                        if upto > Fraction(v, n) * sum(less):
                            break
                share[token] += q[x] / n ** 2
    assert all(abs(a - b) <= Fraction(1, n) for a, b in zip(share, p))
    t = lambda v: torch.tensor([[[float(a) for a in v]] * 2])  # noqa: E731
    for x in range(3):
        for u in (0, 5, 20, 40, 63):
            for v in (0, 31, 63):
                got, kept = plain.verify(t(p), torch.tensor([[x]]), torch.tensor([[u / n, v / n]]), t(q)[:, :1])
                assert int(kept[0]) == (Fraction(u, n) * q[x] < p[x])
                w = p if int(kept[0]) else [max(a - b, 0) for a, b in zip(p, q)]
                first = next(k for k in range(3) if sum(w[:k + 1]) > Fraction(v, n) * sum(w))
                assert got[0].tolist() == ([x, first] if int(kept[0]) else [first, -1])
    assert plain.verify(t(p), torch.tensor([[1]]), torch.tensor([[0.5, 0.0]]), None, torch.tensor([0]))[0].tolist() == [[0, -1]]
    assert plain.verify(torch.zeros(1, 2, 3), torch.tensor([[1]]), torch.tensor([[0.5, 0.5]]))[0].tolist() == [[-1, -1]]
