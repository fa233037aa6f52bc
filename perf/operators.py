"""Performance cases of the operators around a decoder's attention: rotary positions, a cache of keys and
values in pages (16-bit, or quantised to 8 bits as it is written), and attention over that cache.

A program registers the rotation and the cache once (element type, head size, storage), keeps the two
handles, and then calls them at whatever batch, lengths and heads the next step has.  One pass is one
call: a rotation of q and k, or its gradient; storing the new rows of keys and values; reading stored
rows back; attention of one query token per sequence over its pages, with or without a prefix that all
sequences of the batch share.
"""
import math

import torch

own = False

DTYPES = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}
STORED = {"bf16": torch.bfloat16, "f16": torch.float16, "i8": torch.int8, "e4m3": torch.float8_e4m3fn}
LARGEST_CODE = {"i8": 127.0, "e4m3": 448.0}
BYTES = {"bf16": 2, "f16": 2, "f32": 4, "i8": 1, "e4m3": 1}


def listed():
    return [
        # One step of a small batch: a call's latency, not its traffic.
        {"name": "rotary_8_tokens", "kind": "rotary", "T": 8, "q_heads": 32, "kv_heads": 8, "D": 128, "R": 128, "dtype": "bf16", "layout": "half", "scaling": "none", "backward": False, "far": 4096},
        # A packed batch of prompts, an odd number of tokens, part of each head rotated, fp32 activations.
        {"name": "rotary_part_16007", "kind": "rotary", "T": 16007, "q_heads": 12, "kv_heads": 12, "D": 80, "R": 32, "dtype": "f32", "layout": "interleaved", "scaling": "linear", "backward": False, "far": 16384},
        # Training on long sequences: the gradient of the rotation, frequencies scaled by parts.
        {"name": "rotary_backward_32768", "kind": "rotary", "T": 32768, "q_heads": 32, "kv_heads": 8, "D": 128, "R": 128, "dtype": "bf16", "layout": "half", "scaling": "by_parts", "backward": True, "far": 131072},
        # The new token of every sequence of a batch enters a quantised cache.
        {"name": "store_64_tokens_i8", "kind": "store", "T": 64, "kv_heads": 8, "D": 128, "dtype": "bf16", "storage": "i8", "page": 16},
        # A chunk of prompts enters the cache, padded rows among it.
        {"name": "store_40009_tokens_e4m3", "kind": "store", "T": 40009, "kv_heads": 8, "D": 128, "dtype": "bf16", "storage": "e4m3", "page": 64},
        # A short stored prefix comes back for a product that reads dense rows; and a long one.
        {"name": "load_777_tokens_e4m3", "kind": "load", "T": 777, "kv_heads": 4, "D": 64, "dtype": "f16", "storage": "e4m3", "page": 16},
        {"name": "load_65536_tokens_i8", "kind": "load", "T": 65536, "kv_heads": 8, "D": 128, "dtype": "bf16", "storage": "i8", "page": 64},
        # One short conversation: the latency of a step.
        {"name": "attend_1x300_bf16", "kind": "attend", "B": 1, "L": 300, "prefix": 0, "q_heads": 12, "kv_heads": 12, "D": 64, "dtype": "bf16", "storage": "bf16", "page": 16},
        # A served batch with ragged lengths over a quantised cache.
        {"name": "attend_64x8192_i8", "kind": "attend", "B": 64, "L": 8192, "prefix": 0, "q_heads": 32, "kv_heads": 8, "D": 128, "dtype": "bf16", "storage": "i8", "page": 64},
        # Two long documents: few rows, work only along the cache.
        {"name": "attend_2x131072_bf16", "kind": "attend", "B": 2, "L": 131072, "prefix": 0, "q_heads": 64, "kv_heads": 8, "D": 128, "dtype": "bf16", "storage": "bf16", "page": 128},
        # A few questions about one page of instructions; a full batch behind a long one.
        {"name": "prefix_8x1000_f16", "kind": "attend", "B": 8, "L": 130, "prefix": 1000, "q_heads": 16, "kv_heads": 4, "D": 128, "dtype": "f16", "storage": "f16", "page": 16},
        {"name": "prefix_128x16384_i8", "kind": "attend", "B": 128, "L": 512, "prefix": 16384, "q_heads": 64, "kv_heads": 8, "D": 128, "dtype": "bf16", "storage": "i8", "page": 64},
    ]


def _log(rng, lo, hi):
    return max(lo, min(hi, int(round(2.0 ** rng.uniform(math.log2(lo), math.log2(hi))))))


def draw(rng):
    kind = rng.choice(("rotary", "store", "load", "attend", "attend", "prefix"))
    D = rng.choice((64, 80, 128, 128, 256))
    kv = rng.choice((1, 2, 4, 8, 12))
    if kind == "rotary":
        R = D if rng.random() < 0.6 else 2 * rng.randint(4, D // 2)
        q = kv * rng.choice((1, 2, 3, 4, 8))
        return {"kind": kind, "T": _log(rng, 1, min(32768, 32768 * 40 * 128 // ((q + kv) * D))), "q_heads": q, "kv_heads": kv, "D": D, "R": R,
                "dtype": rng.choice(("bf16", "f16", "f32")), "layout": rng.choice(("half", "interleaved")),
                "scaling": rng.choice(("none", "linear", "base", "by_parts")), "backward": rng.random() < 0.4, "far": _log(rng, 64, 1 << 20)}
    dtype = rng.choice(("bf16", "bf16", "f16"))
    storage = rng.choice((dtype, "i8", "e4m3"))
    page = rng.choice((8, 16, 64, 128, 256))
    if kind in ("store", "load"):
        return {"kind": kind, "T": _log(rng, 1, min(65536, 65536 * 8 * 128 // (kv * D))), "kv_heads": kv, "D": D, "dtype": dtype, "storage": storage, "page": page}
    q = kv * rng.choice((1, 2, 4, 5, 8, 16))
    # (most rows of keys and values that a drawn cache holds, and most products of a drawn prefix)
    B = _log(rng, 1, 128)
    rows = 64 * 8192 * 8 * 128 // (B * kv * D)
    if kind == "attend":
        return {"kind": "attend", "B": B, "L": _log(rng, 1, max(1, min(131072, rows // 2))), "prefix": 0, "q_heads": q, "kv_heads": kv, "D": D,
                "dtype": dtype, "storage": storage, "page": page}
    products = 128 * 64 * 16384 * 128 // (B * q * D)
    return {"kind": "attend", "B": B, "L": _log(rng, 1, max(1, min(1024, rows // 8))), "prefix": _log(rng, 100, max(100, min(32768, products // 2))), "q_heads": q,
            "kv_heads": kv, "D": D, "dtype": dtype, "storage": storage, "page": page}


def _frequencies(case):
    """Radians a position of every pair, and the factor on the rotated values (plain numbers that a model's configuration gives)."""
    R, kind = case["R"], case["scaling"]
    base = 10000.0
    if kind == "base":
        base *= 8.0 ** (R / (R - 2.0))
    f = [base ** (-2.0 * j / R) for j in range(R // 2)]
    if kind == "linear":
        f = [x / 4.0 for x in f]
    if kind == "by_parts":              # pairs that turn often in the original length keep their frequency, slow ones are stretched
        whole = [4096.0 * x / (2.0 * math.pi) for x in f]
        keep = [min(1.0, max(0.0, (w - 1.0) / 31.0)) for w in whole]
        f = [x * (k + (1.0 - k) / 16.0) for x, k in zip(f, keep)]
        return f, 0.1 * math.log(16.0) + 1.0
    return f, 1.0


def _generator(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(int(seed))
    return g


def _normal(shape, dtype, g, std=1.0):
    return torch.empty(shape, dtype=torch.float32, device="cuda").normal_(0.0, std, generator=g).to(dtype)


def _lengths(case):
    """Spread over 1..L, the longest among them; in a batch of four and more one sequence has none of its own."""
    B, L = case["B"], case["L"]
    n = [max(1, int(round(L * (((i + 1) * 0.6180339887498949) % 1.0)))) for i in range(B)]
    n[0] = L
    if B >= 4:
        n[3] = 0
    return n


def _rows(shape, g):
    """Keys or values: channels of different size and offset, as projections have them."""
    x = torch.empty(shape, dtype=torch.float32, device="cuda").normal_(0.0, 1.0, generator=g)
    size = torch.empty(shape[-1], dtype=torch.float32, device="cuda").normal_(0.0, 0.4, generator=g).exp_()
    return x.mul_(size).add_(torch.empty(shape[-1], dtype=torch.float32, device="cuda").normal_(0.0, 0.2, generator=g))


def _quantise(x, storage):
    """Codes and scales of rows (the last axis): largest magnitude to the largest code."""
    a = x.abs().amax(-1)
    most = LARGEST_CODE[storage]
    # (divided by a tensor: by a number, torch multiplies with its reciprocal, which is rounded once more)
    whole = torch.full_like(a, most)
    inverse = torch.where(a > 0, whole / a, torch.zeros_like(a))
    y = (x * inverse.unsqueeze(-1)).clamp_(-most, most)
    return (y.round_() if storage == "i8" else y).to(STORED[storage]), a / whole


def _pages(case, pages, g):
    shape = (pages, case["kv_heads"], case["page"], case["D"])
    if case["storage"] not in LARGEST_CODE:
        return [_rows(shape, g).to(STORED[case["storage"]]) for _ in range(2)]
    k, ks = _quantise(_rows(shape, g), case["storage"])
    v, vs = _quantise(_rows(shape, g), case["storage"])
    return [k, v, ks, vs]


def prepare(case, seed):
    g = _generator(seed)
    D, kv = case["D"], case["kv_heads"]
    dtype = DTYPES[case["dtype"]]
    if case["kind"] == "rotary":
        q = case["q_heads"]
        # q and k are parts of one product's rows, as are the keys and values that a cache takes
        x = _normal((case["T"], q + 2 * kv, D), dtype, g)
        positions = torch.randint(0, case["far"], (case["T"],), generator=g, device="cuda", dtype=torch.int32)
        return {"case": case, "positions": positions, "inputs": [x[:, :q], x[:, q:q + kv]],
                "outputs": [torch.empty((case["T"], n, D), dtype=dtype, device="cuda") for n in (q, kv)]}
    page = case["page"]
    if case["kind"] in ("store", "load"):
        T = case["T"]
        pages = -(-T // page) + 3
        slots = torch.arange(T, device="cuda", dtype=torch.int64)
        order = torch.randperm(pages, generator=g, device="cuda")
        slots = order[slots // page] * page + slots % page
        if case["kind"] == "load":
            return {"case": case, "slots": slots, "pages": _pages(case, pages, g),
                    "outputs": [torch.empty((T, kv, D), dtype=dtype, device="cuda") for _ in range(2)]}
        slots[torch.arange(T, device="cuda") % 17 == 16] = -1            # padding rows of the batch
        x = _rows((T, 3 * kv, D), g).to(dtype)
        kept = torch.zeros((pages, kv, page, D), dtype=torch.float32, device="cuda")
        stored = [kept.to(STORED[case["storage"]]) for _ in range(2)]
        if case["storage"] in LARGEST_CODE:
            stored += [torch.zeros((pages, kv, page), dtype=torch.float32, device="cuda") for _ in range(2)]
        return {"case": case, "slots": slots, "inputs": [x[:, kv:2 * kv], x[:, 2 * kv:]], "pages": stored}
    B, n = case["B"], _lengths(case)
    prefix_pages = -(-case["prefix"] // page)
    width = max(1, -(-case["L"] // page))
    lengths = torch.tensor(n, dtype=torch.int32, device="cuda")[torch.randperm(B, generator=g, device="cuda")]
    needed = (lengths.long() + page - 1) // page
    total = sum(-(-m // page) for m in n) + prefix_pages
    order = torch.randperm(total, generator=g, device="cuda").to(torch.int32)
    first = torch.cumsum(needed, 0) - needed
    at = torch.arange(width, device="cuda")
    table = torch.where(at < needed[:, None], order[(prefix_pages + first[:, None] + at).clamp(max=total - 1)], -1).to(torch.int32)
    return {"case": case, "q": _normal((B, case["q_heads"], D), dtype, g), "lengths": lengths, "table": table,
            "prefix_table": order[:prefix_pages].contiguous(), "pages": _pages(case, total, g),
            "out": torch.empty((B, case["q_heads"], D), dtype=dtype, device="cuda")}


# ---- the plain forms -----------------------------------------------------------------------------


def _plain_rotary(state):
    case = state["case"]
    R, sign = case["R"], -1.0 if case["backward"] else 1.0
    f, magnitude = _frequencies(case)
    # (far positions: the angles in 64 bits)
    angle = state["positions"].double()[:, None] * torch.tensor(f, dtype=torch.float64, device="cuda")
    c, s = (magnitude * angle.cos()).float()[:, None], (sign * magnitude * angle.sin()).float()[:, None]
    for x, y in zip(state["inputs"], state["outputs"]):
        z = x.float()
        if case["layout"] == "half":
            a, b = z[..., :R // 2], z[..., R // 2:R]
            turned = torch.cat((a * c - b * s, b * c + a * s, z[..., R:]), -1)
        else:
            a, b = z[..., 0:R:2], z[..., 1:R:2]
            turned = torch.cat((torch.stack((a * c - b * s, b * c + a * s), -1).flatten(-2), z[..., R:]), -1)
        y.copy_(turned)
    return state["outputs"]


def _plain_store(state):
    case = state["case"]
    keep = state["slots"] >= 0
    slots = state["slots"][keep]
    page, place = slots // case["page"], slots % case["page"]
    for i, x in enumerate(state["inputs"]):
        rows = x[keep].float()
        if case["storage"] in LARGEST_CODE:
            codes, scales = _quantise(rows, case["storage"])
            state["pages"][i][page, :, place] = codes
            state["pages"][2 + i][page, :, place] = scales
        else:
            state["pages"][i][page, :, place] = rows.to(STORED[case["storage"]])
    return state["pages"]


def _dense(case, pages, page, place, dtype):
    """Keys and values of the given places, [..., kv_heads, D]."""
    found = [p[page, :, place].to(dtype) for p in pages[:2]]
    if len(pages) == 4:
        found = [x * s[page, :, place].unsqueeze(-1) for x, s in zip(found, pages[2:])]
    return found


def _plain_load(state):
    case = state["case"]
    rows = _dense(case, state["pages"], state["slots"] // case["page"], state["slots"] % case["page"], torch.float32)
    for x, y in zip(rows, state["outputs"]):
        y.copy_(x)
    return state["outputs"]


def _plain_attend(state):
    case = state["case"]
    B, H, kv, D = case["B"], case["q_heads"], case["kv_heads"], case["D"]
    G, scale = H // kv, 1.0 / math.sqrt(D)
    q = state["q"].float().view(B, kv, G, D)
    at = torch.arange(max(1, case["L"]), device="cuda")
    there = at < state["lengths"][:, None]
    page = state["table"][:, at // case["page"]].clamp(min=0).long()
    k, v = _dense(case, state["pages"], page, (at % case["page"]).expand(B, -1), torch.float32)
    k, v = k.permute(0, 2, 3, 1), torch.where(there[..., None, None], v, 0.0).transpose(1, 2)
    scores = torch.matmul(q, k) * scale
    scores = torch.where(there[:, None, None, :], scores, -math.inf)
    if case["prefix"]:
        at = torch.arange(case["prefix"], device="cuda")
        kp, vp = _dense(case, state["pages"], state["prefix_table"][at // case["page"]].long(), at % case["page"], torch.float32)
        shared = torch.matmul(q.transpose(0, 1).reshape(kv, B * G, D), kp.permute(1, 2, 0)) * scale
        scores = torch.cat((shared.view(kv, B, G, -1).transpose(0, 1), scores), -1)
    most = scores.amax(-1, keepdim=True)
    p = torch.exp(scores - torch.where(most > -math.inf, most, 0.0))
    total = p.sum(-1, keepdim=True)
    out = torch.matmul(p[..., case["prefix"]:], v)
    if case["prefix"]:
        mine = p[..., :case["prefix"]].transpose(0, 1).reshape(kv, B * G, -1)
        out = out + torch.matmul(mine, vp.transpose(0, 1)).view(kv, B, G, D).transpose(0, 1)
    state["out"].copy_((out / torch.where(total > 0, total, 1.0)).view(B, H, D))
    return state["out"]


# ---- the framework's calls -----------------------------------------------------------------------

_context = None
_handles = {}


def _handle(case):
    """The registered operator: compiled once in a program's life, whatever batches and lengths follow."""
    global _context
    rotary = case["kind"] == "rotary"
    key = tuple(case[k] for k in (("dtype", "D", "R", "layout", "scaling") if rotary else ("dtype", "D", "storage")))
    if key not in _handles:
        import paper_2103_05288_amd as pkg
        if _context is None:
            _context = pkg.Context(torch.cuda.current_device())
        if rotary:
            frequencies, magnitude = _frequencies(case)
            _handles[key] = _context.register_rotary(case["dtype"], case["D"], frequencies, layout=case["layout"], magnitude=magnitude)
        else:
            _handles[key] = _context.register_cache(case["dtype"], case["D"], storage=case["storage"])
    return _handles[key]


def _own_run(state):
    case = state["case"]
    # (a program keeps its handle and its workspace from step to step)
    handle = state.get("handle")
    if handle is None:
        handle = state["handle"] = _handle(case)
        if case["kind"] == "attend":
            need = handle.workspace_bytes(case["B"], case["q_heads"], case["kv_heads"], state["table"].shape[1] * case["page"], case["prefix"])
            state["workspace"] = torch.empty(max(need, 256), dtype=torch.uint8, device="cuda")
    if case["kind"] == "rotary":
        handle.launch(state["positions"], state["inputs"], state["outputs"], backward=case["backward"])
        return state["outputs"]
    if case["kind"] == "store":
        handle.store(state["inputs"], state["slots"], state["pages"])
        return state["pages"]
    if case["kind"] == "load":
        handle.load(state["slots"], state["pages"], state["outputs"])
        return state["outputs"]
    if case["prefix"]:
        handle.attend(state["q"], state["lengths"], state["table"], state["pages"], state["out"], workspace=state["workspace"],
                      prefix_table=state["prefix_table"], prefix_length=case["prefix"])
    else:
        handle.attend(state["q"], state["lengths"], state["table"], state["pages"], state["out"], workspace=state["workspace"])
    return state["out"]


def run(state):
    if own:
        return _own_run(state)
    return {"rotary": _plain_rotary, "store": _plain_store, "load": _plain_load, "attend": _plain_attend}[state["case"]["kind"]](state)


def work(case):
    D, kv, size = case["D"], case["kv_heads"], BYTES[case["dtype"]]
    if case["kind"] == "rotary":
        elements = case["T"] * (case["q_heads"] + kv) * D
        # (six operations a pair; sine and cosine of a pair's angle once for all heads, counted as 40)
        return {"bytes": 2 * size * elements + 4 * case["T"], "flops": elements / D * case["R"] * 3 + 40 * case["T"] * case["R"] / 2}
    row = D * BYTES[case["storage"]] + (4 if case["storage"] in LARGEST_CODE else 0)     # one stored row of keys or of values
    if case["kind"] in ("store", "load"):
        T = case["T"] - (case["T"] // 17 if case["kind"] == "store" else 0)
        return {"bytes": 2 * T * kv * (row + D * size) + 8 * case["T"], "flops": 3 * 2 * T * kv * D}
    tokens = sum(_lengths(case))
    read = 2 * kv * row * (tokens + case["prefix"]) + 4 * (tokens + case["prefix"]) / case["page"] + 4 * case["B"]
    return {"bytes": read + 2 * case["B"] * case["q_heads"] * D * size, "flops": 4 * case["q_heads"] * D * (tokens + case["B"] * case["prefix"])}


# ---- 64 bits -------------------------------------------------------------------------------------


def exact(case, seed):
    state = prepare(case, seed)
    if case["kind"] == "rotary":
        f, magnitude = _frequencies(case)
        turn = torch.polar(torch.full((1,), magnitude, dtype=torch.float64, device="cuda"),
                           state["positions"].double()[:, None] * torch.tensor(f, dtype=torch.float64, device="cuda"))
        turn = (turn.conj() if case["backward"] else turn)[:, None, :]
        outs = []
        for x in state["inputs"]:
            y = x.double()
            head = y[..., :case["R"]].unflatten(-1, (2, -1)).transpose(-1, -2) if case["layout"] == "half" else y[..., :case["R"]].unflatten(-1, (-1, 2))
            z = torch.view_as_real(torch.view_as_complex(head.contiguous()) * turn)
            y[..., :case["R"]] = (z.transpose(-1, -2) if case["layout"] == "half" else z).flatten(-2)
            outs.append(y)
        return outs
    if case["kind"] == "store":
        live = state["slots"] >= 0
        places = (state["pages"][0].shape[0] * case["page"], case["kv_heads"])
        if len(state["pages"]) == 2:
            outs = []
            for x in state["inputs"]:
                rows = torch.zeros(places + (case["D"],), dtype=torch.float64, device="cuda")
                rows[state["slots"][live]] = x[live].double()
                outs.append(rows.unflatten(0, (-1, case["page"])).transpose(1, 2).contiguous())
            return outs
        # (codes are rounded as the scales are in 32 bits: 64 bits have no value for them)
        outs = [None, None]
        for x in state["inputs"]:
            s = torch.zeros(places, dtype=torch.float64, device="cuda")
            s[state["slots"][live]] = x[live].double().abs().max(-1)[0] / LARGEST_CODE[case["storage"]]
            outs.append(s.unflatten(0, (-1, case["page"])).transpose(1, 2).contiguous())
        return outs
    if case["kind"] == "load":
        outs = []
        for i in range(2):
            x = state["pages"][i].double()
            if len(state["pages"]) == 4:
                x *= state["pages"][2 + i].double()[..., None]
            outs.append(x.transpose(1, 2).flatten(0, 1)[state["slots"]])
        return outs
    B, kv, D, P = case["B"], case["kv_heads"], case["D"], case["prefix"]
    out = torch.zeros((B, kv, case["q_heads"] // kv, D), dtype=torch.float64, device="cuda")
    n, tables = state["lengths"].tolist(), state["table"]

    def rows(table, m):
        """Keys and values of the first m tokens of the pages of a table: [kv_heads, m, D] each."""
        found = []
        for i in range(2):
            x = state["pages"][i][table[:-(-m // case["page"])].long()].double()
            if len(state["pages"]) == 4:
                x *= state["pages"][2 + i][table[:-(-m // case["page"])].long()].double()[..., None]
            found.append(x.transpose(0, 1).flatten(1, 2)[:, :m])
        return found

    shared = rows(state["prefix_table"], P) if P else None
    for b in range(B):
        parts = ([rows(tables[b], n[b])] if n[b] else []) + ([shared] if P else [])
        if parts:
            k, v = (torch.cat([p[i] for p in parts], 1) for i in range(2))
            q = state["q"][b].double().unflatten(0, (kv, -1))
            out[b] = torch.softmax(torch.bmm(q, k.transpose(1, 2).contiguous()) / math.sqrt(D), -1).bmm(v)
    return out.flatten(1, 2)
