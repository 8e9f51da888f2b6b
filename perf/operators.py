"""Workloads of the paged 4-bit cache and of what goes with it: rows written and read back, attention over the pages, the
calls that hand pages out, share, free and pack them, and rotary positions of tokens that have several coordinates.

A case is a dict of plain values whose ``kind`` names what one pass does:

  rotary   queries and keys of new tokens are turned by their positions (time, height, width), or turned back (the gradient)
  rows     new keys and values go into the pages, in 4 bits, and are read back as the values they now stand for
  attend   new queries over the pages of every batch row, and over kept chunk summaries where k > 0
  beams    rows are forked off the first ones, get room for a token each (a shared page that is only part full is copied
           first), their last page is read, and they are given up again
  step     every row gets room for its next tokens, then gives it back
  compact  the pages in use move into a smaller pool

``run`` computes a pass in elementary torch operations, or with the library's calls where ``own`` is set.

The cache format, as both sides read it: 16 tokens of one key-value head are a group of 17 d bytes: the codes of the keys
(16 rows of d / 2 bytes, the element of lower index in the low half), those of the values, then a scale byte for each of
the keys' and of the values' blocks of 32 elements ([16][d / 32][2]).  A code is sign, two bits of exponent and one of
mantissa (0, .5, 1, 1.5, 2, 3, 4, 6); a scale byte s stands for 2^(s - 127), 255 for not-a-number.
"""
import math

import torch

own = False

VALUES = (0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0)
BASE = dict(dtype="bf16", L=1, B=1, H=32, H_kv=32, d=128)
MOST_BYTES, MOST_FLOPS = 2.6e9, 1.15e12


def listed():
    def case(name, kind, **kw):
        return dict(BASE, name=name, kind=kind, **kw)

    def attend(name, **kw):
        return case(name, "attend", **dict(dict(T=4096, Tq=1, page=64, ragged=False, causal=False, window=0, k=0), **kw))

    return [
        # the queries and keys of one token of one layer: the smallest call there is
        case("rotary_token", "rotary", Tq=1, s0=16, s1=24, s2=24, pairs=False, inverse=False, far=4091),
        # a camera frame of 16 x 16 image tokens on 64 streams, 8 key-value heads
        case("rotary_frames_b64", "rotary", B=64, H_kv=8, Tq=256, s0=16, s1=24, s2=24, pairs=False, inverse=False, far=32768),
        # the gradient of a frame's queries and keys in full precision, neighbouring pairs, part of the head turned
        case("rotary_grad_f32", "rotary", dtype="f32", B=4, H=16, H_kv=16, d=64, Tq=197, s0=7, s1=9, s2=10, pairs=True, inverse=True, far=1000000),
        # the next token of 64 streams goes into their pages
        case("rows_token_b64", "rows", B=64, H_kv=8, T=8192, Tn=1, page=64, ragged=True),
        # prompts of four streams, of different lengths and behind what they hold, are written at once
        case("rows_prompts_b4", "rows", B=4, H_kv=8, T=9000, Tn=8000, page=64, ragged=True),
        # a robot's decode step over one layer, at a length that is no multiple of anything
        attend("decode_b1", T=4091, page=32),
        # a served model's layer: 64 streams of all lengths, 4 query heads to a key-value head
        attend("decode_ragged_b64", B=64, H_kv=8, T=8192, ragged=True),
        # all 32 layers of 8 long streams in one call
        attend("decode_32layers_b8", L=32, B=8, H_kv=8, T=8192),
        # a camera frame of one small fp32 layer over the recent window and the kept summaries: how the path is debugged
        attend("frame_f32_small", dtype="f32", B=2, H=4, H_kv=4, d=64, T=1000, Tq=33, page=16, causal=True, window=320, k=16),
        # a frame of 256 image tokens on 16 streams over all that they hold, each token seeing those before it
        attend("frame_b16_causal", B=16, H_kv=8, T=8192, Tq=256, causal=True),
        # one prompt is shared by 16 streams of a 32-layer model that go on from it
        case("beams_16", "beams", L=32, B=16, H_kv=8, T=2061, page=64, sources=1, n=1),
        # the pages of 48 streams of a 4-layer model, a good half of the pool, move into a smaller one
        case("compact_half", "compact", L=4, B=48, H_kv=8, T=4096, page=64, spare=1.7),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    while True:
        kind = rng.choice(("rotary", "rotary", "rows", "rows", "attend", "attend", "attend", "attend", "frame", "frame", "beams", "step", "compact"))
        c = dict(BASE, kind="attend" if kind == "frame" else kind)
        c["dtype"] = "f32" if rng.random() < 0.2 else "bf16"
        c["d"] = 128 if rng.random() < 0.75 else 64
        c["H"] = rng.choice((4, 8, 16, 32, 32))
        c["H_kv"] = c["H"] // rng.choice((1, 2, 4, 4))
        c["L"] = 1 if rng.random() < 0.6 else _log(rng, 2, 32)
        c["B"] = _log(rng, 1, 64)
        if kind == "rotary":
            half = c["d"] // 2
            total = half if rng.random() < 0.7 else rng.randint(3, half)
            c["s0"] = rng.randint(1, total - 2)
            c["s1"] = rng.randint(1, total - c["s0"] - 1)
            c["s2"] = total - c["s0"] - c["s1"]
            c["pairs"], c["inverse"] = rng.random() < 0.4, rng.random() < 0.4
            c["Tq"], c["far"] = _log(rng, 1, 2048), _log(rng, 300, 1000000)
        else:
            c["page"] = rng.choice((16, 32, 64, 64, 128, 256))
            c["T"] = _log(rng, 1, 16384) if kind == "attend" else _log(rng, 300, 16384)
        if kind == "rows":
            c["Tn"], c["ragged"] = min(_log(rng, 1, 8192), c["T"]), rng.random() < 0.6
        if kind in ("attend", "frame"):
            c["Tq"] = 1 if kind == "attend" and rng.random() < 0.8 else min(_log(rng, 2, 300), c["T"])
            c["ragged"], c["causal"] = c["B"] > 1 and rng.random() < 0.6, rng.random() < 0.5
            c["window"] = _log(rng, 32, 600) if rng.random() < 0.25 else 0
            c["k"] = _log(rng, 4, 128) if rng.random() < 0.3 else 0
        if kind in ("beams", "step"):
            c["n"] = _log(rng, 1, 40)
        if kind == "beams":
            c["B"] = max(c["B"], 2)
            c["sources"] = rng.randint(1, (c["B"] + 1) // 2)
        if kind == "compact":
            c["spare"] = round(rng.uniform(1.1, 3.0), 2)
        w = work(c)
        pool = c["L"] * c["B"] * c["H_kv"] * c.get("T", 0) * 17 * c["d"] // 16
        if w["bytes"] > MOST_BYTES or pool > MOST_BYTES or w["flops"] > (5e10 if c["dtype"] == "f32" else MOST_FLOPS):
            continue
        return c


def _pages_of(n, page):
    return -(-n // page)


def _lengths(c):
    """The tokens that each batch row holds: T, or (ragged) lengths from 1 to T, the longest among them."""
    T, B = c["T"], c["B"]
    if not c.get("ragged"):
        return [T] * B
    least = c["Tq"] if c.get("causal") else 1
    return [max(least, T - (T * ((37 * b) % B)) // B) for b in range(B)]


def work(case):
    c, kind = case, case["kind"]
    es, d, S, Sq = (4 if case["dtype"] == "f32" else 2), case["d"], case["L"] * case["H_kv"], case["L"] * case["H"]
    row = 17 * d // 16                                   # a token's key and value of one head, in the pages
    if kind == "rotary":
        n = (S + Sq) * c["B"] * c["Tq"] * d
        return {"bytes": 2 * n * es + 12 * c["B"] * c["Tq"], "flops": 3 * n}
    if kind == "rows":
        n = S * sum(_new_tokens(c))
        return {"bytes": n * 2 * (2 * d * es + row), "flops": 8 * n * d}
    if kind == "attend":
        rows = sum(min(n, c["window"] or n) for n in _lengths(c))
        seen = rows - c["B"] * (c["Tq"] - 1) / 2 if c["causal"] else rows
        seen = max(seen, c["B"])
        kept = c["B"] * c["k"]
        return {"bytes": int(S * (rows * row + kept * 2 * d * es) + 2 * Sq * c["B"] * c["Tq"] * d * es), "flops": int(Sq * c["Tq"] * 4 * d * (seen + kept))}
    cells = c["B"] * 8 * _pages_of(c["T"] + c.get("n", 0), c["page"])         # table entries, there and back
    if kind == "beams":
        copied = (c["B"] - c["sources"]) if c["T"] % c["page"] else 0
        return {"bytes": S * copied * c["page"] * row * 2 + S * (c["B"] - c["sources"]) * (c["T"] % c["page"]) * (row + 2 * d * es) + 2 * cells, "flops": 0}
    if kind == "step":
        return {"bytes": c["B"] * 16 + 4 * c["B"] * _pages_of(c["n"], c["page"]), "flops": 0}
    live = c["B"] * _pages_of(c["T"], c["page"])
    return {"bytes": S * live * c["page"] * row * 2 + cells + 8 * live, "flops": 0}


def _new_tokens(c):
    if not c["ragged"] or c["Tn"] == 1:
        return [c["Tn"]] * c["B"]
    return [max(1, c["Tn"] - (c["Tn"] * ((5 * b) % c["B"])) // (2 * c["B"])) for b in range(c["B"])]


# ---- the format, in torch ----------------------------------------------------------------------------------------------

def _quantise(x):
    """fp32 [..., d] -> codes [..., d] and scale bytes [..., d / 32] (uint8).  The scale is the smallest power of two with
    which the block's largest magnitude rounds to 6 at most; codes are rounded to nearest, ties to even."""
    blk = x.float().reshape(*x.shape[:-1], -1, 32)
    top = blk.abs().amax(-1)
    fine = torch.isfinite(blk).all(-1)
    bits = torch.where(fine, top, torch.zeros_like(top)).contiguous().view(torch.int32)
    s = (((bits + 0x1FFFFF) >> 23) - 2).clamp_(min=2)
    y = blk.abs() * ((254 - s) << 23).view(torch.float32)[..., None]
    code = (y > 0.25).to(torch.uint8)
    for edge, closed in ((0.75, True), (1.25, False), (1.75, True), (2.5, False), (3.5, True), (5.0, False)):
        code += (y >= edge) if closed else (y > edge)
    code += torch.signbit(blk).to(torch.uint8) * 8
    code = torch.where(fine[..., None], code, torch.zeros_like(code))
    return code.reshape(x.shape), torch.where(fine, s, torch.full_like(s, 255)).to(torch.uint8)


def _nibbles(codes):
    return codes[..., 0::2] | (codes[..., 1::2] << 4)


def _store(pool, layer, page, row, K, V):
    """Rows K, V [n, H_kv, d] of one layer into token `row` (0 .. page - 1) of pages `page` (both [n] int64)."""
    d = K.shape[-1]
    for side, x in enumerate((K, V)):
        codes, scale = _quantise(x)
        groups = pool[layer].view(pool.shape[1], pool.shape[2], -1, 17 * d)
        g, r = row // 16, row % 16
        part = groups[..., 8 * d * side:8 * d * (side + 1)].unflatten(-1, (16, d // 2))
        part[page, :, g, r] = _nibbles(codes)
        groups[..., 16 * d:].unflatten(-1, (16, d // 32, 2))[page, :, g, r, :, side] = scale


def _values(codes, scale):
    """Packed codes [..., d / 2] and scale bytes [..., d / 32] -> fp32 [..., d]"""
    lut = torch.tensor(VALUES + tuple(-v for v in VALUES), dtype=torch.float32, device=codes.device)
    s = scale.int()
    factor = torch.where(s == 255, torch.full_like(s, 0x7FC00000), s << 23).view(torch.float32)
    v = lut[torch.stack((codes & 15, codes >> 4), -1).flatten(-2).int()]
    return (v.unflatten(-1, (-1, 32)) * factor[..., None]).flatten(-2)


def _rows(pages, d):
    """Pages [..., H_kv, bytes] -> keys and values [..., H_kv, tokens, d] in fp32"""
    g = pages.unflatten(-1, (-1, 17 * d))
    scale = g[..., 16 * d:].unflatten(-1, (16, d // 32, 2))
    return tuple(_values(g[..., 8 * d * i:8 * d * (i + 1)].unflatten(-1, (16, d // 2)), scale[..., i]).flatten(-3, -2) for i in (0, 1))


# ---- inputs --------------------------------------------------------------------------------------------------------------

def _dtype(c):
    return torch.float32 if c["dtype"] == "f32" else torch.bfloat16


def _normal(g, *shape, scale=1.0, dtype=torch.float32):
    return torch.empty(shape, dtype=dtype, device="cuda").normal_(0.0, scale, generator=g)


def _ints(v):
    return torch.tensor(v, dtype=torch.int32, device="cuda")


def _rotary_inputs(c, g):
    dt, P, T = _dtype(c), c["s0"] + c["s1"] + c["s2"], c["Tq"]
    t = {"Q": _normal(g, c["L"], c["B"], c["H"], T, c["d"], dtype=dt), "K": _normal(g, c["L"], c["B"], c["H_kv"], T, c["d"], dtype=dt)}
    t["freq"] = torch.pow(1.0e4, -torch.arange(P, dtype=torch.float64, device="cuda") / P).float()
    # tokens of frames of 16 x 16, behind the `far` tokens or so that the stream has seen
    i = torch.arange(T, dtype=torch.int64, device="cuda")
    base = torch.randint(0, c["far"] + 1, (1, c["B"], 1), device="cuda", generator=g)
    t["pos"] = (base + torch.stack((i // 256, i // 16 % 16, i % 16))[:, None, :]).to(torch.int32)
    return t


def _table(c, g, held, pages, n_pages, max_pages):
    """A table whose rows hold `pages[b]` pages each, anywhere in the pool."""
    order = torch.randperm(n_pages, generator=g, device="cuda").to(torch.int32)
    table = torch.full((c["B"], max_pages), -1, dtype=torch.int32, device="cuda")
    at = 0
    for b, n in enumerate(pages):
        table[b, :n] = order[at:at + n]
        at += n
    refs = torch.zeros(n_pages, dtype=torch.int32, device="cuda")
    refs[order[:at].long()] = 1
    return table, refs, _ints(held)


def _cache(c, g, held, room, extra_pages=0, fill=True):
    """A pool whose rows hold `held[b]` tokens in pages for `room[b]`; keys with a few channels that stand out, as they do."""
    d, page = c["d"], c["page"]
    pages = [_pages_of(n, page) for n in room]
    max_pages = max(1, max(pages) + _pages_of(c.get("n", 0), page))
    n_pages = max(1, sum(pages) + extra_pages)
    table, refs, length = _table(c, g, held, pages, n_pages, max_pages)
    pool = torch.empty(c["L"], n_pages, c["H_kv"], 17 * d * page // 16, dtype=torch.uint8, device="cuda")
    chan = 1.0 + 3.0 * (torch.rand(d, generator=g, device="cuda") < 0.05)
    step = max(1, (1 << 26) // (c["H_kv"] * page * d))
    for layer in range(c["L"]):
        for p0 in range(0, n_pages if fill else 0, step):
            n = min(step, n_pages - p0)
            groups = pool[layer, p0:p0 + n].view(n, c["H_kv"], page // 16, 17 * d)
            scale = groups[..., 16 * d:].unflatten(-1, (16, d // 32, 2))
            for side in (0, 1):
                x = _normal(g, n, c["H_kv"], page // 16, 16, d)
                codes, s = _quantise(x * chan if side == 0 else x)
                groups[..., 8 * d * side:8 * d * (side + 1)] = _nibbles(codes).flatten(-2)
                scale[..., side] = s
        if not fill:
            pool[layer].random_(0, 250, generator=g)
    return {"pool": pool, "table": table, "refs": refs, "length": length, "n_pages": n_pages, "max_pages": max_pages}


def _make(c, seed):
    """Everything of a case but what only the library's calls take."""
    g = torch.Generator(device="cuda")
    g.manual_seed(int(seed))
    kind, dt, L, B, d = c["kind"], _dtype(c), c["L"], c["B"], c["d"]
    if kind == "rotary":
        return _rotary_inputs(c, g)
    if kind == "rows":
        new = _new_tokens(c)
        before = [max(0, n - m) for n, m in zip(_lengths(c), new)]
        t = _cache(c, g, before, [a + m for a, m in zip(before, new)], fill=False)
        t["K"], t["V"] = (_normal(g, L, B, c["H_kv"], c["Tn"], d, dtype=dt) for _ in range(2))
        t["start"], t["n_new"] = t["length"].clone(), _ints(new)
        return t
    if kind == "attend":
        held = _lengths(c)
        t = _cache(c, g, held, held)
        t["Q"] = _normal(g, L, B, c["H"], c["Tq"], d, dtype=dt)
        t["q_start"] = _ints([n - c["Tq"] for n in held]) if c["causal"] else None
        t["first"] = None
        if c["window"]:
            first = [max(0, n - c["window"]) for n in held]
            t["first"] = _ints(first)
            for b, n in enumerate(first):             # what lies before the window is not held any more
                t["table"][b, :n // c["page"]] = -1
        if c["k"]:
            t["Kc"], t["Vc"] = (_normal(g, L, B, c["H_kv"], c["k"], d, scale=0.25, dtype=dt) for _ in range(2))
            t["count"] = torch.randint((c["k"] + 1) // 2, c["k"] + 1, (L, B, c["H_kv"]), generator=g, device="cuda", dtype=torch.int32)
        return t
    if kind == "beams":
        n_src = c["sources"]
        held = [c["T"] - 3 * b if c["T"] > 3 * b else 1 for b in range(n_src)] + [0] * (B - n_src)
        t = _cache(c, g, held, held, extra_pages=(B - n_src) * (1 + _pages_of(c["n"], c["page"])))
        t["dst"] = torch.arange(n_src, B, dtype=torch.int32, device="cuda")
        t["src"] = t["dst"] % n_src
        t["n_new"] = _ints([0] * n_src + [c["n"]] * (B - n_src))
        t["nil"] = torch.zeros(B, dtype=torch.int32, device="cuda")
        return t
    if kind == "step":
        held = [max(1, c["T"] - (7 * b) % min(c["T"], 300)) for b in range(B)]
        t = _cache(dict(c, L=1), g, held, held, extra_pages=B * (1 + _pages_of(c["n"], c["page"])), fill=False)
        t["n_new"], t["kept"] = _ints([c["n"]] * B), t["length"].clone()
        return t
    live = B * _pages_of(c["T"], c["page"])
    t = _cache(c, g, [c["T"]] * B, [c["T"]] * B, extra_pages=int(live * (c["spare"] - 1.0)), fill=False)
    t["to_pages"] = live + live // 16
    return t


def prepare(case, seed):
    c, s = case, _make(case, seed)
    s["case"] = c
    kind, dt, B, d, zeros = c["kind"], _dtype(c), c["B"], c["d"], torch.zeros
    if kind == "rotary":
        s["Q_out"], s["K_out"] = torch.empty_like(s["Q"]), torch.empty_like(s["K"])
    if kind == "rows":
        s["K_out"], s["V_out"] = torch.zeros_like(s["K"]), torch.zeros_like(s["V"])
    if kind == "attend":
        s["O"] = torch.empty_like(s["Q"])
    if kind == "beams":
        s["K_out"], s["V_out"] = (zeros(c["L"], B, c["H_kv"], c["page"], d, dtype=dt, device="cuda") for _ in range(2))
        part = [0] * B
        held = s["length"].tolist()
        for x, y in zip(s["dst"].tolist(), s["src"].tolist()):
            part[x] = held[y] % c["page"]
        s["part"] = _ints(part)
        s["part_first"] = _ints([0] * c["sources"] + [held[y] - held[y] % c["page"] for y in s["src"].tolist()])
    if kind in ("beams", "step"):
        s["start"], s["status"] = zeros(B, dtype=torch.int32, device="cuda"), zeros(1, dtype=torch.int32, device="cuda")
    if kind == "compact":
        s["to_pool"] = zeros((c["L"], s["to_pages"]) + tuple(s["pool"].shape[2:]), dtype=torch.uint8, device="cuda")
        s["to_table"], s["to_refs"] = torch.empty_like(s["table"]), zeros(s["to_pages"], dtype=torch.int32, device="cuda")
        s["status"] = zeros(1, dtype=torch.int32, device="cuda")
    if own:
        from paper_2509_21354_amd import binding as kb
        L = 1 if kind == "step" else c["L"]
        T = c["Tq"] if kind == "rotary" else c["T"]
        s["kb"] = kb
        s["shape"] = kb.make_shape(L=L, B=B, H=c["H"], H_kv=c["H_kv"], d=d, T=T, T_cap=T, C=32, N_cap=0, W=0, d_sum=32, d_g=64,
                                   dtype=kb.F32 if c["dtype"] == "f32" else kb.BF16)
        if kind == "rotary":
            s["axes"] = kb.make_rotary_axes((c["s0"], c["s1"], c["s2"]), kb.ROTARY_PAIRS if c["pairs"] else kb.ROTARY_HALVES)
        else:
            s["pages"] = kb.make_pages(c["page"], s["n_pages"], s["max_pages"])
        if kind == "attend":
            s["ws"] = kb.alloc_workspace(kb.page_workspace_bytes(kb.OP_PAGE_ATTENTION, s["shape"], s["pages"], c["Tq"]))
        if kind in ("beams", "step"):
            s["ws"] = kb.alloc_workspace(kb.page_workspace_bytes(kb.OP_PAGES_RESERVE, s["shape"], s["pages"], 0))
        if kind == "compact":
            s["to"] = kb.make_pages(c["page"], s["to_pages"], s["max_pages"])
            s["ws"] = kb.alloc_workspace(kb.page_workspace_bytes(kb.OP_PAGES_COMPACT, s["shape"], s["pages"], 0))
    return s


def run(state):
    return (_run_own if own else _run_plain)(state)


# ---- the library's calls ---------------------------------------------------------------------------------------------------

def _run_own(s):
    c, kb, sh = s["case"], s["kb"], s["shape"]
    kind = c["kind"]
    if kind == "rotary":
        kb.kvev_rotary(sh, s["axes"], s["freq"], s["pos"], c["Tq"], s["Q"], s["K"], s["Q_out"], s["K_out"], int(c["inverse"]))
        return {"Q": s["Q_out"], "K": s["K_out"]}
    pg = s["pages"]
    if kind == "rows":
        kb.kvev_page_append(sh, pg, s["K"], s["V"], c["Tn"], s["start"], s["n_new"], s["table"], s["pool"])
        kb.kvev_page_read(sh, pg, s["pool"], s["table"], s["start"], s["n_new"], c["Tn"], s["K_out"], s["V_out"])
        return {"K": s["K_out"], "V": s["V_out"]}
    if kind == "attend":
        kb.kvev_page_attention(sh, pg, s["Q"], c["Tq"], s["pool"], s["table"], s["length"], s["O"], s["ws"], s["first"], s["q_start"],
                               s.get("Kc"), s.get("Vc"), s.get("count"), c["k"])
        return {"O": s["O"]}
    if kind == "beams":
        n = s["dst"].numel()
        kb.kvev_pages_fork(sh, pg, s["src"], s["dst"], n, s["table"], s["length"], s["refs"], s["status"])
        kb.kvev_pages_reserve(sh, pg, s["n_new"], s["table"], s["length"], s["refs"], s["pool"], s["start"], s["status"], s["ws"])
        kb.kvev_page_read(sh, pg, s["pool"], s["table"], s["part_first"], s["part"], c["page"], s["K_out"], s["V_out"])
        out = {"K": s["K_out"], "V": s["V_out"], "table": s["table"].clone(), "length": s["length"].clone(), "refs": s["refs"].clone(),
               "start": s["start"], "status": s["status"]}
        kb.kvev_pages_trim(sh, pg, s["dst"], n, None, s["nil"], s["table"], s["length"], s["refs"])
        return dict(out, refs_after=s["refs"])
    if kind == "step":
        kb.kvev_pages_reserve(sh, pg, s["n_new"], s["table"], s["length"], s["refs"], s["pool"], s["start"], s["status"], s["ws"])
        out = {"table": s["table"].clone(), "length": s["length"].clone(), "refs": s["refs"].clone(), "start": s["start"], "status": s["status"]}
        kb.kvev_pages_trim(sh, pg, None, c["B"], None, s["kept"], s["table"], s["length"], s["refs"])
        return dict(out, refs_after=s["refs"])
    kb.kvev_pages_compact(sh, pg, s["pool"], s["table"], s["refs"], s["to"], s["to_pool"], s["to_table"], s["to_refs"], s["status"], s["ws"])
    return {"pool": s["to_pool"], "table": s["to_table"], "refs": s["to_refs"], "status": s["status"]}


# ---- the plain forms -------------------------------------------------------------------------------------------------------

def _run_plain(s):
    return {"rotary": _plain_rotary, "rows": _plain_rows, "attend": _plain_attend, "beams": _plain_beams, "step": _plain_step,
            "compact": _plain_compact}[s["case"]["kind"]](s)


def _plain_rotary(s):
    c = s["case"]
    P = s["freq"].numel()
    axis = torch.repeat_interleave(torch.arange(3, device="cuda"), torch.tensor((c["s0"], c["s1"], c["s2"]), device="cuda"), output_size=P)
    angle = s["pos"][axis].double() * s["freq"].double()[:, None, None]           # [P, B, T]; far positions want 64 bits
    cos, sin = (f(angle).float().permute(1, 2, 0)[None, :, None] for f in (torch.cos, torch.sin))
    if c["inverse"]:
        sin = -sin
    out = {}
    for name in "QK":
        x, y = s[name].float(), s[name + "_out"]
        a, b = (x[..., 0:2 * P:2], x[..., 1:2 * P:2]) if c["pairs"] else (x[..., :P], x[..., P:2 * P])
        u, v = a * cos - b * sin, a * sin + b * cos
        y[..., :2 * P] = (torch.stack((u, v), -1).flatten(-2) if c["pairs"] else torch.cat((u, v), -1)).to(y.dtype)
        y[..., 2 * P:] = s[name][..., 2 * P:]
        out[name] = y
    return out


def _places(s, first, n, width):
    """Page and row of the tokens first[b] .. first[b] + n[b] - 1 of every batch row, and whether there is one: [B, width]"""
    page = s["case"]["page"]
    i = torch.arange(width, device="cuda")
    at = first[:, None].long() + i
    ok = i < n[:, None]
    at = torch.where(ok, at, torch.zeros_like(at))
    return torch.gather(s["table"].long(), 1, at // page), at % page, ok


def _plain_read(s, first, n, width, K, V):
    c = s["case"]
    page, row, ok = _places(s, first, n, width)
    page = torch.where(ok, page, torch.zeros_like(page))
    d, out = c["d"], (K, V)
    for layer in range(c["L"]):
        groups = s["pool"][layer].unflatten(-1, (-1, 17 * d))
        g, r = row // 16, row % 16
        scale = groups[..., 16 * d:].unflatten(-1, (16, d // 32, 2))[page, :, g, r]
        for side in (0, 1):
            codes = groups[..., 8 * d * side:8 * d * (side + 1)].unflatten(-1, (16, d // 2))[page, :, g, r]
            x = _values(codes, scale[..., side]).permute(0, 2, 1, 3)
            out[side][layer] = torch.where(ok[:, None, :, None], x, out[side][layer].float()).to(K.dtype)


def _plain_rows(s):
    c = s["case"]
    new = s["n_new"].long()
    total = sum(_new_tokens(c))
    b = torch.repeat_interleave(torch.arange(c["B"], device="cuda"), new, output_size=total)      # row and token of each new one
    i = torch.arange(total, device="cuda") - (torch.cumsum(new, 0) - new)[b]
    at = s["start"].long()[b] + i
    page = s["table"].long()[b, at // c["page"]]
    for layer in range(c["L"]):
        _store(s["pool"], layer, page, at % c["page"], s["K"][layer][b, :, i], s["V"][layer][b, :, i])
    _plain_read(s, s["start"], s["n_new"], c["Tn"], s["K_out"], s["V_out"])
    return {"K": s["K_out"], "V": s["V_out"]}


def _plain_attend(s):
    c = s["case"]
    d, page, Tq, H, Hkv, G = c["d"], c["page"], c["Tq"], c["H"], c["H_kv"], c["H"] // c["H_kv"]
    T = s["max_pages"] * page
    t = torch.arange(T, device="cuda")
    step = max(1, (1 << 28) // max(Hkv * T * d, H * Tq * T))
    scale = 1.0 / math.sqrt(d)
    for b0 in range(0, c["B"], step):
        rows = slice(b0, min(c["B"], b0 + step))
        seen = t < s["length"][rows, None]
        if s["first"] is not None:
            seen = seen & (t >= s["first"][rows, None])
        seen = seen[:, None, :].expand(-1, Tq, -1)
        if c["causal"]:
            seen = seen & (t <= (s["q_start"][rows, None] + torch.arange(Tq, device="cuda"))[..., None])
        held = s["table"][rows].clamp(min=0).long()
        n = held.shape[0]
        for layer in range(c["L"]):
            K, V = _rows(s["pool"][layer][held], d)                      # [n, pages, H_kv, page, d]
            K, V = (x.transpose(1, 2).reshape(n, Hkv, T, d) for x in (K, V))
            mask = seen[:, None, None].expand(n, Hkv, G, Tq, T).reshape(n, Hkv, G * Tq, T)
            if c["k"]:
                K, V = torch.cat((s["Kc"][layer, rows].float(), K), 2), torch.cat((s["Vc"][layer, rows].float(), V), 2)
                kept = torch.arange(c["k"], device="cuda") < s["count"][layer, rows][..., None]
                mask = torch.cat((kept[:, :, None].expand(n, Hkv, G * Tq, c["k"]), mask), 3)
            V = torch.where(mask.any(2)[..., None], V, torch.zeros_like(V))
            q = s["Q"][layer, rows].float().reshape(n, Hkv, G * Tq, d) * scale
            x = torch.matmul(q, K.transpose(2, 3).contiguous()).masked_fill_(~mask, float("-inf"))
            top = x.amax(-1, keepdim=True).clamp_(min=-1e30)
            p = torch.exp(x - top)
            o = torch.matmul(p, V) / p.sum(-1, keepdim=True).clamp_(min=1e-30)
            s["O"][layer, rows] = o.reshape(n, H, Tq, d).to(s["O"].dtype)
    return {"O": s["O"]}


def _plain_reserve(s, table, length, refs):
    """Room for n_new tokens in every row: (table, length, refs, start, status), and the pages to copy as (from, to, wanted)."""
    page = s["case"]["page"]
    n_new, n_pages, width = s["n_new"].clamp(min=0).long(), refs.numel(), table.shape[1]
    old = length.long()
    new = old + n_new
    have, want = (old + page - 1) // page, (new + page - 1) // page
    last = torch.gather(table, 1, (old // page).clamp(max=width - 1)[:, None]).squeeze(1).long()
    cow = ((old % page != 0) & (n_new > 0) & (refs[last.clamp(min=0)] > 1)).long()
    need = want - have + cow
    at = torch.cumsum(need, 0) - need
    free = torch.argsort((refs > 0).int(), stable=True)
    enough = need.sum() <= (refs == 0).sum()
    j = torch.arange(width, device="cuda")
    fresh = (j >= have[:, None]) & (j < want[:, None])
    rank = at[:, None] + cow[:, None] + j - have[:, None]
    got = free[rank.clamp(0, n_pages - 1)].to(torch.int32)
    here = (cow > 0)[:, None] & (j == (old // page)[:, None])
    to = free[at.clamp(0, n_pages - 1)]
    after = torch.where(fresh, got, torch.where(here, to[:, None].to(torch.int32), table))
    after = torch.where(enough, after, table)
    used = refs.clone()
    used.index_add_(0, got.flatten().long(), (fresh & enough).flatten().int())
    used.index_add_(0, to, ((cow > 0) & enough).int())
    used.index_add_(0, last.clamp(min=0), -((cow > 0) & enough).int())
    start = torch.where(enough, old, torch.full_like(old, -1)).to(torch.int32)
    status = torch.where(enough, 0, 1).to(torch.int32).reshape(1)
    return after, torch.where(enough, new, old).to(torch.int32), used, start, status, (last, to, (cow > 0) & enough)


def _plain_beams(s):
    table, length, refs = s["table"].clone(), s["length"].clone(), s["refs"].clone()
    src, dst = s["src"].long(), s["dst"].long()
    table[dst], length[dst] = table[src], length[src]
    shared = table[dst]
    refs.index_add_(0, shared.clamp(min=0).flatten().long(), (shared >= 0).flatten().int())
    table, length, refs, start, status, (a, b, wanted) = _plain_reserve(s, table, length, refs)
    b = torch.where(wanted, b, a.clamp(min=0))
    s["pool"][:, b[dst]] = s["pool"][:, a[dst].clamp(min=0)]
    _plain_read(dict(s, table=table), s["part_first"], s["part"], s["case"]["page"], s["K_out"], s["V_out"])
    after = refs.clone()
    given = table[dst]
    after.index_add_(0, given.clamp(min=0).flatten().long(), -(given >= 0).flatten().int())
    return {"K": s["K_out"], "V": s["V_out"], "table": table, "length": length, "refs": refs, "start": start, "status": status, "refs_after": after}


def _plain_step(s):
    table, length, refs, start, status, _ = _plain_reserve(s, s["table"], s["length"], s["refs"])
    j = torch.arange(table.shape[1], device="cuda")
    gone = (j >= ((s["kept"] + s["case"]["page"] - 1) // s["case"]["page"])[:, None]) & (table >= 0)
    after = refs.clone()
    after.index_add_(0, table.clamp(min=0).flatten().long(), -gone.flatten().int())
    return {"table": table, "length": length, "refs": refs, "start": start, "status": status, "refs_after": after}


def _plain_compact(s):
    used = s["refs"] > 0
    rank = torch.cumsum(used.int(), 0) - 1
    n = s["to_pages"]
    order = torch.argsort((~used).int(), stable=True)[:n]
    live = torch.arange(n, device="cuda") < used.sum()
    for layer in range(s["case"]["L"]):
        s["to_pool"][layer] = torch.where(live[:, None, None], s["pool"][layer][order], s["to_pool"][layer])
    s["to_refs"].copy_(torch.where(live, s["refs"][order], torch.zeros_like(s["to_refs"])))
    s["to_table"].copy_(torch.where(s["table"] >= 0, rank[s["table"].clamp(min=0).long()].to(torch.int32), s["table"]))
    return {"pool": s["to_pool"], "table": s["to_table"], "refs": s["to_refs"], "status": s["status"]}


# ---- in 64 bits, from the definitions --------------------------------------------------------------------------------------

def exact(case, seed):
    c, kind = case, case["kind"]
    if kind in ("step", "compact"):
        return None                                    # whole numbers alone
    if kind == "attend" and c["L"] * c["B"] > 700:
        return None
    s = _make(case, seed)
    if kind == "rotary":
        return {n: _exact_rotary(c, s, s[n]) for n in "QK"}
    if kind == "rows":
        out = {}
        for n in "KV":
            ok = torch.arange(c["Tn"], device="cuda") < s["n_new"][:, None]
            out[n] = torch.where(ok[None, :, None, :, None], _exact_rounded(s[n]), torch.zeros((), dtype=torch.float64, device="cuda"))
        return out
    if kind == "attend":
        return {"O": _exact_attend(c, s)}
    K, V = (torch.zeros(c["L"], c["B"], c["H_kv"], c["page"], c["d"], dtype=torch.float64, device="cuda") for _ in range(2))
    for x, y in zip(s["dst"].tolist(), s["src"].tolist()):
        n = int(s["length"][y])
        if n % c["page"]:
            k, v = _exact_page(s["pool"][:, int(s["table"][y, n // c["page"]])], c["d"])
            K[:, x, :, :n % c["page"]], V[:, x, :, :n % c["page"]] = k[..., :n % c["page"], :], v[..., :n % c["page"], :]
    return {"K": K, "V": V, "table": None, "length": None, "refs": None, "start": None, "status": None, "refs_after": None}


def _exact_rotary(c, s, x):
    y = x.double().clone()
    j0 = 0
    P = s["freq"].numel()
    for axis, width in enumerate((c["s0"], c["s1"], c["s2"])):
        for j in range(j0, j0 + width):
            turn = torch.polar(torch.ones((), dtype=torch.float64, device="cuda"), s["pos"][axis].double() * s["freq"][j].double())[None, :, None]
            p, q = (2 * j, 2 * j + 1) if c["pairs"] else (j, j + P)
            z = torch.complex(y[..., p], y[..., q]) * (turn.conj() if c["inverse"] else turn)
            y[..., p], y[..., q] = z.real, z.imag
        j0 += width
    return y


def _exact_rounded(x):
    """The value that the 4-bit block of each element stands for: nearest of the sixteen, the even code where two are as near."""
    blk = x.double().unflatten(-1, (-1, 32))
    top = blk.abs().amax(-1, keepdim=True)
    e = torch.ceil(torch.log2(torch.clamp(top / 7.0, min=2.0 ** -125)))
    e = torch.where(top > 7.0 * torch.exp2(e), e + 1, e)              # (the logarithm rounds)
    e = torch.where(top <= 7.0 * torch.exp2(e - 1), e - 1, e).clamp(min=-125)
    y = (blk / torch.exp2(e)).abs()
    low = torch.clamp(torch.floor(torch.log2(torch.clamp(y, min=1.0))), max=2.0)
    grid = torch.exp2(low - 1.0)                                     # spacing of the codes there: 1/2, 1/2, 1, 2
    return (torch.clamp(torch.round(y / grid) * grid, max=6.0) * torch.exp2(e) * torch.sign(blk)).flatten(-2)


def _exact_page(b, d):
    """Bytes [..., page bytes] -> keys and values [..., tokens, d] in 64 bits"""
    b = b.unflatten(-1, (-1, 17 * d)).long()
    sc = torch.exp2((b[..., 16 * d:] - 127).double()).reshape(*b.shape[:-1], 16, d // 32, 2)
    out = []
    for side in (0, 1):
        by = b[..., side * 8 * d:(side + 1) * 8 * d]
        v = torch.empty(*by.shape, 2, dtype=torch.float64, device=by.device)
        for half in (0, 1):
            n = (by >> (4 * half)) & 15
            exponent, mantissa, sign = (n >> 1) & 3, n & 1, 1 - 2 * (n >> 3)
            v[..., half] = sign * torch.where(exponent == 0, 0.5 * mantissa, (1.0 + 0.5 * mantissa) * torch.exp2(exponent - 1.0))
        v = v.reshape(*by.shape[:-1], 16, d // 32, 32) * sc[..., side, None]
        out.append(v.reshape(*by.shape[:-2], -1, d))
    return out


def _exact_attend(c, s):
    G, page, Tq, d = c["H"] // c["H_kv"], c["page"], c["Tq"], c["d"]
    out = torch.zeros(c["L"], c["B"], c["H"], Tq, d, dtype=torch.float64, device="cuda")
    first = s["first"].tolist() if s["first"] is not None else [0] * c["B"]
    for b, n in enumerate(_lengths(c)):
        p0 = first[b] // page
        ids = s["table"][b, p0:_pages_of(n, page)].long()
        tok = torch.arange(first[b], n, device="cuda")
        hide = None
        if c["causal"]:
            hide = tok[None, :] > (n - Tq + torch.arange(Tq, device="cuda"))[:, None]
        for layer in range(c["L"]):
            k, v = _exact_page(s["pool"][layer, ids], d)             # [pages, H_kv, page, d]
            k, v = (x.transpose(0, 1).reshape(c["H_kv"], -1, d)[:, first[b] - p0 * page:n - p0 * page] for x in (k, v))
            for h in range(c["H_kv"]):
                q = s["Q"][layer, b, h * G:(h + 1) * G].double()
                a = torch.matmul(q.reshape(G * Tq, d), k[h].t()).reshape(G, Tq, -1) / math.sqrt(d)
                if hide is not None:
                    a = a.masked_fill(hide, float("-inf"))
                vals = v[h]
                if c["k"]:
                    m = int(s["count"][layer, b, h])
                    a = torch.cat((a, torch.matmul(q, s["Kc"][layer, b, h, :m].double().t()) / math.sqrt(d)), -1)
                    vals = torch.cat((vals, s["Vc"][layer, b, h, :m].double()), 0)
                w = torch.softmax(a, -1)
                out[layer, b, h * G:(h + 1) * G] = torch.matmul(w.reshape(G * Tq, -1), vals).reshape(G, Tq, d)
    return out
