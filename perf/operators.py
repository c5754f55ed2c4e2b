"""Timed work of the paged KV cache: the operators between a layer's QKV and O
projections, as a serving step calls them.

Three kinds of case: "map" builds a step's block tables and slot maps from
request lengths; "store" normalises and rotates queries and keys and writes
keys and values into cache blocks; "attn" attends one new token a row over the
blocks.  listed() names twelve cases, draw() gives more of the same ranges.

Heads are those of the hidden-4096 and hidden-8192 layer sets (32 or 64 query
and 8 key/value heads of 128) in the listed cases, and other layouts among the
drawn ones.  `run` computes the operators from elementary torch operations in
32 bits, or, where `own` is set, calls the library.

Cache block: K as [kv_heads][row bytes / 64][tokens][64 bytes], then V as
[kv_heads][tokens][head_dim].
"""
import math

import torch

own = False

TYPES = {"fp16": torch.float16, "bf16": torch.bfloat16, "e4m3": torch.float8_e4m3fn}
SIZES = {"fp16": 2, "bf16": 2, "e4m3": 1}


def listed():
    return [
        # a small decode batch: launch and host latency
        {"name": "map_decode_8", "kind": "map", "requests": 8, "new": 1, "ctx": 2000, "tokens": 16,
         "cols": 256, "rows": 8},
        # the largest captured decode batch, padded with idle requests
        {"name": "map_decode_256", "kind": "map", "requests": 256, "new": 1, "ctx": 6000,
         "tokens": 16, "cols": 512, "rows": 256},
        # a burst of prompts admitted at once beside running requests
        {"name": "map_prefill_burst", "kind": "map", "requests": 201, "new": 1100, "ctx": 900,
         "tokens": 32, "cols": 256, "rows": 131072},
        # one user, one token a step
        {"name": "store_decode_1", "kind": "store", "rows": 1, "heads": 32, "kv_heads": 8, "dim": 128,
         "rot": 128, "pairs": "half", "norm": True, "dtype": "fp16", "cache": "fp16", "tokens": 16},
        # a full decode batch of the larger model, no head norms
        {"name": "store_decode_256_bf16", "kind": "store", "rows": 256, "heads": 64, "kv_heads": 8,
         "dim": 128, "rot": 128, "pairs": "half", "norm": False, "dtype": "bf16", "cache": "bf16",
         "tokens": 16},
        # a prompt of ragged length into an 8-bit cache, half of each head rotated in place-pairs
        {"name": "store_prefill_1531_e4m3", "kind": "store", "rows": 1531, "heads": 32, "kv_heads": 8,
         "dim": 128, "rot": 64, "pairs": "adjacent", "norm": True, "dtype": "fp16", "cache": "e4m3",
         "tokens": 32},
        # a long prompt, or several
        {"name": "store_prefill_8192", "kind": "store", "rows": 8192, "heads": 32, "kv_heads": 8,
         "dim": 128, "rot": 128, "pairs": "half", "norm": True, "dtype": "fp16", "cache": "fp16",
         "tokens": 16},
        # one user, a short conversation: latency
        {"name": "attn_1_short", "kind": "attn", "rows": 1, "longest": 777, "shape": "even",
         "heads": 32, "kv_heads": 8, "dim": 128, "dtype": "fp16", "cache": "fp16", "tokens": 16,
         "window": 0, "spare": 0},
        # an ordinary batch of mixed lengths, two rows of it idle
        {"name": "attn_32_mixed", "kind": "attn", "rows": 34, "longest": 4096, "shape": "mixed",
         "heads": 32, "kv_heads": 8, "dim": 128, "dtype": "fp16", "cache": "fp16", "tokens": 16,
         "window": 0, "spare": 0},
        # the largest captured batch of the larger model, short lengths
        {"name": "attn_256_bf16", "kind": "attn", "rows": 256, "longest": 600, "shape": "mixed",
         "heads": 64, "kv_heads": 8, "dim": 128, "dtype": "bf16", "cache": "bf16", "tokens": 32,
         "window": 0, "spare": 0},
        # long documents in an 8-bit cache
        {"name": "attn_16_long_e4m3", "kind": "attn", "rows": 16, "longest": 30011, "shape": "even",
         "heads": 32, "kv_heads": 8, "dim": 128, "dtype": "fp16", "cache": "e4m3", "tokens": 64,
         "window": 0, "spare": 0},
        # one very long request among short ones, blocks spread over more than 4 GiB of the pool:
        # the largest
        {"name": "attn_1_long_among_16", "kind": "attn", "rows": 17, "longest": 131000,
         "shape": "one_long", "heads": 32, "kv_heads": 8, "dim": 128, "dtype": "fp16",
         "cache": "fp16", "tokens": 16, "window": 0, "spare": 80000},
    ]


def _log(rng, lo, hi):
    """A whole number in lo .. hi, spread over the logarithm."""
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    kind = rng.choice(("map", "store", "attn", "attn"))
    tokens = rng.choice((16, 16, 32, 64, 128, 256))
    if kind == "map":
        requests = _log(rng, 1, 2000)
        new = rng.choice((1, 1, _log(rng, 2, 2000)))
        new = max(1, min(new, 200000 // requests))
        ctx = _log(rng, 1, 16000)
        return {"kind": "map", "requests": requests, "new": new, "ctx": ctx, "tokens": tokens,
                "cols": -(-(ctx + new) // tokens) + rng.randrange(9),
                "rows": requests * new + rng.randrange(70)}
    dim = rng.choice((64, 96, 128, 128, 128, 192, 256))
    kv_heads = rng.choice((1, 2, 3, 4, 8, 8, 16))
    group = rng.choice((1, 2, 4, 5, 8, 16, 24))
    cache = rng.choice(("fp16", "bf16", "e4m3"))
    if cache == "e4m3" and dim == 96:
        dim = 128
    dtype = cache if cache != "e4m3" else rng.choice(("fp16", "bf16"))
    case = {"kind": kind, "heads": kv_heads * group, "kv_heads": kv_heads, "dim": dim,
            "dtype": dtype, "cache": cache, "tokens": tokens}
    if kind == "store":
        most = max(1, 8192 * 48 * 128 // ((group + 2) * kv_heads * dim))
        case.update(rows=_log(rng, 1, min(20000, most)), rot=rng.choice((dim, dim, dim // 2)),
                    pairs=rng.choice(("half", "adjacent")), norm=rng.random() < 0.6)
        return case
    # tokens of cache whose bytes the largest listed case allows, kept below it
    shape = rng.choice(("even", "mixed", "one_long"))
    rows = _log(rng, 1, 300)
    most = 120000 * 8 * 128 * 2 // (kv_heads * dim * SIZES[cache])
    longest = _log(rng, 1, max(1, min(most // rows, 40000)))
    case.update(rows=rows, longest=longest, shape=shape, spare=rng.choice((0, 50)),
                window=rng.choice((0, 0, _log(rng, 1, 4096))))
    return case


# ---- inputs -----------------------------------------------------------------------


def _gen(seed, part):
    g = torch.Generator(device="cuda")
    g.manual_seed(1000 * int(seed) + part)
    return g


def _ints(lo, hi, n, g):
    """int32 [n], uniform in lo .. hi."""
    return torch.randint(lo, hi + 1, (n,), generator=g, device="cuda", dtype=torch.int32)


def _block_values(case):
    """Values of one cache block: K and V."""
    return 2 * case["kv_heads"] * case["tokens"] * case["dim"]


def _random_pool(case, blocks, g):
    """Bytes of `blocks` cache blocks of N(0, 1) values."""
    n = blocks * _block_values(case)
    if case["cache"] != "e4m3":
        pool = torch.empty(n, dtype=TYPES[case["cache"]], device="cuda").normal_(generator=g)
    else:
        pool = torch.empty(n, dtype=torch.float16, device="cuda").normal_(generator=g)
        pool = pool.to(torch.float8_e4m3fn)
    return pool.view(torch.uint8)


def _scales(case):
    """Scales of an 8-bit cache's K and V (1 for the 16-bit types)."""
    return (0.0625, 0.125) if case["cache"] == "e4m3" else (1.0, 1.0)


def _prepare_map(case, seed):
    g = _gen(seed, 1)
    requests, tokens = case["requests"], case["tokens"]
    ctx = _ints(case["ctx"] // 4, case["ctx"], requests, g)
    if case["new"] == 1:  # a decode step; a few slots of the batch are idle
        new = (torch.rand(requests, generator=g, device="cuda") > 0.03).to(torch.int32)
    else:  # prompts, whole or in part, beside requests that decode
        new = _ints(case["new"] // 4, case["new"], requests, g).clamp_(min=1)
        ctx[::3] = 0
        new[1::3] = 1
    most = case["cols"] * tokens
    ctx = torch.minimum(ctx, most - new)
    blocks = requests * case["cols"]
    ids = torch.randperm(2 * blocks, generator=g, device="cuda")[:2 * blocks].to(torch.int32)
    table = ids[:blocks].reshape(requests, case["cols"]).clone()
    have = (ctx + tokens - 1) // tokens
    cols = torch.arange(case["cols"], device="cuda", dtype=torch.int32)
    table[cols >= have[:, None]] = -1
    return {"ctx": ctx, "new": new, "table": table, "fresh": ids[blocks:].contiguous()}


def _prepare_store(case, seed):
    g = _gen(seed, 1)
    rows, tokens, dtype = case["rows"], case["tokens"], TYPES[case["dtype"]]
    width = (case["heads"] + 2 * case["kv_heads"]) * case["dim"]
    state = {"qkv": torch.randn((rows, width), generator=g, device="cuda").to(dtype)}
    if rows <= 256:  # a decode step: every row is the next token of a request of its own
        blocks = 2 * rows
        block = torch.randperm(blocks, generator=g, device="cuda")[:rows]
        pos = _ints(0, 32767, rows, g)
        state["slot"] = block * tokens + pos % tokens
    else:  # one prompt from position 0, its blocks anywhere
        blocks = -(-rows // tokens)
        block = torch.randperm(blocks, generator=g, device="cuda")
        pos = torch.arange(rows, device="cuda", dtype=torch.int32)
        state["slot"] = block[(pos // tokens).long()] * tokens + pos % tokens
    state["pos"] = pos
    state["pool"] = _random_pool(case, blocks, g)
    half = case["rot"] // 2
    angle = torch.arange(32768, device="cuda", dtype=torch.float64)[:, None] * torch.exp(
        torch.arange(half, device="cuda", dtype=torch.float64) * (-math.log(1e6) / half))
    state["rope"] = torch.cat((angle.cos(), angle.sin()), 1).float()
    state["wq"] = state["wk"] = None
    if case["norm"]:
        for name in ("wq", "wk"):
            w = 1.0 + 0.1 * torch.randn(case["dim"], generator=g, device="cuda")
            state[name] = w.to(dtype)
    state["q"] = torch.empty((rows, case["heads"], case["dim"]), dtype=dtype, device="cuda")
    return state


def _lengths(case, g):
    rows, longest = case["rows"], case["longest"]
    if case["shape"] == "even":
        lens = _ints(max(1, longest - longest // 8), longest, rows, g)
    else:
        lens = _ints(0, longest if case["shape"] == "mixed" else max(1, longest // 64), rows, g)
        if case["shape"] == "mixed":
            lens[1::17] = 0  # idle rows of a captured batch
    lens[0] = longest
    return lens


def _prepare_attn(case, seed):
    g = _gen(seed, 1)
    rows, tokens, dtype = case["rows"], case["tokens"], TYPES[case["dtype"]]
    lens = _lengths(case, g)
    cols = -(-case["longest"] // tokens)
    need = (lens + tokens - 1) // tokens
    first = torch.cumsum(need, 0) - need
    blocks = int(need.sum()) + case["spare"]
    ids = torch.randperm(blocks, generator=g, device="cuda").to(torch.int32)
    col = torch.arange(cols, device="cuda")
    table = ids[(first[:, None] + col).clamp(max=blocks - 1)]
    table[col >= need[:, None]] = -1
    pool = _random_pool(case, blocks, g)
    # past a request's last token its block holds whatever was there: not always numbers
    kv = pool.view(TYPES[case["cache"]]).view(blocks, 2, -1)
    size = SIZES[case["cache"]]
    k = kv[:, 0].view(blocks, case["kv_heads"], case["dim"] * size // 64, tokens, 64 // size)
    v = kv[:, 1].view(blocks, case["kv_heads"], tokens, case["dim"])
    live = torch.nonzero(lens).flatten()
    last = table[live, (need[live] - 1).long()].long()
    past = torch.arange(tokens, device="cuda") > ((lens[live] - 1) % tokens)[:, None]
    at, t = torch.nonzero(past, as_tuple=True)
    nan = torch.full((), float("nan"), device="cuda")
    bits = {2: torch.int16, 1: torch.uint8}[size]
    nan = nan.to(TYPES[case["cache"]]).view(bits)
    k.view(bits)[last[at], :, :, t] = nan
    v.view(bits)[last[at], :, t] = nan
    shape = (rows, case["heads"], case["dim"])
    kscale = _scales(case)[0]
    return {"q": (torch.randn(shape, generator=g, device="cuda") * (1.5 / kscale)).to(dtype),
            "pool": pool, "table": table, "len": lens,
            "req": torch.arange(rows, device="cuda", dtype=torch.int32),
            "out": torch.empty(shape, dtype=dtype, device="cuda"),
            "lse": torch.empty((rows, case["heads"]), dtype=torch.float32, device="cuda")}


def prepare(case, seed):
    state = {"map": _prepare_map, "store": _prepare_store, "attn": _prepare_attn}[
        case["kind"]](case, seed)
    state["case"] = case
    return state


# ---- one pass: elementary operations -------------------------------------------------


def _plain_map(case, state):
    ctx, new, table = state["ctx"], state["new"], state["table"]
    tokens, rows, fresh = case["tokens"], case["rows"], state["fresh"]
    device = ctx.device
    have = (ctx + tokens - 1) // tokens
    need = (ctx + new + tokens - 1) // tokens - have
    base = torch.cumsum(need, 0) - need
    j = torch.arange(case["cols"], device=device) - have[:, None]
    at = base[:, None] + j
    got = torch.where(at < fresh.numel(), fresh[at.clamp(0, fresh.numel() - 1)], -1)
    table.copy_(torch.where((j >= 0) & (j < need[:, None]), got, table))
    zero = torch.zeros(1, dtype=torch.int64, device=device)
    start = torch.cat((zero, torch.cumsum(new, 0)))
    row = torch.arange(rows, device=device)
    live = row < start[-1]
    req = (torch.searchsorted(start, row, right=True) - 1).clamp(max=case["requests"] - 1)
    pos = torch.where(live, ctx[req] + row - start[req], 0)
    col = pos // tokens
    block = table[req, col.clamp(max=case["cols"] - 1)].long()
    good = live & (col < case["cols"]) & (block >= 0)
    slot = torch.where(good, block * tokens + pos % tokens, -1)
    i32 = torch.int32
    return [table, start.clamp(max=rows).to(i32), ctx + new,
            torch.stack((start[-1], need.sum())).to(i32), pos.to(i32), slot,
            torch.where(live, req, -1).to(i32), torch.where(live, pos + 1, 0).to(i32)]


def _normed(x, w):
    x = x.float()
    if w is None:
        return x
    return x * torch.rsqrt((x * x).mean(-1, keepdim=True) + 1e-6) * w.to(x.dtype)


def _rotated(x, cos, sin, case):
    rot = case["rot"]
    part = x[..., :rot]
    if case["pairs"] == "half":
        a, b = part[..., :rot // 2], part[..., rot // 2:]
        part = torch.cat((a * cos - b * sin, b * cos + a * sin), -1)
    else:
        a, b = part[..., 0::2], part[..., 1::2]
        part = torch.stack((a * cos - b * sin, b * cos + a * sin), -1).flatten(-2)
    return torch.cat((part, x[..., rot:]), -1)


def _coded(x, scale, case):
    """Values as the cache holds them."""
    if case["cache"] == "e4m3":
        x = (x / scale).clamp(-448.0, 448.0)
    return x.to(TYPES[case["cache"]])


def _views(case, pool):
    size = SIZES[case["cache"]]
    blocks = pool.numel() // (_block_values(case) * size)
    kv = pool.view(TYPES[case["cache"]]).view(blocks, 2, -1)
    k = kv[:, 0].view(blocks, case["kv_heads"], case["dim"] * size // 64, case["tokens"], 64 // size)
    return k, kv[:, 1].view(blocks, case["kv_heads"], case["tokens"], case["dim"])


def _plain_store(case, state):
    rows, heads, kv_heads, dim = case["rows"], case["heads"], case["kv_heads"], case["dim"]
    x = state["qkv"].view(rows, heads + 2 * kv_heads, dim)
    half = case["rot"] // 2
    rope = state["rope"][state["pos"].long()][:, None]
    cos, sin = rope[..., :half], rope[..., half:]
    q = _rotated(_normed(x[:, :heads], state["wq"]), cos, sin, case)
    k = _rotated(_normed(x[:, heads:heads + kv_heads], state["wk"]), cos, sin, case)
    v = x[:, heads + kv_heads:].float()
    kscale, vscale = _scales(case)
    kc, vc = _views(case, state["pool"])
    block, t = state["slot"] // case["tokens"], state["slot"] % case["tokens"]
    bits = torch.uint8 if case["cache"] == "e4m3" else torch.int16
    kc.view(bits)[block, :, :, t] = _coded(k, kscale, case).view(bits).view(
        rows, kv_heads, kc.shape[2], kc.shape[4])
    vc.view(bits)[block, :, t] = _coded(v, vscale, case).view(bits)
    state["q"].copy_(q)
    return [state["q"], state["pool"].view(TYPES[case["cache"]])]


def _plain_attn(case, state):
    rows, heads, kv_heads, dim = case["rows"], case["heads"], case["kv_heads"], case["dim"]
    kc, vc = _views(case, state["pool"])
    bits = torch.uint8 if case["cache"] == "e4m3" else torch.int16
    table = state["table"].long().clamp(min=0)
    kscale, vscale = _scales(case)
    k = kc.view(bits)[table].view(TYPES[case["cache"]]).float()  # rows, cols, heads, segment, t, e
    k = k.permute(0, 2, 3, 5, 1, 4).reshape(rows, kv_heads, dim, -1)
    q = state["q"].float().view(rows, kv_heads, heads // kv_heads, dim)
    s = torch.matmul(q, k) * (kscale / math.sqrt(dim))
    del k
    pos = torch.arange(s.shape[-1], device=s.device)
    lens = state["len"][:, None].long()
    live = pos < lens
    if case["window"]:
        live = live & (pos >= lens - case["window"])
    live = live[:, None, None]
    s = torch.where(live, s, float("-inf"))
    top = s.amax(-1, keepdim=True)
    top = torch.where(torch.isinf(top), 0.0, top)
    p = torch.exp(s - top)
    total = p.sum(-1, keepdim=True)
    v = vc.view(bits)[table].view(TYPES[case["cache"]]).float().permute(0, 2, 1, 3, 4)
    v = v.reshape(rows, kv_heads, -1, dim)
    v = torch.where(live[:, 0, :, :, None], v, 0.0)
    o = torch.matmul(p, v) / torch.where(total > 0, total, 1.0) * vscale
    state["out"].copy_(o.reshape(rows, heads, dim))
    state["lse"].copy_((top + torch.log(total)).reshape(rows, heads))
    return [state["out"], state["lse"]]


# ---- one pass: the library -------------------------------------------------------------


def _kept(case, state):
    """What a program keeps from call to call: descriptors, outputs, scratch."""
    if "kept" not in state:
        from paper_2609_34380_amd import dps

        if case["kind"] == "map":
            state["kept"] = dps.make_kv_map(case["requests"], case["rows"], state["ctx"].device)
        else:
            kscale, vscale = _scales(case)
            cache = dps.KvCache(state["pool"], case["tokens"], case["kv_heads"], case["dim"],
                                TYPES[case["cache"]], k_scale=kscale, v_scale=vscale)
            ws = None
            if case["kind"] == "attn":
                need = dps.attn_workspace_bytes(cache, case["rows"], case["heads"])
                ws = torch.empty(max(need, 256), dtype=torch.uint8, device="cuda")
            state["kept"] = (cache, ws)
    return state["kept"]


def _own(case, state):
    from paper_2609_34380_amd import dps

    kept = _kept(case, state)
    if case["kind"] == "map":
        m = dps.kv_map(state["ctx"], state["new"], state["fresh"], state["table"], case["tokens"],
                       out=kept)
        return [state["table"], m.q_start, m.seq_len, m.counts, m.pos, m.slot, m.req, m.kv_len]
    cache, ws = kept
    if case["kind"] == "store":
        dps.kv_store(state["qkv"], cache, state["slot"], case["heads"], pos=state["pos"],
                     rope=state["rope"], q_weight=state["wq"], k_weight=state["wk"], eps=1e-6,
                     adjacent=case["pairs"] == "adjacent", q_out=state["q"])
        return [state["q"], state["pool"].view(TYPES[case["cache"]])]
    dps.attn_decode(state["q"], cache, state["table"], state["len"], req=state["req"],
                    window=case["window"], out=state["out"], lse=state["lse"], workspace=ws)
    return [state["out"], state["lse"]]


def run(state):
    case = state["case"]
    if own:
        return _own(case, state)
    return {"map": _plain_map, "store": _plain_store, "attn": _plain_attn}[case["kind"]](case, state)


# ---- what a pass cannot do without, and what it has to give ------------------------------


def work(case):
    if case["kind"] == "map":
        requests, tokens = case["requests"], case["tokens"]
        live = requests if case["new"] == 1 else requests * case["new"] // 2
        blocks = live // tokens
        # lengths and last blocks in, new blocks in and out, 20 bytes a row and 8 a request out
        return {"bytes": 20 * requests + 8 * blocks + 20 * case["rows"], "flops": 0}
    heads, kv_heads, dim = case["heads"], case["kv_heads"], case["dim"]
    size = SIZES[case["cache"]]
    rows = case["rows"]
    if case["kind"] == "store":
        bytes_ = rows * dim * ((heads + 2 * kv_heads) * 2 + heads * 2 + 2 * kv_heads * size)
        bytes_ += rows * (case["rot"] * 4 + 12)
        return {"bytes": bytes_, "flops": rows * (heads + kv_heads) * dim * 7}
    longest = case["longest"]
    mean = {"even": longest * 15 / 16, "mixed": longest / 2, "one_long": longest / 128}[case["shape"]]
    most = case["window"] or longest
    tokens = min(longest, most) + (rows - 1) * min(mean, most)
    return {"bytes": int(tokens * 2 * kv_heads * dim * size + rows * heads * (4 * dim + 4)),
            "flops": int(4 * tokens * heads * dim)}


def _exact_store(case, state):
    rows, heads, kv_heads, dim = case["rows"], case["heads"], case["kv_heads"], case["dim"]
    half = case["rot"] // 2
    x = state["qkv"].double().reshape(rows, -1, dim)
    angle = state["rope"].double()[state["pos"].long()]
    turn = torch.complex(angle[:, :half], angle[:, half:])[:, None]

    def keyed(part, w):
        if w is not None:
            part = part / (part.square().sum(-1, keepdim=True) / dim + 1e-6).sqrt() * w.double()
        head, rest = part[..., :case["rot"]], part[..., case["rot"]:]
        if case["pairs"] == "half":
            z = torch.complex(head[..., :half].contiguous(), head[..., half:].contiguous()) * turn
            return torch.cat((z.real, z.imag, rest), -1)
        z = torch.view_as_complex(head.contiguous().reshape(rows, -1, half, 2)) * turn
        return torch.cat((torch.view_as_real(z).flatten(-2), rest), -1)

    q = keyed(x[:, :heads], state["wq"])
    k = keyed(x[:, heads:-kv_heads], state["wk"])
    v = x[:, -kv_heads:]
    kscale, vscale = _scales(case)
    if case["cache"] == "e4m3":
        k, v = (k / kscale).clamp(-448, 448), (v / vscale).clamp(-448, 448)
    pool = state["pool"].view(TYPES[case["cache"]]).double()
    # flat place of value (row, head, d) of K and of V
    size, tokens = SIZES[case["cache"]], case["tokens"]
    d = torch.arange(dim, device="cuda")
    h = torch.arange(kv_heads, device="cuda")[:, None]
    block = (state["slot"] // tokens * _block_values(case))[:, None, None]
    t = (state["slot"] % tokens)[:, None, None]
    seg = 64 // size
    pool[block + h * tokens * dim + d // seg * tokens * seg + t * seg + d % seg] = k
    pool[block + (kv_heads + h) * tokens * dim + t * dim + d] = v
    return [q, pool]


def _exact_attn(case, state):
    heads, kv_heads, dim = case["heads"], case["kv_heads"], case["dim"]
    kc, vc = _views(case, state["pool"])
    kscale, vscale = _scales(case)
    out = torch.zeros((case["rows"], heads, dim), dtype=torch.float64, device="cuda")
    lse = torch.full((case["rows"], heads), float("-inf"), dtype=torch.float64, device="cuda")
    for r, n in enumerate(state["len"].tolist()):
        if not n:
            continue
        first = max(0, n - case["window"]) if case["window"] else 0
        blocks = state["table"][r, : -(-n // case["tokens"])].long()
        k = kc[blocks].double().permute(1, 0, 3, 2, 4).reshape(kv_heads, -1, dim)[:, first:n]
        v = vc[blocks].double().permute(1, 0, 2, 3).reshape(kv_heads, -1, dim)[:, first:n]
        q = state["q"][r].double().reshape(kv_heads, -1, dim) * (kscale / math.sqrt(dim))
        for h in range(kv_heads):
            s = q[h] @ k[h].t().contiguous()
            z = torch.logsumexp(s, -1, keepdim=True)
            group = slice(h * q.shape[1], (h + 1) * q.shape[1])
            out[r, group] = torch.exp(s - z) @ v[h] * vscale
            lse[r, group] = z[:, 0]
    return [out, lse]


def exact(case, seed):
    if case["kind"] == "map":
        return None  # whole numbers
    state = prepare(case, seed)
    return (_exact_store if case["kind"] == "store" else _exact_attn)(case, state)
