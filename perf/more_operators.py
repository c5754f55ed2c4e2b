"""Timed work of sequences that branch: the operators of a serving step whose
requests share what they have in common, as beams and several answers to one prompt do.

Four kinds of case: "attn" attends one new token a row over the paged cache, rows of
a group over the blocks of a common prefix and then their own; "beam" picks
the next beams from logits over the vocabulary; "fork" gives every surviving
sequence the block table of its parent, with a block of its own to write into;
"move" compacts the cache: blocks to other places, and the tables after them.
listed() names twelve cases, draw() gives more of the same ranges.

`run` computes the operators from elementary torch operations (32 bits; the beams'
scores in 64, where two may lie closer than 32 can tell), or, where `own` is set, calls
the library.

Cache block: K as [kv_heads][row bytes / 64][tokens][64 bytes], then V as
[kv_heads][tokens][head_dim].
"""
import math

import torch

own = False

TYPES = {"fp16": torch.float16, "bf16": torch.bfloat16, "fp32": torch.float32,
         "e4m3": torch.float8_e4m3fn}
SIZES = {"fp16": 2, "bf16": 2, "fp32": 4, "e4m3": 1}
END = 2  # the token that ends a sequence


def listed():
    return [
        # four answers to one short prompt: latency
        {"name": "attn_4_answers", "kind": "attn", "rows": 4, "groups": 1, "shared": 992, "own": 40,
         "heads": 32, "kv_heads": 8, "dim": 128, "dtype": "fp16", "cache": "fp16", "tokens": 16},
        # an ordinary batch: several prompts of mixed lengths with a few answers each, two idle rows
        {"name": "attn_34_mixed", "kind": "attn", "rows": 34, "groups": 5, "shared": 3000, "own": 300,
         "heads": 32, "kv_heads": 8, "dim": 128, "dtype": "bf16", "cache": "bf16", "tokens": 32},
        # eight documents under eight beams each, in an 8-bit cache
        {"name": "attn_64_beams_e4m3", "kind": "attn", "rows": 64, "groups": 8, "shared": 12000,
         "own": 128, "heads": 32, "kv_heads": 8, "dim": 128, "dtype": "fp16", "cache": "e4m3",
         "tokens": 64},
        # the largest captured batch of the larger model under one long system prompt: the largest
        {"name": "attn_256_one_prompt", "kind": "attn", "rows": 256, "groups": 1, "shared": 16384,
         "own": 600, "heads": 64, "kv_heads": 8, "dim": 128, "dtype": "fp16", "cache": "fp16",
         "tokens": 16},
        # one request with four beams: latency
        {"name": "beam_1_by_4", "kind": "beam", "batch": 1, "beams": 4, "vocab": 32000, "keep": 4,
         "dtype": "fp16", "masked": False, "step": 5},
        # a batch of beams, twice as many candidates as beams, most tokens ruled out in some rows
        {"name": "beam_16_by_8", "kind": "beam", "batch": 16, "beams": 8, "vocab": 131072,
         "keep": 16, "dtype": "bf16", "masked": True, "step": 40},
        # many requests over a vocabulary of odd size, logits in 32 bits
        {"name": "beam_64_by_8_fp32", "kind": "beam", "batch": 64, "beams": 8, "vocab": 100003,
         "keep": 8, "dtype": "fp32", "masked": False, "step": 40},
        # the beams of one request: latency
        {"name": "fork_8", "kind": "fork", "requests": 8, "beams": 8, "longest": 2000, "tokens": 16,
         "cols": 256, "kv_heads": 8, "dim": 128, "cache": "fp16"},
        # the largest captured batch, beams of 32 requests
        {"name": "fork_256", "kind": "fork", "requests": 256, "beams": 8, "longest": 4000,
         "tokens": 16, "cols": 512, "kv_heads": 8, "dim": 128, "cache": "fp16"},
        # many rows with long tables, small blocks of an 8-bit cache
        {"name": "fork_1000_wide", "kind": "fork", "requests": 1000, "beams": 20, "longest": 20000,
         "tokens": 16, "cols": 1300, "kv_heads": 2, "dim": 64, "cache": "e4m3"},
        # a few blocks out of the way of one residual
        {"name": "move_40", "kind": "move", "moves": 40, "blocks": 800, "requests": 32, "cols": 64,
         "tokens": 16, "kv_heads": 8, "dim": 128, "cache": "fp16"},
        # a fragmented cache compacted at once
        {"name": "move_3000", "kind": "move", "moves": 3000, "blocks": 9000, "requests": 256,
         "cols": 512, "tokens": 16, "kv_heads": 8, "dim": 128, "cache": "bf16"},
    ]


def _log(rng, lo, hi):
    """A whole number in lo .. hi, spread over the logarithm."""
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    kind = rng.choice(("attn", "attn", "beam", "fork", "move"))
    tokens = rng.choice((16, 16, 32, 64, 128, 256))
    if kind == "beam":
        beams = _log(rng, 1, 40)
        vocab = _log(rng, 50, 200000)
        batch = _log(rng, 1, max(1, min(100, 40000000 // (beams * vocab))))
        return {"kind": kind, "batch": batch, "beams": beams, "vocab": vocab,
                "keep": rng.choice((beams, 2 * beams, rng.randint(1, 64))),
                "dtype": rng.choice(("fp16", "bf16", "fp32")), "masked": rng.random() < 0.4,
                "step": rng.choice((0, 40))}
    dim = rng.choice((64, 96, 128, 128, 128, 192, 256))
    kv_heads = rng.choice((1, 2, 3, 4, 8, 8, 16))
    cache = rng.choice(("fp16", "bf16", "e4m3"))
    if cache == "e4m3" and dim == 96:
        dim = 128
    case = {"kind": kind, "kv_heads": kv_heads, "dim": dim, "cache": cache, "tokens": tokens}
    if kind == "attn":
        group = rng.choice((1, 2, 4, 5, 8, 16, 24))
        rows = _log(rng, 1, 300)
        # below the largest listed case: its products, and a cache of 1 GB
        most = 16000 * 256 * 64 * 128 // (rows * kv_heads * group * dim)
        most = min(most, 250000 * 8 * 128 * 2 // (kv_heads * dim * SIZES[cache]) // rows, 60000)
        shared = _log(rng, 1, max(1, most))
        case.update(rows=rows, groups=_log(rng, 1, max(1, rows // 2)), shared=shared,
                    own=_log(rng, 1, max(1, min(2000, most))), heads=kv_heads * group,
                    dtype=cache if cache != "e4m3" else rng.choice(("fp16", "bf16")))
        return case
    block = 2 * kv_heads * tokens * dim * SIZES[cache]
    if kind == "fork":
        beams = _log(rng, 1, 32)
        requests = beams * _log(rng, 1, max(1, 600 // beams))
        # distinct blocks in 500 MB: a prompt's, and two for each row
        most = max(3, 500000000 // block - 4 * requests) * beams // requests
        longest = _log(rng, 2, max(2, min(30000, most * tokens)))
        case.update(requests=requests, beams=beams, longest=longest,
                    cols=-(-longest // tokens) + rng.randrange(9))
        return case
    blocks = _log(rng, 16, max(17, 600000000 // block))
    requests = _log(rng, 1, 300)
    case.update(blocks=blocks, moves=_log(rng, 1, max(1, blocks // 3)), requests=requests,
                cols=rng.randint(1, 600))
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


def _views(case, pool):
    """K [blocks][kv_heads][segments][tokens][64 bytes] and V [blocks][kv_heads][tokens][dim]
    as whole numbers of the elements' size."""
    size = SIZES[case["cache"]]
    blocks = pool.numel() // (_block_values(case) * size)
    bits = torch.int16 if size == 2 else torch.uint8
    kv = pool.view(bits).view(blocks, 2, -1)
    k = kv[:, 0].view(blocks, case["kv_heads"], case["dim"] * size // 64, case["tokens"], 64 // size)
    return k, kv[:, 1].view(blocks, case["kv_heads"], case["tokens"], case["dim"])


def _prepare_attn(case, seed):
    g = _gen(seed, 1)
    rows, groups, tokens, dtype = case["rows"], case["groups"], case["tokens"], TYPES[case["dtype"]]
    # groups of uneven size side by side; in larger batches a few rows after the last are in none
    alone = rows // 16 if rows > groups + 8 else 0
    inside = rows - alone
    cuts = torch.randperm(inside - 1, generator=g, device="cuda")[:groups - 1].sort().values + 1
    group_start = torch.cat((torch.zeros(1, device="cuda", dtype=torch.int64), cuts,
                             torch.full((1,), inside, device="cuda"))).to(torch.int32)
    # rows share whole blocks
    shared = _ints(case["shared"] // 2, case["shared"], groups, g) // tokens * tokens
    shared[0] = case["shared"] // tokens * tokens
    row = torch.arange(rows, device="cuda")
    of = (torch.searchsorted(group_start, row, right=True) - 1).clamp(max=groups - 1)
    member = row < inside
    start = torch.where(member, shared[of], 0)
    lens = start + _ints(1, case["own"], rows, g)
    lens[1::17] = 0  # idle rows of a captured batch
    lens[0] = start[0] + case["own"]
    cols = -(-(case["shared"] + case["own"]) // tokens)
    # block ids: the prompts', then each row's own
    before = start // tokens
    mine = ((lens + tokens - 1) // tokens - before).clamp(min=0)
    prompt = shared // tokens
    prompt_first = torch.cumsum(prompt, 0) - prompt
    prompts = int(prompt.sum())
    first = prompts + torch.cumsum(mine, 0) - mine
    blocks = prompts + int(mine.sum()) + 3
    ids = torch.randperm(blocks, generator=g, device="cuda").to(torch.int32)
    col = torch.arange(cols, device="cuda")
    at = torch.where(col < before[:, None], prompt_first[of][:, None] + col,
                     first[:, None] + col - before[:, None])
    table = ids[at.clamp(max=blocks - 1)]
    table[col >= ((lens + tokens - 1) // tokens)[:, None]] = -1
    pool = _random_pool(case, blocks, g)
    # past a request's last token its block holds whatever was there: not always numbers
    k, v = _views(case, pool)
    live = torch.nonzero(lens).flatten()
    last = table[live, ((lens[live] - 1) // tokens).long()].long()
    past = torch.arange(tokens, device="cuda") > ((lens[live] - 1) % tokens)[:, None]
    b, t = torch.nonzero(past & (mine[live] > 0)[:, None], as_tuple=True)
    nan = {"fp16": 0x7E00, "bf16": 0x7FC0, "e4m3": 0x7F}[case["cache"]]
    k[last[b], :, :, t] = nan
    v[last[b], :, t] = nan
    shape = (rows, case["heads"], case["dim"])
    kscale = _scales(case)[0]
    return {"q": (torch.randn(shape, generator=g, device="cuda") * (1.5 / kscale)).to(dtype),
            "pool": pool, "table": table, "len": lens, "group_start": group_start,
            "shared": shared, "most": int((group_start[1:] - group_start[:-1]).max()),
            "out": torch.empty(shape, dtype=dtype, device="cuda"),
            "lse": torch.empty((rows, case["heads"]), dtype=torch.float32, device="cuda")}


def _prepare_beam(case, seed):
    g = _gen(seed, 1)
    rows, vocab = case["batch"] * case["beams"], case["vocab"]
    logits = (torch.randn((rows, vocab), generator=g, device="cuda") * 2.5).to(TYPES[case["dtype"]])
    if case["masked"]:  # a grammar leaves some rows few tokens; elsewhere the type's lowest value does it
        few = torch.rand((rows, vocab), generator=g, device="cuda") * vocab < 5
        kind = torch.randint(0, 4, (rows, 1), generator=g, device="cuda")
        logits.masked_fill_(~few & (kind == 0), float("-inf"))
        logits.masked_fill_(~few & (kind == 1), torch.finfo(logits.dtype).min)
    score = torch.zeros(rows, device="cuda")
    done = torch.zeros(rows, dtype=torch.uint8, device="cuda")
    if case["step"]:  # beams in the order of their scores, some of them at their end
        score = -torch.rand((case["batch"], case["beams"]), generator=g, device="cuda") * 8
        score = score.sort(-1, descending=True).values.flatten() - 0.7 * case["step"]
        done = (torch.rand(rows, generator=g, device="cuda") < 0.1).to(torch.uint8)
    else:  # the first step: all beams are alike, one of them counts
        score.view(case["batch"], case["beams"])[:, 1:] = float("-inf")
    return {"logits": logits, "score": score, "done": done}


def _prepare_fork(case, seed):
    g = _gen(seed, 1)
    requests, beams, tokens, cols = (case[n] for n in ("requests", "beams", "tokens", "cols"))
    prompts = requests // beams
    # beams of one prompt are equally long; they share all of it but the last two blocks
    lens = _ints(max(1, case["longest"] // 4), case["longest"], prompts, g)
    lens[0] = case["longest"]
    lens = lens.repeat_interleave(beams)
    have = (lens + tokens - 1) // tokens
    common = (have - 2).clamp(min=0)
    prompt = common.view(prompts, beams)[:, 0]
    prompt_first = (torch.cumsum(prompt, 0) - prompt).repeat_interleave(beams)
    total = int(prompt.sum())
    mine = have - common
    first = total + torch.cumsum(mine, 0) - mine
    used = total + int(mine.sum())
    blocks = prompts * -(-case["longest"] // tokens) + 4 * requests  # whatever the lengths are
    ids = torch.randperm(blocks, generator=g, device="cuda").to(torch.int32)
    col = torch.arange(cols, device="cuda")
    at = torch.where(col < common[:, None], prompt_first[:, None] + col,
                     first[:, None] + col - common[:, None])
    table = ids[at.clamp(max=blocks - 1)]
    table[col >= have[:, None]] = -1
    # a beam goes on from one of its prompt's beams; a few requests have ended
    parent = torch.randint(0, beams, (requests,), generator=g, device="cuda")
    parent = (parent + torch.arange(requests, device="cuda") // beams * beams).to(torch.int32)
    parent[torch.rand(requests, generator=g, device="cuda") < 0.03] = -1
    return {"parent": parent, "len": lens, "table": table, "blocks": blocks,
            "fresh": ids[used:used + requests].contiguous(), "pool": _random_pool(case, blocks, g)}


def _prepare_move(case, seed):
    g = _gen(seed, 1)
    blocks, moves = case["blocks"], case["moves"]
    ids = torch.randperm(blocks, generator=g, device="cuda")
    # block ids of the tables, some shared; those that move, ascending, and free places
    held = ids[:blocks - moves]
    src = held[:moves].sort().values.to(torch.int32)
    dst = ids[blocks - moves:].sort().values.to(torch.int32)
    n = case["requests"] * case["cols"]
    pick = torch.randint(0, held.numel(), (n,), generator=g, device="cuda")
    table = held[pick].to(torch.int32).view(case["requests"], case["cols"])
    table[torch.rand(table.shape, generator=g, device="cuda") < 0.3] = -1
    return {"src": src, "dst": dst, "table": table.contiguous(),
            "pool": _random_pool(case, blocks, g)}


def prepare(case, seed):
    state = {"attn": _prepare_attn, "beam": _prepare_beam, "fork": _prepare_fork,
             "move": _prepare_move}[case["kind"]](case, seed)
    state["case"] = case
    return state


# ---- one pass: elementary operations -------------------------------------------------


def _rows_of(state, rows):
    """Group of each row and the tokens that it shares (0: in no group, or shorter)."""
    group_start, shared = state["group_start"], state["shared"]
    row = torch.arange(rows, device="cuda")
    of = (torch.searchsorted(group_start, row, right=True) - 1).clamp(max=shared.numel() - 1)
    start = torch.where(row < group_start[-1], shared[of], 0)
    return of, torch.where(state["len"] >= start, start, 0)


def _plain_attn(case, state):
    rows, heads, kv_heads, dim = case["rows"], case["heads"], case["kv_heads"], case["dim"]
    tokens, most, group = case["tokens"], state["most"], heads // kv_heads
    kc, vc = _views(case, state["pool"])
    kscale, vscale = _scales(case)
    kind = TYPES[case["cache"]]
    of, start = _rows_of(state, rows)
    q = state["q"].float().view(rows, kv_heads, group, dim) * (kscale / math.sqrt(dim))

    def keys(table):  # [n, cols] block ids -> [n, kv_heads, dim, positions]
        k = kc[table].view(kind).float()
        return k.permute(0, 2, 3, 5, 1, 4).reshape(table.shape[0], kv_heads, dim, -1)

    def values(table, live):
        v = vc[table].view(kind).float().permute(0, 2, 1, 3, 4)
        return torch.where(live[:, None, :, None], v.reshape(table.shape[0], kv_heads, -1, dim), 0.0)

    def scores(q, k, live):
        s = torch.where(live, torch.matmul(q, k), float("-inf"))
        top = s.amax(-1, keepdim=True)
        top = torch.where(torch.isinf(top), 0.0, top)
        p = torch.exp(s - top)
        return p, top, p.sum(-1, keepdim=True)

    # the prefixes: all rows of a group at once
    first, shared = state["group_start"][:-1].long(), state["shared"]
    cols = max(1, case["shared"] // tokens)
    member = first[:, None] + torch.arange(most, device="cuda")
    member = member.clamp(max=rows - 1)
    live = torch.arange(cols * tokens, device="cuda") < shared[:, None]
    # a group's first row may be idle: its blocks are those of any row that is not
    has = (start[member] > 0) & (of[member] == torch.arange(first.numel(), device="cuda")[:, None])
    lead = member.gather(1, has.int().argmax(1, keepdim=True))[:, 0]
    table = state["table"][lead][:, :cols].long().clamp(min=0)
    qg = q[member].transpose(1, 2).reshape(first.numel(), kv_heads, most * group, dim)
    p, top, total = scores(qg, keys(table), live[:, None, None])
    o = torch.matmul(p, values(table, live))
    del p

    def by_row(x):
        x = x.view(first.numel(), kv_heads, most, group, -1)
        x = x[of, :, (torch.arange(rows, device="cuda") - first[of]).clamp(0, most - 1)]
        return x.reshape(rows, kv_heads, group, -1)

    o, top, total = by_row(o), by_row(top), by_row(total)
    sharing = (start > 0)[:, None, None, None]
    total = torch.where(sharing, total, 0.0)
    o = torch.where(sharing, o, 0.0)

    # each row's own tokens
    cols = -(-case["own"] // tokens)
    at = start[:, None] // tokens + torch.arange(cols, device="cuda")
    inside = at < state["table"].shape[1]
    table = state["table"].gather(1, at.clamp(max=state["table"].shape[1] - 1).long()).long()
    live = start[:, None] + torch.arange(cols * tokens, device="cuda") < state["len"][:, None]
    live = live & inside.repeat_interleave(tokens, 1)
    table = table.clamp(min=0)
    p, top2, total2 = scores(q, keys(table), live[:, None, None])
    o2 = torch.matmul(p, values(table, live))
    both = torch.maximum(torch.where(total > 0, top, float("-inf")),
                         torch.where(total2 > 0, top2, float("-inf")))
    both = torch.where(torch.isinf(both), 0.0, both)
    a, b = torch.exp(top - both), torch.exp(top2 - both)
    a, b = torch.where(total > 0, a, 0.0), torch.where(total2 > 0, b, 0.0)
    total = total * a + total2 * b
    o = (o * a + o2 * b) / torch.where(total > 0, total, 1.0) * vscale
    state["out"].copy_(o.reshape(rows, heads, dim))
    state["lse"].copy_((both + torch.log(total)).reshape(rows, heads))
    return [state["out"], state["lse"]]


def _plain_beam(case, state):
    batch, beams, vocab, keep = (case[n] for n in ("batch", "beams", "vocab", "keep"))
    logits = state["logits"].double()
    top = logits.amax(-1, keepdim=True)
    top = torch.where(torch.isinf(top), 0.0, top)
    s = logits - (top + torch.log(torch.exp(logits - top).sum(-1, keepdim=True)))
    s = state["score"].double()[:, None] + torch.where(torch.isnan(s), float("-inf"), s)
    # a beam at its end goes on as it is
    done = state["done"][:, None] != 0
    token = torch.arange(vocab, device="cuda")
    stays = torch.where(token == min(END, vocab - 1), state["score"].double()[:, None], float("-inf"))
    s = torch.where(done, stays, s).view(batch, -1)
    # the `keep` best; of equal ones those that come first
    n = min(keep, s.shape[1])
    least = torch.topk(s, n, dim=1).values[:, -1:]
    more, same = s > least, s == least
    room = n - more.sum(1, keepdim=True)
    taken = more | (same & (torch.cumsum(same, 1) <= room))
    at = torch.arange(s.shape[1], device="cuda")
    at = torch.topk(torch.where(taken, at, s.shape[1]), n, dim=1, largest=False, sorted=True).values
    best = s.gather(1, at)
    best, order = torch.sort(best, dim=1, descending=True, stable=True)
    at = at.gather(1, order)
    none = torch.isinf(best)
    parent = torch.where(none, -1, at // vocab + torch.arange(batch, device="cuda")[:, None] * beams)
    token = torch.where(none, -1, at % vocab)
    ended = (token == min(END, vocab - 1)) | (state["done"][parent.clamp(min=0)] != 0)
    pad = (0, keep - n)
    whole = lambda x, v: torch.nn.functional.pad(x, pad, value=v)
    return [whole(best, float("-inf")).float(), whole(parent, -1).int(), whole(token, -1).int(),
            whole((ended & ~none).to(torch.uint8), 0)]


def _copy_blocks(case, pool, src, dst, tokens):
    """The first tokens[i] tokens of block src[i] to block dst[i]."""
    live = torch.arange(case["tokens"], device="cuda") < tokens[:, None]
    for part, axis in zip(_views(case, pool), (3, 2)):
        shape = [1] * part.dim()
        shape[0], shape[axis] = live.shape
        part[dst] = torch.where(live.view(shape), part[src], part[dst])


def _bits(state):
    return state["pool"].view(torch.int32)


def _plain_fork(case, state):
    parent, table, fresh, tokens = state["parent"].long(), state["table"], state["fresh"], case["tokens"]
    requests, cols, blocks = case["requests"], case["cols"], state["blocks"]
    has = parent >= 0
    of = parent.clamp(min=0)
    lens = torch.where(has, state["len"][of], 0)
    have = (lens + tokens - 1) // tokens
    col = torch.arange(cols, device="cuda")
    new = torch.where(col < have[:, None], table[of], -1)
    # the first child of a parent goes on in its last block, the others in a copy of it
    row = torch.arange(requests, device="cuda")
    eldest = torch.full((requests,), requests, device="cuda")
    eldest = eldest.scatter_reduce(0, of, torch.where(has, row, requests), "amin")
    copies = has & (lens % tokens != 0) & (eldest[of] != row)
    rank = torch.cumsum(copies, 0) - 1
    block = fresh[rank.clamp(0, fresh.numel() - 1)]
    last = (have - 1).clamp(min=0).long()[:, None]
    old = new.gather(1, last)[:, 0]
    new = new.scatter(1, last, torch.where(copies, block, old)[:, None])
    n = copies.sum()
    # the list of copies, in the order of the rows
    place = torch.where(copies, rank, requests)
    listed_ = lambda x: torch.full((requests + 1,), -1, dtype=torch.int32, device="cuda").scatter(
        0, place, x.int())[:requests]
    src, dst, part = listed_(old), listed_(block), listed_(lens % tokens)
    none = row >= n
    src, dst, part = (torch.where(none, -1, x) for x in (src, dst, part))
    # blocks of the old tables that no new one holds
    held = lambda t: torch.zeros(blocks + 1, dtype=torch.bool, device="cuda").index_fill(
        0, torch.where(t >= 0, t, blocks).flatten().long(), True)[:blocks]
    free = held(table) & ~held(new)
    where = torch.where(free, torch.cumsum(free, 0) - 1, blocks)
    freed = torch.full((blocks + 1,), -1, dtype=torch.int32, device="cuda").scatter(
        0, where, torch.arange(blocks, device="cuda", dtype=torch.int32))
    freed[blocks] = -1
    live = torch.nonzero(src >= 0)[:, 0]
    _copy_blocks(case, state["pool"], src[live].long(), dst[live].long(), part[live])
    return [new.int(), lens.int(), src, dst, part, freed[:blocks],
            torch.stack((n, free.sum())).int(), _bits(state)]


def _plain_move(case, state):
    src, dst, table = state["src"], state["dst"], state["table"]
    _copy_blocks(case, state["pool"], src.long(), dst.long(),
                 torch.full((case["moves"],), case["tokens"], device="cuda"))
    to = torch.arange(-1, case["blocks"], device="cuda", dtype=torch.int32)
    to[src.long() + 1] = dst
    table.copy_(to[table.long() + 1])
    return [table, _bits(state)]


# ---- one pass: the library -------------------------------------------------------------


def _kept(case, state):
    """What a program keeps from call to call: descriptors, outputs, scratch."""
    if "kept" not in state:
        from paper_2609_34380_amd import dps

        scratch = lambda need: torch.empty(max(need, 256), dtype=torch.uint8, device="cuda")
        if case["kind"] == "beam":
            state["kept"] = (dps.make_beam_step(case["batch"], case["keep"], "cuda"),
                             scratch(dps.beam_workspace_bytes(case["batch"], case["beams"],
                                                              case["vocab"], case["keep"])))
            return state["kept"]
        kscale, vscale = _scales(case)
        cache = dps.KvCache(state["pool"], case["tokens"], case["kv_heads"], case["dim"],
                            TYPES[case["cache"]], k_scale=kscale, v_scale=vscale)
        out = ws = None
        if case["kind"] == "attn":
            ws = scratch(dps.attn_shared_workspace_bytes(cache, case["rows"], case["heads"],
                                                         case["groups"]))
        elif case["kind"] == "fork":
            out = dps.make_kv_fork(case["requests"], case["cols"], state["blocks"], "cuda")
            ws = scratch(dps.kv_fork_workspace_bytes(case["requests"], state["blocks"]))
        state["kept"] = (cache, out, ws)
    return state["kept"]


def _own(case, state):
    from paper_2609_34380_amd import dps

    if case["kind"] == "beam":
        out, ws = _kept(case, state)
        dps.beam_select(state["logits"], state["score"], case["beams"], keep=case["keep"],
                        done=state["done"], end=min(END, case["vocab"] - 1), out=out, workspace=ws)
        return [out.score, out.parent, out.token, out.done]
    cache, out, ws = _kept(case, state)
    if case["kind"] == "attn":
        dps.attn_shared(state["q"], cache, state["table"], state["len"], state["group_start"],
                        state["shared"], out=state["out"], lse=state["lse"], workspace=ws)
        return [state["out"], state["lse"]]
    if case["kind"] == "fork":
        f = dps.kv_fork(state["parent"], state["len"], state["table"], state["fresh"],
                        case["tokens"], state["blocks"], out=out, workspace=ws)
        dps.kv_copy(cache, f.src, f.dst, tokens=f.tokens, count=f.counts)
        return [f.table, f.seq_len, f.src, f.dst, f.tokens, f.freed, f.counts, _bits(state)]
    dps.kv_copy(cache, state["src"], state["dst"])
    dps.kv_remap(state["table"], state["src"], state["dst"])
    return [state["table"], _bits(state)]


def run(state):
    case = state["case"]
    if own:
        return _own(case, state)
    return {"attn": _plain_attn, "beam": _plain_beam, "fork": _plain_fork,
            "move": _plain_move}[case["kind"]](case, state)


# ---- what a pass cannot do without, and what it has to give ------------------------------


def work(case):
    if case["kind"] == "beam":
        rows = case["batch"] * case["beams"]
        return {"bytes": rows * (case["vocab"] * SIZES[case["dtype"]] + 5) +
                case["batch"] * case["keep"] * 13, "flops": 4 * rows * case["vocab"]}
    size, token = SIZES[case["cache"]], 2 * case["kv_heads"] * case["dim"]
    if case["kind"] == "attn":
        rows, heads, dim = case["rows"], case["heads"], case["dim"]
        shared, own_ = case["shared"] * (0.75 + 0.25 / case["groups"]), case["own"] / 2
        tokens = case["groups"] * shared + rows * own_
        return {"bytes": int(tokens * token * size + rows * heads * (4 * dim + 4)),
                "flops": int(4 * rows * (shared + own_) * heads * dim)}
    if case["kind"] == "fork":
        requests = case["requests"]
        copies = requests * 0.6 * case["tokens"] / 2  # tokens in the last blocks that are copied
        return {"bytes": int(8 * requests * case["cols"] + 24 * requests + 2 * copies * token * size),
                "flops": 0}
    return {"bytes": 8 * case["requests"] * case["cols"] + 8 * case["moves"] +
            2 * case["moves"] * case["tokens"] * token * size, "flops": 0}


def _exact_attn(case, state):
    heads, kv_heads, dim = case["heads"], case["kv_heads"], case["dim"]
    kc, vc = _views(case, state["pool"])
    kscale, vscale = _scales(case)
    kind = TYPES[case["cache"]]
    out = torch.zeros((case["rows"], heads, dim), dtype=torch.float64, device="cuda")
    lse = torch.full((case["rows"], heads), float("-inf"), dtype=torch.float64, device="cuda")
    for r, n in enumerate(state["len"].tolist()):
        if not n:
            continue
        blocks = state["table"][r, : -(-n // case["tokens"])].long()
        k = kc[blocks].view(kind).double().permute(1, 0, 3, 2, 4).reshape(kv_heads, -1, dim)[:, :n]
        v = vc[blocks].view(kind).double().permute(1, 0, 2, 3).reshape(kv_heads, -1, dim)[:, :n]
        q = state["q"][r].double().reshape(kv_heads, -1, dim) * (kscale / math.sqrt(dim))
        s = torch.matmul(q, k.transpose(1, 2).contiguous())
        z = torch.logsumexp(s, -1, keepdim=True)
        out[r] = (torch.matmul(torch.exp(s - z), v.contiguous()) * vscale).reshape(heads, dim)
        lse[r] = z.reshape(heads)
    return [out, lse]


def _exact_beam(case, state):
    batch, beams, keep = case["batch"], case["beams"], case["keep"]
    x = state["logits"].double()
    s = state["score"].double()[:, None] + x - torch.logsumexp(x, -1, keepdim=True)
    over = state["done"] != 0
    s[over] = float("-inf")
    s[over, min(END, case["vocab"] - 1)] = state["score"].double()[over]
    s = s.nan_to_num(nan=float("-inf")).view(batch, -1)
    best = torch.full((batch, keep), float("-inf"), dtype=torch.float64, device="cuda")
    n = min(keep, s.shape[1])
    best[:, :n] = torch.topk(s, n, dim=1, sorted=True).values
    return [best, None, None, None]


def exact(case, seed):
    if case["kind"] in ("fork", "move"):
        return None  # whole numbers
    state = prepare(case, seed)
    return (_exact_attn if case["kind"] == "attn" else _exact_beam)(case, state)
