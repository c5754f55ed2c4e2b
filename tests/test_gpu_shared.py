"""Attention of rows that share prefixes, on the GPU, against the definition in 64 bits
on the CPU: every row attends its tokens through its own table row, whatever is shared."""
import math

import numpy as np
import pytest
import torch

from gpu_helpers import DEV
from paper_2609_34380_amd import dps
from test_gpu_kv_cache import BF16, E4M3, F16, Cache, attn_oracle, check_attn, rnd

pytestmark = pytest.mark.gpu


def i32(a):
    return torch.tensor(np.array(a), dtype=torch.int32)


class Batch:
    """Groups [(L, [own tokens of each row])], rows alone after them: a cache that holds
    every row's tokens, NaN everywhere else.  Whole blocks of a prefix are shared; what is
    left of it lies in a block of each row's own, as after a fork."""

    def __init__(self, groups, alone, dtype, cdtype, dim, kv_heads, group, tokens, seed=0,
                 offset=0, gap=0, kmul=1.0, qmul=1.0):
        rng = np.random.default_rng(seed)
        self.group_start, self.shared, self.len = [0], [], []
        plan = []                                   # of each row: (group, own tokens)
        for g, (n, own) in enumerate(groups):
            self.shared.append(n)
            self.group_start.append(self.group_start[-1] + len(own))
            plan += [(g, m) for m in own]
        plan += [(None, m) for m in alone]
        total = [0 if m is None else m + (self.shared[g] if g is not None else 0)
                 for g, m in plan]                  # None: an idle row
        self.len = total
        whole = [n // tokens for n, _ in groups]
        cols = max(1, max(-(-n // tokens) for n in total + self.shared)) + 1
        need = [-(-n // tokens) for n in total]
        blocks = sum(whole) + sum(need) + 3
        ids = rng.permutation(blocks)
        scales = (0.05, 0.02) if cdtype == E4M3 else (1.0, 1.0)
        self.cache = Cache(blocks, tokens, kv_heads, dim, cdtype, *scales, offset=offset, gap=gap)
        self.table = torch.full((len(plan), cols), -1, dtype=torch.int32)
        at = 0
        common = []
        for w in whole:
            common.append(ids[at:at + w])
            at += w
        for r, (g, m) in enumerate(plan):
            if m is None:
                continue
            first = whole[g] if g is not None else 0
            row = list(common[g]) if g is not None else []
            row += list(ids[at:at + need[r] - first])
            at += need[r] - first
            self.table[r, :need[r]] = i32(row)
            n = self.shared[g] if g is not None else 0
            t = torch.arange(total[r])
            slot = self.table[r].long()[t // tokens] * tokens + t % tokens
            k = torch.cat((rnd(n, kv_heads, dim, seed=seed + 10 + (g or 0)),
                           rnd(m, kv_heads, dim, seed=seed + 100 + r)))
            v = torch.cat((rnd(n, kv_heads, dim, seed=seed + 50 + (g or 0)),
                           rnd(m, kv_heads, dim, seed=seed + 1000 + r)))
            self.cache.place(slot, k / scales[0] * kmul, v / scales[1])
        self.q = (rnd(len(plan), kv_heads * group, dim, seed=seed + 3) * qmul).to(dtype)

    def run(self, lens=None, group_start=None, shared=None, req=None, table=None, scale=None, **kw):
        """Checks the call against the definition; returns its results."""
        q = self.q
        lens = i32(self.len if lens is None else lens)
        table = self.table if table is None else table
        starts = i32(self.group_start if group_start is None else group_start)
        shared = i32(self.shared if shared is None else shared)
        rq = i32(range(q.shape[0])) if req is None else i32(req)
        cache = self.cache.up()
        groups = shared.numel()
        need = dps.attn_shared_workspace_bytes(cache, q.shape[0], q.shape[1], groups)
        ws = torch.full((need + 256,), 0xFF, dtype=torch.uint8, device=DEV)
        lse = torch.full(q.shape[:2], 5.0, device=DEV)
        got = dps.attn_shared(q.to(DEV), cache, table.to(DEV), lens.to(DEV), starts.to(DEV),
                              shared.to(DEV), req=None if req is None else rq.to(DEV), scale=scale,
                              lse=lse, workspace=ws, **kw)
        torch.cuda.synchronize()
        assert bool((ws[need:] == 0xFF).all())
        want = attn_oracle(q, self.cache, table, lens, rq,
                           q.shape[2] ** -0.5 if scale is None else scale, 0)
        check_attn(got, lse, want, q.dtype)
        return got, lse


KINDS = [
    # dtype, cache, dim, kv_heads, group, tokens
    (F16, F16, 128, 2, 4, 16), (BF16, BF16, 128, 1, 8, 32), (F16, E4M3, 128, 2, 4, 64),
    (BF16, E4M3, 64, 1, 2, 16), (F16, F16, 64, 3, 1, 16), (F16, F16, 96, 1, 5, 16),
    (BF16, BF16, 96, 2, 3, 128), (F16, F16, 192, 1, 4, 16), (BF16, E4M3, 192, 1, 16, 32),
    (F16, F16, 256, 1, 2, 16), (F16, E4M3, 256, 1, 8, 256), (BF16, BF16, 256, 1, 24, 16),
]


@pytest.mark.parametrize("dtype,cdtype,dim,kv_heads,group,tokens", KINDS)
def test_kinds(dtype, cdtype, dim, kv_heads, group, tokens):
    """Every type and width, prefixes that end in the middle of a tile and a block."""
    args = (dtype, cdtype, dim, kv_heads, group, tokens)
    Batch([(5 * tokens, [1, 7, 33]), (77, [4, None, 1, 60]), (0, [9, 2])], [40, None], *args).run()
    Batch([(300, [3 + i for i in range(9)])], [], *args, seed=1).run()
    Batch([(129, [2, 50, None, 1] * 9)], [5], *args, seed=2).run()


@pytest.mark.parametrize("n", [1, 15, 16, 17, 31, 32, 33, 64, 127, 128, 129, 1000, 4097])
def test_prefix_lengths(n):
    Batch([(n, [1, 40, 2])], [], F16, F16, 64, 1, 4, 16, seed=n).run()


@pytest.mark.parametrize("group", [1, 2, 3, 7, 16, 17, 24, 32, 33, 40, 71])
@pytest.mark.parametrize("rows", [2, 5, 33])
def test_query_heads(group, rows):
    """Columns of one, two and more tiles, rows that do not divide them, passes."""
    own = [1 + 5 * i % 23 for i in range(rows)]
    Batch([(70, own)], [], F16, F16, 64, 1, group, 16, seed=group).run()
    if rows == 5:
        Batch([(70, own), (33, [4, 4])], [3], BF16, BF16, 128, 2, group, 32, seed=group).run()


@pytest.mark.parametrize("groups", [1, 3, 63, 64, 65, 256, 257, 1024])
def test_many_groups(groups):
    rng = np.random.default_rng(groups)
    spec = [(int(rng.integers(0, 70)), [int(x) for x in rng.integers(1, 9, rng.integers(0, 4))])
            for _ in range(groups)]
    spec[0] = (40, [3, 5])
    Batch(spec, [7, 30], F16, F16, 64, 1, 2, 16, seed=groups).run()


def test_work_is_cut_anywhere():
    """Long and short groups on one line, items of one tile and of hundreds."""
    Batch([(5000, [3, 9, 1, 1, 30]), (20, [5] * 40), (900, [2, 2]), (31, [1])], [600],
          F16, F16, 64, 2, 4, 16).run()
    Batch([(64, [1] * 200), (2500, [4] * 70)], [], F16, F16, 64, 1, 8, 16, seed=4).run()
    Batch([(1500, [900, 3, 2000])], [1800], F16, E4M3, 64, 1, 4, 16, seed=5).run()


def test_same_as_attn_decode():
    b = Batch([(640, [3, 20, 5, 8]), (96, [2, 2, None])], [50], F16, F16, 128, 2, 4, 16)
    got, lse = b.run()
    cache, dev = b.cache.up(), lambda x: x.to(DEV)
    one = torch.empty_like(lse)
    ref = dps.attn_decode(dev(b.q), cache, dev(b.table), dev(i32(b.len)), lse=one)
    assert torch.equal(torch.isinf(lse), torch.isinf(one))
    fine = ~torch.isinf(one)
    assert bool(((lse - one).abs()[fine] <= 2.0 ** -18 * (1 + one.abs()[fine])).all())
    # both are one rounding and some 2^-17 of weights of size 1 away from the definition
    assert bool(((got - ref).float().abs() <= 2.0 ** -10 * ref.float().abs() + 2.0 ** -13).all())
    # and the same call gives the same bits
    again, lse2 = b.run()
    assert torch.equal(got, again) and torch.equal(lse, lse2)


def test_rows_that_cannot_share():
    """Idle and shorter rows, rows without a table row, first rows of that kind: each
    attends what it has, through its own table row."""
    b = Batch([(200, [5, 30, 1, 12]), (64, [3, 3, 3])], [20], F16, F16, 64, 2, 4, 16)
    lens = list(b.len)
    for r, n in ((0, 0), (0, 199), (0, 200), (0, -4), (1, 17), (4, 10), (6, 64)):
        cut = list(lens)
        cut[r] = n
        b.run(lens=cut)
    b.run(lens=[0] * 8)
    b.run(lens=[190, 100, 0, 3, 64, 65, 66, 20])
    b.run(req=[0, 1, 2, 3, 4, 5, 6, 7])
    b.run(req=[-1, 1, 2, 3, 99, 5, 6, 7])
    b.run(req=[0, -1, 2, 8, 4, 5, 6, -7])
    b.run(req=[-1] * 8)


def test_rows_in_another_order():
    """Table rows through req, several rows of one request."""
    b = Batch([(150, [4, 9, 30]), (48, [2, 2])], [20], BF16, BF16, 128, 1, 4, 16)
    req = [2, 0, 1, 4, 3, 5]
    lens = [b.len[r] for r in req]
    b.run(req=req, lens=lens)
    b.run(req=[0, 0, 0, 3, 3, 5], lens=[154, 153, 151, 50, 49, 20])


def test_groups_that_do_not_fit():
    """Nothing is shared where group_start does not ascend within the rows, and by a group
    whose prefix no row can have."""
    b = Batch([(96, [5, 3, 1]), (64, [3, 3])], [20], F16, F16, 64, 1, 4, 16)
    for starts in ([0, 5, 3], [-1, 3, 5], [0, 3, 7], [3, 3, 2], [0, -2 ** 31, 5],
                   [0, 3, 2 ** 31 - 1], [2 ** 31 - 1, -2 ** 31, 0]):
        b.run(group_start=starts)
    for shared in ([-5, 64], [0, 0], [2 ** 31 - 1, 64], [96, 10000], [96, -2 ** 31]):
        b.run(shared=shared)
    b.run(group_start=[0, 0, 0])                # empty groups
    b.run(group_start=[3, 5, 5], shared=[64, 7])
    b.run(group_start=[3, 3, 5], shared=[7, 64])
    b.run(group_start=[0], shared=[])           # no groups
    b.run(shared=[90, 33])                      # less than they have in common


def test_lost_blocks():
    """Prefix and own blocks that are not in the cache are left out, for all rows."""
    b = Batch([(160, [5, 30, 1])], [], F16, F16, 64, 1, 4, 16)
    for cols, lost in (((2,), -1), ((0, 9), 10 ** 6), ((10,), -1), (range(10), -1)):
        t = b.table.clone()
        for c in cols:
            t[:, c] = lost
        b.run(table=t)
    t = torch.full_like(b.table, -1)
    b.run(table=t)


@pytest.mark.parametrize("case", ["large", "tiny", "negative", "one"])
def test_score_ranges(case):
    """Large and tiny scores; one part of a row far above the other."""
    kw = {"large": dict(kmul=30.0, qmul=30.0), "tiny": dict(kmul=1e-3), "negative": {}, "one": {}}
    b = Batch([(200, [40, 3, 100])], [9], F16, F16, 64, 1, 4, 16, seed=7, **kw[case])
    if case == "one":
        for r in range(3):                     # own tokens against the prefix, and the reverse
            t = torch.arange(b.len[r])[200:] if r < 2 else torch.arange(200)
            slot = b.table[r].long()[t // 16] * 16 + t % 16
            k, v = b.cache.fetch(slot)
            if r < 2:
                b.cache.place(slot, k * 40, v)
    b.run(scale=-0.2 if case == "negative" else None)


def test_values_beyond_the_prefix_and_rows():
    """What lies behind a row's tokens, and an infinite value of one row's own, stay out
    of the others."""
    b = Batch([(72, [5, 9, 6])], [], F16, F16, 64, 1, 4, 16)
    clean, _ = b.run()
    slot = int(b.table[1, 76 // 16]) * 16 + 76 % 16
    k, v = b.cache.fetch([slot])
    v[0, 0, 5] = math.inf
    b.cache.place([slot], k, v)
    cache, dev = b.cache.up(), lambda x: x.to(DEV)
    got = dps.attn_shared(dev(b.q), cache, dev(b.table), dev(i32(b.len)), dev(i32([0, 3])),
                          dev(i32([72])))
    assert torch.equal(got[0], clean[0]) and torch.equal(got[2], clean[2])
    bad = ~torch.isfinite(got[1].float())
    assert bool(bad[:, 5].all()) and int(bad.sum()) == 4


def test_strides_offset_and_streams():
    b = Batch([(100, [5, 9, 6]), (33, [1, 2])], [17], BF16, BF16, 128, 2, 4, 16, offset=64, gap=32)
    want, _ = b.run()
    rows, heads, dim = b.q.shape
    room = torch.full((rows, heads * dim + 40), 7.0, dtype=BF16, device=DEV)
    q = room[:, :heads * dim].copy_(b.q.reshape(rows, -1)).view(rows, heads * dim)
    q = q.as_strided((rows, heads, dim), (heads * dim + 40, dim, 1))
    out = torch.full((rows, heads * dim + 8), 7.0, dtype=BF16, device=DEV)
    view = out.as_strided((rows, heads, dim), (heads * dim + 8, dim, 1))
    cache, dev = b.cache.up(), lambda x: x.to(DEV)
    args = [dev(b.table), dev(i32(b.len)), dev(i32(b.group_start)), dev(i32(b.shared))]
    torch.cuda.synchronize()
    stream = torch.cuda.Stream()
    with torch.cuda.stream(stream):
        got = dps.attn_shared(q, cache, *args, out=view)
    stream.synchronize()
    assert got is view and torch.equal(view, want)
    assert bool((out[:, heads * dim:] == 7.0).all())


def test_in_a_graph():
    """One captured call for groups and lengths that change between replays, two graphs on
    one workspace, and an eager call in between."""
    b = Batch([(130, [5, 9, 6, 30]), (64, [1, 2, 8])], [17, 4], F16, F16, 64, 2, 4, 16)
    cache, dev = b.cache.up(), lambda x: x.to(DEV)
    q, table = dev(b.q), dev(b.table)
    lens, starts, shared = dev(i32(b.len)), dev(i32(b.group_start)), dev(i32(b.shared))
    need = dps.attn_shared_workspace_bytes(cache, 9, 8, 2)
    ws = torch.empty(need, dtype=torch.uint8, device=DEV)
    outs = [torch.empty_like(q) for _ in range(2)]
    call = lambda out: dps.attn_shared(q, cache, table, lens, starts, shared, out=out, workspace=ws)
    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(stream):
        call(outs[0])
    stream.synchronize()
    graphs = []
    for out in outs:
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g, stream=stream):
            call(out)
        graphs.append(g)
    for t, (n, s, m) in enumerate(((b.len, [0, 4, 7], [130, 64]), (b.len, [0, 4, 4], [100, 64]),
                                   ([0] * 9, [0, 4, 7], [130, 64]), (b.len, [0, 0, 0], [0, 0]),
                                   ([133, 20, 0, 150, 65, 64, 70, 10, 4], [0, 4, 7], [130, 64]))):
        lens.copy_(i32(n))
        starts.copy_(i32(s))
        shared.copy_(i32(m))
        ws.fill_(0xFF)
        torch.cuda.synchronize()
        graphs[0].replay()
        graphs[1].replay()
        torch.cuda.synchronize()
        eager = dps.attn_shared(q, cache, table, lens, starts, shared)
        torch.cuda.synchronize()
        want = attn_oracle(b.q, b.cache, b.table, i32(n), i32(range(9)), 64 ** -0.5, 0)
        for out in outs:
            assert torch.equal(out, eager)
        check_attn(eager, None, want, F16)


def test_beyond_4_gib():
    """Shared and own blocks on both sides of 4 GiB."""
    tokens, kv_heads, dim = 256, 8, 128
    size = 2 * kv_heads * tokens * dim * 2
    blocks = (5 << 30) // size
    pool = torch.empty(blocks * size, dtype=torch.uint8, device=DEV)
    cache = dps.KvCache(pool, tokens, kv_heads, dim, F16)
    ids = [[blocks - 1, 3, blocks - 5], [blocks - 1, 3, 9]]
    small = Cache(5, tokens, kv_heads, dim, F16)
    places = {blocks - 1: 0, 3: 1, blocks - 5: 2, 9: 3}
    for j in range(4):
        slot = torch.arange(tokens) + j * tokens
        small.place(slot, rnd(tokens, kv_heads, dim, seed=j), rnd(tokens, kv_heads, dim, seed=20 + j))
    for big, at in places.items():
        pool[big * size:(big + 1) * size] = small.host[at * size:(at + 1) * size].to(DEV)
    q = rnd(2, 16, dim, seed=5).to(F16)
    lens = i32([2 * tokens + 90, 2 * tokens + 201])
    got = dps.attn_shared(q.to(DEV), cache, i32(ids).to(DEV), lens.to(DEV), i32([0, 2]).to(DEV),
                          i32([2 * tokens]).to(DEV))
    table = i32([[places[b] for b in row] for row in ids])
    want = attn_oracle(q, small, table, lens, i32([0, 1]), dim ** -0.5, 0)
    check_attn(got, None, want, F16)


def test_empty_and_refused_calls():
    b = Batch([(32, [5, 9])], [], F16, F16, 64, 1, 4, 16)
    cache, dev = b.cache.up(), lambda x: x.to(DEV)
    q, table, lens = dev(b.q), dev(b.table), dev(i32(b.len))
    starts, shared = dev(i32([0, 2])), dev(i32([32]))
    none = dps.attn_shared(q[:0], cache, table, lens[:0], dev(i32([0])), shared[:0])
    assert none.shape == (0, 4, 64)
    for bad in (lambda: dps.attn_shared(q, cache, table, lens[:1], starts, shared),
                lambda: dps.attn_shared(q, cache, table, lens, starts[:1], shared),
                lambda: dps.attn_shared(q, cache, table, lens, starts.long(), shared),
                lambda: dps.attn_shared(q, cache, table, lens, starts, shared.cpu()),
                lambda: dps.attn_shared(q.float(), cache, table, lens, starts, shared),
                lambda: dps.attn_shared(q, cache, table, lens, starts, shared, req=lens[:1]),
                lambda: dps.attn_shared(q, cache, table, lens, starts, shared,
                                        lse=torch.empty(2, 3, device=DEV))):
        with pytest.raises(ValueError):
            bad()
    with pytest.raises(dps.DpsError):
        dps.attn_shared(q, cache, table, lens, starts, shared,
                        workspace=torch.empty(64, dtype=torch.uint8, device=DEV))


@pytest.mark.parametrize("dtype,cdtype,dim,kv_heads,group,tokens", KINDS)
def test_many_columns(dtype, cdtype, dim, kv_heads, group, tokens):
    """Groups of 150 columns and more, three and one: tiles through LDS, for every type and
    width; last items of one row, and of as many columns as go into a wave and more."""
    args = (dtype, cdtype, dim, kv_heads, group, tokens)
    rows = -(-150 // group)
    own = [(None if i % 11 == 4 else 1 + 5 * i % 23) for i in range(2 * rows)]
    Batch([(333, own[:rows]), (64, own[:rows + 1]), (700, own[1:rows])], [7], *args, seed=4).run()
    Batch([(515, own[:rows * 2])], [], *args, seed=5).run()


@pytest.mark.parametrize("dtype,cdtype,dim,kv_heads,group,groups", [
    (F16, F16, 128, 4, 8, [(3300, 20)]), (BF16, BF16, 128, 4, 8, [(2900, 17), (700, 5)]),
    (F16, E4M3, 128, 2, 16, [(5000, 11)]), (BF16, E4M3, 192, 4, 4, [(1500, 1), (3000, 30)]),
    (F16, F16, 64, 4, 32, [(4001, 6)]), (F16, F16, 192, 4, 4, [(2100, 11)]),
    (BF16, BF16, 256, 2, 16, [(3000, 3)]), (F16, F16, 96, 4, 8, [(2500, 13), (2500, 13)]),
])
def test_items_side_by_side(dtype, cdtype, dim, kv_heads, group, groups):
    """One or two groups of several items, which get whole blocks with the same tokens."""
    Batch([(n, [3 * i % 40 + 1 if i % 7 != 2 else None for i in range(rows)])
           for n, rows in groups], [9], dtype, cdtype, dim, kv_heads, group, 32, seed=dim).run()


@pytest.mark.parametrize("cdtype,dim,rows,heads,tiles", [(E4M3, 64, 2, 32, 2 ** 16),
                                                         (F16, 192, 4, 16, 2 ** 17)])
def test_longest_prefix(cdtype, dim, rows, heads, tiles):
    """Rows under 2^31 - 256 tokens, all of them in one block: a token counts as often as the
    block is named.  Sums grow over up to `tiles` tiles, each of which rounds them (and what
    the matrix cores hold, 4 times) to 2^-24 of themselves."""
    tokens, cols = 256, 2 ** 23 - 1
    scales = (0.05, 0.02) if cdtype == E4M3 else (1.0, 1.0)
    c = Cache(1, tokens, 1, dim, cdtype, *scales)
    k, v = rnd(tokens, 1, dim, seed=1), 1 + 0.5 * rnd(tokens, 1, dim, seed=2)
    c.place(torch.arange(tokens), k / scales[0], v / scales[1])
    q = rnd(rows, heads, dim, seed=3).to(F16)
    one = torch.zeros(1, dtype=torch.int32)
    want, lse64 = attn_oracle(q, c, one[:, None], torch.tensor([tokens] * rows),
                              torch.zeros(rows).int(), dim ** -0.5, 0)[:2]
    table = torch.zeros((1, cols), dtype=torch.int32, device=DEV)
    n = i32([cols * tokens]).to(DEV)
    lse = torch.empty((rows, heads), device=DEV)
    got = dps.attn_shared(q.to(DEV), c.up(), table, n.repeat(rows), i32([0, rows]).to(DEV), n,
                          req=torch.zeros(rows, dtype=torch.int32, device=DEV), lse=lse)
    step = tiles * 2.0 ** -24
    err = (got.cpu().double() - want).abs().max()
    assert err <= 5 * step * float(v.abs().max()) + 2.0 ** -10, err
    assert float((lse.cpu().double() - lse64 - math.log(cols)).abs().max()) <= 2 * step
