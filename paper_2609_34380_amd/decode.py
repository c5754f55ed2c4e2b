"""The attention half of a decoder layer on nested weights, over KV blocks of the
shared region (Sec. IV-B "Shared Region": one memory that residual planes and
paged KV blocks take turns in).

    PagedBatch      the requests of a serving loop: KV blocks from a SUM
                    manager, block tables and slot maps built on the GPU
    AttentionLayer  QKV product, head norms with rotation into the cache,
                    attention, O product, in the precision mode of the pass
    Beams           beam search over the slots of a PagedBatch: several answers
                    to one prompt share its blocks, which are read once for all

Everything an AttentionLayer and PagedBatch.map() enqueue reads lengths, tables
and slots on the device, so a step can be captured (graphs.ModeGraphs) and
replayed while requests grow.

Run as a program (python -m paper_2609_34380_amd.decode), it decodes with a small
layer until KV blocks push the residuals out, goes on in fast mode, and returns
to full mode once the requests end and the residuals are restored; with the argument
"beams" the requests are beams of two prompts, and blocks that end up scattered over the
units are moved together so that the residuals can return.
"""
import sys

import torch

from . import dps


class PagedBatch:
    """`batch` slots for requests of up to max_tokens tokens (rounded up to whole
    blocks: self.max_tokens), their KV blocks (of block_tokens tokens) from `sums`.  A
    step takes at most `rows` new tokens.

    grow() does a step's host work (blocks, lengths to the device), map() enqueues
    the GPU's; the results are in self.step (a dps.KvMap) and self.table.  Each grow()
    is followed by its map(), or by one replay of a graph that holds it, before the
    next: the blocks of a step that is not mapped reach no table.  Several new tokens of
    a slot are rows that the attention serves one by one, each over all tokens before it.

    Steps may run on other streams than grow(): its copies wait for the work of every
    stream that map() was called on, also to capture it, and are complete when it
    returns.  Before the next grow(), fork() or compact() a caller waits for a graph replayed
    elsewhere than on the stream of its capture.

    fork() lets slots go on from other slots, sharing their whole blocks.  It and compact()
    come between steps, after all that reads self.step is enqueued.  With groups > 0
    (the most groups of rows that one step's attention treats as one) grow() also finds
    which neighbouring rows share their first blocks: self.group_start and
    self.shared_len, for dps.attn_shared."""

    def __init__(self, sums, batch, max_tokens, block_tokens, rows=None, device="cuda", groups=0):
        self.sums, self.block_tokens, self.groups = sums, block_tokens, groups
        self.lengths = [0] * batch           # tokens in the cache, after the last step
        self.blocks = [[] for _ in range(batch)]
        columns = -(-max_tokens // block_tokens)
        self.max_tokens = columns * block_tokens
        i32 = dict(dtype=torch.int32, device=device)
        self.table = torch.full((batch, columns), -1, **i32)
        # a step's lengths, and the counts that its map() writes: below 0 before it has run
        self._lengths = torch.zeros(2 * batch + 2, **i32)
        self.ctx_len, self.new_len = self._lengths[:batch], self._lengths[batch:2 * batch]
        self.rows = batch if rows is None else rows
        # a step never takes more than a block a slot and what its rows fill
        self.fresh = torch.full((batch + self.rows // block_tokens + 1,), -1, **i32)
        self.step = dps.make_kv_map(batch, self.rows, self.ctx_len.device)
        self.step = self.step._replace(counts=self._lengths[2 * batch:])
        # that the buffers were filled on, or map() was called on
        self._streams = [torch.cuda.current_stream(self.table.device)]
        self._unmapped = set()               # slots that grew since the last map()
        self._grown = set()                  # slots of the last step, whoever mapped it
        self._captured = False               # map() is in a graph: replays are not seen here
        self._forks = 0                      # > 0: slots may have blocks in common
        self._group_key = None               # of the groups that are on the device
        self.wake = False                    # what forks have freed lets residuals return
        self.group_start, self.shared_len = (torch.zeros(n, **i32) for n in (groups + 1, groups))

    def grow(self, new):
        """new[r] tokens join slot r in the coming step.  Takes the blocks they need
        (which may evict residuals: look at sums.mode afterwards) and brings the
        lengths to the device on the current stream, once the steps before have read
        theirs (the host waits for that).  False, with nothing changed, if no room is
        left."""
        if len(new) != len(self.lengths) or min(new) < 0 or sum(new) > self.rows:
            raise ValueError("one count of new tokens a slot, at most %d in all" % self.rows)
        need = []
        for had, n in zip(self.lengths, new):
            if had + n > self.max_tokens:
                raise ValueError("a request outgrows its table row")
            need.append(-(-(had + n) // self.block_tokens) - -(-had // self.block_tokens))
        try:
            self._mapped()
        except RuntimeError:
            c = self.sums.counts()
            if sum(need) > (c["free"] + c["backed"]) * self.sums.blocks_per_unit + c["free_blocks"]:
                return False
            raise
        taken = self.sums.alloc(sum(need))
        if taken is None:
            return False
        self._after_steps()
        if self.groups:
            self._group([r for r, n in enumerate(new) for _ in range(n)])
        self._lengths.copy_(torch.tensor([*self.lengths, *new, -1, -1], dtype=torch.int32))
        if taken:
            self.fresh[:len(taken)].copy_(torch.tensor(taken, dtype=torch.int32))
        at = 0
        for r, n in enumerate(need):
            self.blocks[r] += taken[at:at + n]
            at += n
            self.lengths[r] += new[r]
        self._unmapped = {r for r, n in enumerate(new) if n}
        self._grown = set(self._unmapped)
        return True

    def _after_steps(self):
        """Work enqueued from here on comes after every step: it replaces what they read."""
        here = torch.cuda.current_stream(self.table.device)
        for stream in self._streams:
            if stream != here:
                here.wait_stream(stream)
        return here

    def _group(self, slots):
        """The groups of a step whose rows are those slots': neighbours with the same first
        block, and the blocks, full before the step, that all of them have in common."""
        key = (slots, self._forks)
        if key == self._group_key:
            return
        # rows of one slot share what it holds, which grows from step to step
        self._group_key = key if len(set(slots)) == len(slots) else None
        starts, lengths = [], []
        row = 0
        while self._forks and row < len(slots) and len(starts) < self.groups:
            first = self.blocks[slots[row]]
            end, common = row + 1, self.lengths[slots[row]] // self.block_tokens
            while end < len(slots) and common and self.blocks[slots[end]][:1] == first[:1]:
                other = self.blocks[slots[end]][:self.lengths[slots[end]] // self.block_tokens]
                common = next((i for i, (a, b) in enumerate(zip(first[:common], other)) if a != b),
                              min(common, len(other)))
                end += 1
            if end > row + 1 or starts:     # (between groups a row by itself is one, too)
                starts.append(row)
                lengths.append(common * self.block_tokens if end > row + 1 else 0)
            row = end
        pad = self.groups - len(starts)
        starts += [row if starts else 0] * (pad + 1)
        self.group_start.copy_(torch.tensor(starts, dtype=torch.int32))
        self.shared_len.copy_(torch.tensor(lengths + [0] * pad, dtype=torch.int32))

    def _mapped(self):
        if self._unmapped and not self._captured:
            raise RuntimeError("the tokens of the last grow() are not mapped")

    def _between_steps(self):
        """Refuses what would come between a step's grow() and its map(), which may be in a
        graph: the step's blocks are in no table yet.  Returns the current stream."""
        self._mapped()
        here = self._after_steps()
        if self._captured and self._grown and int(self.step.counts[0]) < 0:
            raise RuntimeError("the tokens of the last grow() are not mapped")
        return here

    def map(self):
        """Enqueue the step's block tables and slot maps."""
        stream = torch.cuda.current_stream(self.table.device)
        if stream not in self._streams:
            self._streams.append(stream)
        self._captured = self._captured or torch.cuda.is_current_stream_capturing()
        self._unmapped.clear()
        return dps.kv_map(self.ctx_len, self.new_len, self.fresh, self.table, self.block_tokens,
                          out=self.step)

    def _ours(self, caches):
        """Every block that the manager hands out has to be one of each cache's."""
        blocks = self.sums.n_units * self.sums.blocks_per_unit
        for cache in caches:
            if cache.block_tokens != self.block_tokens or cache.n_blocks < blocks:
                raise ValueError("a cache has other blocks than the batch")

    def fork(self, parents, caches):
        """Slot r goes on from slot parents[r] (an int32 device tensor, or a list; -1: the
        slot is empty from now on), for all slots at once: shared whole blocks, and a copy
        of a last block that has room, in each of `caches` (every layer's).  Takes the
        blocks of the copies (False, with nothing changed, if no room is left) and gives
        back those that no slot holds any more; where residuals wait for units that became
        free, self.wake turns True, and stays so until the caller, who wakes their restore, has
        set it back.  Waits for the steps before, as grow() does, and for the copies."""
        here = self._between_steps()
        self._ours(caches)
        given = torch.is_tensor(parents)
        if given and not (parents.dtype == torch.int32 and parents.device == self.table.device and
                          parents.is_contiguous() and parents.dim() == 1):
            raise ValueError("parents must be a list, or a contiguous int32 tensor beside the table")
        host = parents.tolist() if given else list(parents)
        if len(host) != len(self.lengths) or max(host) >= len(host):
            raise ValueError("one parent a slot, a slot or -1")
        copied, seen = [], set()
        for r, p in enumerate(host):
            if p >= 0 and p in seen and self.lengths[p] % self.block_tokens:
                copied.append(r)
            seen.add(p)
        taken = self.sums.alloc(len(copied))
        if taken is None:
            return False
        i32 = dict(dtype=torch.int32, device=self.table.device)
        try:
            if not given:
                parents = torch.tensor(host, **i32)
            # no blocks for kv_fork to list: a table row names what its slot's earlier requests
            # held, too, which may be another holder's by now; what nothing holds any more is
            # known here
            out = dps.make_kv_fork(len(host), self.table.shape[1], 0, self.table.device)
            f = dps.kv_fork(parents, torch.tensor(self.lengths, **i32), self.table,
                            torch.tensor(taken, **i32), self.block_tokens, 0, out=out)
            for cache in caches:
                dps.kv_copy(cache, f.src, f.dst, tokens=f.tokens, count=f.counts)
            self.table.copy_(f.table)      # where captured steps look for it
        except Exception:
            here.synchronize()             # copies may be under way
            self.wake = self.sums.free(taken) or self.wake
            raise
        fresh = dict(zip(copied, taken))
        blocks = [list(self.blocks[p]) if p >= 0 else [] for p in host]
        for r, block in fresh.items():
            blocks[r][-1] = block
        freed = {b for x in self.blocks for b in x} - {b for x in blocks for b in x}
        self.lengths = [self.lengths[p] if p >= 0 else 0 for p in host]
        self.blocks, self._forks = blocks, self._forks + 1
        here.synchronize()
        self.wake = (bool(freed) and self.sums.free(sorted(freed))) or self.wake
        return True

    def compact(self, caches, max_moves=1 << 16):
        """Moves blocks of nearly empty units together (dps.SumManager.compact), in each of
        `caches`, so that units become free: True when residuals wait for them.  Units in
        which others than this batch have blocks stay as they are.  Waits for the steps before
        and for the moves."""
        here = self._between_steps()
        self._ours(caches)
        ours, per = {b for blocks in self.blocks for b in blocks}, self.sums.blocks_per_unit
        moves = list(zip(*self.sums.compact(max_moves)))
        others = {s // per for s, _ in moves if s not in ours}
        left = [d for s, d in moves if s // per in others]
        if left:
            self.sums.free(left)
        src, dst = ([m[i] for m in moves if m[0] // per not in others] for i in range(2))
        if not src:
            return False
        i32 = dict(dtype=torch.int32, device=self.table.device)
        try:
            s, d = torch.tensor(src, **i32), torch.tensor(dst, **i32)
            for cache in caches:
                dps.kv_copy(cache, s, d)
            dps.kv_remap(self.table, s, d)
        except Exception:
            here.synchronize()
            self.sums.free(dst)
            raise
        to = dict(zip(src, dst))
        self.blocks = [[to.get(b, b) for b in blocks] for blocks in self.blocks]
        here.synchronize()
        return self.sums.free(src)

    def end(self, slot):
        """The request of a slot ends: its blocks go back, but for those it shares.  True
        when residuals wait for the units that became free.  The steps that use the blocks,
        the one that grow() has just prepared among them, must have completed: a restore
        worker copies on a stream of its own."""
        mine = self.blocks[slot]
        self.blocks[slot], self.lengths[slot] = [], 0
        self._group_key = None              # the slot's next request shares nothing
        if self._forks:
            others = {b for blocks in self.blocks for b in blocks}
            mine = [b for b in mine if b not in others]
        self._unmapped.discard(slot)
        self._grown.discard(slot)
        return self.sums.free(mine) if mine else False


class AttentionLayer:
    """Attention of a decoder layer: qkv and o are dps.NestedWeight, cache the
    layer's dps.KvCache (FP16 or E4M3), rope the rotation table (of the batch's
    max_tokens positions: past its end rows are NaN); q_weight and k_weight (FP16
    [head_dim]) the head norms' weights, or None without norms.  Made for steps of
    decode tokens: a prompt's rows are taken, at the cost of reading the cache anew for
    each.  groups: those of the batch (PagedBatch), whose shared blocks are then read once
    (without a window).  The buffers between the products are the layer's own, so one call
    runs at a time: calls on several streams are ordered by the caller."""

    def __init__(self, qkv, o, cache, heads, rope, q_weight=None, k_weight=None, rows=256,
                 window=0, groups=0):
        self.qkv, self.o, self.cache, self.heads, self.rope = qkv, o, cache, heads, rope
        self.q_weight, self.k_weight, self.window = q_weight, k_weight, window
        dim, device = cache.head_dim, qkv.hi.device
        f16 = dict(dtype=torch.float16, device=device)
        self._qkv = torch.empty((rows, qkv.n), **f16)
        self._q = torch.empty((rows, heads, dim), **f16)
        self._a = torch.empty((rows, heads, dim), **f16)
        if groups and window:
            raise ValueError("rows that share blocks have no window")
        self.groups = groups
        need = max([256, dps.attn_workspace_bytes(cache, rows, heads)] +
                   [dps.attn_shared_workspace_bytes(cache, m, heads, groups)
                    for m in range(1, rows + 1) if groups] +
                   [dps.workspace_bytes(mode, dps.ACT_FP16, m, w.n, w.k)
                    for mode in (dps.MODE_FULL, dps.MODE_FAST) for w in (qkv, o)
                    for m in range(1, rows + 1)])
        self._ws = torch.empty(need, dtype=torch.uint8, device=device)

    def __call__(self, x, batch, mode, out=None):
        """One step of rows x ([rows][hidden] FP16) as batch.step maps them."""
        rows, step = x.shape[0], batch.step
        if rows != step.pos.shape[0]:
            raise ValueError("x has %d rows, the step's map %d" % (rows, step.pos.shape[0]))
        if self.groups != batch.groups:
            raise ValueError("the layer is for %d groups, the batch has %d" %
                             (self.groups, batch.groups))
        qkv, q, a = self._qkv[:rows], self._q[:rows], self._a[:rows]
        dps.linear(x, self.qkv, mode, out=qkv, workspace=self._ws)
        dps.kv_store(qkv, self.cache, step.slot, self.heads, pos=step.pos, rope=self.rope,
                     q_weight=self.q_weight, k_weight=self.k_weight, q_out=q)
        if self.groups:
            dps.attn_shared(q, self.cache, batch.table, step.kv_len, batch.group_start,
                            batch.shared_len, req=step.req, out=a, workspace=self._ws)
        else:
            dps.attn_decode(q, self.cache, batch.table, step.kv_len, req=step.req, out=a,
                            window=self.window, workspace=self._ws)
        return dps.linear(a.view(rows, -1), self.o, mode, out=out, workspace=self._ws)


class Beams:
    """Beam search over the slots of a PagedBatch, `beams` slots a request: pick() takes
    the logits of a step's rows (a new token in every slot), gives every slot the beam it
    goes on with (PagedBatch.fork: look at the batch's wake then), and returns the tokens of
    the next step.  caches: every layer's.  end: the token that ends a beam (-1: none).
    Ended beams keep their slots, and slots for which there is no beam are empty and have no
    score; both take tokens like the others, whose logits do not count."""

    def __init__(self, batch, caches, beams, vocab, end=-1):
        slots = len(batch.lengths)
        if slots % beams:
            raise ValueError("the batch's slots must be a multiple of beams")
        device = batch.table.device
        self.batch, self.caches, self.beams, self.end = batch, caches, beams, end
        # at first the beams of a request are alike, and one of them counts
        self.score = torch.full((slots // beams, beams), float("-inf"), device=device)
        self.score[:, 0] = 0.0
        self.done = torch.zeros(slots, dtype=torch.uint8, device=device)
        self.tokens = [[] for _ in range(slots)]
        self._step = dps.make_beam_step(slots // beams, beams, device)
        self._ws = torch.empty(max(1, dps.beam_workspace_bytes(slots // beams, beams, vocab, beams)),
                               dtype=torch.uint8, device=device)

    def pick(self, logits):
        """int32 [slots] tokens (-1: no beam), or None if no room is left for the copies of
        blocks that the beams need."""
        step = dps.beam_select(logits, self.score.view(-1), self.beams,
                               done=self.done if self.end >= 0 else None, end=self.end,
                               out=self._step, workspace=self._ws)
        if not self.batch.fork(step.parent.view(-1), self.caches):
            return None
        self.score.copy_(step.score)
        self.done.copy_(step.done.view(-1))
        parents, tokens = step.parent.view(-1).tolist(), step.token.view(-1).clone()
        self.tokens = [self.tokens[p] + [t] if p >= 0 else []
                       for p, t in zip(parents, tokens.tolist())]
        return tokens


def rope_table(max_pos, rot, base=10000.0, device="cuda"):
    """float32 [max_pos][rot]: cosines then sines of pos * base^(-2i / rot)."""
    i = torch.arange(rot // 2, dtype=torch.float64, device=device)
    pos = torch.arange(max_pos, dtype=torch.float64, device=device)[:, None]
    angle = pos * base ** (-2 * i / rot)
    return torch.cat((angle.cos(), angle.sin()), 1).float()


class SharedLayer:
    """A small layer whose two residuals share `units` units of 2 MiB with its KV
    blocks: hidden 1024, 16 query and 4 key/value heads of 64."""

    HIDDEN, HEADS, KV_HEADS, DIM, TOKENS = 1024, 16, 4, 64, 16
    UNIT, LOG2_CHUNK = 2 << 20, 16

    def __init__(self, units=4, batch=4, max_tokens=4096, seed=0, device="cuda", groups=0):
        from . import workloads

        block = 2 * self.KV_HEADS * self.TOKENS * self.DIM * 2
        self.pool = torch.zeros(units * self.UNIT, dtype=torch.uint8, device=device)
        self.sums = dps.SumManager(units, self.UNIT // block, 2)
        shapes = (((self.HEADS + 2 * self.KV_HEADS) * self.DIM, self.HIDDEN),
                  (self.HIDDEN, self.HEADS * self.DIM))
        self.weights, self.nested, targets = [], [], []
        per_unit = self.UNIT >> self.LOG2_CHUNK
        for r, (n, k) in enumerate(shapes):
            w = workloads.weight_fp16(n, k, seed=seed + r)
            chunks = -(-n * k // (1 << self.LOG2_CHUNK))
            slots = self.sums.slots(r, per_unit, chunks).to(device)
            nw = dps.split(w.to(device), dps.Residual(self.pool, slots, self.LOG2_CHUNK))
            self.weights.append(w)
            self.nested.append(nw)
            targets.append((dps.backup(nw.residual, n * k), n * k, nw.residual))
        torch.cuda.synchronize()   # the backups are complete
        self.worker = dps.RestoreWorker(self.sums, targets, per_unit)
        self.batch = PagedBatch(self.sums, batch, max_tokens, self.TOKENS, device=device,
                                groups=groups)
        self.q_weight = torch.ones(self.DIM, dtype=torch.float16, device=device)
        self.rope = rope_table(self.batch.max_tokens, self.DIM, device=device)
        cache = dps.KvCache(self.pool, self.TOKENS, self.KV_HEADS, self.DIM, torch.float16)
        self.layer = AttentionLayer(*self.nested, cache, self.HEADS, self.rope,
                                    self.q_weight, self.q_weight, rows=batch, groups=groups)
        self.cache = cache

    def decode(self, x, new):
        """One token (new[r] = 1) of each active slot; x holds their rows first.  The
        mode is the SUM manager's once the step's blocks are taken."""
        if not self.batch.grow(new):
            return None
        self.batch.map()
        return self.layer(x, self.batch, self.sums.mode)

    def close(self):
        self.worker.close()


def main(steps=1600):
    shared = SharedLayer()
    x = torch.randn(4, SharedLayer.HIDDEN, device="cuda").to(torch.float16)
    names = {dps.MODE_FULL: "full", dps.MODE_FAST: "fast"}
    mode = None
    for t in range(steps):
        y = shared.decode(x, [1] * 4)
        if y is None:
            print("step %d: no room for more KV blocks" % t)
            break
        if shared.sums.mode != mode:
            mode = shared.sums.mode
            print("step %d: %s mode, %s" % (t, names[mode], shared.sums.counts()))
    torch.cuda.synchronize()
    print("%d tokens a request, |y| %.3f" % (shared.batch.lengths[0], y.float().norm()
                                             if y is not None else float("nan")))
    if any([shared.batch.end(r) for r in range(4)]):
        shared.worker.kick()
    shared.worker.wait_idle()
    print("requests ended, residuals restored: %s mode" % names[shared.sums.mode])
    shared.close()


def main_beams(steps=2000, requests=2, beams=4, vocab=32000, prompt=400):
    """Prompts of `prompt` tokens, then beams over a vocabulary until their blocks evict a
    residual, and one beam that is left."""
    slots = requests * beams
    shared = SharedLayer(batch=slots, groups=requests)
    gen = torch.Generator(device="cuda").manual_seed(1)
    head = torch.randn((vocab, SharedLayer.HIDDEN), device="cuda", generator=gen).to(torch.float16)
    embed = torch.randn((vocab, SharedLayer.HIDDEN), device="cuda", generator=gen).to(torch.float16)
    names = {dps.MODE_FULL: "full", dps.MODE_FAST: "fast"}
    search, batch, mode = Beams(shared.batch, [shared.cache], beams, vocab), shared.batch, None
    x = torch.zeros((slots, SharedLayer.HIDDEN), dtype=torch.float16, device="cuda")
    for t in range(prompt):   # in each request's first slot
        x[:requests] = embed[t % vocab:t % vocab + requests]
        y = shared.decode(x, ([1] + [0] * (beams - 1)) * requests)
    batch.fork([r // beams * beams for r in range(slots)], [shared.cache])
    y = y[:requests].repeat_interleave(beams, 0)
    for t in range(steps):
        token = search.pick(y @ head.t())
        if token is None:
            print("step %d: no room for more KV blocks" % t)
            break
        if batch.wake:
            batch.wake = False
            shared.worker.kick()
        y = shared.decode(embed[token.long().clamp(min=0)], [1] * slots)
        if y is None:
            print("step %d: no room for more KV blocks" % t)
            break
        if shared.sums.mode != mode:
            mode = shared.sums.mode
            print("step %d: %s mode, %s" % (t, names[mode], shared.sums.counts()))
    torch.cuda.synchronize()
    print("%d beams of %d tokens in %d blocks, %d of them shared" %
          (slots, batch.lengths[0], len({b for x in batch.blocks for b in x}),
           int(batch.shared_len.sum()) // batch.block_tokens))
    wake = any([batch.end(r) for r in range(1, slots)])
    if batch.compact([shared.cache]) or wake or batch.wake:
        shared.worker.kick()
    shared.worker.wait_idle()
    print("one beam is left, its blocks together: %s mode, %s" %
          (names[shared.sums.mode], shared.sums.counts()))
    shared.close()


if __name__ == "__main__":
    main_beams() if sys.argv[1:] == ["beams"] else main()
