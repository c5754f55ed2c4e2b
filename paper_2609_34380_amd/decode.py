"""The attention half of a decoder layer on nested weights, over KV blocks of the
shared region (Sec. IV-B "Shared Region": one memory that residual planes and
paged KV blocks take turns in).

    PagedBatch      the requests of a serving loop: KV blocks from a SUM
                    manager, block tables and slot maps built on the GPU
    AttentionLayer  QKV product, head norms with rotation into the cache,
                    attention, O product, in the precision mode of the pass

Everything an AttentionLayer and PagedBatch.map() enqueue reads lengths, tables
and slots on the device, so a step can be captured (graphs.ModeGraphs) and
replayed while requests grow.

Run as a program (python -m paper_2609_34380_amd.decode), it decodes with a small
layer until KV blocks push the residuals out, goes on in fast mode, and returns
to full mode once the requests end and the residuals are restored.
"""
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
    returns.  Before the next grow() a caller waits for a graph replayed elsewhere than
    on the stream of its capture."""

    def __init__(self, sums, batch, max_tokens, block_tokens, rows=None, device="cuda"):
        self.sums, self.block_tokens = sums, block_tokens
        self.lengths = [0] * batch           # tokens in the cache, after the last step
        self.blocks = [[] for _ in range(batch)]
        columns = -(-max_tokens // block_tokens)
        self.max_tokens = columns * block_tokens
        i32 = dict(dtype=torch.int32, device=device)
        self.table = torch.full((batch, columns), -1, **i32)
        self.ctx_len, self.new_len = torch.zeros(batch, **i32), torch.zeros(batch, **i32)
        self.rows = batch if rows is None else rows
        # a step never takes more than a block a slot and what its rows fill
        self.fresh = torch.full((batch + self.rows // block_tokens + 1,), -1, **i32)
        self.step = dps.make_kv_map(batch, self.rows, self.ctx_len.device)
        # that the buffers were filled on, or map() was called on
        self._streams = [torch.cuda.current_stream(self.table.device)]
        self._unmapped = set()               # slots that grew since the last map()
        self._captured = False               # map() is in a graph: replays are not seen here

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
        taken = self.sums.alloc(sum(need))
        if taken is None:
            return False
        if self._unmapped and not self._captured:
            self.sums.free(taken)
            raise RuntimeError("the tokens of the last grow() are not mapped")
        here = torch.cuda.current_stream(self.table.device)
        for stream in self._streams:   # earlier steps read what is replaced here
            if stream != here:
                here.wait_stream(stream)
        self.ctx_len.copy_(torch.tensor(self.lengths, dtype=torch.int32))
        self.new_len.copy_(torch.tensor(new, dtype=torch.int32))
        if taken:
            self.fresh[:len(taken)].copy_(torch.tensor(taken, dtype=torch.int32))
        at = 0
        for r, n in enumerate(need):
            self.blocks[r] += taken[at:at + n]
            at += n
            self.lengths[r] += new[r]
        self._unmapped = {r for r, n in enumerate(new) if n}
        return True

    def map(self):
        """Enqueue the step's block tables and slot maps."""
        stream = torch.cuda.current_stream(self.table.device)
        if stream not in self._streams:
            self._streams.append(stream)
        self._captured = self._captured or torch.cuda.is_current_stream_capturing()
        self._unmapped.clear()
        return dps.kv_map(self.ctx_len, self.new_len, self.fresh, self.table, self.block_tokens,
                          out=self.step)

    def end(self, slot):
        """The request of a slot ends: its blocks go back.  True when residuals wait
        for the units that became free.  The steps that use the blocks, the one that
        grow() has just prepared among them, must have completed: a restore worker
        copies on a stream of its own."""
        wake = self.sums.free(self.blocks[slot]) if self.blocks[slot] else False
        self.blocks[slot], self.lengths[slot] = [], 0
        self._unmapped.discard(slot)
        return wake


class AttentionLayer:
    """Attention of a decoder layer: qkv and o are dps.NestedWeight, cache the
    layer's dps.KvCache (FP16 or E4M3), rope the rotation table (of the batch's
    max_tokens positions: past its end rows are NaN); q_weight and k_weight (FP16
    [head_dim]) the head norms' weights, or None without norms.  Made for steps of
    decode tokens: a prompt's rows are taken, at the cost of reading the cache anew for
    each.  The buffers between the products are the layer's own, so one call runs at a
    time: calls on several streams are ordered by the caller."""

    def __init__(self, qkv, o, cache, heads, rope, q_weight=None, k_weight=None, rows=256,
                 window=0):
        self.qkv, self.o, self.cache, self.heads, self.rope = qkv, o, cache, heads, rope
        self.q_weight, self.k_weight, self.window = q_weight, k_weight, window
        dim, device = cache.head_dim, qkv.hi.device
        f16 = dict(dtype=torch.float16, device=device)
        self._qkv = torch.empty((rows, qkv.n), **f16)
        self._q = torch.empty((rows, heads, dim), **f16)
        self._a = torch.empty((rows, heads, dim), **f16)
        need = max([256, dps.attn_workspace_bytes(cache, rows, heads)] +
                   [dps.workspace_bytes(mode, dps.ACT_FP16, m, w.n, w.k)
                    for mode in (dps.MODE_FULL, dps.MODE_FAST) for w in (qkv, o)
                    for m in range(1, rows + 1)])
        self._ws = torch.empty(need, dtype=torch.uint8, device=device)

    def __call__(self, x, batch, mode, out=None):
        """One step of rows x ([rows][hidden] FP16) as batch.step maps them."""
        rows, step = x.shape[0], batch.step
        if rows != step.pos.shape[0]:
            raise ValueError("x has %d rows, the step's map %d" % (rows, step.pos.shape[0]))
        qkv, q, a = self._qkv[:rows], self._q[:rows], self._a[:rows]
        dps.linear(x, self.qkv, mode, out=qkv, workspace=self._ws)
        dps.kv_store(qkv, self.cache, step.slot, self.heads, pos=step.pos, rope=self.rope,
                     q_weight=self.q_weight, k_weight=self.k_weight, q_out=q)
        dps.attn_decode(q, self.cache, batch.table, step.kv_len, req=step.req, out=a,
                        window=self.window, workspace=self._ws)
        return dps.linear(a.view(rows, -1), self.o, mode, out=out, workspace=self._ws)


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

    def __init__(self, units=4, batch=4, max_tokens=4096, seed=0, device="cuda"):
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
        self.batch = PagedBatch(self.sums, batch, max_tokens, self.TOKENS, device=device)
        self.q_weight = torch.ones(self.DIM, dtype=torch.float16, device=device)
        self.rope = rope_table(self.batch.max_tokens, self.DIM, device=device)
        cache = dps.KvCache(self.pool, self.TOKENS, self.KV_HEADS, self.DIM, torch.float16)
        self.layer = AttentionLayer(*self.nested, cache, self.HEADS, self.rope,
                                    self.q_weight, self.q_weight, rows=batch)

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


if __name__ == "__main__":
    main()
