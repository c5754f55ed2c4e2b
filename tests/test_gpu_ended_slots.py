"""Sequences that branch after others have ended: the ended slots' rows of the device's
table still name blocks that are nobody's, or another batch's."""
import random

import pytest
import torch

from gpu_helpers import DEV
from paper_2609_34380_amd import decode, dps, graphs
from test_gpu_beams import check_blocks, fork_ref
from test_gpu_decode import Layer64, close

pytestmark = pytest.mark.gpu


class Slots:
    """A shared layer and its definition, stepped together."""

    def __init__(self, slots, seed, groups=0):
        self.shared = decode.SharedLayer(units=4, batch=slots, groups=groups)
        self.batch, self.ref = self.shared.batch, Layer64(self.shared, slots)
        self.gen = torch.Generator().manual_seed(seed)

    def step(self, new):
        active = [r for r, n in enumerate(new) if n]
        x = torch.zeros(len(new), 1024, dtype=torch.float16)
        x[:len(active)] = torch.randn(len(active), 1024, generator=self.gen).to(torch.float16)
        y = self.shared.decode(x.to(DEV), new)
        if active:
            close(y[:len(active)], self.ref.step(x[:len(active)], active, self.shared.sums.mode))

    def fork(self, parents):
        assert self.batch.fork(parents, [self.shared.cache])
        fork_ref(self.ref, parents)

    def end(self, slot):
        torch.cuda.synchronize()
        self.batch.end(slot)
        self.ref.k[slot], self.ref.v[slot] = [], []


def test_fork_after_a_slot_has_ended():
    s = Slots(2, 1)
    try:
        for _ in range(20):
            s.step([0, 1])
        for _ in range(35):
            s.step([1, 0])
        s.end(1)
        for parents in ([0, -1], [0, 0], [1, 0]):
            s.fork(parents)
            check_blocks(s.batch)
            s.step([1 if p >= 0 else 0 for p in parents])
            check_blocks(s.batch)
    finally:
        torch.cuda.synchronize()
        s.shared.close()


def test_another_holder_of_the_manager():
    """What an ended slot gave back is another holder's when the batch forks."""
    s = Slots(2, 2)
    try:
        sums = s.shared.sums
        for _ in range(40):
            s.step([1, 1])
        before = set(s.batch.blocks[0])
        s.end(0)
        theirs = sums.alloc(3)
        assert before == set(theirs)
        s.fork([-1, 1])
        s.step([0, 1])
        more = sums.alloc(5)
        assert not set(more) & (set(theirs) | set(s.batch.blocks[1]))
        sums.free(theirs + more)
        check_blocks(s.batch)
    finally:
        torch.cuda.synchronize()
        s.shared.close()


def test_moves_beside_another_holder():
    """Another holder's blocks in the unit that is nearly empty: they and their bytes stay."""
    s = Slots(4, 3)
    try:
        sums, pool = s.shared.sums, s.shared.pool
        per = sums.blocks_per_unit
        for _ in range(16 * per // 4):
            s.step([1, 1, 1, 1])                        # one unit
        theirs = sums.alloc(3)                          # the next one's first
        block = pool.numel() // (sums.n_units * per)
        for b in theirs:
            pool[b * block:(b + 1) * block] = 0x5A
        s.end(0)
        assert not s.batch.compact([s.shared.cache])
        s.step([0, 1, 1, 1])
        assert all(bool((pool[b * block:(b + 1) * block] == 0x5A).all()) for b in theirs)
        assert not set(sums.alloc(20)) & (set(theirs) | {b for x in s.batch.blocks for b in x})
    finally:
        torch.cuda.synchronize()
        s.shared.close()


@pytest.mark.parametrize("seed", range(3))
def test_random_ends_and_forks(seed):
    """Ends, forks, moves and steps in any order, with none or several of a kind together."""
    rng = random.Random(seed)
    slots = 4
    s = Slots(slots, seed, groups=2)
    try:
        after_end = 0
        ended = False
        for _ in range(120):
            op = rng.random()
            if op < 0.2:
                after_end += ended
                s.fork([rng.choice([-1] + list(range(slots)) * 2) for _ in range(slots)])
                ended = False
            elif op < 0.35:
                s.end(rng.randrange(slots))
                ended = True
            elif op < 0.4:
                s.batch.compact([s.shared.cache])
            else:
                s.step([int(rng.random() < 0.8) for _ in range(slots)])
                ended = False
            check_blocks(s.batch)
        assert after_end > 1
    finally:
        torch.cuda.synchronize()
        s.shared.close()


def test_fork_and_compact_wait_for_the_replay():
    """A step is grown, and its map() and layer are in a graph: until the replay its blocks
    are in no table, and fork and compact are refused; after it they do what they always do."""
    s = Slots(3, 4, groups=2)
    try:
        batch, shared = s.batch, s.shared
        x = torch.zeros(3, 1024, dtype=torch.float16, device=DEV)
        y = {m: torch.zeros_like(x) for m in graphs.ModeGraphs.MODES}

        def step(m, mode):
            batch.map()
            shared.layer(x, batch, mode, out=y[mode])

        steps = graphs.ModeGraphs(step, (3,))
        steps.capture()
        torch.cuda.synchronize()
        for t in range(60):
            assert batch.grow([1, 1, 1])
            table, lengths, counts = batch.table.clone(), list(batch.lengths), shared.sums.counts()
            for call in (lambda: batch.fork([0, 0, 2], [shared.cache]),
                         lambda: batch.compact([shared.cache])):
                with pytest.raises(RuntimeError):
                    call()
            assert torch.equal(table, batch.table) and lengths == batch.lengths
            assert counts == shared.sums.counts()
            x.copy_(torch.randn(3, 1024, generator=s.gen).to(torch.float16))
            steps.stream.wait_stream(torch.cuda.current_stream())
            with torch.cuda.stream(steps.stream):
                steps.replay(3, shared.sums.mode)
            torch.cuda.synchronize()
            close(y[shared.sums.mode], s.ref.step(x.cpu(), [0, 1, 2], shared.sums.mode))
            check_blocks(batch)
            if t % 7 == 6:
                s.fork([t % 3, 1, 0])
            elif t % 11 == 10:
                s.end(t % 3)
                batch.compact([shared.cache])
            check_blocks(batch)
    finally:
        torch.cuda.synchronize()
        s.shared.close()


@pytest.mark.parametrize("rows,cols", [(3, 20), (64, 700)])
def test_fork_without_blocks_to_list(rows, cols):
    """n_blocks = 0: tables and copies as ever, nothing freed (small and large tables)."""
    gen = torch.Generator().manual_seed(rows)
    table = torch.randperm(rows * cols, generator=gen).int().view(rows, cols)
    lens = torch.randint(1, cols * 16, (rows,), generator=gen).int()
    parent = torch.randint(0, rows, (rows,), generator=gen).int()
    fresh = torch.arange(rows, dtype=torch.int32) + rows * cols
    got = [dps.kv_fork(parent.to(DEV), lens.to(DEV), table.to(DEV), fresh.to(DEV), 16, n)
           for n in (0, rows * cols + rows)]
    for name in ("table", "seq_len", "src", "dst", "tokens"):
        assert torch.equal(*[getattr(f, name) for f in got]), name
    assert got[0].counts.tolist() == [int(got[1].counts[0]), 0] and got[0].freed.numel() == 0
    assert int(got[1].counts[1]) > 0
