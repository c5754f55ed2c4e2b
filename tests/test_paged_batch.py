"""PagedBatch and Beams on the host: the real bookkeeping and SUM manager, with the
kernels replaced by their definitions on CPU tensors and a cache whose tokens are
numbers of their own, so that every slot's history can be read back."""
import random

import numpy as np
import pytest
import torch

from paper_2609_34380_amd import decode, dps
from test_gpu_branch import fork_oracle

TOKENS = 4  # of a block


class Cache:
    """One layer's blocks, a number a token."""

    def __init__(self, n_blocks):
        self.block_tokens, self.n_blocks = TOKENS, n_blocks
        self.tokens = np.full((n_blocks, TOKENS), -1)


class Stream:
    """The one there is."""

    def wait_stream(self, other):
        raise AssertionError("there is no other")

    def synchronize(self):
        pass


class Host:
    """The entry points that PagedBatch calls, and the capture of map()."""

    def __init__(self):
        self.recorded = None     # calls of a capture under way
        self.log = []            # names of the calls made
        self.fail = None         # the name of a call that is refused

    def enter(self, name):
        if self.fail == name:
            raise ValueError("refused")
        self.log.append(name)

    def map(self, ctx_len, new_len, fresh, table, block_tokens, out=None):
        def run():
            at = row = 0
            for r, (c, n) in enumerate(zip(ctx_len.tolist(), new_len.tolist())):
                have, need = -(-c // block_tokens), -(-(c + n) // block_tokens)
                for col in range(have, need):
                    table[r, col] = fresh[at]
                    at += 1
                out.seq_len[r] = c + n
                for i in range(n):
                    pos = c + i
                    out.slot[row] = int(table[r, pos // block_tokens]) * block_tokens + \
                        pos % block_tokens
                    out.req[row] = r
                    out.pos[row] = pos
                    row += 1
            out.slot[row:] = out.req[row:] = -1
            out.counts[0], out.counts[1] = row, at
        if self.recorded is not None:
            self.recorded.append(run)
        else:
            run()
        return out

    def fork(self, parent, seq_len, table, fresh, block_tokens, n_blocks, out=None, workspace=None):
        self.enter("fork")
        f = fork_oracle(parent.tolist(), seq_len.numpy(), table.numpy(), fresh.tolist(), block_tokens,
                        n_blocks, out.freed.shape[0])
        for to, x in zip(out, f):
            to.copy_(torch.as_tensor(np.array(x), dtype=torch.int32).view(to.shape))
        return out

    def copy(self, cache, src, dst, tokens=None, count=None):
        self.enter("copy")
        n = src.shape[0] if count is None else int(count[0])
        for i in range(n):
            s, d = int(src[i]), int(dst[i])
            part = TOKENS if tokens is None else int(tokens[i])
            cache.tokens[d, :part] = cache.tokens[s, :part]

    def remap(self, table, src, dst):
        self.enter("remap")
        to = dict(zip(src.tolist(), dst.tolist()))
        flat = table.view(-1)
        for i, b in enumerate(flat.tolist()):
            flat[i] = to.get(b, b)
        return table


@pytest.fixture
def host(monkeypatch):
    h, stream = Host(), Stream()
    monkeypatch.setattr(torch.cuda, "current_stream", lambda device=None: stream)
    monkeypatch.setattr(torch.cuda, "is_current_stream_capturing", lambda: h.recorded is not None)
    monkeypatch.setattr(dps, "kv_map", h.map)
    monkeypatch.setattr(dps, "kv_fork", h.fork)
    monkeypatch.setattr(dps, "kv_copy", h.copy)
    monkeypatch.setattr(dps, "kv_remap", h.remap)
    return h


class Life:
    """A batch over a cache, and what every slot's tokens have to be."""

    count = 0

    def __init__(self, sums, slots, columns=16, groups=0, rows=None):
        self.batch = decode.PagedBatch(sums, slots, columns * TOKENS, TOKENS, rows=rows,
                                       device="cpu", groups=groups)
        self.cache = Cache(sums.n_units * sums.blocks_per_unit)
        self.want = [[] for _ in range(slots)]

    def store(self):
        """What a step's layer stores: a new number in every row's slot."""
        step = self.batch.step
        for slot, req in zip(step.slot.tolist(), step.req.tolist()):
            if req >= 0:
                Life.count += 1
                self.cache.tokens.reshape(-1)[slot] = Life.count
                self.want[req].append(Life.count)

    def step(self, new):
        if not self.batch.grow(new):
            return False
        self.batch.map()
        self.store()
        return True

    def fork(self, parents):
        if not self.batch.fork(parents, [self.cache]):
            return False
        self.want = [list(self.want[p]) if p >= 0 else [] for p in parents]
        return True

    def end(self, slot):
        self.want[slot] = []
        return self.batch.end(slot)

    def check(self):
        b = self.batch
        for r, want in enumerate(self.want):
            assert b.lengths[r] == len(want)
            blocks = b.blocks[r]
            assert len(blocks) == -(-len(want) // TOKENS)
            assert b.table[r, :len(blocks)].tolist() == blocks
            got = self.cache.tokens[blocks].reshape(-1)[:len(want)] if blocks else []
            assert list(got) == want, r


def held(*lives):
    return [{b for blocks in life.batch.blocks for b in blocks} for life in lives]


def check(sums, *lives):
    """Each batch's histories, no block in two batches, and none that the manager has given
    out and nobody holds, or the other way round."""
    for life in lives:
        life.check()
    sets = held(*lives)
    every = set().union(*sets)
    assert len(every) == sum(len(s) for s in sets)
    c, per = sums.counts(), sums.blocks_per_unit
    assert len(every) == (c["full"] + c["avail"]) * per - c["free_blocks"]


# ---- slots that end before others go on -------------------------------------------------


def test_fork_after_a_slot_has_ended(host):
    """The simplest case: the ended slot's blocks are no longer anybody's."""
    sums = dps.SumManager(2, 8, 0)
    a = Life(sums, 2)
    for _ in range(6):
        a.step([0, 1])
    for _ in range(9):
        a.step([1, 0])
    a.end(1)
    assert a.fork([0, -1])
    check(sums, a)
    assert a.fork([0, 0])
    check(sums, a)
    a.step([1, 1])
    check(sums, a)


def test_one_request_of_two_has_ended(host):
    """Two prompts of two beams: the first request ends, the second's beams go on."""
    sums = dps.SumManager(2, 16, 0)
    a = Life(sums, 4)
    for t in range(14):
        a.step([1, 0, 1 if t < 10 else 0, 0])
    assert a.fork([0, 0, 2, 2])
    for _ in range(5):
        a.step([1] * 4)
    a.end(0)
    a.end(1)
    for parents in ([-1, -1, 3, 3], [-1, -1, 2, 3], [2, 2, 2, 3]):
        assert a.fork(parents)
        check(sums, a)
        a.step([1 if p >= 0 else 0 for p in parents])
        check(sums, a)


def test_fork_frees_nothing_of_another_batch(host):
    """Two batches on one manager: the second takes the blocks that the first one's slot has
    given back, and keeps them when the first forks."""
    sums = dps.SumManager(2, 8, 0)
    a, b = Life(sums, 2), Life(sums, 1)
    for _ in range(14):
        a.step([1, 0])
    for _ in range(3):
        a.step([0, 1])
    a.end(0)
    for _ in range(15):
        b.step([1])
    assert held(b)[0] & set(range(4))
    assert a.fork([-1, 1])
    check(sums, a, b)
    assert not set(sums.alloc(4)) & (held(a)[0] | held(b)[0])


@pytest.mark.parametrize("seed", range(40))
def test_random_lives(host, seed):
    """Two batches on one manager whose slots grow, fork, change places and end at random,
    in any order, until the manager has no room and on from there."""
    rng = random.Random(seed)
    sums = dps.SumManager(rng.randint(2, 5), rng.choice((4, 8, 16)), rng.randint(0, 2))
    lives = [Life(sums, rng.randint(2, 5), groups=rng.choice((0, 2))) for _ in range(2)]
    for _ in range(200):
        a = rng.choice(lives)
        slots = len(a.want)
        op = rng.random()
        if op < 0.25:
            a.fork([rng.choice([-1] + list(range(slots)) * 2) for _ in range(slots)])
        elif op < 0.45:
            a.end(rng.randrange(slots))
        elif all(n < a.batch.max_tokens for n in a.batch.lengths):
            a.step([int(rng.random() < 0.8) for _ in range(slots)])
        check(sums, *lives)


# ---- moves, beside other holders of blocks ----------------------------------------------


def test_compact_leaves_another_holders_blocks(host):
    """The unit to empty holds another batch's blocks: they stay where its table says, and the
    places that the plan had taken for them are free again."""
    sums = dps.SumManager(2, 8, 0)
    a, b = Life(sums, 2), Life(sums, 1)
    for new, n in (([1, 0], 20), ([0, 1], 12)):    # blocks 0 .. 4 and 5 .. 7
        for _ in range(n):
            a.step(new)
    for _ in range(8):
        b.step([1])                                # 8 and 9
    a.end(1)
    before = sums.counts()
    assert not a.batch.compact([a.cache])
    assert sums.counts() == before and b.batch.blocks == [[8, 9]]
    check(sums, a, b)
    assert "copy" not in host.log
    assert not set(sums.alloc(9)) & {0, 1, 2, 3, 4, 8, 9}


def test_compact_moves_the_units_that_are_its_own(host):
    """Of two units to empty one holds another batch's block: the other is emptied, and the
    residual that waits for it is reported."""
    sums = dps.SumManager(3, 8, 1)
    a, b = Life(sums, 3), Life(sums, 1)
    for r, n in ((0, 20), (1, 12), (2, 8), (1, 24)):   # 8 .. 12, 13 .. 15, 16 and 17, 18 .. 23
        for _ in range(n):
            a.step([int(i == r) for i in range(3)])
    b.step([1])                                    # 0, where the residual was
    assert sums.mode == dps.MODE_FAST and b.batch.blocks == [[0]]
    a.end(1)
    assert a.batch.compact([a.cache])
    assert a.batch.blocks[2] == [14, 15] and b.batch.blocks == [[0]]
    check(sums, a, b)
    assert sums.unit_state(2) == dps.UNIT_FREE
    assert not set(sums.alloc(9)) & (held(a)[0] | {0})


def test_compact_of_one_batch_frees_whole_units(host):
    sums = dps.SumManager(3, 8, 1)
    a = Life(sums, 3)
    for _ in range(32):
        a.step([1, 1, 1])
    assert sums.mode == dps.MODE_FAST
    a.end(0)
    a.end(2)
    assert sums.counts()["free"] == 0
    assert a.batch.compact([a.cache])
    check(sums, a)
    assert sums.counts()["free"] == 2


@pytest.mark.parametrize("seed", range(30))
def test_random_lives_with_moves(host, seed):
    rng = random.Random(1000 + seed)
    sums = dps.SumManager(rng.randint(2, 5), rng.choice((4, 8)), rng.randint(0, 2))
    lives = [Life(sums, rng.randint(1, 4)) for _ in range(rng.randint(1, 3))]
    for _ in range(200):
        a = rng.choice(lives)
        slots = len(a.want)
        op = rng.random()
        if op < 0.15:
            a.fork([rng.choice([-1] + list(range(slots)) * 2) for _ in range(slots)])
        elif op < 0.3:
            a.end(rng.randrange(slots))
        elif op < 0.45:
            a.batch.compact([a.cache], rng.choice((1, 3, 1000)))
        elif all(n < a.batch.max_tokens for n in a.batch.lengths):
            a.step([int(rng.random() < 0.8) for _ in range(slots)])
        check(sums, *lives)


# ---- between a step's grow() and the replay of its captured map() --------------------------


class Captured(Life):
    """Its map() is captured once; a step replays it."""

    def capture(self, host):
        host.recorded = self.recorded = []
        self.batch.map()
        host.recorded = None

    def replay(self):
        for run in self.recorded:
            run()
        self.store()


def same_again(a, host):
    """Nothing has changed when a call is refused."""
    b, log = a.batch, list(host.log)
    state = lambda: (list(b.lengths), [list(x) for x in b.blocks], b.table.tolist(),
                     b.sums.counts(), a.cache.tokens.tolist(), b.ctx_len.tolist(),
                     b.new_len.tolist())
    before = state()
    for call in (lambda: b.fork([0, 0, 1], [a.cache]), lambda: b.compact([a.cache])):
        with pytest.raises(RuntimeError):
            call()
        assert state() == before and host.log == log


@pytest.mark.parametrize("eager_first", [True, False])
def test_fork_and_compact_wait_for_the_replay(host, eager_first):
    sums = dps.SumManager(3, 8, 0)
    a = Captured(sums, 3)
    if eager_first:
        for _ in range(3):
            a.step([1, 1, 1])
    a.capture(host)
    for t in range(30):
        assert a.batch.grow([1, int(t < 20), 1])
        same_again(a, host)
        a.replay()
        check(sums, a)
        if t == 20:
            a.end(1)
            a.batch.compact([a.cache])
        elif t % 3 == 0:
            assert a.fork([0, 2, 0])
        check(sums, a)


def test_capture_after_grow(host):
    """The step that was grown before the capture still has to be replayed."""
    a = Captured(dps.SumManager(2, 8, 0), 3)
    assert a.batch.grow([1, 1, 0])
    a.capture(host)
    same_again(a, host)
    a.replay()
    assert a.fork([0, 1, 0])
    a.check()


def test_an_eager_map_beside_a_capture(host):
    a = Captured(dps.SumManager(2, 8, 0), 3)
    a.capture(host)
    assert a.step([1, 0, 1])
    assert a.fork([0, 2, 0])
    a.check()
    assert a.batch.grow([0, 0, 0])          # nothing to map
    assert a.fork([0, 0, 0])
    a.check()


def test_the_same_lengths_as_in_the_step_before(host):
    """A slot whose new length is what the last step left in the step's arrays."""
    a = Captured(dps.SumManager(2, 8, 0), 3)
    a.capture(host)
    for new in ([1, 1, 1], [1, 0, 0]):
        assert a.batch.grow(new)
        a.replay()
    assert a.fork([1, 1, 2])                # lengths 1, 1, 1; the step's arrays say 2, 1, 1
    assert a.batch.grow([1, 0, 0])
    same_again(a, host)
    a.replay()
    check(a.batch.sums, a)


def test_the_slot_that_grew_has_ended(host):
    a = Captured(dps.SumManager(2, 8, 0), 3)
    a.capture(host)
    assert a.batch.grow([1, 0, 0])
    a.end(0)
    assert a.fork([0, 1, 2])
    a.check()


# ---- calls that are refused below -------------------------------------------------------------


@pytest.mark.parametrize("name", ["fork", "copy", "remap"])
def test_a_refused_call_changes_nothing(host, name):
    """An entry point that refuses its arguments (tensors of another device than the current
    one, too many rows): tables, lists and the manager's blocks are what they were."""
    sums = dps.SumManager(2, 8, 0)
    a = Life(sums, 3)
    for t in range(22):
        a.step([1, int(t < 13), 1])
    a.end(1)
    a.end(2)
    b = a.batch
    state = lambda: (list(b.lengths), [list(x) for x in b.blocks], b.table.tolist(), sums.counts())
    before = state()
    host.fail = name
    calls = [lambda: b.fork([0, 0, 1], [a.cache]), lambda: b.compact([a.cache])]
    for call in {"fork": calls[:1], "copy": calls, "remap": calls[1:]}[name]:
        with pytest.raises(ValueError):
            call()
        assert state() == before
    host.fail = None
    assert a.fork([0, 0, 1])
    check(sums, a)
    b.compact([a.cache])
    check(sums, a)


# ---- residuals that wait ----------------------------------------------------------------------


def test_wake_stays_until_it_is_looked_at(host):
    """A fork frees a unit that an evicted residual waits for; the ones after it free none."""
    sums = dps.SumManager(2, 4, 2)
    a = Life(sums, 2)
    for _ in range(16):
        a.step([1, 1])
    assert sums.mode == dps.MODE_FAST and not a.batch.wake
    assert a.fork([-1, 1])
    assert not a.batch.wake              # every other block: no whole unit
    a.batch.compact([a.cache])
    for _ in range(16):
        a.step([1, 0])
    assert a.fork([-1, 1]) and a.batch.wake
    for _ in range(3):
        assert a.fork([-1, 1]) and a.batch.wake
    a.batch.wake = False
    assert a.fork([-1, 1]) and not a.batch.wake


def test_a_grow_that_is_refused_evicts_nothing(host):
    """A step that is refused takes no blocks, and so evicts nothing."""
    sums = dps.SumManager(2, 4, 1)
    a = Life(sums, 2, rows=20)
    for _ in range(15):
        a.step([1, 0])
    assert a.batch.grow([1, 0]) and sums.mode == dps.MODE_FULL
    with pytest.raises(RuntimeError):
        a.batch.grow([0, 1])
    assert sums.mode == dps.MODE_FULL and a.batch.lengths == [16, 0]
    assert not a.batch.grow([0, 17])         # no room for it anyway
    assert sums.mode == dps.MODE_FULL and a.batch.lengths == [16, 0]


# ---- beams ------------------------------------------------------------------------------------


class Picks:
    """beam_select that hands out given parents and tokens, in the buffers it is given."""

    def __init__(self, picks):
        self.picks = list(picks)

    def __call__(self, logits, score, beams, keep=None, done=None, end=-1, out=None, workspace=None):
        parent, token = self.picks.pop(0)
        out.score.fill_(-1.0)
        out.parent.copy_(torch.tensor(parent, dtype=torch.int32).view(out.parent.shape))
        out.token.copy_(torch.tensor(token, dtype=torch.int32).view(out.token.shape))
        out.done.zero_()
        return out


def test_picked_tokens_stay(host, monkeypatch):
    """What pick() returned is still what it was after the next pick()."""
    monkeypatch.setattr(dps, "beam_select", Picks([([0, 0], [5, 6]), ([1, 0], [7, 8])]))
    a = Life(dps.SumManager(2, 8, 0), 2)
    search = decode.Beams(a.batch, [a.cache], 2, 100)
    a.step([1, 1])
    first = search.pick(torch.zeros(2, 100))
    a.step([1, 1])
    second = search.pick(torch.zeros(2, 100))
    assert first.tolist() == [5, 6] and second.tolist() == [7, 8]
    assert search.tokens == [[6, 7], [5, 8]]
