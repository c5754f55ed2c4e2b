"""Sequences that branch, end to end: a layer over shared blocks, beams picked from its
outputs, slots forked, blocks moved together and residuals back, against the layer's
definition in 64 bits with a history of its own for every slot."""
import random

import numpy as np
import pytest
import torch

from gpu_helpers import DEV
from paper_2609_34380_amd import decode, dps
from test_gpu_branch import beam_oracle
from test_gpu_decode import Layer64, close

pytestmark = pytest.mark.gpu


def fork_ref(ref, parents):
    ref.k, ref.v = ([list(h[p]) if p >= 0 else [] for p in parents] for h in (ref.k, ref.v))


def check_blocks(batch):
    """Every slot's table row is its host list; only whole blocks are shared; the manager
    has handed out what is in them and nothing else."""
    table = batch.table.tolist()
    owners = {}
    for r, blocks in enumerate(batch.blocks):
        n = -(-batch.lengths[r] // batch.block_tokens)
        assert len(blocks) == n and table[r][:n] == blocks
        for i, b in enumerate(blocks):
            owners.setdefault(b, []).append((r, i))
    for b, held in owners.items():
        if len(held) > 1:
            assert len({i for _, i in held}) == 1
            assert all((i + 1) * batch.block_tokens <= batch.lengths[r] for r, i in held)
    c = batch.sums.counts()
    per = batch.sums.blocks_per_unit
    assert len(owners) == c["full"] * per + c["avail"] * per - c["free_blocks"]


def test_beam_search_over_a_layer():
    """Two requests of three beams: prompts of different lengths, twenty picks."""
    beams, slots, vocab = 3, 6, 2000
    shared = decode.SharedLayer(units=4, batch=slots, groups=2)
    try:
        batch, ref = shared.batch, Layer64(shared, slots)
        gen = torch.Generator().manual_seed(5)
        rand = lambda *s: torch.randn(*s, generator=gen).to(torch.float16)
        head, embed = rand(vocab, 1024), rand(vocab, 1024)
        y = None
        for t in range(41):                       # 41 tokens, and 23 in the other slot
            active = [0, 3] if t < 23 else [0]
            x = torch.zeros(slots, 1024, dtype=torch.float16)
            x[:len(active)] = rand(len(active), 1024)
            out = shared.decode(x.to(DEV), [1 if r in active else 0 for r in range(slots)])
            close(out[:len(active)], ref.step(x[:len(active)], active, dps.MODE_FULL))
            if t == 22:
                y3 = out[1].clone()
        y0 = out[0]
        assert batch.fork([0, 0, 0, 3, 3, 3], [shared.cache])
        fork_ref(ref, [0, 0, 0, 3, 3, 3])
        check_blocks(batch)
        y = torch.stack([y0] * 3 + [y3] * 3)
        search = decode.Beams(batch, [shared.cache], beams, vocab, end=7)
        score, done = np.array([0.0, -np.inf, -np.inf] * 2, np.float32), np.zeros(slots)
        grouped = False
        for t in range(20):
            logits = y.float().cpu() @ head.float().t() / 16
            want = beam_oracle(logits.double().numpy(), score, beams, beams, done, 7)
            token = search.pick(logits.to(DEV))
            parents = want[1].reshape(-1)
            assert token.tolist() == want[2].reshape(-1).tolist()
            assert search.done.tolist() == want[3].reshape(-1).tolist()
            fork_ref(ref, parents)
            check_blocks(batch)
            score, done = search.score.cpu().numpy().reshape(-1), want[3].reshape(-1)
            x = embed[token.cpu().long()]
            y = shared.decode(x.to(DEV), [1] * slots)
            assert batch.group_start.tolist() == [0, 3, 6]
            grouped = grouped or batch.shared_len.tolist() == [32, 16]
            close(y, ref.step(x, list(range(slots)), shared.sums.mode))
        assert grouped
        assert all(len(t) == 20 for t in search.tokens)
        for r in range(slots):
            batch.end(r)
        c = shared.sums.counts()
        assert c["avail"] == c["full"] == 0
    finally:
        shared.close()


@pytest.mark.parametrize("seed", range(3))
def test_random_life(seed):
    """Slots grow, fork, change places and end at random, with compaction in between; the
    layer's outputs stay those of every slot's own history."""
    rng = random.Random(seed)
    slots = 5
    shared = decode.SharedLayer(units=4, batch=slots, groups=rng.choice((1, 3, 5)))
    try:
        batch, ref = shared.batch, Layer64(shared, slots)
        gen = torch.Generator().manual_seed(seed)
        for t in range(60):
            op = rng.random()
            if op < 0.15:
                parents = [rng.choice([-1] + list(range(slots)) * 2) for _ in range(slots)]
                assert batch.fork(parents if rng.random() < 0.5 else
                                  torch.tensor(parents, dtype=torch.int32, device=DEV), [shared.cache])
                fork_ref(ref, parents)
            elif op < 0.2:
                r = rng.randrange(slots)
                torch.cuda.synchronize()
                batch.end(r)
                ref.k[r], ref.v[r] = [], []
            elif op < 0.3:
                batch.compact([shared.cache], rng.choice((2, 1000)))
            active = [r for r in range(slots) if rng.random() < 0.8]
            x = torch.zeros(slots, 1024, dtype=torch.float16)
            x[:len(active)] = torch.randn(len(active), 1024, generator=gen).to(torch.float16)
            y = shared.decode(x.to(DEV), [1 if r in active else 0 for r in range(slots)])
            if active:
                close(y[:len(active)], ref.step(x[:len(active)], active, shared.sums.mode))
            check_blocks(batch)
    finally:
        shared.close()


def test_another_request_in_a_slot_of_a_group():
    """A slot that shared a prefix ends; the request that comes after it grows past that
    prefix's length with the same slots in every step."""
    shared = decode.SharedLayer(units=4, batch=3, groups=2)
    try:
        batch, ref = shared.batch, Layer64(shared, 3)
        gen = torch.Generator().manual_seed(11)

        def step(active):
            x = torch.zeros(3, 1024, dtype=torch.float16)
            x[:len(active)] = torch.randn(len(active), 1024, generator=gen).to(torch.float16)
            y = shared.decode(x.to(DEV), [1 if r in active else 0 for r in range(3)])
            close(y[:len(active)], ref.step(x[:len(active)], active, shared.sums.mode))

        for _ in range(35):
            step([0])
        assert batch.fork([0, 0, 0], [shared.cache])
        fork_ref(ref, [0, 0, 0])
        step([0, 1, 2])
        assert batch.shared_len.tolist() == [32, 0]
        for slot in (1, 0):
            torch.cuda.synchronize()
            batch.end(slot)
            ref.k[slot], ref.v[slot] = [], []
            for _ in range(40):
                step([0, 1, 2])
            assert batch.shared_len.tolist() == [0, 0]
            check_blocks(batch)
    finally:
        shared.close()


def test_compaction_brings_full_mode_back():
    """Blocks of slots that live on are scattered over the units that evicted residuals
    wait for; together they leave one free, and the outputs stay what they were."""
    shared = decode.SharedLayer(units=3, batch=4, max_tokens=4096, groups=4)
    try:
        batch, sums = shared.batch, shared.sums
        x = torch.randn(4, 1024, generator=torch.Generator().manual_seed(1)).to(torch.float16).to(DEV)
        t = 0
        while sums.mode == dps.MODE_FULL:
            assert shared.decode(x, [1] * 4) is not None
            t += 1
        for _ in range(40):
            shared.decode(x, [1] * 4)
        torch.cuda.synchronize()
        for r in (0, 2, 3):
            batch.end(r)
        assert sums.counts()["free"] == 0
        # slot 1 attends the same keys and values before and after the move
        q = torch.randn(1, 16, 64, generator=torch.Generator().manual_seed(2)).to(torch.float16).to(DEV)
        n = torch.tensor([batch.lengths[1]], dtype=torch.int32, device=DEV)
        attend = lambda: dps.attn_decode(q, shared.cache, batch.table, n, req=torch.ones_like(n))
        before = attend()
        assert batch.compact([shared.cache])
        check_blocks(batch)
        assert torch.equal(before, attend())
        shared.worker.kick()
        shared.worker.wait_idle()
        assert sums.mode == dps.MODE_FULL and sums.counts()["evicted"] == 0
        assert torch.equal(before, attend())
    finally:
        shared.close()


def test_refusals():
    shared = decode.SharedLayer(units=4, batch=3)
    try:
        batch = shared.batch
        with pytest.raises(ValueError):
            batch.fork([0, 0], [shared.cache])
        with pytest.raises(ValueError):
            batch.fork([0, 3, 1], [shared.cache])
        for bad in (torch.int64, torch.float32):
            with pytest.raises(ValueError):
                batch.fork(torch.zeros(3, dtype=bad, device=DEV), [shared.cache])
        with pytest.raises(ValueError):
            batch.fork(torch.zeros(3, dtype=torch.int32), [shared.cache])
        pool = torch.zeros(1 << 20, dtype=torch.uint8, device=DEV)
        for tokens in (shared.TOKENS, 2 * shared.TOKENS):    # too few blocks, others
            cache = dps.KvCache(pool, tokens, 8, 128, torch.float16)
            for call in (lambda: batch.fork([0, 0, 0], [cache]), lambda: batch.compact([cache])):
                with pytest.raises(ValueError):
                    call()
        assert sum(shared.sums.counts()[n] for n in ("avail", "full")) == 0   # nothing taken
        assert batch.grow([1, 0, 0])
        with pytest.raises(RuntimeError):
            batch.fork([0, 0, 0], [shared.cache])
        with pytest.raises(RuntimeError):
            batch.compact([shared.cache])
        batch.map()
        assert not batch.compact([shared.cache])
        with pytest.raises(ValueError):
            decode.Beams(batch, [shared.cache], 2, 100)
        with pytest.raises(ValueError):
            decode.AttentionLayer(*shared.nested, shared.cache, 16, shared.rope, groups=1, window=4)
        other = decode.AttentionLayer(*shared.nested, shared.cache, 16, shared.rope, rows=3, groups=2)
        with pytest.raises(ValueError):
            other(torch.zeros(3, 1024, dtype=torch.float16, device=DEV), batch, dps.MODE_FULL)
    finally:
        shared.close()
