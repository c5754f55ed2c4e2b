"""The attention half of a decoder layer, end to end: nested products, step maps,
the store and the attention over KV blocks that share memory with the residuals.
Checked against the layer's definition in 64 bits on the CPU (rounded to FP16
where the layer stores FP16), through eviction, fast mode and restore, and from a
captured graph."""
import numpy as np
import pytest
import torch

from gpu_helpers import DEV
from paper_2609_34380_amd import decode, dps, graphs

pytestmark = pytest.mark.gpu

FULL, FAST = dps.MODE_FULL, dps.MODE_FAST


def f16(x):
    return x.to(torch.float16).double()


class Layer64:
    """The layer in 64 bits, its own history of keys and values."""

    def __init__(self, shared, batch):
        self.w = [w.double() for w in shared.weights]
        # fast mode multiplies by the upper bytes: two mantissa bits of each word
        self.fast = [(w.view(torch.int16) & -256).view(torch.float16).double()
                     for w in shared.weights]
        self.rope = shared.rope.cpu().double()
        self.s = shared
        self.k = [[] for _ in range(batch)]
        self.v = [[] for _ in range(batch)]

    def step(self, x, active, mode):
        s, half = self.s, self.s.DIM // 2
        wqkv, wo = self.w if mode == FULL else self.fast
        qkv = f16(x.double() @ wqkv.t()).view(len(active), -1, s.DIM)
        out = []
        for row, r in enumerate(active):
            cs, sn = self.rope[len(self.k[r])][:half], self.rope[len(self.k[r])][half:]

            def turned(h):
                h = h / torch.sqrt((h ** 2).mean(-1, keepdim=True) + 1e-6)
                a, b = h[:, :half], h[:, half:]
                return f16(torch.cat((a * cs - b * sn, b * cs + a * sn), 1))

            q = turned(qkv[row, :s.HEADS])
            self.k[r].append(turned(qkv[row, s.HEADS:s.HEADS + s.KV_HEADS]))
            self.v[r].append(qkv[row, s.HEADS + s.KV_HEADS:])
            k = torch.stack(self.k[r], 1).repeat_interleave(s.HEADS // s.KV_HEADS, 0)
            v = torch.stack(self.v[r], 1).repeat_interleave(s.HEADS // s.KV_HEADS, 0)
            p = torch.softmax((k * q[:, None]).sum(-1) * s.DIM ** -0.5, 1)
            out.append(f16((p[..., None] * v).sum(1)).reshape(-1))
        return torch.stack(out) @ wo.t()


def close(y, want):
    """Four stored FP16 results on the way, 2^-11 of their size each at most."""
    err = float((y.cpu().double() - want).norm() / want.norm())
    assert err <= 4 * 2.0 ** -11, err


def test_layer_through_eviction_and_restore():
    shared = decode.SharedLayer(units=4, batch=4)
    try:
        ref = Layer64(shared, 4)
        gen = torch.Generator().manual_seed(3)
        modes = []
        for t in range(40):
            # slot 2 is idle, slot 3 joins late
            new = [1, 1, 0, 1 if t > 7 else 0]
            if t == 20:   # another tenant fills the free units: the residuals go
                taken = []
                while shared.sums.mode == FULL:
                    taken += shared.sums.alloc(64)
            active = [r for r in range(4) if new[r]]
            x = torch.randn(4, shared.HIDDEN, generator=gen).to(torch.float16)
            y = shared.decode(x.to(DEV), new)
            mode = shared.sums.mode
            modes.append(mode)
            close(y[:len(active)], ref.step(x[:len(active)], active, mode))
            # rows of the graph's batch that no request uses attend nothing
            assert bool((y[len(active):] == 0).all())
            if t == 30:   # it leaves, a unit of its own is free: the residual comes back there
                assert shared.sums.free(taken)
                shared.worker.kick()
                shared.worker.wait_idle()
        assert modes[0] == FULL and modes[25] == FAST and modes[-1] == FULL
    finally:
        torch.cuda.synchronize()
        shared.close()


def test_captured_step_replays_as_requests_grow():
    """Map, products, store and attention in one graph per mode; lengths, block ids
    and inputs change between the replays."""
    shared = decode.SharedLayer(units=4, batch=4, seed=9)
    eager = decode.SharedLayer(units=4, batch=4, seed=9)
    try:
        x = torch.zeros(4, shared.HIDDEN, dtype=torch.float16, device=DEV)
        y = {m: torch.zeros_like(x) for m in graphs.ModeGraphs.MODES}

        def step(m, mode):
            shared.batch.map()
            shared.layer(x, shared.batch, mode, out=y[mode])

        mg = graphs.ModeGraphs(step, (4,)).capture()   # runs with no request active
        gen = torch.Generator().manual_seed(4)
        for t in range(24):
            mode = FULL if t % 3 else FAST
            new = [1, t % 2, 1, 0 if t < 5 else 1]
            x.copy_(torch.randn(4, shared.HIDDEN, generator=gen).to(torch.float16))
            assert shared.batch.grow(new) and eager.batch.grow(new)
            eager.batch.map()
            want = eager.layer(x, eager.batch, mode)
            torch.cuda.synchronize()
            mg.replay(4, mode)
            torch.cuda.synchronize()
            assert torch.equal(y[mode], want)
        assert shared.batch.lengths == eager.batch.lengths == [24, 12, 24, 19]
    finally:
        torch.cuda.synchronize()
        shared.close()
        eager.close()


def test_batch_refusals():
    sums = dps.SumManager(1, 4, 0)
    batch = decode.PagedBatch(sums, 2, 48, 16, rows=40)
    with pytest.raises(ValueError):
        batch.grow([1])
    with pytest.raises(ValueError):
        batch.grow([40, 1])
    assert batch.grow([33, 1]) and batch.lengths == [33, 1]
    with pytest.raises(ValueError):
        batch.grow([16, 0])
    assert not batch.grow([0, 16]) and batch.lengths == [33, 1]   # four blocks, all taken
    batch.map()
    assert batch.step.q_start.tolist() == [0, 33, 34] and batch.step.counts.tolist() == [34, 4]
    assert not batch.end(0) and batch.grow([0, 16])
    batch.map()
    assert batch.step.pos[:16].tolist() == list(range(1, 17))
    assert np.unique(batch.table[1, :2].cpu().numpy()).size == 2
