"""Steps of a paged batch whose host work, graphs and requests come in other orders than
one after the other on one stream."""
import pytest
import torch

from gpu_helpers import DEV
from paper_2609_34380_amd import decode, dps, graphs

pytestmark = pytest.mark.gpu

FULL, FAST = dps.MODE_FULL, dps.MODE_FAST


def news(t):
    return [1, t % 2, 1, 0 if t < 5 else 1]


@pytest.mark.parametrize("captured", [True, False])
def test_grow_waits_for_steps_on_another_stream(captured):
    """Every step is held up on its stream while the host goes on to the next grow():
    the step still sees its own lengths and blocks.  Nothing else orders the two."""
    slow, plain = (decode.SharedLayer(units=4, batch=4, seed=9) for _ in range(2))
    try:
        gen = torch.Generator().manual_seed(4)
        xs = torch.randn(40, 4, slow.HIDDEN, generator=gen).to(torch.float16).to(DEV)
        want = []
        for t in range(40):
            assert plain.batch.grow(news(t))
            plain.batch.map()
            want.append(plain.layer(xs[t], plain.batch, FULL if t % 3 else FAST).clone())
        x = torch.zeros_like(xs[0])
        y = {m: torch.zeros_like(x) for m in graphs.ModeGraphs.MODES}

        def step(m, mode):
            slow.batch.map()
            slow.layer(x, slow.batch, mode, out=y[mode])

        steps = graphs.ModeGraphs(step, (4,))
        if captured:
            steps.capture()
        torch.cuda.synchronize()
        got = []
        for t in range(40):
            mode = FULL if t % 3 else FAST
            assert slow.batch.grow(news(t))
            with torch.cuda.stream(steps.stream):
                torch.cuda._sleep(1_000_000)
                x.copy_(xs[t])
                if captured:
                    steps.replay(4, mode)
                else:
                    step(4, mode)
                got.append(y[mode].clone())
        torch.cuda.synchronize()
        assert slow.batch.lengths == plain.batch.lengths
        for t in range(40):
            assert torch.equal(got[t], want[t]), t
    finally:
        torch.cuda.synchronize()
        slow.close()
        plain.close()


def test_grow_again_before_map_is_refused():
    """The blocks of a step that was never mapped would be in no table: the slot's next
    rows would read what an earlier request left there."""
    sums = dps.SumManager(1, 8, 0)
    batch = decode.PagedBatch(sums, 2, 64, 16)
    assert batch.grow([1, 0])
    free = sums.counts()["free_blocks"]
    for new in ([0, 1], [1, 1], [0, 0]):
        with pytest.raises(RuntimeError):
            batch.grow(new)
    assert batch.lengths == [1, 0] and sums.counts()["free_blocks"] == free
    batch.map()
    assert batch.step.slot.tolist()[0] == batch.blocks[0][0] * 16
    assert batch.grow([0, 0]) and batch.grow([0, 1])     # nothing to map between these
    batch.map()
    assert batch.step.slot.tolist()[0] == batch.blocks[1][0] * 16
    assert batch.grow([1, 1])
    batch.map()
    assert batch.step.slot.tolist() == [b[0] * 16 + 1 for b in batch.blocks]
    assert batch.grow([1, 0])
    batch.end(0)                                         # the only slot that grew is gone
    assert batch.grow([0, 1])


def test_shared_layer_to_its_batchs_last_token():
    """max_tokens inside a block: the positions up to the block's end are rotated too."""
    short, wide = (decode.SharedLayer(units=4, batch=1, max_tokens=n, seed=2) for n in (21, 4096))
    try:
        gen = torch.Generator().manual_seed(5)
        for t in range(32):
            x = torch.randn(1, short.HIDDEN, generator=gen).to(torch.float16).to(DEV)
            got, want = short.decode(x, [1]), wide.decode(x, [1])
            assert bool(torch.isfinite(want).all()) and torch.equal(got, want), t
        with pytest.raises(ValueError):
            short.decode(x, [1])
    finally:
        torch.cuda.synchronize()
        short.close()
        wide.close()
