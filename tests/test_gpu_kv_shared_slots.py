"""Rows of one store that name the same slot: what the slot then holds comes from these
rows, piece by piece, and nothing else is touched."""
import pytest
import torch

from gpu_helpers import DEV
from paper_2609_34380_amd import dps

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", [torch.float16, torch.float8_e4m3fn])
def test_rows_of_one_slot(dtype):
    rows, tokens, heads, dim = 64, 16, 2, 128
    x = torch.randn(rows, 3 * heads * dim, generator=torch.Generator().manual_seed(1))
    x = x.to(torch.float16).to(DEV)
    slot = torch.arange(rows, device=DEV)
    slot[40:] = slot[:24]                      # 24 slots named twice
    block = 2 * heads * tokens * dim * dtype.itemsize

    def stored(part):
        pool = torch.full((5 * block,), 0x55, dtype=torch.uint8, device=DEV)
        cache = dps.KvCache(pool, tokens, heads, dim, dtype)
        dps.kv_store(x[part], cache, slot[part], heads)
        return pool.view(-1, 8 * dtype.itemsize).cpu()

    first, last, both = stored(slice(0, 40)), stored(slice(24, 64)), stored(slice(0, 64))
    one = (both == first).all(1)
    assert bool((one | (both == last).all(1)).all())
    named_once = stored(slice(24, 40))
    untouched = (named_once == 0x55).all(1)
    assert torch.equal(both[~untouched], named_once[~untouched])
    assert bool((both.view(5, -1)[3:] == 0x55).all())
