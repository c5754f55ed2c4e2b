"""A layer and a batch that were made for different numbers of groups."""
import pytest
import torch

from gpu_helpers import DEV
from paper_2609_34380_amd import decode, dps

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("groups", [0, 2])
def test_other_groups_are_refused_before_anything_is_stored(groups):
    shared = decode.SharedLayer(units=4, batch=3, groups=1)
    try:
        other = decode.AttentionLayer(*shared.nested, shared.cache, 16, shared.rope, rows=3,
                                      groups=groups)
        assert shared.batch.grow([1, 1, 1])
        shared.batch.map()
        before = shared.pool.clone()
        x = torch.randn(3, 1024, generator=torch.Generator().manual_seed(1)).to(torch.float16).to(DEV)
        with pytest.raises(ValueError):
            other(x, shared.batch, dps.MODE_FULL)
        assert torch.equal(before, shared.pool)
        shared.layer(x, shared.batch, dps.MODE_FULL)
        assert not torch.equal(before, shared.pool)
    finally:
        torch.cuda.synchronize()
        shared.close()
