"""A head_dim that no row has is refused as other bad arguments are, before anything is made of it."""
import pytest
import torch

from paper_2406_11016_amd import paged_cache
from paper_2406_11016_amd.binding import SpecVerifyError


@pytest.mark.parametrize("head_dim", [0, -8, -64, 12])
def test_head_dims_that_there_are_not(head_dim):
    with pytest.raises(SpecVerifyError, match="head_dim"):
        paged_cache._page4(16 * 34, head_dim, None)
    cache, slots = torch.zeros(2, 1, 16 * 34, dtype=torch.uint8), torch.zeros(1, 2, dtype=torch.int32)
    with pytest.raises(SpecVerifyError, match="head_dim"):
        paged_cache.read4(cache, cache, slots, head_dim, torch.float16)


@pytest.mark.gpu
def test_tensors_without_values_are_refused():
    if not torch.cuda.is_available():
        pytest.fail("no GPU visible")
    cache = torch.zeros(2, 1, 16 * 34, dtype=torch.uint8, device="cuda")
    slots = torch.zeros(1, 2, dtype=torch.int32, device="cuda")
    x = torch.zeros(1, 2, 1, 0, dtype=torch.float16, device="cuda")
    for call in (lambda: paged_cache.append4(x, x, cache, cache.clone(), slots),
                 lambda: paged_cache.read4(cache, cache, slots, out=(x, x.clone())),
                 lambda: paged_cache.attend4(x, cache, cache, slots, slots[0, :1])):
        with pytest.raises(SpecVerifyError, match="head_dim"):
            call()
