"""Whose page a cache in 4 bits has: its bytes fit several head_dims, so the functions hold it against a page size that they
are given."""
import pytest
import torch

from paper_2406_11016_amd import paged_cache
from paper_2406_11016_amd.binding import SpecVerifyError


def test_the_page_size_that_the_bytes_give():
    # rows of 34, 68 and 136 bytes: what is one page for one head_dim is another for another
    size = 32 * 68
    assert paged_cache._page4(size, 128, None) == 32 and paged_cache._page4(size, 64, None) == 64
    assert paged_cache._page4(size, 256, None) == 16 and paged_cache._page4(16 * 43, 80, 16) == 16
    for head_dim, page in ((128, 16), (64, 32), (256, 32), (128, 64), (128, 0)):
        with pytest.raises(SpecVerifyError, match="page_size"):
            paged_cache._page4(size, head_dim, page)
    with pytest.raises(SpecVerifyError, match="no whole number"):
        paged_cache._page4(size, 96, None)


@pytest.mark.gpu
def test_a_cache_of_another_head_dim_is_refused():
    if not torch.cuda.is_available():
        pytest.fail("no GPU visible")
    P, K, dev = 32, 2, "cuda"
    cache = [torch.zeros(6, K, P * paged_cache.row_bytes4(128), dtype=torch.uint8, device=dev) for _ in range(2)]
    before = [c.clone() for c in cache]
    slots = torch.zeros(1, 1, dtype=torch.int32, device=dev)
    table, lengths = torch.zeros(1, 1, dtype=torch.int32, device=dev), torch.zeros(1, dtype=torch.int32, device=dev)

    def x(D):
        return torch.ones(1, 1, K, D, dtype=torch.float16, device=dev)

    for D in (64, 256):
        for call in (lambda: paged_cache.append4(x(D), x(D), *cache, slots, page_size=P),
                     lambda: paged_cache.read4(*cache, slots, D, torch.float16, page_size=P),
                     lambda: paged_cache.read4(*cache, slots, out=(x(D), x(D)), page_size=P),
                     lambda: paged_cache.attend4(x(D), *cache, table, lengths, page_size=P)):
            with pytest.raises(SpecVerifyError, match="page_size"):
                call()
    assert all(torch.equal(a, b) for a, b in zip(cache, before))
    # and the right one is taken
    paged_cache.append4(x(128), 2 * x(128), *cache, slots, page_size=P)
    k, v = paged_cache.read4(*cache, slots, 128, torch.float16, page_size=P)
    out = paged_cache.attend4(x(128), *cache, table, lengths, page_size=P)
    assert torch.equal(k, x(128)) and torch.equal(v, 2 * x(128)) and torch.equal(out, v)
