"""PagedCache against what it is handed: caches that its tables do not describe,
a prefix on pages of the program's choice, another device's loop, arguments
that no kernel takes."""
import pytest
import torch

from paper_2406_11016_amd import paged_cache
from paper_2406_11016_amd.binding import SpecVerifyError
from paper_2406_11016_amd.paged_cache import PagedCache

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def gpu():
    if not torch.cuda.is_available():
        pytest.fail("no GPU visible")
    paged_cache.load_library()
    torch.cuda.init()


def _zeros(*shape):
    return torch.zeros(*shape, dtype=torch.float16, device="cuda")


def test_storage_that_the_tables_do_not_describe():
    """Slots and tables count in the tables' pages: other pages, or fewer, would be other places."""
    cache = PagedCache(2, num_pages=8, page_size=32, max_pages=3, max_new=4, prefix_pages=1)
    cache.set_prefix(10)
    cache.plan(4)
    kv, q, prefix = _zeros(2, 4, 2, 64), _zeros(2, 4, 4, 64), _zeros(1, 10, 2, 64)
    for shape in ((16, 2, 16, 64), (4, 2, 64, 64), (7, 2, 32, 64), (8, 2, 16, 64)):
        other = _zeros(*shape), _zeros(*shape)
        for call in (lambda: cache.append(kv, kv, *other), lambda: cache.attend(q, *other),
                     lambda: cache.append_prefix(prefix, prefix, *other)):
            with pytest.raises(SpecVerifyError, match="pages"):
                call()
    with pytest.raises(SpecVerifyError):
        cache.attend(q, _zeros(8, 2, 32), _zeros(8, 2, 32))
    for pages in (8, 9):                   # (a cache may have more than the tables name)
        own = _zeros(pages, 2, 32, 64), _zeros(pages, 2, 32, 64)
        cache.append_prefix(prefix, prefix, *own)
        cache.append(kv, kv, *own)
        assert not cache.attend(q, *own).any()
