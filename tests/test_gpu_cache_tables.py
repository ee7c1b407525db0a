"""PagedCache against what it is handed: caches that its tables do not describe,
a prefix on pages of the program's choice, another device's loop, arguments
that no kernel takes."""
import pytest
import torch

from paper_2406_11016_amd import paged_cache
from paper_2406_11016_amd.binding import SpecVerifyError
from paper_2406_11016_amd.decode_loop import DecodeLoop
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


def _ints(*x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


def test_reset_keeps_the_prefix_where_the_program_put_it():
    """A prefix on pages of the program's choice: reset() hands out all others, in ascending order, and none of those."""
    N, P, B, M = 12, 16, 3, 4
    for prefix in ((7, 2), (11,), (0, 1), ()):
        reserved = _ints(*prefix)
        cache = PagedCache.over(_ints(*[0] * B), _ints(*[0] * B), _ints(*[0] * B),
                                torch.full((B, M), -1, dtype=torch.int32, device="cuda"),
                                torch.empty(N, dtype=torch.int32, device="cuda"), _ints(0), page_size=P, max_new=3 * P,
                                prefix_table=reserved)
        for _ in range(2):
            cache.reset()
            rest = [p for p in range(N - 1, -1, -1) if p not in prefix]
            assert int(cache.free_count) == len(rest)
            assert cache.free_pages.tolist() == rest + [-1] * len(prefix)
            assert cache.lengths.tolist() == cache.counts.tolist() == cache.held.tolist() == [0] * B
            assert (cache.block_table == -1).all()
            cache.plan(3 * P)              # 9 pages, of the 10 or more that there are
            used = cache.block_table[cache.block_table >= 0].tolist()
            assert sorted(used) == sorted(rest)[:9] and cache.counts.tolist() == [3 * P] * B


def test_a_loop_on_another_device_than_its_cache():
    class Other:
        batch, max_new, device = 2, 5, torch.device("cuda", torch.cuda.current_device() + 1)

    for device in ("cuda", f"cuda:{torch.cuda.current_device()}"):
        with pytest.raises(ValueError, match="the cache must serve"):
            DecodeLoop(2, 100, "f32", gamma0=1, gamma_max=4, cache=Other(), device=device)


def test_reset_in_a_graph():
    """Of the tables' own order; a prefix on pages of the program's choice is refused there."""
    tables = [torch.zeros(2, dtype=torch.int32, device="cuda") for _ in range(3)]
    rows, free = torch.zeros(2, 3, dtype=torch.int32, device="cuda"), torch.zeros(9, dtype=torch.int32, device="cuda")
    kinds = {}
    for name, prefix in (("none", None), ("chosen", _ints(4, 2))):
        kinds[name] = PagedCache.over(*tables, rows, free, _ints(0), page_size=16, max_new=4, prefix_table=prefix)
    kinds["first"] = PagedCache(2, num_pages=9, page_size=16, max_pages=3, max_new=4, prefix_pages=2)
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    for name in ("none", "first"):
        cache = kinds[name]
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g, stream=side):
            cache.reset()
        for _ in range(3):
            cache.plan(4)
            torch.cuda.synchronize()
            g.replay()
            torch.cuda.synchronize()
            first = cache.prefix_table.numel()
            assert int(cache.free_count) == 9 - first
            assert cache.free_pages.tolist() == list(range(8, first - 1, -1)) + [-1] * first
    with torch.cuda.stream(side):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g, stream=side):
            with pytest.raises(SpecVerifyError, match="captured"):
                kinds["chosen"].reset()
            kinds["none"].reset()
    torch.cuda.synchronize()
