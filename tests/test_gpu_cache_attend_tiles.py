"""The cache's attention over several row tiles of a sequence: bad pages, and
values that only some tokens see."""
import pytest
import torch

from paper_2406_11016_amd import paged_cache
from tests.test_gpu_cache_attend import KEPT, check, make

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def gpu():
    if not torch.cuda.is_available():
        pytest.fail("no GPU visible")
    paged_cache.load_library()
    torch.cuda.init()


# batch, new tokens, heads, key/value heads, head_dim, page size: one tile to many, pooled and joined prefixes
SHAPES = [(3, 257, 4, 1, 64, 16), (2, 300, 8, 2, 128, 32), (3, 40, 4, 2, 256, 16), (300, 64, 4, 2, 80, 16),
          (70, 128, 8, 4, 128, 64)]


@pytest.mark.parametrize("prefix", [0, 100])
@pytest.mark.parametrize("shape", SHAPES, ids=str)
def test_a_bad_page_makes_all_of_its_sequence_nan(shape, prefix):
    """Also where only the last tokens see it; behind the last token's page nothing is looked at."""
    B, n, H, K, D, P = shape
    lengths = [(37 * b) % 90 for b in range(B)]
    counts = [n - b % 3 for b in range(B)]
    x = make(B, n, H, K, D, P, prefix, lengths, counts, "bf16", seed=n)
    q, k, v, table, at, count, prefix_table = x

    def run():
        out = torch.full_like(q, KEPT)
        paged_cache.attend(q, k, v, table, at, count, prefix_table=prefix_table, prefix_len=prefix, out=out)
        return out

    clean = check(x, prefix, "bf16") if B < 10 else run()
    assert torch.isfinite(clean).all()
    others = [b for b in range(B) if b != 1]
    last = (lengths[1] + counts[1] - 1) // P
    for page in (last, lengths[1] // P, 0):
        for word in (-1, k.shape[0]):
            saved = table[1, page].clone()
            table[1, page] = word
            out = run()
            table[1, page] = saved
            assert torch.isnan(out[1, :counts[1]]).all(), (page, word)
            assert (out[1, counts[1]:] == KEPT).all() and torch.equal(out[others], clean[others]), (page, word)
    if last + 1 < table.shape[1]:
        table[1, last + 1] = -7
        assert torch.equal(run(), clean)
