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


# tasks of 32, 64 and 128 rows, several to a sequence; the last shape's run over the prefix themselves
SPECIAL = [(2, 20, 8, 1, 64, 16), (2, 20, 8, 1, 128, 32), (2, 50, 8, 2, 80, 16), (2, 6, 4, 1, 256, 16), (2, 9, 2, 2, 96, 16),
           (70, 128, 8, 4, 128, 64), (64, 16, 8, 2, 256, 32)]


@pytest.mark.parametrize("dtype", ["f16", "bf16"])
@pytest.mark.parametrize("prefix", [0, 40, 128])
@pytest.mark.parametrize("shape", SPECIAL, ids=str)
def test_special_values_of_later_tokens(shape, prefix, dtype):
    """An infinity or NaN in token 3's key or value: tokens 0 to 2 of its sequence and the others are what they were, and
    later tokens get it (their weights here are far from 0)."""
    B, n, H, K, D, P = shape
    lengths, counts = [125] + [(29 * b) % 70 for b in range(1, B)], [n] * B
    x = make(B, n, H, K, D, P, prefix, lengths, counts, dtype, seed=n, spread=0.2)
    q, k, v, table, at, count, prefix_table = x

    def run():
        out = torch.full_like(q, KEPT)
        paged_cache.attend(q, k, v, table, at, count, prefix_table=prefix_table, prefix_len=prefix, out=out)
        return out

    clean = check(x, prefix, dtype) if B < 10 else run()
    G, token = H // K, lengths[0] + 3
    page, off = int(table[0][token // P]), token % P
    cols = [1, 33, D - 1]
    rest = [d for d in range(D) if d not in cols]
    for what in (float("nan"), float("inf"), float("-inf")):
        saved = v[page, 0, off].clone()
        v[page, 0, off, cols] = what
        out = run()
        v[page, 0, off] = saved
        assert torch.equal(out[0, :3], clean[0, :3]) and torch.equal(out[1:], clean[1:]), what
        if K > 1:
            assert torch.equal(out[0, :, G:], clean[0, :, G:])
        got = out[0, 3:, :G]
        assert torch.equal(got[..., rest], clean[0, 3:, :G][..., rest]), what
        assert (torch.isnan(got[..., cols]) if what != what else got[..., cols].float() == what).all(), what
        saved = k[page, 0, off].clone()
        k[page, 0, off] = what
        out = run()
        k[page, 0, off] = saved
        assert torch.equal(out[0, :3], clean[0, :3]) and torch.equal(out[1:], clean[1:]), what
        if what != what:
            assert torch.isnan(out[0, 3:, :G]).all()
    # both signs at once, and in a key that all tokens see
    v[page, 0, off, 1] = float("inf")
    page, off = int(table[0][0]), 0
    v[page, 0, off, 1] = float("-inf")
    v[page, 0, off, 33] = float("inf")
    out = run()
    assert torch.isnan(out[0, 3:, :G, 1]).all() and (out[0, :3, :G, 1].float() == float("-inf")).all()
    assert (out[0, :, :G, 33].float() == float("inf")).all() and torch.equal(out[1:], clean[1:])


@pytest.mark.parametrize("dtype", ["f16", "bf16"])
@pytest.mark.parametrize("prefix", [0, 300])
def test_infinite_values_of_keys_without_weight(prefix, dtype):
    """A key that every token sees, with an infinite value and a weight that is 0 in the storage type: NaN or infinity
    in that place of the head dimension, and nowhere else."""
    x = make(2, 3, 2, 1, 64, 16, prefix, [400, 30], [3, 3], dtype, seed=3)
    q, k, v, table, at, count, prefix_table = x
    clean = check(x, prefix, dtype)
    page = int(prefix_table[1] if prefix else table[0][1])
    k[page, 0, 2] = 0.0
    out0 = torch.full_like(q, KEPT)
    q[..., 0] = 1.0
    k[:, :, :, 0] = torch.nan_to_num(k[:, :, :, 0], 0.0)
    k[page, 0, 2, 0] = -1000.0
    paged_cache.attend(q, k, v, table, at, count, prefix_table=prefix_table, prefix_len=prefix, scale=1.0, out=out0)
    v[page, 0, 2, 5] = float("inf")
    out = paged_cache.attend(q, k, v, table, at, count, prefix_table=prefix_table, prefix_len=prefix, scale=1.0)
    rest = [d for d in range(64) if d != 5]
    hit = [0, 1] if prefix else [0]
    assert torch.equal(out[..., rest], out0[..., rest]) and clean.shape == out.shape
    assert not torch.isfinite(out[hit][..., 5]).any()
    if not prefix:
        assert torch.equal(out[1], out0[1])
