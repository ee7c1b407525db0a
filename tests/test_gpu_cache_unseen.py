"""What a token does not see has no influence on it, to the last bit: keys and values of later tokens and other sequences'
queries, however large, where the rows share tiles with those that do see them.  Caches of 16 and of 4 bits."""
import pytest
import torch

from paper_2406_11016_amd import paged_cache
from tests.cache_util import TORCH_DTYPES
from tests.test_gpu_cache4_attend import KEPT, Batch4

pytestmark = pytest.mark.gpu
# new tokens, query and key/value heads, head_dim: rows of one tile to many
SHAPES = [(4, 2, 1, 64), (9, 4, 2, 128), (10, 3, 1, 80), (12, 4, 1, 128), (40, 2, 1, 96), (140, 2, 1, 64), (4, 4, 1, 256), (24, 2, 1, 256)]


@pytest.fixture(scope="module", autouse=True)
def gpu():
    if not torch.cuda.is_available():
        pytest.fail("no GPU visible")
    paged_cache.load_library()
    torch.cuda.init()


def run(x, bits, **more):
    if bits == 4:
        return x.run(**more)
    out = torch.full(x.q.shape, KEPT, dtype=x.q.dtype, device="cuda")
    return paged_cache.attend(x.q, x.k, x.v, x.table, x.lengths, x.counts, prefix_table=x.prefix_table, prefix_len=x.prefix, out=out,
                              **more)


def same(a, b):
    return torch.equal(torch.nan_to_num(a), torch.nan_to_num(b)) and torch.equal(torch.isnan(a), torch.isnan(b))


@pytest.mark.parametrize("bits", [16, 4])
@pytest.mark.parametrize("dtype", ["f16", "bf16"])
@pytest.mark.parametrize("prefix", [0, 130])
@pytest.mark.parametrize("shape", SHAPES, ids=str)
def test_keys_of_later_tokens(shape, prefix, dtype, bits):
    n, H, K, D = shape
    lengths = [190, 61]
    x = Batch4(2, n, H, K, D, 16, prefix, lengths, [n, n], dtype, seed=n)
    x.q.abs_()
    t = TORCH_DTYPES[dtype]
    k, v, k4 = x.k, x.v, x.k4
    slots = torch.arange(k.shape[0] * 16, dtype=torch.int32, device="cuda")[None]
    for scale in (D ** -0.5, 300.0):              # (the second's scores are far from zero)
        clean = run(x, bits, scale=scale)
        for first in sorted({1, n // 2, n - 1}):
            for key in (8.0, -8.0, 200.0, 5e4, float("inf"), float("-inf"), float("nan")):
                x.k, x.k4 = k.clone(), torch.zeros_like(k4)
                for token in range(lengths[0] + first, lengths[0] + n):
                    x.k[int(x.table[0, token // 16]), :, token % 16] = key
                rows = x.k.permute(0, 2, 1, 3).reshape(1, -1, K, D)
                paged_cache.append4(rows, rows, x.k4, torch.empty_like(x.k4), slots)
                out = run(x, bits, scale=scale)
                assert torch.equal(out[0, :first], clean[0, :first]) and torch.equal(out[1], clean[1]), (scale, first, key)
                # (an infinite key is held as NaN in 4 bits)
                if key != key or (bits == 4 and abs(key) == float("inf")):
                    assert torch.isnan(out[0, first:]).all()
        x.k, x.v, x.k4 = k, v, k4
    assert t == x.q.dtype


@pytest.mark.parametrize("bits", [16, 4])
@pytest.mark.parametrize("dtype", ["f16", "bf16"])
@pytest.mark.parametrize("shape", SHAPES[:5] + SHAPES[6:], ids=str)
def test_queries_of_other_sequences(shape, dtype, bits):
    """In tiles of the prefix, which rows of all sequences share."""
    n, H, K, D = shape
    x = Batch4(6, n, H, K, D, 16, 500, [20, 0, 77, 130, 5, 64], [n, max(1, n // 2), n, 1, n, n], dtype, seed=n)
    clean = run(x, bits)
    q = x.q.clone()
    for by in (3.0, 40.0, 1000.0, float("inf"), float("nan")):
        for others in ([0], [1, 4], [5]):
            x.q = q.clone()
            for b in others:
                x.q[b] = x.q[b] * by
            out = run(x, bits)
            rest = [b for b in range(6) if b not in others]
            assert same(out[rest], clean[rest]), (by, others)
