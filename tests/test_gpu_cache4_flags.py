"""The attention over a cache in 4 bits where a workgroup has several tasks of few rows: sequences with a page that there is
not, with a length that cannot be, or with a block that is NaN, among hundreds of others, which stay as they were."""
import numpy as np
import pytest
import torch

from paper_2406_11016_amd import paged_cache
from tests.cache_util import TORCH_DTYPES
from tests.test_gpu_cache4_attend import KEPT, Batch4
from tests.test_gpu_cache_attend import make

pytestmark = pytest.mark.gpu
P = 16
# kv_heads, group, new tokens, head_dim: one, two and three row tiles of 16, and one at head_dim 256
SHAPES = [(4, 4, 1, 128), (4, 4, 4, 64), (3, 4, 7, 80), (4, 4, 8, 128), (3, 4, 11, 64), (2, 4, 12, 96), (4, 1, 36, 128), (3, 4, 4, 256)]


@pytest.fixture(scope="module", autouse=True)
def gpu():
    if not torch.cuda.is_available():
        pytest.fail("no GPU visible")
    paged_cache.load_library()
    torch.cuda.init()


class Large(Batch4):
    """Hundreds of sequences, whose caches are packed on the GPU."""

    def __init__(self, B, n, H, K, D, prefix, lengths, counts, dtype, seed):
        x = make(B, n, H, K, D, P, prefix, lengths, counts, dtype, seed)
        self.q, k, v, self.table, self.lengths, self.counts, self.prefix_table = x
        self.P, self.D, self.dtype, self.prefix = P, D, dtype, prefix
        N = k.shape[0]
        self.k4, self.v4 = (torch.zeros(N, K, P * paged_cache.row_bytes4(D), dtype=torch.uint8, device="cuda") for _ in range(2))
        slots = torch.arange(N * P, dtype=torch.int32, device="cuda")[None]
        paged_cache.append4(*(c.permute(0, 2, 1, 3).reshape(1, N * P, K, D) for c in (k, v)), self.k4, self.v4, slots)
        self.k, self.v = (c.view(N, P, K, D).permute(0, 2, 1, 3)
                          for c in paged_cache.read4(self.k4, self.v4, slots, D, TORCH_DTYPES[dtype]))


def batch(shape, long, prefix, dtype):
    """400 sequences: 800 to 1,600 tasks for 512 workgroups at most.  `long`: one is so long that the table has more units than
    tasks are left whole with, and that borders cut its tasks."""
    K, G, n, D = shape
    B = 400
    lengths = [(37 * b) % 200 for b in range(B)]
    if long:
        lengths[11] = 1500
    counts = [max(1, n - b % 3) if b % 17 else 0 for b in range(B)]
    x = Large(B, n, K * G, K, D, prefix, lengths, counts, dtype, seed=D + n)
    assert (x.table.shape[1] * P <= 1024) != long
    return x, lengths, counts


def exactly(out, clean, counts, chosen):
    """NaN are the rows of the chosen sequences and no others."""
    for b in chosen:
        assert torch.isnan(out[b, :counts[b]]).all() and (out[b, counts[b]:] == KEPT).all(), b
    others = sorted(set(range(len(counts))) - set(chosen))
    assert torch.equal(out[others], clean[others])


@pytest.mark.parametrize("long", [False, True])
@pytest.mark.parametrize("prefix", [0, 100])
@pytest.mark.parametrize("shape", SHAPES, ids=str)
def test_bad_pages_among_many_tasks(shape, prefix, long):
    x, lengths, counts = batch(shape, long, prefix, "bf16" if shape[2] % 2 else "f16")
    clean = x.run()
    assert torch.isfinite(clean).all()
    rng = np.random.default_rng(shape[2])
    live = [b for b in range(len(counts)) if counts[b] > 0]
    # a few; every second one; runs of neighbours (tasks after one another); all but a few; the one that borders cut
    for chosen in (rng.choice(live, 9, replace=False), live[::2], live[100:140] + live[141:143],
                   sorted(set(live) - set(rng.choice(live, 7, replace=False).tolist())), [11]):
        saved = x.table.clone()
        for i, b in enumerate(chosen):
            pages = (lengths[b] + counts[b] - 1) // P + 1
            x.table[b, (0, pages - 1, pages // 2)[i % 3]] = (-1, x.k4.shape[0], 1 << 30)[i // 3 % 3]
        for _ in range(2):
            exactly(x.run(), clean, counts, [int(b) for b in chosen])
        x.table.copy_(saved)
        assert torch.equal(x.run(), clean)


@pytest.mark.parametrize("long", [False, True])
@pytest.mark.parametrize("prefix", [0, 100])
@pytest.mark.parametrize("shape", SHAPES[1::2], ids=str)
def test_bad_lengths_among_many_tasks(shape, prefix, long):
    """(Other lengths share the work out otherwise, so the other sequences are held to the definition.)"""
    x, lengths, counts = batch(shape, long, prefix, "f16" if shape[2] % 2 else "bf16")
    chosen = [b for b in range(len(counts)) if counts[b] > 0 and (b % 7 == 3 or 200 <= b < 220)]
    for i, b in enumerate(chosen):
        x.lengths[b] = (-1, x.table.shape[1] * P, (1 << 31) - 1, -(1 << 31))[i % 4]
    out = x.run()
    for b in chosen:
        assert torch.isnan(out[b, :counts[b]]).all() and (out[b, counts[b]:] == KEPT).all(), b
        x.lengths[b] = lengths[b]   # (what the definition is then asked of, it is not compared with)
    x.check(shape, out=out, without=chosen)


@pytest.mark.parametrize("long", [False, True])
@pytest.mark.parametrize("shape", SHAPES, ids=str)
def test_nan_blocks_among_many_tasks(shape, long):
    """Of a value of the last token's, which the others of its sequence do not see, or of the first one's."""
    x, lengths, counts = batch(shape, long, 0, "bf16")
    K, G, n, D = shape
    clean = x.run()
    blocks = -(-D // 32)
    chosen = [b for b in range(len(counts)) if counts[b] > 0 and (b % 5 == 1 or 300 <= b < 320)]
    want = clean.clone()
    for i, b in enumerate(chosen):
        last = i % 2 == 0
        token, head, block = lengths[b] + counts[b] - 1 if last else 0, i % K, i % blocks
        page = int(x.table[b, token // P])
        x.v4[page, head, P * D // 2 + token % P * blocks + block] = 255
        want[b, counts[b] - 1 if last else 0:counts[b], head * G:(head + 1) * G, 32 * block:32 * block + 32] = float("nan")
    out = x.run()
    assert torch.equal(torch.isnan(out), torch.isnan(want))
    assert torch.equal(torch.nan_to_num(out), torch.nan_to_num(want))
