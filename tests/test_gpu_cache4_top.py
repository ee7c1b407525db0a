"""The cache in 4 bits at the top of the storage types' range: finite numbers are held as finite ones, by the write, by the
read and by the attention."""
import numpy as np
import pytest
import torch

from paper_2406_11016_amd import paged_cache
from tests import cache4_util as C4
from tests.cache_util import TORCH_DTYPES
from tests.test_gpu_cache4_attend import Batch4

pytestmark = pytest.mark.gpu
TOP = {"f16": 57344.0, "bf16": 1.75 * 2.0 ** 127}   # from here on 4 times a block's scale is not a number of the type


@pytest.fixture(scope="module", autouse=True)
def gpu():
    if not torch.cuda.is_available():
        pytest.fail("no GPU visible")
    paged_cache.load_library()
    torch.cuda.init()


@pytest.mark.parametrize("dtype", ["f16", "bf16"])
def test_a_finite_number_is_read_back_as_one(dtype):
    """Every finite number as its block's largest, at each place of it, beside smaller ones: off by a fifth of the largest
    at most, by a quarter from TOP on, or by a quarter of the least scale."""
    t = TORCH_DTYPES[dtype]
    every = torch.arange(65536, dtype=torch.int32, device="cuda").to(torch.int16).view(t)
    every = every[torch.isfinite(every)]
    n = every.numel()
    x = (every.double()[:, None] * torch.linspace(-0.99, 0.99, 32, device="cuda", dtype=torch.float64)).to(t)
    x[torch.arange(n, device="cuda"), torch.arange(n, device="cuda") % 32] = every
    x = x.view(1, n // 2, 1, 64)
    slots = torch.arange(n // 2, dtype=torch.int32, device="cuda")[None]
    caches = [torch.zeros(-(-n // 2 // 64), 1, 64 * 34, dtype=torch.uint8, device="cuda") for _ in range(2)]
    paged_cache.append4(x, -x, *caches, slots)
    k, v = paged_cache.read4(*caches, slots, 64, t)
    assert torch.isfinite(k).all() and torch.equal(v, -k)
    blocks, held = x.double().view(-1, 32), k.double().view(-1, 32)
    largest = blocks.abs().amax(-1, keepdim=True)
    top = largest >= TOP[dtype]
    assert int(top.sum()) > 60
    bound = torch.where(top, largest / 4, largest / 5).clamp(min=2.0 ** C4.LEAST[t] / 4)
    assert ((held - blocks).abs() <= bound).all()
    assert (held.abs().amax(-1, keepdim=True)[top] == 6 / 7 * TOP[dtype]).all()


# rows of one, two and three direct tiles, of many, and of both kinds at head_dim 256
@pytest.mark.parametrize("dtype", ["f16", "bf16"])
@pytest.mark.parametrize("shape", [(2, 2, 4, 1, 64), (2, 7, 8, 2, 128), (2, 12, 4, 1, 96), (2, 40, 4, 1, 128), (2, 3, 4, 1, 256),
                                   (2, 20, 4, 1, 256)], ids=str)
@pytest.mark.parametrize("prefix", [0, 90])
def test_attention_to_the_largest_numbers(shape, prefix, dtype):
    """Keys and values beyond TOP, of every token's past and of the last tokens, which some rows do not see: the outputs
    are those of the values that are held, finite as these are."""
    B, n, H, K, D = shape
    x = Batch4(B, n, H, K, D, 16, prefix, [100, 7], [n, n], dtype, seed=n + D, spread=0.2)
    k, v = x.k.clone(), x.v.clone()
    large = float(torch.finfo(k.dtype).max)
    q_small = 4.0 / large if dtype == "f16" else 2.0 ** -126
    x.q[..., 3] = q_small                                        # (scores of a few units)
    k[..., 3] = torch.where(torch.isnan(k[..., 3]), k[..., 3], 0.0)
    for b, tokens in enumerate(([5, 100 + n // 2, 100 + n - 1], [7])):
        for i, token in enumerate(tokens):
            page, off = int(x.table[b][token // 16]), token % 16
            k[page, :, off, 3] = large if i % 2 == 0 else -large * 0.9
            v[page, :, off, D - 5] = -large if i % 2 == 0 else large
    N = k.shape[0]
    slots = torch.arange(N * 16, dtype=torch.int32, device="cuda")[None]
    rows = [c.permute(0, 2, 1, 3).reshape(1, N * 16, K, D) for c in (k, v)]
    paged_cache.append4(*rows, x.k4, x.v4, slots)
    x.values()
    out = x.check()
    assert torch.isfinite(out).all()
    for b in range(B):
        assert np.isfinite(out[b].double().cpu().numpy()).all()
        assert float(out[b, -1].abs().max()) > large * 2.0 ** -20
