"""A program that makes its cache and plans its prompts on the current stream,
behind long work there, and starts the loop at once, as the usage shows it."""
import pytest
import torch

from paper_2406_11016_amd import paged_cache
from paper_2406_11016_amd import workloads as W
from paper_2406_11016_amd.decode_loop import DecodeLoop, SyntheticSteps
from paper_2406_11016_amd.paged_cache import PagedCache

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def gpu():
    if not torch.cuda.is_available():
        pytest.fail("no GPU visible")
    paged_cache.load_library()
    torch.cuda.init()


@pytest.mark.parametrize("native", [False, True])
def test_a_program_on_the_current_stream(native):
    B, prompts = 3, [5, 30, 16]
    w = W.WORKLOADS["exact_b1_g5_v51865_f32"].with_(batch=B, vocab=1009)
    steps = SyntheticSteps(w, 6, 4)
    new = torch.tensor(prompts, dtype=torch.int32, device="cuda")
    ended = torch.tensor([0, 1, 0], dtype=torch.int32, device="cuda")
    some = torch.tensor([0, 7, 0], dtype=torch.int32, device="cuda")
    big = torch.empty(1 << 28, dtype=torch.uint8, device="cuda")

    def busy():
        for i in range(200):           # 256 MiB each: several ms
            big.fill_(i % 256)

    torch.cuda.synchronize()
    for _ in range(3):
        busy()
        cache = PagedCache(B, num_pages=48, page_size=16, max_pages=12, max_new=30, device="cuda")
        cache.plan(30, new_tokens=new)
        loop = DecodeLoop(B, 1009, "f32", gamma0=3, gamma_max=6, cache=cache, native=native)
        stats = loop.run(steps, 3)
        last = stats.accepted[-1]
        # between runs, on the current stream again; then the loop at once
        busy()
        cache.plan(7, new_tokens=some, accepted_len=loop.acc, release=ended)
        loop.program_planned()
        stats2 = loop.run(steps, 2)
        kept = [prompts[b] + sum(int(a[b]) + 1 for a in stats.accepted) for b in range(B)]
        kept[1] = 7
        kept = [k + int(stats2.accepted[0][b]) + 1 for b, k in enumerate(kept)]
        # no synchronisation: the current stream follows the loop's
        assert cache.lengths.tolist() == kept, last
        assert int((cache.block_table >= 0).sum()) + int(cache.free_count) == 48
        loop.close()
