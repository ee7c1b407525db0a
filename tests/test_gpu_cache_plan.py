"""The paged cache's tables and writes (spec_cache_init, spec_cache_plan,
spec_cache_append) against a plain host model: whole numbers and copies, so
every result has to be equal."""
import numpy as np
import pytest
import torch

from paper_2406_11016_amd import paged_cache
from paper_2406_11016_amd.paged_cache import PagedCache
from tests.cache_util import TORCH_DTYPES, PlanReference

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def gpu():
    if not torch.cuda.is_available():
        pytest.fail("no GPU visible")
    paged_cache.load_library()
    torch.cuda.init()


def _dev(x):
    return None if x is None else torch.tensor(x, dtype=torch.int32, device="cuda")


def _same(cache, ref, got, want, label):
    slots, positions = (x.cpu().numpy() for x in got)
    assert np.array_equal(slots, want[0]), (label, np.argwhere(slots != want[0])[:4], slots, want[0])
    assert np.array_equal(positions, want[1]), label
    assert cache.lengths.tolist() == ref.lengths, label
    assert cache.counts.tolist() == ref.counts, label
    assert cache.held.tolist() == [len(r) for r in ref.rows], label
    assert np.array_equal(cache.block_table.cpu().numpy(), ref.table()), label
    assert int(cache.free_count) == len(ref.free), label
    assert cache.free_pages.tolist() == ref.below, label


# (batch, max_new, page size, pages a sequence, pages of the pool over those that all could hold, reserved pages)
SHAPES = [(1, 1, 16, 3, 0, 0), (1, 6, 16, 7, 2, 3), (3, 21, 64, 2, 0, 1), (64, 9, 16, 12, 0, 5), (17, 300, 32, 13, 0, 0),
          (70, 130, 16, 11, 0, 2), (1025, 3, 16, 3, 7, 0), (4096, 2, 128, 2, 0, 0)]


@pytest.mark.parametrize("shape", SHAPES, ids=["b%d_n%d_p%d" % s[:3] for s in SHAPES])
def test_steps_match_the_host_model(shape):
    """Steps with accepted lengths (the sentinel among them), fewer new tokens than the padding, ended sequences,
    and values that cannot be right, until pages run out and are given back."""
    B, n, P, M, spare, reserved = shape
    rng = np.random.default_rng(B * 1000 + n)
    N = max(1, (2 * B * M) // 3) + spare + reserved      # too few for all sequences at their longest
    cache = PagedCache(B, num_pages=N, page_size=P, max_pages=M, max_new=n, prefix_pages=reserved)
    ref = PlanReference(B, N, P, M, reserved)
    cache.set_prefix(min(reserved * P, 5))
    for step in range(12):
        k = int(rng.integers(1, n + 1)) if step % 3 else n
        new = None if step % 4 == 1 else [int(x) for x in rng.integers(0, k + 1, B)]
        accepted = None if step % 5 == 0 else [int(rng.integers(-1, max(c, 1))) for c in ref.counts]
        release = None if step % 3 == 0 else [int(x) for x in (rng.random(B) < (0.5 if step == 8 else 0.1)) * 3]
        if accepted is not None and step % 2:
            accepted[rng.integers(B)] = int(ref.counts[0]) + 2     # outside, for some
            accepted[rng.integers(B)] = -2
        if new is not None and step % 3 == 2:
            new[rng.integers(B)] = k + 1
            new[rng.integers(B)] = -1
        want = ref.plan(k, accepted, new, release, cache.prefix_len)
        got = cache.plan(k, new_tokens=_dev(new), accepted_len=_dev(accepted), release=_dev(release))
        _same(cache, ref, got, want, (shape, step))
    assert -1 in ref.counts      # the pool did run out, or a value was refused
    cache.reset()
    ref = PlanReference(B, N, P, M, reserved)
    _same(cache, ref, cache.plan(1), ref.plan(1, base=cache.prefix_len), (shape, "reset"))


def test_prompts_then_decoding():
    """Prompts of several hundred pages in one step, and steps behind them (the kernel with its own slots)."""
    B, n, P = 40, 1500, 16
    cache = PagedCache(B, num_pages=5000, page_size=P, max_pages=130, max_new=n)
    ref = PlanReference(B, 5000, P, 130)
    rng = np.random.default_rng(3)
    new = [int(x) for x in rng.integers(0, n + 1, B)]
    _same(cache, ref, cache.plan(n, new_tokens=_dev(new)), ref.plan(n, None, new), "prompts")
    for step in range(6):
        accepted = None if step == 0 else [int(rng.integers(-1, 9)) for _ in range(B)]
        release = [1 if (b + step) % 11 == 0 else 0 for b in range(B)]
        _same(cache, ref, cache.plan(9, accepted_len=_dev(accepted), release=_dev(release)),
              ref.plan(9, accepted, None, release), step)


def test_plan_over_a_programs_tables_and_corrupt_ones():
    """Words that cannot be right are not followed out of the tables; the other sequences are served."""
    B, M, P, N = 4, 3, 16, 9
    held, table = _dev([1, 7, -3, 2]), torch.full((B, M), -1, dtype=torch.int32, device="cuda")
    table[0, 0], table[1, 0], table[3, 0], table[3, 1] = 4, 99, 5, 1 << 30
    lengths = _dev([7, 2000000000, -5, 20])
    free = _dev([0, 1, 2, 3, 6, 7, 8, -1, -1])
    cache = PagedCache.over(lengths, _dev([0, 0, 0, 0]), held, table, free, _dev([7]), page_size=P, max_new=4)
    slots, _ = cache.plan(4, release=_dev([0, 1, 0, 0]))
    # sequence 1 gives back 3 entries (its table's): 99, -1, -1; then needs a page: the last of them, -1
    assert slots[0].tolist() == [4 * P + 7 + i for i in range(4)]
    assert slots[1].tolist() == [-1] * 4
    assert slots[2].tolist() == [-1] * 4 and cache.counts.tolist() == [4, 4, -1, 4]
    assert slots[3].tolist() == [-1] * 4                       # a page outside the cache: no slot
    cache = PagedCache.over(_dev([0] * B), _dev([0] * B), _dev([0] * B), table.fill_(-1), free, _dev([1 << 29]),
                            page_size=P, max_new=4)
    cache.plan(4)
    assert int(cache.free_count) == N - B


@pytest.mark.parametrize("dtype", ["f16", "bf16"])
@pytest.mark.parametrize("shape", [(1, 1, 1, 64, 16), (3, 7, 2, 80, 32), (5, 40, 8, 128, 16), (2, 300, 1, 256, 128),
                                   (2, 3, 3, 8, 1024)], ids=str)
def test_append_writes_the_named_slots_only(shape, dtype):
    B, n, H, D, P = shape
    t = TORCH_DTYPES[dtype]
    gen = torch.Generator(device="cuda").manual_seed(n)
    N = -(-B * n // P) + 2
    fused = torch.randn(B, n, 2 * H + 3, D, generator=gen, device="cuda").to(t)     # a fused projection's rows
    k, v = fused[:, :, 1:1 + H], fused[:, :, 2 + H:2 + 2 * H]
    both = torch.randn(N, 2, H, P, D, generator=gen, device="cuda").to(t)           # K and V pages alternate
    k_cache, v_cache = both[:, 0], both[:, 1]
    slots = torch.randperm(N * P, generator=gen, device="cuda")[:B * n].to(torch.int32).view(B, n)
    slots[0, n // 2] = -1
    if B > 1:
        slots[1, -1] = N * P            # outside the cache
        slots[1, 0] = -(1 << 31)
    want = both.clone()
    live = (slots >= 0) & (slots < N * P)
    at = slots[live].long()
    want[at // P, 0, :, at % P] = k[live]
    want[at // P, 1, :, at % P] = v[live]
    paged_cache.append(k, v, k_cache, v_cache, slots)
    torch.cuda.synchronize()
    assert torch.equal(both.view(torch.int16), want.view(torch.int16))


def test_plan_and_append_replay_in_a_graph():
    """A captured step (plan, append) replays as its eager twin goes, with eager work in between."""
    B, n, H, D, P = 6, 5, 2, 64, 16
    caches = [PagedCache(B, num_pages=80, page_size=P, max_pages=12, max_new=n) for _ in range(2)]
    stores = [tuple(torch.zeros(80, H, P, D, dtype=torch.float16, device="cuda") for _ in range(2)) for _ in range(2)]
    k = torch.zeros(B, n, H, D, dtype=torch.float16, device="cuda")
    v = torch.zeros_like(k)
    accepted, release = _dev([-1] * B), _dev([0] * B)
    side = torch.cuda.Stream()
    g = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(g, stream=side):
        caches[0].plan(n, accepted_len=accepted, release=release)
        caches[0].append(k, v, *stores[0])
    torch.cuda.synchronize()
    gen = torch.Generator(device="cuda").manual_seed(1)
    for step in range(6):
        accepted.copy_(torch.randint(-1, n, (B,), generator=gen, device="cuda"))
        release.copy_((torch.rand(B, generator=gen, device="cuda") < 0.2).int())
        k.normal_(generator=gen)
        v.normal_(generator=gen)
        g.replay()
        caches[1].plan(n, accepted_len=accepted, release=release)
        caches[1].append(k, v, *stores[1])
        torch.cuda.synchronize()
        for name in ("lengths", "counts", "held", "block_table", "free_pages", "free_count", "slots", "positions"):
            assert torch.equal(getattr(caches[0], name), getattr(caches[1], name)), (step, name)
        for x, y in zip(*stores):
            assert torch.equal(x, y), step
