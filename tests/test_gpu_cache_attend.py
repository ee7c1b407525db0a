"""The cache's attention (spec_cache_attend) against its definition in 64 bits,
within the bounds of tests/cache_util.py.  Everything that a call must not read
is NaN: entries behind a sequence's last token, pages of nobody, rows of q
behind a sequence's count; rows of the output there keep what they held."""
import numpy as np
import pytest
import torch

from paper_2406_11016_amd import paged_cache
from paper_2406_11016_amd.binding import SpecVerifyError
from paper_2406_11016_amd.paged_cache import PagedCache
from tests.cache_util import TORCH_DTYPES, attend_bound, attend_reference

pytestmark = pytest.mark.gpu
KEPT = 7.0   # what rows of the output hold that no call may write


@pytest.fixture(scope="module", autouse=True)
def gpu():
    if not torch.cuda.is_available():
        pytest.fail("no GPU visible")
    paged_cache.load_library()
    torch.cuda.init()


def make(B, n, H, K, D, P, prefix, lengths, counts, dtype, seed, spread=1.0):
    """A batch's tensors, NaN wherever nothing may be read."""
    t = TORCH_DTYPES[dtype]
    gen = torch.Generator(device="cuda").manual_seed(seed)
    M = max(1, max(-(-(l + max(c, 0)) // P) for l, c in zip(lengths, counts)))
    shared = -(-prefix // P)
    N = B * M + shared + 1
    order = torch.randperm(N, generator=gen, device="cuda").to(torch.int32)
    table = order[:B * M].view(B, M).clone()
    prefix_table = order[B * M:B * M + shared].clone()
    k = torch.full((N, K, P, D), float("nan"), dtype=t, device="cuda")
    v = k.clone()

    def fill(pages, count):
        if count <= 0:
            return
        at = torch.arange(count, device="cuda")
        for c, s in ((k, spread), (v, 1.0)):
            c[pages[at // P].long(), :, at % P] = (torch.randn(count, K, D, generator=gen, device="cuda") * s).to(t)

    for b in range(B):
        if counts[b] > 0:
            fill(table[b], lengths[b] + counts[b])
            table[b, -(-(lengths[b] + counts[b]) // P):] = -1
    fill(prefix_table, prefix)
    q = torch.full((B, n, H, D), float("nan"), dtype=t, device="cuda")
    for b in range(B):
        if counts[b] > 0:
            q[b, :counts[b]] = torch.randn(counts[b], H, D, generator=gen, device="cuda").to(t)
    ints = [torch.tensor(x, dtype=torch.int32, device="cuda") for x in (lengths, counts)]
    return q, k, v, table.contiguous(), ints[0], ints[1], prefix_table


def check(x, prefix, dtype, scale=None, label="", **more):
    q, k, v, table, lengths, counts, prefix_table = x
    out = more.pop("out", None)
    if out is None:
        out = torch.full(q.shape, KEPT, dtype=q.dtype, device="cuda")
    paged_cache.attend(q, k, v, table, lengths, counts, prefix_table=prefix_table, prefix_len=prefix, scale=scale, out=out,
                       **more)
    torch.cuda.synchronize()
    D = q.shape[3]
    c = counts.tolist()
    want, size, product = attend_reference(q, k, v, table.cpu().numpy(), lengths.tolist(), c,
                                           prefix_table.cpu().numpy(), prefix, D ** -0.5 if scale is None else scale)
    keys = prefix + max(int(l) + max(m, 0) for l, m in zip(lengths.tolist(), c))
    bound = attend_bound(size, product, dtype, D, keys, float(torch.nan_to_num(v.float(), 0.0).abs().max()))
    got = out.double().cpu().numpy()
    for b, m in enumerate(c):
        m = max(m, 0)
        assert np.all(got[b, m:] == KEPT), (label, b, "rows behind the last token")
        bad = ~(np.abs(got[b, :m] - want[b, :m]) <= bound[b, :m])
        assert not bad.any(), (label, b, np.argwhere(bad)[:4], got[b, :m][bad][:4], want[b, :m][bad][:4],
                               bound[b, :m][bad][:4])
    return out


# heads, key/value heads, head_dim
HEADS = [(4, 4, 64), (14, 2, 64), (6, 3, 80), (2, 1, 96), (8, 2, 128), (7, 1, 128), (8, 8, 128), (8, 1, 256), (2, 2, 256)]


@pytest.mark.parametrize("dtype", ["f16", "bf16"])
@pytest.mark.parametrize("heads", HEADS, ids=["h%dx%d_d%d" % h for h in HEADS])
def test_heads(heads, dtype):
    H, K, D = heads
    for n, prefix, lengths, counts in [(1, 0, [0], [1]), (5, 0, [1, 130, 0], [5, 3, 1]), (6, 77, [0, 40], [6, 2]),
                                       (21, 300, [255, 3, 129, 64], [21, 20, 1, 0])]:
        x = make(len(lengths), n, H, K, D, 16, prefix, lengths, counts, dtype, seed=n)
        check(x, prefix, dtype, label=(heads, n, prefix))


LENGTHS = [0, 1, 15, 16, 17, 126, 127, 128, 129, 255, 256, 1000]


@pytest.mark.parametrize("page", [16, 32, 64, 128, 512, 1024])
def test_lengths_around_pages_and_tiles(page):
    """Every border of a page, a run, a tile; with every count, without a prefix and with prefixes of odd lengths."""
    for n in (1, 2, 9):
        counts = [1 + (i * 5) % n for i in range(len(LENGTHS))]
        for prefix in (0, 1, 127, 128, 129, 640):
            x = make(len(LENGTHS), n, 4, 2, 64, page, prefix, LENGTHS, counts, "bf16", seed=page + n + prefix)
            check(x, prefix, "bf16", label=(page, n, prefix))


@pytest.mark.parametrize("n", [1, 7, 8, 9, 15, 16, 17, 31, 33, 64, 65, 130, 257])
def test_new_tokens_around_row_tiles(n):
    """32, 64 and 128 rows a task, and tasks of several tiles; pooled and joined prefixes."""
    for H, K, D, dtype in ((4, 1, 128, "bf16"), (3, 3, 64, "f16"), (10, 2, 80, "bf16"), (4, 2, 256, "f16")):
        for prefix in (0, 200):
            x = make(3, n, H, K, D, 32, prefix, [5, 0, 300], [n, max(1, n // 2), n], dtype, seed=n)
            check(x, prefix, dtype, label=(n, H, K, D, prefix))


def test_long_sequences_and_prefixes():
    """Tasks cut among many workgroups: one long sequence, a long prefix of one, and both beside short ones."""
    for B, n, H, K, D, prefix, lengths, dtype in [
            (1, 1, 2, 1, 128, 0, [70001], "bf16"), (1, 5, 4, 4, 64, 40007, [0], "f16"), (1, 130, 2, 1, 128, 0, [9000], "f16"),
            (5, 3, 4, 2, 128, 20000, [1, 30000, 0, 5, 4000], "bf16"), (2, 300, 4, 2, 64, 5000, [3000, 10], "bf16")]:
        x = make(B, n, H, K, D, 64, prefix, lengths, [n] * B, dtype, seed=B + n)
        check(x, prefix, dtype, label=(B, n, prefix))


@pytest.mark.parametrize("prefix", [0, 130])
def test_many_sequences(prefix):
    """More sequences than threads, some without tokens."""
    B = 300
    x = make(B, 2, 2, 1, 64, 16, prefix, [(b * 7) % 90 for b in range(B)], [(b % 4) - 1 for b in range(B)], "bf16", seed=4)
    check(x, prefix, "bf16")
    B = 4096
    x = make(B, 1, 1, 1, 64, 16, prefix, [b % 17 for b in range(B)], [b % 2 for b in range(B)], "f16", seed=5)
    check(x, prefix, "f16")


@pytest.mark.parametrize("prefix", [0, 40])
@pytest.mark.parametrize("B,D", [(4096, 128), (2048, 256)])
def test_largest_batches(B, D, prefix):
    """The batch's sums take the most LDS beside the tiles."""
    x = make(B, 1, 1, 1, D, 16, prefix, [b % 13 for b in range(B)], [b % 3 - 1 for b in range(B)], "bf16", seed=6)
    check(x, prefix, "bf16")
    if D == 256:
        with pytest.raises(SpecVerifyError, match="invalid sizes"):
            paged_cache.new_attend_workspace(B + 1, 1, 1, 1, D, "cuda")


@pytest.mark.parametrize("B,n,H,K,D,P", [(32, 128, 8, 8, 64, 16), (16, 125, 16, 16, 128, 32), (64, 16, 8, 2, 256, 64),
                                         (33, 37, 24, 8, 80, 16), (130, 500, 2, 1, 96, 128)])
@pytest.mark.parametrize("prefix", [1, 64, 333])
def test_tasks_that_run_over_the_prefix_themselves(B, n, H, K, D, P, prefix):
    """Many sequences with nearly full row tiles; some have fewer tokens, or none, or nothing cached."""
    counts = [n if b % 4 else max(0, n - 9 * b) for b in range(B)]
    x = make(B, n, H, K, D, P, prefix, [(37 * b) % 150 for b in range(B)], counts, "bf16" if B % 2 else "f16", seed=B)
    check(x, prefix, "bf16" if B % 2 else "f16")


@pytest.mark.parametrize("n", [1, 5, 30])
@pytest.mark.parametrize("H,K,D", [(8, 1, 256), (4, 2, 128), (2, 1, 80)])
def test_rows_of_many_parts(H, K, D, n):
    """One long sequence, or a few behind a long prefix: a row's keys are shared out to most workgroups."""
    x = make(1, n, H, K, D, 64, 0, [20011], [n], "bf16", seed=n)
    check(x, 0, "bf16")
    x = make(3, n, H, K, D, 64, 15005, [300, 0, 9000], [n, 0, max(1, n - 2)], "f16", seed=n)
    check(x, 15005, "f16")


def test_more_rows_than_a_launch_has_waves_in_one_dimension():
    """4096 x 513 x 32 rows of q, of which four sequences have a few tokens."""
    if torch.cuda.mem_get_info()[0] < 80 << 30:
        pytest.skip("needs 60 GB of memory")
    B, n, H, D = 4096, 513, 32, 64
    some = [0, 1, 2049, B - 1]
    x = make(len(some), n, H, H, D, 16, 20, [5, 0, 30, 17], [3, 1, 2, 5], "bf16", seed=11)
    q, k, v, table, lengths, counts, prefix_table = x
    at = torch.tensor(some, device="cuda")

    def spread(small, fill):
        big = torch.full((B, *small.shape[1:]), fill, dtype=small.dtype, device="cuda")
        big[at] = small
        return big

    out = torch.full((B, n, H, D), KEPT, dtype=q.dtype, device="cuda")
    paged_cache.attend(spread(q, float("nan")), k, v, spread(table, -1), spread(lengths, 3), spread(counts, 0),
                       prefix_table=prefix_table, prefix_len=20, out=out)
    want, size, product = attend_reference(q, k, v, table.cpu().numpy(), lengths.tolist(), counts.tolist(),
                                           prefix_table.cpu().numpy(), 20, D ** -0.5)
    bound = attend_bound(size, product, "bf16", D, 60, float(torch.nan_to_num(v.float(), 0.0).abs().max()))
    got = out[at].double().cpu().numpy()
    for i, m in enumerate(counts.tolist()):
        assert np.all(np.abs(got[i, :m] - want[i, :m]) <= bound[i, :m]), some[i]
    for b in range(B):
        first = counts[some.index(b)].item() if b in some else 0
        assert bool((out[b, first:] == KEPT).all()), b


def test_nothing_to_do():
    x = make(3, 4, 4, 2, 64, 16, 100, [5, 6, 7], [0, -1, 0], "bf16", seed=1)
    check(x, 100, "bf16")


def test_without_counts_and_with_scales():
    x = make(2, 3, 4, 2, 128, 16, 50, [30, 8], [3, 3], "bf16", seed=2)
    q, k, v, table, lengths, counts, prefix_table = x
    a = paged_cache.attend(q, k, v, table, lengths, counts, prefix_table=prefix_table, prefix_len=50)
    b = paged_cache.attend(q, k, v, table, lengths, prefix_table=prefix_table, prefix_len=50)
    assert torch.equal(a, b)
    for scale in (1e-6, 0.5, 1.0):
        check(x, 50, "bf16", scale=scale)


@pytest.mark.parametrize("prefix", [0, 200])
def test_rising_and_far_apart_scores(prefix):
    """Scores that rise along the keys (each tile a new maximum, by more and by less than the step that is let pass)
    and reach far from zero: the weights stay relative to a maximum."""
    for rise in (0.01, 0.2, 3.0):
        x = make(2, 4, 4, 1, 64, 16, prefix, [700, 90], [4, 4], "bf16", seed=3)
        q, k, v, table, lengths, counts, prefix_table = x
        q.fill_(1.0)
        for b in range(2):
            L = int(lengths[b]) + 4
            at = torch.arange(L, device="cuda")
            ramp = ((prefix + at) * rise / 8).to(k.dtype)
            k[table[b][at // 16].long(), :, at % 16] = ramp[:, None, None].expand(L, 1, 64)
        if prefix:
            at = torch.arange(prefix, device="cuda")
            k[prefix_table[at // 16].long(), :, at % 16] = (at * rise / 8).to(k.dtype)[:, None, None].expand(prefix, 1, 64)
        check(x, prefix, "bf16", label=rise)


@pytest.mark.parametrize("dtype", ["f16", "bf16"])
def test_values_that_a_token_does_not_see(dtype):
    """An infinity or NaN in a later token's key or value leaves earlier tokens as they are, and reaches the others."""
    low = torch.finfo(TORCH_DTYPES[dtype]).min
    for what in (float("nan"), float("inf"), float("-inf"), low):
        for D, H, K, n in ((64, 4, 2, 6), (128, 8, 1, 6), (80, 2, 2, 6), (256, 4, 1, 20)):
            x = make(2, n, H, K, D, 16, 40, [125, 3], [n, n], dtype, seed=6)
            q, k, v, table, lengths, counts, prefix_table = x
            clean = check(x, 40, dtype)
            at = int(lengths[0]) + 3                       # token 3 of sequence 0
            page, off = int(table[0][at // 16]), at % 16
            saved = v[page, :, off].clone()
            v[page, 0, off, 1] = what
            v[page, 0, off, D - 1] = what
            dirty = torch.full_like(clean, KEPT)
            paged_cache.attend(q, k, v, table, lengths, counts, prefix_table=prefix_table, prefix_len=40, out=dirty)
            assert torch.equal(dirty[0, :3], clean[0, :3]) and torch.equal(dirty[1], clean[1]), (what, D)
            G = H // K
            others = [d for d in range(D) if d not in (1, D - 1)]
            assert torch.equal(dirty[0, 3:, :G][..., others], clean[0, 3:, :G][..., others])
            if what != low:
                assert not torch.isfinite(dirty[0, 3:, :G][..., [1, D - 1]]).any()
                if what == what:
                    assert (dirty[0, 3:, :G][..., [1, D - 1]].float() == what).all()
            if K > 1:
                assert torch.equal(dirty[0, :, G:], clean[0, :, G:])
            v[page, :, off] = saved
            k[page, :, off] = what
            paged_cache.attend(q, k, v, table, lengths, counts, prefix_table=prefix_table, prefix_len=40, out=dirty)
            assert torch.equal(dirty[0, :3], clean[0, :3]) and torch.equal(dirty[1], clean[1]), (what, D)
            if what != what:
                assert torch.isnan(dirty[0, 3:]).all()


def test_infinite_scores():
    """Keys whose score is -inf have no weight; a row with +inf is NaN, as in the definition."""
    x = make(1, 2, 2, 1, 64, 16, 0, [300], [2], "bf16", seed=8)
    q, k, v, table, lengths, counts, prefix_table = x
    q.abs_()
    at = torch.arange(300, device="cuda")
    k[table[0][at[::3] // 16].long(), :, at[::3] % 16] = float("-inf")
    out = paged_cache.attend(q, k, v, table, lengths, counts)
    kk = k.clone()
    want, _, _ = attend_reference(q, torch.where(torch.isinf(kk), -3e4, kk.float()).to(torch.float32), v, table.cpu().numpy(),
                                  [300], [2], None, 0, 0.125)
    assert torch.isfinite(out).all() and np.allclose(out.double().cpu().numpy(), want, rtol=0, atol=0.02)
    k[table[0, 3].long(), 0, 5] = float("inf")
    assert torch.isnan(paged_cache.attend(q, k, v, table, lengths, counts)).all()


def test_bad_tables_make_their_sequence_nan():
    x = make(4, 3, 4, 2, 64, 16, 60, [200, 30, 70, 9], [3, 3, 2, 3], "bf16", seed=9)
    q, k, v, table, lengths, counts, prefix_table = x
    clean = check(x, 60, "bf16")

    def run():
        out = torch.full_like(clean, KEPT)
        paged_cache.attend(q, k, v, table, lengths, counts, prefix_table=prefix_table, prefix_len=60, out=out)
        return out

    for word in (-1, k.shape[0], 1 << 30, -(1 << 31)):
        saved = table[0, 5].clone()
        table[0, 5] = word
        out = run()
        assert torch.isnan(out[0]).all() and torch.equal(out[1:], clean[1:]), word
        table[0, 5] = saved
        table[1, 3] = word                 # behind its last token's page: not looked at
        assert torch.equal(run(), clean)
        saved = prefix_table[1].clone()
        prefix_table[1] = word
        out = run()
        for b, m in enumerate(counts.tolist()):
            assert torch.isnan(out[b, :m]).all() and (out[b, m:] == KEPT).all()
        prefix_table[1] = saved
    for tensor, word, whole in ((lengths, -1, 3), (lengths, table.shape[1] * 16 - 1, 3), (lengths, (1 << 31) - 1, 3),
                                (counts, 4, 3), (counts, (1 << 31) - 1, 3)):
        saved = tensor[1].clone()
        tensor[1] = word
        out = run()
        assert torch.isnan(out[1]).all() and torch.equal(out[[0, 2, 3]], clean[[0, 2, 3]]), word
        tensor[1] = saved
    for prefix in (0, 60):                 # joined, too
        lengths[2] = -7
        out = torch.full_like(clean, KEPT)
        paged_cache.attend(q, k, v, table, lengths, counts, prefix_table=prefix_table, prefix_len=prefix, out=out)
        assert torch.isnan(out[2, :2]).all() and (out[2, 2:] == KEPT).all()


def test_strides_and_layouts():
    """q from a fused projection, an output that is a view, K and V in alternating pages, 16-byte aligned starts."""
    x = make(3, 5, 8, 2, 128, 32, 90, [10, 200, 0], [5, 4, 2], "bf16", seed=11)
    q, k, v, table, lengths, counts, prefix_table = x
    plain = check(x, 90, "bf16")
    fused = torch.full((3, 5, 13, 136), float("nan"), dtype=q.dtype, device="cuda")
    fused[:, :, 3:11, 8:] = q
    both = torch.stack([k, v], 1)
    token_major = torch.full((5, 3, 9, 144), KEPT, dtype=q.dtype, device="cuda")
    out = token_major.permute(1, 0, 2, 3)[:, :, 1:, 8:136]
    paged_cache.attend(fused[:, :, 3:11, 8:], both[:, 0], both[:, 1], table, lengths, counts, prefix_table=prefix_table,
                       prefix_len=90, out=out)
    assert torch.equal(out, plain)
    assert (token_major[..., :8] == KEPT).all() and (token_major[..., 136:] == KEPT).all()
    assert (token_major[:, :, 0] == KEPT).all()


def test_offsets_past_32_bits():
    """Pages whose entries lie behind 2^31 elements (2^32 bytes) of the caches."""
    K, P, D = 8, 1024, 128
    N = (1 << 31) // (K * P * D) + 3
    k = torch.empty(N, K, P, D, dtype=torch.bfloat16, device="cuda")
    v = torch.empty_like(k)
    cache = PagedCache(2, num_pages=N, page_size=P, max_pages=2, max_new=1100, prefix_pages=1)
    cache.set_prefix(1000)
    cache.free_pages[:4] = torch.tensor([3, N - 3, N - 2, N - 1], dtype=torch.int32)
    cache.free_count.fill_(4)
    gen = torch.Generator(device="cuda").manual_seed(12)

    def rand(*shape):
        return torch.randn(*shape, generator=gen, device="cuda").to(torch.bfloat16)

    cache.append_prefix(rand(1, 1000, K, D), rand(1, 1000, K, D), k, v)
    new = torch.tensor([1100, 900], dtype=torch.int32, device="cuda")
    slots, positions = cache.plan(1100, new_tokens=new)
    assert int(slots.max()) >= (N - 2) * P and positions[0, :2].tolist() == [1000, 1001]
    cache.append(rand(2, 1100, K, D), rand(2, 1100, K, D), k, v)
    cache.plan(3)                          # the prompts stay
    cache.append(rand(2, 3, K, D), rand(2, 3, K, D), k, v)
    q = rand(2, 3, K, D)
    out = cache.attend(q, k, v)
    want, size, product = attend_reference(q, k, v, cache.block_table.cpu().numpy(), cache.lengths.tolist(), [3, 3],
                                           cache.prefix_table.cpu().numpy(), 1000, D ** -0.5)
    assert np.all(np.abs(out.double().cpu().numpy() - want) <= attend_bound(size, product, "bf16", D, 2103, 6.0))


def test_other_streams_and_graphs():
    """Two captured calls that share a workspace, replayed in turn with eager calls between, on other streams."""
    xs = [make(4, 3, 8, 2, 128, 16, p, [40, 300, 0, 77], [3, 2, 3, 1], "bf16", seed=20 + p) for p in (0, 333)]
    size = paged_cache.attend_workspace_bytes(4, 3, 8, 2, 128)
    shared = torch.full((size,), 255, dtype=torch.uint8, device="cuda")
    eager = [check(x, p, "bf16") for x, p in zip(xs, (0, 333))]
    outs = [torch.full_like(e, KEPT) for e in eager]
    graphs = []
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    for (q, k, v, table, lengths, counts, prefix_table), p, out in zip(xs, (0, 333), outs):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g, stream=side):
            paged_cache.attend(q, k, v, table, lengths, counts, prefix_table=prefix_table, prefix_len=p, out=out,
                               workspace=shared)
        graphs.append(g)
    torch.cuda.synchronize()
    for rep in range(4):
        for g, out, e in zip(graphs, outs, eager):
            out.fill_(KEPT)
            g.replay()
            torch.cuda.synchronize()
            assert torch.equal(out, e), rep
        with torch.cuda.stream(side):
            again = check(xs[rep % 2], (0, 333)[rep % 2], "bf16", workspace=shared)
        assert torch.equal(again, eager[rep % 2])
        # new lengths under a captured call
        if rep == 2:
            xs[1][4][1] -= 100
            eager[1] = check(xs[1], 333, "bf16")


@pytest.mark.parametrize("seed", range(6))
def test_drawn_batches(seed):
    """Sizes, layouts and lengths by chance."""
    rng = np.random.default_rng(seed)
    for _ in range(6):
        K = int(rng.integers(1, 5))
        H, D = K * int(rng.integers(1, 9)), int(rng.choice([64, 80, 96, 128, 256]))
        B, n = int(rng.integers(1, 20)), int(rng.choice([1, 2, 5, 9, 21, 40]))
        P, prefix = int(rng.choice([16, 32, 64, 256])), int(rng.choice([0, 0, 1, 50, 500, 3000]))
        lengths = [int(x) for x in rng.integers(0, rng.choice([2, 40, 900]), B)]
        counts = [int(x) for x in rng.integers(-1, n + 1, B)]
        dtype = str(rng.choice(["f16", "bf16"]))
        x = make(B, n, H, K, D, P, prefix, lengths, counts, dtype, seed=seed, spread=float(rng.choice([0.2, 1.0, 4.0])))
        check(x, prefix, dtype, label=(seed, B, n, H, K, D, P, prefix))
