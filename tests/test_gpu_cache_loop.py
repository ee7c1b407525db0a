"""The cache's operators together, as a decoder runs them: a prefix that all
sequences share, prompts, and the decoding loop's steps, in which the plan goes
by what was verified.  Each step's attention is checked against the dense
attention of the tokens that each sequence has kept, gathered on the host."""
import numpy as np
import pytest
import torch

from paper_2406_11016_amd import binding, paged_cache
from paper_2406_11016_amd import workloads as W
from paper_2406_11016_amd.decode_loop import DecodeLoop, SyntheticSteps
from paper_2406_11016_amd.paged_cache import PagedCache
from tests.cache_util import attend_bound

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def gpu():
    if not torch.cuda.is_available():
        pytest.fail("no GPU visible")
    paged_cache.load_library()
    torch.cuda.init()


H, K, D, DTYPE = 4, 2, 64, torch.bfloat16


def _dense(q, keys, values, first):
    """Attention of tokens that follow `first` ones to everything up to themselves, 64 bits; and with |v|."""
    n = q.shape[0]
    out, size, product = np.zeros((n, H, D)), np.zeros((n, H, D)), 0.0
    seen = np.arange(len(keys))[None] <= first + np.arange(n)[:, None]
    for h in range(H):
        k, v = keys[:, h // (H // K)], values[:, h // (H // K)]
        z = q[:, h] @ k.T / 8.0
        product = max(product, (np.abs(q[:, h]) @ np.abs(k).T).max() / 8.0)
        z = np.where(seen, z, -np.inf)
        w = np.exp(z - z.max(-1, keepdims=True))
        w /= w.sum(-1, keepdims=True)
        out[:, h], size[:, h] = w @ v, w @ np.abs(v)
    return out, size, product


class Model:
    """Two layers' attention of random queries, keys and values; the host keeps what each sequence holds."""

    def __init__(self, loop, steps, prefix, prompts, seed):
        self.loop, self.steps = loop, steps
        self.gen = torch.Generator(device="cuda").manual_seed(seed)
        cache = loop.cache
        self.layers = [cache.new_storage(K, D, DTYPE) for _ in range(2)]
        for pair in self.layers:
            for x in pair:
                x.fill_(float("nan"))
        self.held = [[[] for _ in range(cache.batch)] for _ in self.layers]   # (k, v) rows by layer and sequence
        self.pending = None
        B = cache.batch
        with torch.cuda.stream(loop.stream):
            for l, pair in enumerate(self.layers):
                k, v = self.rand(1, prefix, K), self.rand(1, prefix, K)
                cache.append_prefix(k, v, *pair)
                rows = list(zip(k[0].double().cpu().numpy(), v[0].double().cpu().numpy()))
                for b in range(B):
                    self.held[l][b] += rows
            cache.set_prefix(prefix)
            new = torch.tensor(prompts, dtype=torch.int32, device="cuda")
            cache.plan(max(prompts), new_tokens=new)
            self.step_tokens(max(prompts), prompts)
        self.keep([p - 1 for p in prompts])

    def rand(self, *shape):
        return torch.randn(*shape, D, generator=self.gen, device="cuda").to(DTYPE)

    def step_tokens(self, n, counts):
        """One pass of n tokens a sequence through both layers, checked."""
        cache, B = self.loop.cache, self.loop.cache.batch
        self.pending = []
        for l, pair in enumerate(self.layers):
            q, k, v = self.rand(B, n, H), self.rand(B, n, K), self.rand(B, n, K)
            cache.append(k, v, *pair)
            out = cache.attend(q, *pair)
            self.pending.append((k.double().cpu().numpy(), v.double().cpu().numpy()))
            q, out = q.double().cpu().numpy(), out.double().cpu().numpy()
            positions = cache.positions.cpu().numpy()
            for b in range(B):
                m, held = counts[b], self.held[l][b]
                assert positions[b].tolist() == [len(held) + i for i in range(m)] + [-1] * (n - m)
                if m == 0:
                    continue
                rows = held + list(zip(self.pending[l][0][b, :m], self.pending[l][1][b, :m]))
                keys, values = (np.stack([r[x] for r in rows]) for x in (0, 1))
                want, size, product = _dense(q[b, :m], keys, values, len(held))
                bound = attend_bound(size, product, "bf16", D, len(rows), 6.0)
                assert np.all(np.abs(out[b, :m] - want) <= bound), (l, b, np.abs(out[b, :m] - want).max())

    def keep(self, accepted):
        for l in range(2):
            for b, a in enumerate(accepted):
                for i in range(a + 1):
                    self.held[l][b].append((self.pending[l][0][b, i], self.pending[l][1][b, i]))
        self.pending = None

    def __call__(self, loop, i, gamma):
        if self.pending is not None:
            self.keep(loop.acc.tolist())          # (what the last step accepted)
        with torch.cuda.stream(loop.stream):
            self.step_tokens(gamma + 1, [gamma + 1] * loop.cache.batch)
        self.steps(loop, i, gamma)


@pytest.mark.parametrize("native,graphs", [(False, False), (True, False), (False, True)])
def test_decoding_with_a_cache(native, graphs):
    B, prefix, prompts = 5, 37, [3, 30, 16, 1, 9]
    w = W.WORKLOADS["exact_b1_g5_v51865_f32"].with_(batch=B, vocab=1009)
    cache = PagedCache(B, num_pages=64, page_size=16, max_pages=12, max_new=30, prefix_pages=3)
    loop = DecodeLoop(B, 1009, "f32", gamma0=3, gamma_max=6, cache=cache, native=native, use_graphs=graphs)
    model = Model(loop, SyntheticSteps(w, 6, 4), prefix, prompts, seed=5)
    stats = loop.run(model, 7)
    assert stats.iterations == 7 and any(int(a.min()) >= 0 for a in stats.accepted)
    model.keep(loop.acc.tolist())
    # two sequences end; new ones with prompts take their places
    release = torch.tensor([0, 1, 0, 0, 1], dtype=torch.int32, device="cuda")
    new = [0, 20, 0, 0, 5]
    with torch.cuda.stream(loop.stream):
        cache.plan(20, new_tokens=torch.tensor(new, dtype=torch.int32, device="cuda"), accepted_len=loop.acc,
                   release=release)
        for held in model.held:
            for b in (1, 4):
                del held[b][prefix:]
        model.step_tokens(20, new)
    model.keep([n - 1 for n in new])
    loop.program_planned()
    stats = loop.run(model, 4, stats)
    assert stats.iterations == 11
    lengths = [prefix + int(x) for x in cache.lengths]
    assert lengths == [len(h) for h in model.held[0]]       # (the last step's tokens are not kept yet)
    assert int((cache.block_table >= 0).sum()) + int(cache.free_count) == 64 - 3
    loop.close()


def test_refusals_on_the_device():
    B, n = 2, 3
    cache = PagedCache(B, num_pages=8, page_size=16, max_pages=3, max_new=n)
    k_cache, v_cache = cache.new_storage(2, 64, torch.float16)
    k_cache.zero_(), v_cache.zero_()
    q = torch.zeros(B, n, 4, 64, dtype=torch.float16, device="cuda")
    k = torch.zeros(B, n, 2, 64, dtype=torch.float16, device="cuda")
    acc = torch.zeros(B, dtype=torch.int32, device="cuda")
    bad = [
        lambda: cache.plan(0), lambda: cache.plan(n + 1), lambda: cache.plan(n, accepted_len=acc.long()),
        lambda: cache.plan(n, new_tokens=acc[:1]), lambda: cache.plan(n, release=acc.cpu()),
        lambda: cache.set_prefix(1), lambda: cache.new_storage(2, 64, torch.float32),
        lambda: cache.append(k, k[:, :2], k_cache, v_cache), lambda: cache.append(k.bfloat16(), k, k_cache, v_cache),
        lambda: cache.append(k[:, :, :1], k[:, :, :1], k_cache, v_cache),
        lambda: cache.append(k.transpose(2, 3), k.transpose(2, 3), k_cache, v_cache),
        lambda: cache.append(k, k, k_cache, v_cache[:4]), lambda: cache.append(k, k, k_cache[:, :, ::2], v_cache[:, :, ::2]),
        lambda: cache.append_prefix(k[:1], k[:1], k_cache, v_cache),
        lambda: cache.attend(q[..., :32], k_cache, v_cache), lambda: cache.attend(q.float(), k_cache, v_cache),
        lambda: cache.attend(q[:, :, :3], k_cache, v_cache), lambda: cache.attend(q, k_cache, v_cache, scale=0.0),
        lambda: cache.attend(q, k_cache, v_cache, out=q[:1]), lambda: cache.attend(q, k_cache, v_cache, out=q.float()),
        lambda: cache.attend(torch.zeros(B, n, 4, 68, dtype=torch.float16, device="cuda")[..., 4:], k_cache, v_cache),
        lambda: paged_cache.attend(q, k_cache, v_cache, cache.block_table, cache.lengths[:1]),
        lambda: paged_cache.attend(q, k_cache, v_cache, cache.block_table.long(), cache.lengths),
        lambda: paged_cache.attend(q, k_cache, v_cache, cache.block_table, cache.lengths, prefix_len=3),
        lambda: paged_cache.attend(q, k_cache, v_cache, cache.block_table, cache.lengths, prefix_len=17,
                                   prefix_table=cache.block_table[0, :1]),
        lambda: paged_cache.attend(q, k_cache, v_cache, cache.block_table, cache.lengths,
                                   workspace=torch.zeros(64, dtype=torch.uint8, device="cuda")),
        lambda: PagedCache.over(cache.lengths, cache.counts, cache.held, cache.block_table, cache.free_pages,
                                cache.free_count, page_size=24, max_new=2),
        lambda: PagedCache.over(cache.lengths, cache.counts, cache.held, cache.block_table.t(), cache.free_pages,
                                cache.free_count, page_size=16, max_new=2),
    ]
    for i, f in enumerate(bad):
        with pytest.raises(binding.SpecVerifyError):
            f()
            pytest.fail(f"call {i} was not refused")
    cache.plan(n)
    cache.append(k, k, k_cache, v_cache)
    assert not cache.attend(q, k_cache, v_cache).any()


def test_workspaces_of_steps_of_many_sizes():
    """A workspace for each power of two of bytes serves all sizes of a step; the results are attend()'s."""
    cache = PagedCache(2, num_pages=16, page_size=16, max_pages=6, max_new=80)
    gen = torch.Generator(device="cuda").manual_seed(3)
    k, v = (torch.randn(16, K, 16, D, device="cuda", generator=gen).to(DTYPE) for _ in range(2))
    ended = torch.ones(2, dtype=torch.int32, device="cuda")
    for n in range(1, 81):
        cache.plan(n, release=ended)
        q = torch.randn(2, n, H, D, device="cuda", generator=gen).to(DTYPE)
        want = paged_cache.attend(q, k, v, cache.block_table, cache.lengths, cache.counts)
        assert torch.equal(cache.attend(q, k, v), want)
    assert len(cache._workspaces) <= 8
    with pytest.raises(binding.SpecVerifyError, match="q must be"):
        cache.attend(q[0], k, v)
