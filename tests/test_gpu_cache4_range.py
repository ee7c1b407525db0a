"""The attention over a cache in 4 bits at the ends of its types' ranges, and over runs of many units: scores far from
zero, their last bits, small weights of large values, large values, long tasks of few rows."""
import numpy as np
import pytest
import torch

from paper_2406_11016_amd import paged_cache
from tests import cache4_util as C4
from tests.cache_util import TORCH_DTYPES, attend_bound, attend_reference

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def gpu():
    if not torch.cuda.is_available():
        pytest.fail("no GPU visible")
    paged_cache.load_library()
    torch.cuda.init()


def _ints(x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


class Sequences:
    """Sequences one after the other in their pages; keys of zeros, values at random, both as 4 bits hold them."""

    def __init__(self, n, H, D, P, lengths, dtype, seed, prefix=0):
        self.t, self.n, self.P, self.D, self.lengths, self.prefix = TORCH_DTYPES[dtype], n, P, D, lengths, prefix
        gen = torch.Generator(device="cuda").manual_seed(seed)
        B, M, self.shared = len(lengths), -(-(max(lengths) + n) // P), -(-prefix // P)
        order = torch.randperm(B * M + self.shared, generator=gen, device="cuda").to(torch.int32)
        self.table, self.prefix_table = order[:B * M].view(B, M).contiguous(), order[B * M:].contiguous()
        self.k = torch.zeros(B * M + self.shared, 1, P, D, dtype=self.t, device="cuda")
        self.v = torch.randn(B * M + self.shared, 1, P, D, generator=gen, device="cuda").to(self.t)
        self.q = torch.zeros(B, n, H, D, dtype=self.t, device="cuda")

    def at(self, b, j):
        """Pages and places of tokens j of sequence b, the prefix's first."""
        own = j - self.prefix
        pages = self.table[b][own.clamp(min=0) // self.P]
        if self.shared:
            pages = torch.where(own >= 0, pages, self.prefix_table[(j // self.P).clamp(max=self.shared - 1)])
        return pages.long(), torch.where(own >= 0, own, j) % self.P

    def run(self, scale):
        k4, v4 = C4.pack(self.k), C4.pack(self.v)
        self.k, self.v = C4.unpack(k4, self.P, self.D, self.t), C4.unpack(v4, self.P, self.D, self.t)
        return paged_cache.attend4(self.q, k4, v4, self.table, _ints(self.lengths), prefix_table=self.prefix_table,
                                   prefix_len=self.prefix, scale=scale)

    def repeat(self, B):
        """B sequences of the first one's pages."""
        self.table, self.q = self.table.expand(B, -1).contiguous(), self.q.expand(B, -1, -1, -1).contiguous()
        self.lengths = self.lengths * B


NUMBERS = np.array([-6.0, -4, -3, -2, -1.5, -1, -0.5, 0, 0.5, 1, 1.5, 2, 3, 4, 6])
SHAPES = [(1, 64, 16, 0, [9000]), (3, 128, 16, 150, [300, 0]), (9, 80, 32, 0, [700, 5, 64]), (2, 256, 64, 2000, [900]),
          (12, 96, 16, 0, [300, 40]), (40, 128, 64, 0, [500, 200])]


@pytest.mark.parametrize("dtype", ["f16", "bf16"])
@pytest.mark.parametrize("n,D,P,prefix,lengths", SHAPES, ids=str)
def test_far_scores_choose_the_nearest_key(n, D, P, prefix, lengths, dtype):
    """With scores that are a scale of 2^7 and more times halves of small whole numbers, exact in fp32, a weight is
    1 / (number of keys with the highest score), or at most exp(-64) of that.  One head looks for the highest number, one
    for the lowest, one for the highest beside a term of -240 and one has all scores 0.  Bound: weights and output rounded,
    u each, and 2 (keys + 64) roundings of 2^-24."""
    u = torch.finfo(TORCH_DTYPES[dtype]).eps / 2
    for scale in (2.0 ** 7, 2.0 ** 13, 2.0 ** 24, 2.0 ** 40, 2.0 ** 96, 9e29):
        x = Sequences(n, 4, D, P, lengths, dtype, n, prefix)
        x.q[:, :, 0, 0], x.q[:, :, 1, 0] = 1.0, -1.0
        x.q[:, :, 2, 0], x.q[:, :, 2, 32] = 1.0, -40.0
        rng = np.random.default_rng(n)
        shared = rng.choice(NUMBERS, prefix)
        every = []
        for b, length in enumerate(lengths):
            numbers = np.concatenate([shared, rng.choice(NUMBERS, length + n)])
            pages, at = x.at(b, torch.arange(len(numbers), device="cuda"))
            x.k[pages, 0, at, 0] = torch.tensor(numbers, device="cuda").to(x.t)
            x.k[pages, 0, at, 32] = 6.0
            every.append(numbers)
        out = x.run(scale).double().cpu()
        keys = prefix + max(lengths) + n
        for b, numbers in enumerate(every):
            pages, at = x.at(b, torch.arange(len(numbers), device="cuda"))
            assert np.array_equal(x.k[pages, 0, at, 0].double().cpu().numpy(), numbers)
            values = x.v[pages, 0, at].double().cpu()
            for i in range(n):
                seen = numbers[:prefix + lengths[b] + i + 1]
                for h, score in enumerate((seen, -seen, seen - 240, 0 * seen)):
                    best = np.flatnonzero(score == score.max())
                    want, most = values[best].mean(0), values[best].abs().mean(0).max()
                    bound = (2 * u * (1 + u) + 2 * (keys + 64) * 2.0 ** -24) * most + (2.0 ** -24 if dtype == "f16" else 0.0)
                    assert ((out[b, i, h] - want).abs() <= bound).all(), (scale, b, i, h)


@pytest.mark.parametrize("dtype", ["f16", "bf16"])
@pytest.mark.parametrize("n,prefix", [(2, 0), (2, 130), (11, 0), (40, 0)])
@pytest.mark.parametrize("steps", [1.0, 3.0, 6.0, 12.0])
def test_rises_of_the_last_bit_of_far_scores(dtype, n, prefix, steps):
    """Scores 4096 + j 2^-11, exact in fp32, one last bit apart, which is `steps` in log2 units.  600 sequences of one set of
    pages, so that a workgroup has most of a sequence's units.  Bound: exact scores; a weight's argument (at most 6 steps,
    72) is off by 4 roundings of 2^-24, scale's among them, so the weights by 2^-15 of themselves, twice; weights and output
    rounded; 2 (keys + 64) roundings of 2^-24 of the sums; fp16 weights below 2^-14 next to 2^7, 2^-32 of the largest each."""
    D, B, length = 128, 600, 400
    x = Sequences(n, 2, D, 16, [length], dtype, 9, prefix)
    x.q[:, :, :, 0], x.q[:, :, :, 32] = 64.0, 2.0 ** -11
    scale = steps * 2.0 ** 11 * float(np.log(2.0))
    j = torch.arange(prefix + length + n, device="cuda")
    pages, at = x.at(0, j)
    x.k[pages, 0, at, 0] = 64.0
    x.k[pages, 0, at, 32] = torch.tensor([0.0, 1, 2, 3, 4, 6], device="cuda")[(j // 64) % 6].to(x.t)
    x.repeat(B)
    out = x.run(scale).double()
    u, keys = torch.finfo(x.t).eps / 2, prefix + length + n
    for i in range(n):
        seen = slice(0, prefix + length + i + 1)
        z = x.k[pages[seen], 0, at[seen]].double() @ x.q[0, i].double().t()
        w = torch.softmax(z * float(np.float32(scale)), 0)
        values = x.v[pages[seen], 0, at[seen]].double()
        want, size = w.t() @ values, w.t() @ values.abs()
        bound = (2 * u * (1 + u) + 2 * 2.0 ** -15 + 2 * (keys + 64) * 2.0 ** -24) * size + \
            (keys * 2.0 ** -32 * 6.0 + 2.0 ** -25 if dtype == "f16" else 0.0)
        wrong = ~((out[:, i] - want).abs() <= bound)
        assert not wrong.any(), (i, wrong.nonzero()[:3].tolist())


@pytest.mark.parametrize("n", [1, 40])
@pytest.mark.parametrize("prefix", [0, 1000])
def test_small_fp16_weights_of_large_values_count(prefix, n):
    """One key of value 0 and a thousand others of weight exp(-18) and exp(-20), 2^-26 and 2^-29.  Bound as in the 16-bit
    attention's test: the output rounded; scores exact; 2 (keys + 64) roundings; weights next to 2^7 off by 2^-32 each."""
    B, own = 600, 0 if prefix else 1000
    x = Sequences(n, 1, 64, 64, [own], "f16", 1, prefix)
    x.q[:, :, 0, 0] = x.q[:, :, 0, 32] = 1.0
    count = 1000 + n
    j = torch.arange(count, device="cuda")
    pages, at = x.at(0, j)
    score = torch.where(j % 2 == 0, -18.0, -20.0)
    x.k[pages, 0, at, 0] = -16.0
    x.k[pages, 0, at, 32] = (score + 16).to(x.t)
    large = torch.tensor([8192.0, 16384, 24576, 49152], device="cuda")[j * 7 % 4]
    x.v[pages, 0, at] = large[:, None].expand(count, 64).to(x.t)
    x.k[pages[500], 0, at[500]], x.v[pages[500], 0, at[500]], score[500] = 0.0, 0.0, 0.0
    for i in range(1000, count):                              # (the new tokens)
        x.k[pages[i], 0, at[i], 0], x.k[pages[i], 0, at[i], 32], x.v[pages[i], 0, at[i]] = -32.0, 0.0, 0.0
        score[i] = -32.0
    x.repeat(B)
    out = x.run(1.0).double()
    values = x.v[pages, 0, at].double()
    assert torch.equal(values[:500, 0].float(), large[:500])
    want = torch.softmax(score.double()[:1001], 0) @ values[:1001]
    assert float(want.min()) > 0.1
    bound = (2.0 ** -11 + 2 * (count + 64) * 2.0 ** -24) * want + 2.0 ** -32 * values.sum(0)
    assert ((out[:, 0, 0] - want).abs() <= bound).all(), (out[0, 0, 0, :4], want[:4])


@pytest.mark.parametrize("prefix", [0, 300])
@pytest.mark.parametrize("n,D", [(1, 64), (6, 128), (30, 128), (40, 96)])
def test_large_values_do_not_overflow(n, D, prefix):
    """bfloat16 values of 1.3e38 and less, of one sign or both, under scores that rise.  Bound: weights and output rounded, u
    each, of the sum of w |v|, and 2 (keys + 64) roundings of 2^-24."""
    lengths = [900, 20]
    x = Sequences(n, 2, D, 16, lengths, "bf16", 2, prefix)
    x.q[:, :, :, 0], x.q[:, :, 1, 32] = 1.0, 1.0
    steps = torch.tensor([0.0, 1, 2, 3, 4, 6], device="cuda")
    for b, length in enumerate(lengths):
        j = torch.arange(prefix + length + n, device="cuda")
        pages, at = x.at(b, j)
        x.k[pages, 0, at, 0], x.k[pages, 0, at, 32] = steps[(j // 64) % 6].to(x.t), -steps[(j // 64) % 6].to(x.t)
        x.v[pages, 0, at] = 1.5 * 2.0 ** 126
        x.v[pages, 0, at, 1] = torch.where(j % 2 == 0, 1.5 * 2.0 ** 126, -2.0 ** 126).to(x.t)
        x.v[pages, 0, at, 32:] = 1.0
    out = x.run(1.0).double().cpu()
    u = 2.0 ** -8
    for b, length in enumerate(lengths):
        for i in range(n):
            j = torch.arange(prefix + length + i + 1, device="cuda")
            pages, at = x.at(b, j)
            for h in range(2):
                w = torch.softmax(x.k[pages, 0, at].double() @ x.q[b, i, h].double(), 0)
                values = x.v[pages, 0, at].double()
                want, size = (w @ values).cpu(), (w @ values.abs()).cpu()
                bound = (2 * u * (1 + u) + 2 * (len(j) + 64) * 2.0 ** -24) * size
                assert ((out[b, i, h] - want).abs() <= bound).all(), (b, i, h, out[b, i, h, :3], want[:3])


@pytest.mark.parametrize("n,H,D,dtype", [(1, 8, 128, "bf16"), (2, 4, 64, "f16"), (9, 4, 80, "f16"), (12, 4, 128, "bf16"),
                                         (3, 4, 256, "f16")])
def test_long_runs_of_one_task(n, H, D, dtype):
    """300 long sequences that share pages, two key/value heads: a workgroup's run of one task is longer than the pages that
    it looks up at a time.  Three of the sequences against the reference."""
    K, P, B = 2, 64, 300
    gen = torch.Generator(device="cuda").manual_seed(n)
    lengths = [5000 - 7 * b for b in range(B)]
    M = -(-(5000 + n) // P)
    t = TORCH_DTYPES[dtype]
    k4, v4 = (C4.pack(torch.randn(M, K, P, D, generator=gen, device="cuda").to(t)) for _ in range(2))
    table = torch.stack([torch.randperm(M, generator=gen, device="cuda") for _ in range(B)]).to(torch.int32)
    q = torch.randn(B, n, H, D, generator=gen, device="cuda").to(t)
    out = paged_cache.attend4(q, k4, v4, table, _ints(lengths)).double().cpu().numpy()
    k, v = C4.unpack(k4, P, D, dtype), C4.unpack(v4, P, D, dtype)
    for b in (0, 137, B - 1):
        want, size, product = attend_reference(q[b:b + 1], k, v, table[b:b + 1].cpu().numpy(), [lengths[b]], [n], None, 0,
                                               D ** -0.5)
        bound = attend_bound(size, product, dtype, D, lengths[b] + n, float(v.float().abs().max()))
        assert (np.abs(out[b:b + 1] - want) <= bound).all(), b
