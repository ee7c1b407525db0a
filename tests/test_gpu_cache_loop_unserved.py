"""The decoding loop with a cache whose pages do not suffice: a sequence that a
plan cannot serve takes no part in that step, and resumes where its cache ends
when there are pages."""
import numpy as np
import pytest
import torch

from paper_2406_11016_amd import paged_cache
from paper_2406_11016_amd import workloads as W
from paper_2406_11016_amd.decode_loop import DecodeLoop, SyntheticSteps
from paper_2406_11016_amd.paged_cache import PagedCache
from tests.test_gpu_cache_loop import Model

pytestmark = pytest.mark.gpu
B, PREFIX, PROMPTS = 4, 21, [5, 30, 16, 1]


@pytest.fixture(scope="module", autouse=True)
def gpu():
    if not torch.cuda.is_available():
        pytest.fail("no GPU visible")
    paged_cache.load_library()
    torch.cuda.init()


class Short(Model):
    """Goes by what each plan gave."""

    def __call__(self, loop, i, gamma):
        if self.pending is not None:
            self.keep(loop.acc.tolist())
        self.plans.append(loop.cache.counts.tolist())
        with torch.cuda.stream(loop.stream):
            self.step_tokens(gamma + 1, [max(c, 0) for c in self.plans[-1]])
        self.steps(loop, i, gamma)


def _check(stats, plans):
    """Results and tokens of the sequences that were served, and no others."""
    tokens = 0
    for i, counts in enumerate(plans):
        for b, c in enumerate(counts):
            assert (c < 0) == bool(stats.unserved[i][b])
            if c < 0:
                assert stats.accepted[i][b] == -1 and stats.next_tokens[i][b] == -1, (i, b)
            else:
                assert c == stats.gammas[i] + 1 and stats.next_tokens[i][b] >= 0
                tokens += int(stats.accepted[i][b]) + 1
        if i + 1 < len(plans) and -1 in counts:
            assert stats.gammas[i + 1] == max(stats.gammas[i] - 1, 1)      # not every draft was accepted
    assert stats.tokens == tokens and len(stats.unserved) == len(plans) == stats.iterations


@pytest.mark.parametrize("native,graphs", [(False, False), (True, False), (False, True), (True, True)])
@pytest.mark.parametrize("pages,max_pages", [(8, 12), (40, 3)], ids=["pool", "table"])
def test_sequences_without_pages_wait(native, graphs, pages, max_pages):
    """The pool runs out, or the longest sequences reach the table's width; then one ends and others go on."""
    w = W.WORKLOADS["exact_b1_g5_v51865_f32"].with_(batch=B, vocab=1009)
    cache = PagedCache(B, num_pages=pages, page_size=16, max_pages=max_pages, max_new=30, prefix_pages=2)
    torch.cuda.synchronize()
    loop = DecodeLoop(B, 1009, "f32", gamma0=3, gamma_max=6, cache=cache, native=native, use_graphs=graphs)
    model = Short(loop, SyntheticSteps(w, 6, 4), PREFIX, PROMPTS, seed=7)
    model.plans = []
    stats = loop.run(model, 20)
    assert any(-1 in p and max(p) > 0 for p in model.plans)
    _check(stats, model.plans)
    model.keep(loop.acc.tolist())
    assert loop.acc.tolist() == stats.accepted[-1].tolist()
    # sequence 1 ends, and a short one takes its place; everyone else's last tokens stay
    new = [0, 2, 0, 0]
    with torch.cuda.stream(loop.stream):
        cache.plan(2, new_tokens=torch.tensor(new, dtype=torch.int32, device="cuda"), accepted_len=loop.acc,
                   release=torch.tensor([0, 1, 0, 0], dtype=torch.int32, device="cuda"))
        for held in model.held:
            del held[1][PREFIX:]
        got = [max(c, 0) for c in cache.counts.tolist()]
        model.step_tokens(2, got)
    model.keep([c - 1 for c in got])
    loop.program_planned()
    model.plans = []
    stats = loop.run(model, 3)
    assert model.plans[0][1] > 0
    _check(stats, model.plans)
    assert [PREFIX + int(x) for x in cache.lengths] == [len(h) for h in model.held[0]]
    loop.close()


def test_a_loop_without_a_cache_reports_none():
    w = W.WORKLOADS["exact_b1_g5_v51865_f32"].with_(batch=2, vocab=1009)
    loop = DecodeLoop(2, 1009, "f32", gamma0=3, gamma_max=6)
    stats = loop.run(SyntheticSteps(w, 6, 4), 3)
    assert stats.unserved == [] and all(np.all(a >= 0) for a in stats.accepted)
