"""The decoding loop with a cache when a step does not complete: the producer
raises, or the step's results are not valid.  Nothing of that step's plan stays
in the cache, and every later step's attention is that of the tokens that were
accepted (checked by the model of test_gpu_cache_loop)."""
import numpy as np
import pytest
import torch

from paper_2406_11016_amd import binding, paged_cache
from paper_2406_11016_amd import workloads as W
from paper_2406_11016_amd.decode_loop import DecodeLoop, SyntheticSteps
from paper_2406_11016_amd.paged_cache import PagedCache
from tests.test_gpu_cache_loop import Model

pytestmark = pytest.mark.gpu
B, PREFIX, PROMPTS, PAGES = 4, 21, [5, 30, 16, 1], 64


@pytest.fixture(scope="module", autouse=True)
def gpu():
    if not torch.cuda.is_available():
        pytest.fail("no GPU visible")
    paged_cache.load_library()
    torch.cuda.init()


class Stop(Exception):
    pass


def _model(native, graphs, seed=5):
    w = W.WORKLOADS["exact_b1_g5_v51865_f32"].with_(batch=B, vocab=1009)
    cache = PagedCache(B, num_pages=PAGES, page_size=16, max_pages=12, max_new=30, prefix_pages=2)
    torch.cuda.synchronize()
    loop = DecodeLoop(B, 1009, "f32", gamma0=3, gamma_max=6, cache=cache, native=native, use_graphs=graphs)
    return Model(loop, SyntheticSteps(w, 6, 4), PREFIX, PROMPTS, seed)


def _settle(model):
    """What the steps so far accepted, on the model's side."""
    if model.pending is not None:
        model.keep(model.loop.acc.tolist())


def _lengths_agree(model):
    cache = model.loop.cache
    assert [PREFIX + int(x) for x in cache.lengths] == [len(h) for h in model.held[0]]
    assert int((cache.block_table >= 0).sum()) + int(cache.free_count) == PAGES - 2


def _producer_raises(model, monkeypatch):
    def producer(loop, i, gamma):
        _settle(model)             # (the plan before this producer kept them)
        raise Stop

    with pytest.raises(Stop):
        model.loop.run(producer, 1)


def _step_raises(model, monkeypatch):
    """The step runs, but what it left is not valid."""
    loop = model.loop

    def collect():
        torch.cuda.synchronize()
        raise binding.WorkspaceTimeoutError("as after a wait that timed out")

    def step(handle, gamma):
        real(handle, gamma)
        raise binding.WorkspaceTimeoutError("as after a wait that timed out")

    real = binding.loop_step
    with monkeypatch.context() as m:
        m.setattr(loop, "collect", collect)
        m.setattr(binding, "loop_step", step)
        with pytest.raises(binding.WorkspaceTimeoutError):
            loop.run(model, 1)
    model.pending = None


KINDS = [(False, False), (True, False), (False, True)]


@pytest.mark.parametrize("native,graphs", KINDS, ids=["python", "native", "graphs"])
@pytest.mark.parametrize("before", [0, 3])
@pytest.mark.parametrize("fail", [_producer_raises, _step_raises], ids=["producer", "step"])
def test_nothing_stays_of_a_step_that_did_not_complete(native, graphs, before, fail, monkeypatch):
    model = _model(native, graphs)
    loop = model.loop
    if before:
        loop.run(model, before)
    for _ in range(2):             # (also right after one another)
        fail(model, monkeypatch)
    model.pending = None
    stats = loop.run(model, 4)
    assert any(int(a.max()) > 0 for a in stats.accepted)
    _settle(model)
    # the program plans for itself after another such step
    fail(model, monkeypatch)
    model.pending = None
    new = [4, 0, 20, 0]
    with torch.cuda.stream(loop.stream):
        loop.cache.plan(20, new_tokens=torch.tensor(new, dtype=torch.int32, device="cuda"), accepted_len=loop.acc)
        model.step_tokens(20, new)
    model.keep([n - 1 for n in new])
    loop.program_planned()
    loop.run(model, 2)
    _lengths_agree(model)
    loop.close()


def test_steps_driven_by_hand():
    """plan_cache, launch and collect without run(): a plan without a step, and one whose step left the error flag."""
    model = _model(False, False)
    loop = model.loop
    for kind in ("ok", "no step", "ok", "flag", "ok", "ok"):
        loop.plan_cache(3)
        _settle(model)
        model.pending = None
        with torch.cuda.stream(loop.stream):
            model.step_tokens(4, [4] * B)
            model.steps(loop, 0, 3)
        if kind == "no step":
            model.pending = None
            continue
        loop.launch(3)
        if kind == "flag":
            with torch.cuda.stream(loop.stream):
                loop.ws[binding.ERROR_FLAG_OFFSET:binding.ERROR_FLAG_OFFSET + 4].view(torch.int32).fill_(1)
            with pytest.raises(binding.SpecVerifyError):
                loop.collect()
            loop.reset_workspace()
            model.pending = None
        else:
            loop.collect()
    _lengths_agree(model)
    loop.close()


@pytest.mark.parametrize("graphs", [False, True])
def test_capturing_between_runs_leaves_the_accepted_lengths(graphs):
    """capture_all() checks each call's arguments by running it; the last step's results stay what they are."""
    model = _model(False, graphs)
    loop = model.loop
    stats = loop.run(model, 3)
    loop.uniforms.fill_(1.0)       # (a step on the buffers as they are now would accept other lengths)
    loop.tokens.fill_(3)
    torch.cuda.synchronize()
    loop.capture_all()
    torch.cuda.synchronize()
    assert loop.acc.tolist() == stats.accepted[-1].tolist() and loop.nxt.tolist() == stats.next_tokens[-1].tolist()
    _settle(model)
    model.pending = None
    loop.run(model, 2)
    _lengths_agree(model)
    loop.close()
