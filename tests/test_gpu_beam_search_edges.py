"""Beam searches with groups that have fewer continuations than beams, or none."""
import math

import pytest

from tests.gpu_common import log, require_gpu
from tests.test_gpu_decoding_steps import Search

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def env():
    torch = require_gpu()
    from paper_2608_01785_amd import binding
    ctx = binding.Context(0, budgets=(128, 256))
    yield torch, binding, ctx
    torch.cuda.synchronize()
    ctx.close()


def with_tokens(s, tokens, end, beams, groups, max_new):
    """A search as `s`, whose head gives every other token no probability."""
    from paper_2608_01785_amd.answer import AnswerHead
    from paper_2608_01785_amd.beams import BeamSearch
    torch, head = s.torch, s.head
    bias = torch.full((head.vocab,), -math.inf, dtype=torch.bfloat16, device="cuda")
    bias[tokens] = 0
    only = AnswerHead(s.ctx, head.gain, (head.w, head.w_scale), bias, max_rows=head.max_rows)
    return BeamSearch(s.ctx, s.shape, s.w, only, s.search.embed, beams, groups, 50, max_new, end)


def steps_of(search):
    steps = 1
    while search.step():
        steps += 1
    return steps


def test_search_ends_where_nothing_goes_on(env):
    """One group whose only token ends it, one of rows that have no distribution."""
    torch, b, ctx = env
    log("[beam search] an ended group and one of NaN")
    s = Search(env, 3, 2, 40, 50, 6, seed=96)
    x, offsets = s.prompts([30, 20])
    search = with_tokens(s, [7], 7, 3, 2, 6)
    search.start(x, offsets)
    assert steps_of(search) == 1
    bad = x.clone()
    bad[offsets[1]:] = math.nan
    torch.cuda.synchronize()
    search.start(bad, offsets)
    assert steps_of(search) == 1
    first, second = search.results()
    assert first[0].tokens == [7] and first[0].finished and first[0].score == 0
    for beam in first[1:] + second:
        assert beam.tokens == [] and beam.score == -math.inf and not beam.finished


def test_search_goes_on_beside_a_group_without_continuations(env):
    """The other group's beams are those that it finds alone."""
    torch, b, ctx = env
    log("[beam search] a group of NaN beside another")
    s = Search(env, 3, 2, 40, 50, 6, seed=97)
    x, offsets = s.prompts([30, 20])
    bad = x.clone()
    bad[offsets[1]:] = math.nan
    torch.cuda.synchronize()
    s.search.start(bad, offsets)
    assert steps_of(s.search) == 6
    results = s.search.results()
    assert all(beam.tokens == [] and beam.score == -math.inf for beam in results[1])
    s.search.start(x, offsets)
    assert steps_of(s.search) == 6
    assert s.search.results()[0] == results[0]


def test_search_of_fewer_continuations_than_beams(env):
    """Two tokens, one of which ends: after t steps there are t ended sequences and one that goes on."""
    torch, b, ctx = env
    log("[beam search] two tokens, five beams")
    s = Search(env, 5, 1, 40, 50, 4, seed=98)
    x, offsets = s.prompts([25])
    search = with_tokens(s, [3, 9], 9, 5, 1, 4)
    search.start(x, offsets)
    assert steps_of(search) == 4
    got = sorted(tuple(beam.tokens) for beam in search.results()[0])
    assert got == sorted([(9,), (3, 9), (3, 3, 9), (3, 3, 3, 9), (3, 3, 3, 3)])


@pytest.mark.parametrize("closed", [True, False])
def test_a_search_given_back_after_its_context(env, closed):
    """Its buffers, pinned ones among them, outlive the context's streams: closed before, or held by nothing else."""
    import gc
    torch, b, _ = env
    ctx = b.Context(0, budgets=(128,))
    log(f"[beam search] given back after its context, closed {closed}")
    s = Search((torch, b, ctx), 3, 1, 40, 50, 3, seed=99)
    x, offsets = s.prompts([25])
    s.search.start(x, offsets)
    assert steps_of(s.search) == 3
    want = s.search.results()
    torch.cuda.synchronize()
    if closed:
        ctx.close()
    del ctx, s, x
    gc.collect()
    for _ in range(3):
        pinned = torch.full((64,), 5.0).pin_memory()
        assert float(pinned.cuda().sum()) == 320.0
    torch.cuda.synchronize()
    again = Search(env, 3, 1, 40, 50, 3, seed=99)
    x, offsets = again.prompts([25])
    again.search.start(x, offsets)
    assert steps_of(again.search) == 3
    assert again.search.results() == want


def test_results_before_a_start(env):
    s = Search(env, 2, 2, 50, 20, 3)
    assert s.search.results() == []
    x, offsets = s.prompts([20, 5])
    s.search.start(x, offsets)
    assert [len(g) for g in s.search.results()] == [2, 2]


def test_results_are_the_callers(env):
    """What is done to them leaves the search as it is."""
    s = Search(env, 3, 1, 40, 50, 5, seed=100)
    x, offsets = s.prompts([25])
    s.search.start(x, offsets)
    assert steps_of(s.search) == 5
    want = s.search.results()
    s.search.start(x, offsets)
    for _ in range(4):
        for beam in s.search.results()[0]:
            beam.tokens.append(-5)
        assert s.search.step()
    assert s.search.results() == want


def test_pages_of_a_search(env):
    """Free are those that no beam lists: during a search, after it, and after another start."""
    torch, b, ctx = env
    beams, page = 4, 64
    s = Search(env, beams, 3, 500, 130, 9, seed=101)
    rows, per_seq = 3 * beams, -(-(130 + 9) // page)

    def check():
        table, lens = s.search.pages.table(list(range(rows)))
        used = {int(table[i, j]) for i in range(rows) for j in range(-(-int(lens[i]) // page))}
        assert s.search.pages.free_count() == rows * per_seq - len(used)
        return len(used)
    assert check() == 0
    x, offsets = s.prompts([70, 5, 130])
    s.search.start(x, offsets)
    assert check() == 2 + 1 + 3      # the prompts' pages, each listed by its beams
    while s.search.step():
        # A group's whole pages are shared; each beam's last one is its own, or its siblings' after the fork.
        assert 6 <= check() <= (1 + beams) + beams + (2 + beams)
    x, offsets = s.prompts([64])
    s.search.start(x, offsets)
    assert check() == 1
    s.search.step()
    assert 2 <= check() <= 1 + beams
