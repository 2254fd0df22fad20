"""Beam search without a GPU: when a step has nothing to do, and what a start refuses before it touches anything."""
from types import SimpleNamespace

import pytest

torch = pytest.importorskip("torch")

from paper_2608_01785_amd.beams import BeamSearch   # noqa: E402


class Untouched:
    """Stands for what a call must not reach."""

    def __getattr__(self, name):
        raise AssertionError(f"{name} was reached")


def search(parents, finished, max_new=9, steps=1):
    """A search after a selection with these parents and finished flags [groups][beams]."""
    s = object.__new__(BeamSearch)
    s.beams, s.max_new, s.steps, s.ready, s.groups = len(parents[0]), max_new, steps, True, len(parents)
    # One group more than there are: what an earlier search left.
    s.at = 0
    parents, finished = (torch.tensor(x + [[0] * s.beams], dtype=t) for x, t in (
        (parents, torch.int32), (finished, torch.uint8)))
    s.host = parents, parents, [finished, 1 - finished]
    s.pages = Untouched()
    return s


@pytest.mark.parametrize("parents,finished", [
    ([[0, 1, 2]], [[1, 1, 1]]),
    ([[0, -1, -1]], [[1, 0, 0]]),                        # an ended beam, and no continuation beside it
    ([[-1, -1]], [[0, 0]]),                              # nothing at all: rows without a distribution
    ([[0, 1], [0, -1], [-1, -1]], [[1, 1], [1, 0], [0, 0]]),
])
def test_a_step_with_nothing_to_continue(parents, finished):
    assert search(parents, finished).step() is False


@pytest.mark.parametrize("parents,finished", [
    ([[0, 1, 2]], [[1, 0, 1]]), ([[0, -1]], [[0, 0]]), ([[0, 1], [0, -1]], [[0, 1], [1, 0]]),
])
def test_a_step_with_something_to_continue(parents, finished):
    with pytest.raises(AssertionError, match="reserve was reached"):
        search(parents, finished).step()
    assert search(parents, finished, max_new=1).step() is False   # but no token left


@pytest.mark.parametrize("x,text", [
    (torch.zeros((5, 8)), "float32"), (torch.zeros((5, 8), dtype=torch.float16), "float16"),
    (torch.zeros((5, 8), dtype=torch.int8), "int8"), (torch.zeros((5, 8), dtype=torch.bfloat16, device="meta"), "meta"),
    (torch.zeros((8, 5), dtype=torch.bfloat16).t(), "contiguous"),
    (torch.zeros((10, 8), dtype=torch.bfloat16)[::2], "contiguous"),
])
def test_a_start_refuses_rows_of_another_kind(x, text):
    s = search([[0]], [[0]])
    s.max_groups, s.max_prompt, s.shape = 2, 5, SimpleNamespace(hidden=8)
    s.x, s.torch_stream = torch.zeros((2, 8), dtype=torch.bfloat16), Untouched()
    for offsets in ([0, 5], [0, 2, 5]):
        with pytest.raises(ValueError, match=text):
            s.start(x, offsets)
    assert s.ready and s.groups == 1   # the search before goes on
