"""Numbers that do not fit the library's 32 bits, handed to the calls of decoding on a shared cache: refused, not cut."""
import numpy as np
import pytest

from paper_2608_01785_amd import workloads as W

BIG = 2 ** 32


@pytest.fixture(scope="module")
def b():
    from paper_2608_01785_amd import binding
    binding.lib()
    return binding


@pytest.mark.parametrize("at", range(4))
def test_pages_of_too_many(b, at):
    for n in (BIG + 4, BIG + 64):
        args = [4, 64, 2, 3]
        args[at] = n
        with pytest.raises(b.HorizonError):
            b.Pages(*args)


@pytest.mark.parametrize("make", [list, np.array, lambda x: np.array(x)[:, None].repeat(2, 1)[:, 0],
                                  lambda x: [np.int64(v) for v in x]])
def test_lists_of_pages(b, make):
    p = b.Pages(4, 64, 2, 3)
    p.reserve(make([0]), make([65]))
    for call in (lambda: p.reserve(make([BIG]), make([1])), lambda: p.reserve(make([0]), make([BIG + 1])),
                 lambda: p.reserve(make([0]), make([1 - BIG])), lambda: p.fork(make([BIG + 1]), make([0])),
                 lambda: p.fork(make([1]), make([BIG])), lambda: p.table(make([BIG])), lambda: p.shared(make([BIG]))):
        with pytest.raises((ValueError, OverflowError)):
            call()
    table, lens = p.table([0, 1])
    assert lens.tolist() == [65, 0] and table.tolist() == [[0, 1, 0], [0, 0, 0]] and p.free_count() == 2


def test_fractions_are_no_pages(b):
    p = b.Pages(4, 64, 2, 3)
    for values in (np.array([0.5]), np.array([np.nan]), [0.5], (0.5,), [np.float32(1)], [[0.5]]):
        with pytest.raises(ValueError):
            p.reserve([0], values)
    assert p.free_count() == 4


def test_lists_of_copies(b):
    for values in (np.array([BIG]), np.array([0.5]), np.array([np.nan]), [BIG], [0.5]):
        with pytest.raises(ValueError, match="32-bit"):
            b._host_ints(values, "src")
    for values in ([3, 0], np.array([3, 0]), np.array([3, 9, 0], np.uint8)[::2]):
        keep, address = b._host_ints(values, "src")
        assert list(keep) == [3, 0] and address


def test_room_for_moves_is_what_there_are_pages(b):
    p = b.Pages(4, 64, 2, 3)
    p.reserve([0, 1], [64, 64])
    p.release([0])
    assert p.compact(10 ** 12) == ([1], [0], [64])


def test_workspaces_of_too_many(b):
    shape = W.TINY
    for bad in ((BIG + 3, 10, 64, 0, 1), (3, 10, BIG + 64, 0, 1), (3, 10, 64, BIG, 1), (3, 10, 64, 0, BIG + 1)):
        with pytest.raises(b.HorizonError):
            b.hs_workspace_size_prefix(shape, *bad)
    assert b.hs_workspace_size_prefix(shape, 3, BIG + 10, 64, 0, 1) > b.hs_workspace_size_prefix(shape, 3, 10, 64, 0, 1)


def test_block_tables(b):
    for table in (np.array([[0, BIG + 1]]), np.array([[0.0, 1.5]])):
        with pytest.raises(ValueError, match="32-bit"):
            b._kv_struct(([1], [2], 4, 64, table))
    for table in ([[0, BIG + 1]], [[0.0, 1.5]]):
        with pytest.raises(ValueError, match="32-bit"):
            b._kv_struct(([1], [2], 4, 64, table))
    for table in (np.array([[0, 3], [1, -1]]), np.array([[0, 3], [1, -1]], np.int32), [[0, 3], [1, -1]]):
        s = b._kv_struct(([1], [2], 4, 64, table))
        assert [s.block_table[i] for i in range(4)] == [0, 3, 1, -1] and s.pages_per_seq == 2
