"""Attention behind shared prefixes, in each of its kernels: keys that no weight falls on, and what is wrong with one row.

A score of -inf is a weight of zero.  The whole tiles, ranges and splits of such keys lie before, between and behind
finite ones here; a row that has no other key has no distribution and is NaN.
"""
import math

import numpy as np
import pytest

from oracle import decoding as ref
from tests.gpu_common import log, require_gpu
from tests.test_gpu_decoding import HALF, Prefix

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def env():
    torch = require_gpu()
    from paper_2608_01785_amd import binding
    ctx = binding.Context(0, budgets=(64, 256))
    yield torch, binding, ctx
    torch.cuda.synchronize()
    ctx.close()


ROWS, REST = [3, 4], [5, 70, 1, 9, 200, 3, 64]

# One launch over everything; 16 and 32 columns a block; 128, of either head size.
CASES = {
    "short": (dict(prefix=[40, 65], rest=[5, 30, 1, 9, 20, 3, 24], heads=(28, 4, 128)), None),
    "16": (dict(prefix=[700, 900], rest=REST, heads=(4, 2, 64)), 16),
    "32": (dict(prefix=[700, 900], rest=REST, heads=(28, 4, 128)), 32),
    "wide": (dict(prefix=[700, 900], rest=REST, heads=(40, 1, 128)), 128),
    "wide64": (dict(prefix=[700, 900], rest=REST, heads=(64, 1, 64)), 128),
}


def columns_of_a_block(heads, rows):
    columns = sum(rows) * heads[0] // heads[1]
    return 16 if columns <= 16 * len(rows) else 32 if columns <= 128 * len(rows) else 128


@pytest.fixture(params=[(name, dtype) for name in CASES for dtype in ("f16", "bf16")], ids="-".join)
def case(request, env):
    name, dtype = request.param
    args, columns = CASES[name]
    if columns is not None:   # more than one launch's worth of tiles, in blocks of that width
        assert max(args["prefix"]) > 32 * 16 and columns_of_a_block(args["heads"], ROWS) == columns
    log(f"[prefix edges] {name} {dtype}")
    return Prefix(env, ROWS, page=64, dtype=dtype, seed=21, poison=False, **args)


def keys_of(s, row, first, last):
    """(slots, positions in them) of positions [first, last) of a row, those of the prefix in its group's pages."""
    g = next(g for g in range(len(s.prefix)) if s.offsets[g] <= row < s.offsets[g + 1])
    at = np.arange(first, last)
    slots = np.where(at < s.prefix[g], s.table[s.offsets[g]][at // s.page], s.table[row][at // s.page])
    return s.torch.as_tensor(slots).cuda(), s.torch.as_tensor(at % s.page).cuda()


def put(s, row, first, last, value):
    """`value` in one dimension of the keys [first, last); every query is at least 0.5 there."""
    slots, at = keys_of(s, row, first, last)
    s.k[slots, :, at, 3] = value


def positive_queries(s):
    hq, _, dh = s.heads
    q = s.q.unflatten(1, (hq, dh))
    q[:, :, 3] = q[:, :, 3].abs() + 0.5


def run(s):
    s.torch.cuda.synchronize()
    s.call()
    s.torch.cuda.synchronize()
    return s.out.double().cpu().numpy()


def check_without(s, rows):
    """Against the float64 formula; the tolerance of Prefix.check with the scores' errors from the finite keys."""
    hq, _, dh = s.heads
    q = s.q.double().cpu().numpy().reshape(s.n, hq, dh)
    k, v = s.k.double().cpu().numpy(), s.v.double().cpu().numpy()
    o, a, slack = ref.prefix_attention(q, k, v, s.table, s.lens, s.offsets, s.prefix)
    kmax = np.sqrt((np.where(np.isfinite(k), k, 0) ** 2).sum(-1).max())
    score = 2.0 ** -24 * dh * np.sqrt((q ** 2).sum(-1)) * kmax / math.sqrt(dh)
    keys = np.asarray(s.lens, np.float64)[:, None, None]
    tol = (np.abs(o) * HALF[s.dtype] + a * (2.0 ** -11 + 2 * score[..., None] + 2.0 ** -20 + keys * 2.0 ** -24)
           + slack[..., None] + 2.0 ** -25)
    got = s.out.double().cpu().numpy().reshape(o.shape)
    assert np.all(np.isfinite(got[rows]))
    bad = np.abs(got - o)[rows] > tol[rows]
    assert not bad.any(), (np.argwhere(bad)[:3], np.abs(got - o)[rows][bad][:3], tol[rows][bad][:3])


def test_keys_at_minus_infinity(case):
    s = case
    positive_queries(s)
    p = s.prefix
    hidden = [(0, 0, 33), (0, p[0] - 5, p[0]),               # a wavefront's first tile, and the prefix's end
              (3, 0, p[1] - 2),                              # all but two keys of a prefix: whole splits
              (2, p[0], s.lens[2]), (5, p[1], s.lens[5]),    # everything that two rows have to themselves
              (1, p[0], s.lens[1] - 1), (4, p[1] + 1, s.lens[4])]
    for row, first, last in hidden:
        put(s, row, first, last, -60000.0)
    # The weights of these keys are zero too, after at least one multiplication by zero.
    want = run(s)
    for row, first, last in hidden:
        put(s, row, first, last, -math.inf)
    got = run(s)
    assert np.all(np.isfinite(got)), np.argwhere(~np.isfinite(got))[:3]
    check_without(s, list(range(s.n)))
    assert (got == want).all()


def test_a_row_without_any_weight_is_nan(case):
    """Its prefix and its own keys, all at -inf; another group's rows keep their bits."""
    s = case
    positive_queries(s)
    want = run(s)
    put(s, 3, 0, s.prefix[1], -math.inf)
    for row in (4, 6):
        put(s, row, s.prefix[1], s.lens[row], -math.inf)
    got = run(s)
    assert np.isnan(got[[4, 6]]).all()
    assert (got[:3] == want[:3]).all()
    check_without(s, [0, 1, 2, 3, 5])


def test_many_splits_at_minus_infinity(env):
    """More splits than a wavefront of the join adds up at a time; with one wavefront a row, and with four."""
    for rows, heads, dtype in ((2, (28, 4, 128), "f16"), (40, (32, 1, 128), "f16"), (9, (32, 1, 64), "bf16")):
        log(f"[prefix edges] {rows} rows, {heads}, {dtype}")
        s = Prefix(env, [rows], [6000], [1] * rows, heads, 512, dtype, seed=22, poison=False)
        positive_queries(s)
        for hidden in ((0, 5990), (3, 6000)):
            put(s, 0, 0, 6000, 0.0)
            put(s, 0, *hidden, -math.inf)
            run(s)
            check_without(s, list(range(rows)))


def test_wrong_lengths_and_slots(case):
    s = case
    clean = run(s)
    prefix, table, lens = list(s.prefix), s.table.copy(), list(s.lens)
    s.table[1, (s.lens[1] - 1) // 64] = s.k.shape[0]   # beyond the cache: keys of row 1 alone
    s.table[4, (s.lens[4] - 1) // 64] = -5
    s.lens[2] = prefix[0] - 1                   # shorter than its prefix
    s.lens[5] = prefix[1] + s.max_rest + 1      # beyond the bound
    s.lens[6] = 64 * s.table.shape[1] + 1       # beyond the table (and the bound)
    s.upload()
    got = run(s)
    for i in range(7):
        assert np.isnan(got[i]).all() if i in (1, 2, 4, 5, 6) else (got[i] == clean[i]).all(), i
    # A page inside a prefix, and the one that it ends in: all rows of the group.
    for group, page in ((0, prefix[0] // 128), (1, (prefix[1] - 1) // 64)):
        s.table, s.lens = table.copy(), list(lens)
        s.table[s.offsets[group], page] = 10 ** 6
        s.upload()
        got = run(s)
        mine = np.arange(s.offsets[group], s.offsets[group + 1])
        rest = np.setdiff1d(np.arange(7), mine)
        assert np.isnan(got[mine]).all() and (got[rest] == clean[rest]).all(), group
    s.table = table
    s.prefix = [max(prefix) + 1, -1]            # beyond its bound, negative
    s.upload()
    assert np.isnan(run(s)).all()


def test_nan_stays_with_its_rows(case):
    """In one row's own keys, values and query, the rows beside it in the same products keep their bits."""
    s = case
    clean = run(s)
    slots, at = keys_of(s, 4, s.lens[4] - 1, s.lens[4])
    s.v[slots, :, at // 32, :, at % 32] = math.nan
    put(s, 1, s.lens[1] - 1, s.lens[1], math.nan)
    s.q[5] = math.nan
    got = run(s)
    for i in range(7):
        assert np.isnan(got[i]).all() if i in (1, 4, 5) else (got[i] == clean[i]).all(), i


def test_an_end_token_beyond_32_bits_is_refused(env):
    from tests.test_gpu_decoding import Beams
    torch, b, ctx = env
    for end in (2 ** 32 + 5, 5 - 2 ** 32):
        s = Beams(env, 2, 3, 100, 4, end=5)
        s.end = end
        with pytest.raises(b.HorizonError, match="end_token"):
            s.call()
