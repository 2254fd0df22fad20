"""Decoding on a shared cache, without a GPU: refusals (no context, fake pointers) and the pages' bookkeeping."""
import ctypes

import numpy as np
import pytest

P = 0x10000000   # fake device addresses, far apart and never dereferenced
INVALID, UNSUPPORTED, BUDGET, WORKSPACE = 1, 2, 3, 4


@pytest.fixture(scope="module")
def b():
    from paper_2608_01785_amd import binding
    binding.lib()
    return binding


def beam(b, **kw):
    a = dict(z=P, t=0, ld=64, groups=2, beams=4, vocab=64, scores=2 * P, fin=3 * P, end=1, k=8, os=4 * P, op=5 * P,
             ot=6 * P, of=7 * P, ws=8 * P, wsb=1 << 30, cus=256)
    a.update(kw)
    st = b.lib().hs_beam_select(None, a["z"], a["t"], a["ld"], a["groups"], a["beams"], a["vocab"], a["scores"],
                                a["fin"], a["end"], a["k"], a["os"], a["op"], a["ot"], a["of"], a["cus"], None, a["ws"],
                                a["wsb"])
    return st, b.hs_last_error()


def _i32(x):
    return None if x is None else (ctypes.c_int32 * max(len(x), 1))(*x)


def copy(b, **kw):
    a = dict(k=[P, 2 * P], v=[3 * P, 4 * P], slots=8, page=128, layers=2, hkv=4, dh=64, src=[0, 0], dst=[1, 2],
             pos=[5, 128], n=None)
    a.update(kw)
    arr = [None if x is None else (ctypes.c_void_p * len(x))(*x) for x in (a["k"], a["v"])]
    kv = b.KvCache(*(ctypes.cast(x, ctypes.POINTER(ctypes.c_void_p)) for x in arr), a["slots"], a["page"], None, 0)
    n = len(a["src"] or []) if a["n"] is None else a["n"]
    st = b.lib().hs_cache_copy(None, ctypes.byref(kv), a["layers"], a["hkv"], a["dh"], _i32(a["src"]), _i32(a["dst"]),
                               _i32(a["pos"]), n, 256, None)
    return st, b.hs_last_error()


def prefix(b, **kw):
    a = dict(q=P, t=2, ldq=256, o=2 * P, ldo=256, hq=4, hkv=2, dh=64, k=3 * P, v=4 * P, slots=8, page=64, tab=5 * P,
             pps=4, lens=6 * P, n=3, off=7 * P, pre=8 * P, g=2, mp=128, mr=100, ws=9 * P, wsb=1 << 28, cus=256)
    a.update(kw)
    st = b.lib().hs_prefix_attention(None, a["q"], a["t"], a["ldq"], a["o"], a["ldo"], a["hq"], a["hkv"], a["dh"],
                                     a["k"], a["v"], a["slots"], a["page"], a["tab"], a["pps"], a["lens"], a["n"],
                                     a["off"], a["pre"], a["g"], a["mp"], a["mr"], a["cus"], None, a["ws"], a["wsb"])
    return st, b.hs_last_error()


REFUSED = [
    (beam, dict(t=3), INVALID, "type"),
    (beam, dict(groups=-1), INVALID, "groups"),
    (beam, dict(beams=0), INVALID, "beams"),
    (beam, dict(beams=65), UNSUPPORTED, "at most 64"),
    (beam, dict(k=0), INVALID, "selected"),
    (beam, dict(k=65), UNSUPPORTED, "at most 64"),
    (beam, dict(vocab=0), INVALID, "vocabulary"),
    (beam, dict(groups=2 ** 31 - 1), UNSUPPORTED, "rows"),
    (beam, dict(groups=(1 << 20) + 1), UNSUPPORTED, "rows"),
    (beam, dict(ld=63), INVALID, "stride"),
    (beam, dict(z=None), INVALID, "logits is null"),
    (beam, dict(z=P + 2), INVALID, "aligned"),
    (beam, dict(scores=None), INVALID, "scores is null"),
    (beam, dict(os=None), INVALID, "out_scores is null"),
    (beam, dict(op=None), INVALID, "out_parents is null"),
    (beam, dict(ot=None), INVALID, "out_tokens is null"),
    (beam, dict(ot=6 * P + 2), INVALID, "aligned"),
    (beam, dict(end=64), INVALID, "end_token"),
    (beam, dict(end=-2), INVALID, "end_token"),
    (beam, dict(end=-1), INVALID, "need an end_token"),
    (beam, dict(os=2 * P), INVALID, "overlap"),
    (beam, dict(of=3 * P + 7), INVALID, "overlap"),
    (beam, dict(ot=5 * P + 60), INVALID, "overlap"),
    (beam, dict(op=P + 7 * 64 * 4 + 252), INVALID, "overlap"),
    (beam, dict(ws=4 * P - 16), INVALID, "overlap"),
    (beam, dict(ws=None), WORKSPACE, "null"),
    (beam, dict(ws=8 * P + 8), INVALID, "aligned"),
    (beam, dict(wsb=16), WORKSPACE, "needed"),
    (beam, dict(), INVALID, "context is null"),
    (beam, dict(cus=0), BUDGET, "budget"),
    (prefix, dict(cus=-5), BUDGET, "budget"),
    (beam, dict(cus=100000), INVALID, "context is null"),
    (prefix, dict(cus=100000), INVALID, "context is null"),
    (beam, dict(fin=None, end=-1, of=None), INVALID, "context is null"),
    (beam, dict(groups=0, z=None, scores=None, fin=None, os=None, op=None, ot=None, of=None, ws=None), INVALID,
     "context is null"),
    (copy, dict(k=None), INVALID, "cache is null"),
    (copy, dict(k=[P, 0]), INVALID, "layer 1"),
    (copy, dict(v=[P + 8, P]), INVALID, "aligned"),
    (copy, dict(layers=0), INVALID, "n_layers"),
    (copy, dict(hkv=0), INVALID, "heads"),
    (copy, dict(hkv=1025), UNSUPPORTED, "heads"),
    (copy, dict(dh=96), UNSUPPORTED, "head_dim"),
    (copy, dict(slots=0), INVALID, "slots"),
    (copy, dict(page=96), INVALID, "multiple of 64"),
    (copy, dict(page=2 ** 31 - 64, hkv=1024, dh=128), UNSUPPORTED, "exceeds"),
    (copy, dict(slots=(1 << 28) + 1), UNSUPPORTED, "slots"),
    (copy, dict(n=-1), INVALID, "copies"),
    (copy, dict(src=None, n=2), INVALID, "null"),
    (copy, dict(dst=None), INVALID, "null"),
    (copy, dict(src=[0, 8]), INVALID, "outside"),
    (copy, dict(dst=[-1, 2]), INVALID, "outside"),
    (copy, dict(pos=[5, 129]), INVALID, "positions"),
    (copy, dict(pos=[-1, 3]), INVALID, "positions"),
    (copy, dict(dst=[3, 3]), INVALID, "two copies"),
    (copy, dict(src=[0, 1], dst=[1, 2]), INVALID, "source and a destination"),
    (copy, dict(src=[4, 5], dst=[4, 6]), INVALID, "source and a destination"),
    (copy, dict(), INVALID, "context is null"),
    (copy, dict(src=[], dst=[], pos=[]), INVALID, "context is null"),
    (copy, dict(pos=None), INVALID, "context is null"),
    (prefix, dict(t=0), INVALID, "type"),
    (prefix, dict(dh=96), UNSUPPORTED, "head_dim"),
    (prefix, dict(hkv=0), INVALID, "heads"),
    (prefix, dict(hq=3), INVALID, "query heads"),
    (prefix, dict(hq=0), INVALID, "query heads"),
    (prefix, dict(hq=130, ldq=8320, ldo=8320), UNSUPPORTED, "at most 64"),
    (prefix, dict(n=-1), INVALID, "rows"),
    (prefix, dict(mp=-1), INVALID, "prefixes"),
    (prefix, dict(mr=-1), INVALID, "prefixes"),
    (prefix, dict(mp=2 ** 31 - 1), UNSUPPORTED, "keys"),
    (prefix, dict(n=2 ** 31 - 1), UNSUPPORTED, "rows"),
    (prefix, dict(slots=0), INVALID, "slots"),
    (prefix, dict(slots=2 ** 31 - 1), UNSUPPORTED, "slots"),
    (prefix, dict(page=32), INVALID, "multiple of 64"),
    (prefix, dict(pps=0), INVALID, "pages_per_seq"),
    (prefix, dict(g=-1), INVALID, "n_groups"),
    (prefix, dict(g=1 << 25, mp=0, mr=3), UNSUPPORTED, "blocks"),
    (prefix, dict(g=1 << 24), UNSUPPORTED, "blocks"),
    (prefix, dict(ldq=255), INVALID, "stride"),
    (prefix, dict(ldq=260), INVALID, "multiple of 8"),
    (prefix, dict(q=P + 8), INVALID, "aligned"),
    (prefix, dict(o=2 * P + 1), INVALID, "aligned"),
    (prefix, dict(ldo=255), INVALID, "stride"),
    (prefix, dict(k=None), INVALID, "cache is null"),
    (prefix, dict(v=4 * P + 8), INVALID, "aligned"),
    (prefix, dict(tab=None), INVALID, "block_table is null"),
    (prefix, dict(lens=None), INVALID, "lens is null"),
    (prefix, dict(off=None), INVALID, "group_offsets is null"),
    (prefix, dict(pre=None), INVALID, "prefix_lens is null"),
    (prefix, dict(tab=5 * P + 2), INVALID, "aligned"),
    (prefix, dict(o=P + 512), INVALID, "overlap"),
    (prefix, dict(o=3 * P + 8 * 64 * 2 * 64 * 2 - 2), INVALID, "overlap"),
    (prefix, dict(ws=2 * P - 16), INVALID, "overlap"),
    (prefix, dict(ws=None), WORKSPACE, "null"),
    (prefix, dict(wsb=64), WORKSPACE, "needed"),
    (prefix, dict(), INVALID, "context is null"),
    (prefix, dict(g=0, off=None, pre=None), INVALID, "context is null"),
    (prefix, dict(n=0, q=None, o=None, k=None, v=None, tab=None, lens=None, ws=None), INVALID, "context is null"),
]


@pytest.mark.parametrize("call,bad,status,text", REFUSED)
def test_refused_before_any_gpu_work(b, call, bad, status, text):
    st, msg = call(b, **bad)
    assert st == status and text in msg, (st, msg)


def test_workspaces_cover_smaller_calls(b):
    """One that was sized for the largest call holds every smaller one."""
    for select in (1, 5, 64):
        most = b.hs_beam_select_workspace_size(64, 8, 50001, select)
        for groups in (1, 2, 7, 33, 64):
            for beams in (1, 3, 8):
                assert b.hs_beam_select_workspace_size(groups, beams, 50001, select) <= most, (groups, beams)
    for heads in ((28, 4, 128), (16, 16, 64), (64, 1, 128)):
        most = b.hs_prefix_attention_workspace_size(*heads, 200, 20000, 3000)
        for n in (1, 3, 16, 77, 200):
            for p in (0, 1, 255, 4096, 20000):
                for r in (0, 1, 257, 3000):
                    assert b.hs_prefix_attention_workspace_size(*heads, n, p, r) <= most, (n, p, r)
    assert b.hs_prefix_attention_workspace_size(28, 4, 128, 0, 4096, 100) == 0


def test_partial_results_of_beams_fit_the_workspace(b):
    states = b.lib().hs_beam_select_states
    states.restype = ctypes.c_uint64
    rng = np.random.default_rng(2)
    for _ in range(20000):
        groups, beams = int(np.exp(rng.uniform(0, np.log(1000)))), int(rng.integers(1, 65))
        vocab, select = int(np.exp(rng.uniform(0, np.log(300000)))), int(rng.integers(1, 65))
        size = b.hs_beam_select_workspace_size(groups, beams, vocab, select)
        for cus in (1, 64, 160, 256):
            less = int(rng.integers(1, groups + 1))
            for g, elem in ((groups, 2), (groups, 4), (less, 2), (less, 4)):
                assert states(g * beams, vocab, elem, select, cus) <= size, (groups, g, beams, vocab, select, cus)


def test_partial_states_fit_the_workspace(b):
    """Every grouping and budget of a call, and of smaller ones, writes no more than its workspace holds."""
    states = b.lib().hs_prefix_attention_states
    states.restype = ctypes.c_uint64
    rng = np.random.default_rng(1)
    for heads in ((28, 4, 128), (16, 16, 64), (64, 1, 128), (4, 2, 64), (1, 1, 64)):
        for _ in range(4000):
            n = int(np.exp(rng.uniform(0, np.log(600))))
            p, r = (int(np.exp(rng.uniform(0, np.log(200000)))) - 1 for _ in range(2))
            size = b.hs_prefix_attention_workspace_size(*heads, n, p, r)
            for cus in (1, 64, 160, 256):
                m, g = int(rng.integers(1, n + 1)), int(rng.integers(0, n + 2))
                less = int(rng.integers(0, p + 1)), int(rng.integers(0, r + 1))
                assert states(n, g, p if g else 0, r, *heads, cus) <= size, (heads, n, g, p, r, cus)
                assert states(m, g, less[0] if g else 0, less[1], *heads, cus) <= size, (heads, n, m, g, p, r, less, cus)


# ---------------------------------------------------------------------------- pages

class Model:
    """Sequences as lists of values, pages as the arrays that a cache would hold."""

    def __init__(self, b, n_pages, page, max_seqs, per_seq):
        self.pages = b.Pages(n_pages, page, max_seqs, per_seq)
        self.n_pages, self.page, self.per_seq, self.n = n_pages, page, per_seq, max_seqs
        self.held = np.full((n_pages, page), -1, np.int64)
        self.seqs = [[] for _ in range(max_seqs)]
        self.next = 0

    def move(self, copies):
        src, dst, positions = copies
        assert not set(dst) & set(src) and len(set(dst)) == len(dst)
        for s, d, n in zip(src, dst, positions):
            assert 0 < n <= self.page
            self.held[d] = -7   # what a copy leaves there beyond its positions is nobody's
            self.held[d, :n] = self.held[s, :n]

    def reserve(self, seqs, add):
        before = [len(self.seqs[s]) for s in seqs]
        self.move(self.pages.reserve(seqs, add))
        table, lens = self.pages.table(seqs)
        for i, (s, n) in enumerate(zip(seqs, add)):
            assert lens[i] == before[i] + n
            for p in range(before[i], before[i] + n):
                self.held[table[i, p // self.page], p % self.page] = self.next
                self.seqs[s].append(self.next)
                self.next += 1

    def fork(self, seqs, parents):
        self.pages.fork(seqs, parents)
        old = [list(s) for s in self.seqs]
        for s, p in zip(seqs, parents):
            self.seqs[s] = list(old[p]) if p >= 0 else []

    def compact(self, room):
        self.move(self.pages.compact(room))

    def check(self):
        everyone = list(range(self.n))
        table, lens = self.pages.table(everyone)
        used = set()
        for s in everyone:
            assert lens[s] == len(self.seqs[s])
            n = -(-int(lens[s]) // self.page)
            assert np.all(table[s, n:] == 0)
            used |= set(table[s, :n].tolist())
            got = [self.held[table[s, p // self.page], p % self.page] for p in range(int(lens[s]))]
            assert got == self.seqs[s], s
        assert self.pages.free_count() == self.n_pages - len(used)
        for group in ([0], [0, 1], everyone):
            want = min(len(self.seqs[s]) // self.page for s in group)
            for j in range(want):
                if len({int(table[s, j]) for s in group}) > 1:
                    want = j
                    break
            assert self.pages.shared(group) == want * self.page
        return used


@pytest.mark.parametrize("seed", range(6))
def test_pages_hold_what_sequences_hold(b, seed):
    rng = np.random.default_rng(seed)
    m = Model(b, n_pages=40, page=64, max_seqs=7, per_seq=6)
    for step in range(150):
        what = rng.integers(0, 5)
        seqs = rng.permutation(m.n)[:rng.integers(0, m.n + 1)].tolist()
        if what <= 1:
            add = [int(rng.choice((0, 1, 3, 63, 64, 65, 130))) for _ in seqs]
            try:
                m.reserve(seqs, add)
            except b.HorizonError as e:
                assert e.status in (INVALID, WORKSPACE)   # too long, or no free pages: nothing changed
        elif what == 2:
            m.fork(seqs, [int(rng.integers(-1, m.n)) for _ in seqs])
        elif what == 3:
            m.fork(seqs, [int(rng.integers(0, m.n)) for _ in seqs])
        else:
            m.compact(int(rng.integers(0, 12)))
        m.check()
    m.compact(40)
    used = m.check()
    assert used == set(range(len(used)))   # dense
    m.pages.release(list(range(m.n)))
    assert m.pages.free_count() == 40


def test_a_step_of_beams(b):
    """Beams share their prompt; a fork copies only the partly filled page, and the last user keeps it."""
    p = b.Pages(20, 64, 4, 5)
    assert p.reserve([0], [100]) == ([], [], [])
    p.fork([1, 2, 3], [0, 0, 0])
    assert p.free_count() == 18 and p.shared([0, 1, 2, 3]) == 64
    src, dst, n = p.reserve([0, 1, 2, 3], [1] * 4)
    assert src == [1, 1, 1] and dst == [2, 3, 4] and n == [36] * 3
    table, lens = p.table([0, 1, 2, 3])
    assert table[:, :2].tolist() == [[0, 2], [0, 3], [0, 4], [0, 1]] and lens.tolist() == [101] * 4
    p.fork([0, 1, 2, 3], [2, 2, 0, 0])    # parents as they were before the call
    table, _ = p.table([0, 1, 2, 3])
    assert table[:, :2].tolist() == [[0, 4], [0, 4], [0, 2], [0, 2]] and p.free_count() == 17
    # A whole last page is shared as it is.
    q = b.Pages(4, 64, 2, 3)
    q.reserve([0], [64])
    q.fork([1], [0])
    assert q.reserve([0, 1], [1, 1]) == ([], [], []) and q.shared([0, 1]) == 64 and q.free_count() == 1


def test_pages_refusals(b):
    for bad in ((0, 64, 1, 1), (4, 96, 1, 1), (4, 64, 0, 1), (4, 64, 1, 0), (4, 0, 1, 1)):
        with pytest.raises(b.HorizonError):
            b.Pages(*bad)
    for bad in (((1 << 28) + 1, 64, 1, 1), (4, 64, (1 << 24) + 1, 1)):
        with pytest.raises(b.HorizonError, match="at most"):
            b.Pages(*bad)
    with pytest.raises(b.HorizonError, match="positions a sequence"):
        b.Pages(4, 1 << 20, 1, 1 << 20)
    p = b.Pages(4, 64, 2, 3)
    p.reserve([0], [65])
    for call, text in ((lambda: p.reserve([0, 0], [1, 1]), "twice"), (lambda: p.reserve([2], [1]), "outside"),
                       (lambda: p.reserve([0], [-1]), "add"), (lambda: p.reserve([0], [200]), "beyond its 3 pages"),
                       (lambda: p.reserve([0, 1], [64, 129]), "free"), (lambda: p.fork([0], [2]), "parent"),
                       (lambda: p.fork([0, 0], [1, 1]), "twice"), (lambda: p.compact(-1), "room"),
                       (lambda: p.shared([]), "no sequences"), (lambda: p.table([-1]), "outside")):
        with pytest.raises(b.HorizonError, match=text):
            call()
    table, lens = p.table([0, 1])
    assert lens.tolist() == [65, 0] and table.tolist() == [[0, 1, 0], [0, 0, 0]] and p.free_count() == 2
    with pytest.raises(ValueError, match="parents"):
        p.fork([0], [1, 1])
    L = b.lib()
    n = ctypes.c_int32(0)
    for call in (lambda: L.hs_pages_create(4, 64, 1, 1, None), lambda: L.hs_pages_free_count(None, ctypes.byref(n)),
                 lambda: L.hs_pages_fork(None, None, None, 0), lambda: L.hs_pages_table(None, None, 0, None, None),
                 lambda: L.hs_pages_fork(p.handle, None, None, 1),
                 lambda: L.hs_pages_compact(p.handle, 1, None, None, None, ctypes.byref(n)),
                 lambda: L.hs_pages_shared(p.handle, _i32([0]), 1, None)):
        assert call() == INVALID
    assert L.hs_pages_destroy(None) == 0
