"""Decoding on a shared cache on the GPU: selection over beams, copies, attention behind shared prefixes, against
float64.

Tolerances.  A rounding is off by at most half a step (fp16 2^-11, bf16 2^-8, fp32 2^-24 of the value).

Beams: the sum of e^(z - m) is fp32.  An exponent's argument is rounded at |z - m| log2(e), which moves the term by
|z - m| 2^-24 of itself, and on average over the row's distribution by D 2^-24, D the mean distance; the exponential
(2^-22) and at most 32 additions in a row and over the lanes add 36 steps.  So log S is within (D + 40) 2^-24, and a
value is rounded once more when it is written.

Attention: with A = sum w |v| / sum w, an output is off by its own rounding, by the weights' (2^-11 A, and below 2^-14,
where fp16 has steps of 2^-24, half a step of each: the oracle's slack), by the scores' fp32 sums (dh 2^-24 |q| |k|
/ sqrt(dh) in the exponent, of each weight and of their sum), the exponential and its argument (2^-20), and by fp32 sums over the
keys (n 2^-24 A).
"""
import math

import numpy as np
import pytest

from oracle import decoding as ref
from tests.gpu_common import log, require_gpu

pytestmark = pytest.mark.gpu

HALF = {"f32": 2.0 ** -24, "f16": 2.0 ** -11, "bf16": 2.0 ** -8}


@pytest.fixture(scope="module")
def env():
    torch = require_gpu()
    from paper_2608_01785_amd import binding
    ctx = binding.Context(0, budgets=(64, 128, 256))
    yield torch, binding, ctx
    torch.cuda.synchronize()
    ctx.close()


def _type(torch, name):
    return {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}[name]


def _gen(torch, seed):
    return torch.Generator(device="cuda").manual_seed(seed)


# ---------------------------------------------------------------------------- beams

class Beams:
    """Inputs, outputs and workspace of one selection; rows start `pad` elements apart from each other's ends."""

    def __init__(self, env, groups, beams, vocab, select, dtype="f32", pad=0, first=0, seed=1, end=-1, finished=False,
                 masked=0.0):
        self.torch, self.b, self.ctx = env
        torch = self.torch
        gen = _gen(torch, seed)
        self.groups, self.beams, self.vocab, self.select, self.end = groups, beams, vocab, select, end
        rows = groups * beams
        store = torch.full((rows * (vocab + pad) + first + 8,), float("nan"), dtype=_type(torch, dtype), device="cuda")
        self.z = store[first:first + rows * (vocab + pad)].view(rows, vocab + pad)[:, :vocab]
        z = torch.randn((rows, vocab), generator=gen, device="cuda") * 2.5
        z.scatter_add_(1, torch.randint(0, vocab, (rows, 1), generator=gen, device="cuda"),
                       12 * torch.rand((rows, 1), generator=gen, device="cuda"))
        if masked:
            z.masked_fill_(torch.rand((rows, vocab), generator=gen, device="cuda") < masked, -math.inf)
        self.z.copy_(z)
        self.scores = -30 * torch.rand((groups, 1), generator=gen, device="cuda") - 4 * torch.rand(
            (groups, beams), generator=gen, device="cuda")
        self.finished = None
        if finished:
            u = torch.rand((groups, beams), generator=gen, device="cuda")
            self.finished = (u < 0.3).to(torch.uint8) * 5   # any non-zero entry
            self.scores.masked_fill_(u > 0.75, -math.inf)

        def new(t, fill):
            return torch.full((groups, select), fill, dtype=t, device="cuda")
        self.out = dict(out_scores=new(torch.float32, 7.0), out_parents=new(torch.int32, 77),
                        out_tokens=new(torch.int32, 777), out_finished=new(torch.uint8, 9))
        self.ws = torch.full((max(1, self.b.hs_beam_select_workspace_size(groups, beams, vocab, select)),), 255,
                             dtype=torch.uint8, device="cuda")
        torch.cuda.synchronize()

    def call(self, cus=256, stream=None):
        self.b.hs_beam_select(self.ctx, self.z, self.scores, self.out["out_scores"], self.out["out_parents"],
                              self.out["out_tokens"], finished=self.finished, out_finished=self.out["out_finished"],
                              end_token=self.end, cu_budget=cus, stream=stream, workspace=self.ws)
        return self

    def check(self, exact_order=False):
        self.torch.cuda.synchronize()
        z = self.z.double().cpu().numpy()
        scores = self.scores.cpu().numpy()
        fin = None if self.finished is None else self.finished.cpu().numpy()
        got = {n: t.cpu().numpy() for n, t in self.out.items()}
        close = 0
        for g in range(self.groups):
            rows = slice(g * self.beams, (g + 1) * self.beams)
            values, distance = ref.beam_values(z[rows], scores[g], None if fin is None else fin[g], self.end)
            tol = (distance.max() + 40) * 2.0 ** -24
            want = ref.beam_select(values, z[rows], self.select)
            for i, (v, b, t) in enumerate(want):
                at = (g, i)
                gb, gt, gs = int(got["out_parents"][at]), int(got["out_tokens"][at]), float(got["out_scores"][at])
                if v == -np.inf:
                    assert (gb, gt, gs, got["out_finished"][at]) == (-1, -1, -np.inf, 0), (at, gb, gt, gs)
                    continue
                if (gb, gt) != (b, t):
                    # Only a value closer than both sides' errors may stand here, and none of its own beam.
                    assert not exact_order and gb != b and abs(values[gb, gt] - v) <= 2 * tol, (at, (gb, gt), (b, t))
                    close += 1
                assert abs(gs - v) <= 2 * tol + abs(v) * HALF["f32"], (at, gs, v)
                done = (fin is not None and fin[g, gb] != 0) or (self.end >= 0 and gt == self.end)
                assert got["out_finished"][at] == done, at
            pairs = list(zip(got["out_parents"][g].tolist(), got["out_tokens"][g].tolist()))
            live = [p for p in pairs if p[0] >= 0]
            assert len(set(live)) == len(live)
        return close


BEAMS = [
    # groups, beams, vocab, select: one of everything, lists longer than the vocabulary, split and whole rows, and
    # enough rows for one wavefront each.
    (1, 1, 1, 1), (1, 1, 1, 3), (2, 3, 2, 64), (1, 4, 777, 4), (3, 1, 5000, 64), (1, 4, 32000, 8), (5, 7, 4097, 14),
    (2, 64, 1500, 64), (1, 1, 131072, 5), (1, 2, 160001, 64), (40, 8, 2048, 16), (300, 8, 1031, 9), (129, 16, 700, 2),
]


@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("groups,beams,vocab,select", BEAMS)
def test_selection(env, groups, beams, vocab, select, dtype):
    seed = groups + beams + vocab + select
    log(f"[beam] {groups} x {beams}, vocabulary {vocab}, {select} selected, {dtype}")
    Beams(env, groups, beams, vocab, select, dtype, pad=seed % 3, first=seed % 5, seed=seed).call().check()


@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("masked", [0.0, 0.6, 0.999, 1.0])
def test_finished_empty_and_masked_beams(env, dtype, masked):
    log(f"[beam] finished and empty beams, masked {masked}, {dtype}")
    s = Beams(env, 30, 5, 3001, 10, dtype, pad=1, seed=5, end=3000, finished=True, masked=masked)
    s.call().check()


@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
def test_equal_values_go_to_the_lower_beam_and_token(env, dtype):
    """Rows alike in every bit: whole groups of equal values, at odd row starts too."""
    torch = env[0]
    for vocab, pad in ((50, 0), (5000, 3), (40000, 1)):
        s = Beams(env, 2, 5, vocab, 30, dtype, pad=pad, seed=3)
        s.z.copy_((s.z[:1].float() / 2).round().expand_as(s.z))   # many equal logits
        s.scores.fill_(-1.5)
        torch.cuda.synchronize()
        s.call().check()
        got = s.out["out_parents"].cpu()
        # Each value stands 5 times, beam after beam, where all its tokens fit.
        z = s.z[0].float().cpu()
        top = int((z == z.max()).sum())
        if top <= 6:
            want = sum(([b] * top for b in range(5)), [])[:30]
            assert got[0, :len(want)].tolist() == want and got[1, :len(want)].tolist() == want
    s = Beams(env, 1, 3, 9000, 64, dtype, seed=4)
    s.z.fill_(1.0)
    s.scores.copy_(torch.tensor([[-2.0, -1.0, -2.0]]))
    torch.cuda.synchronize()
    s.call().check(exact_order=True)
    assert s.out["out_tokens"].cpu().tolist() == [list(range(64))]


@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
def test_rows_without_a_distribution(env, dtype):
    torch = env[0]
    for vocab in (200, 20000):
        s = Beams(env, 3, 4, vocab, 6, dtype, seed=6)
        s.z[0, vocab // 2] = float("nan")
        s.z[2, vocab - 1] = math.inf
        s.z[5] = -math.inf
        s.z[6] = float("-nan")
        s.z[8:12] = -math.inf
        s.z[9, 3] = math.inf
        s.scores[1, 3] = float("nan")
        s.scores[1, 0] = -math.inf
        torch.cuda.synchronize()
        s.call().check()
        parents = s.out["out_parents"].cpu()
        assert set(parents[0].tolist()) <= {1, 3} and torch.all(parents[1:] == -1)


@pytest.mark.parametrize("select", [4, 60])
def test_scores_that_swallow_the_logits(env, select):
    """Beyond 2^60 every continuation of a beam has one value: its logits' order is left, then the lower beam's."""
    torch = env[0]
    s = Beams(env, 1, 3, 2000, select, "f32", seed=20)
    s.scores.copy_(torch.tensor([[-2e30, -1e30, -1e30]]))
    torch.cuda.synchronize()
    s.call()
    torch.cuda.synchronize()
    want = torch.sort(s.z[1], descending=True, stable=True).indices[:select].tolist()
    assert s.out["out_tokens"][0].tolist() == want and s.out["out_parents"][0].tolist() == [1] * select
    s.scores.fill_(math.inf)
    torch.cuda.synchronize()
    s.call()
    torch.cuda.synchronize()
    want = torch.sort(s.z[0], descending=True, stable=True).indices[:select].tolist()
    assert s.out["out_tokens"][0].tolist() == want and s.out["out_parents"][0].tolist() == [0] * select
    assert torch.all(s.out["out_scores"] == math.inf)


def test_far_scores_and_certain_tokens(env):
    """A token with all the probability: its distance from 0 counts; logits beyond 2^20; scores from many steps."""
    torch = env[0]
    s = Beams(env, 2, 4, 3000, 8, "f32", seed=8)
    s.z[0, 7] = 40.0
    s.z[1] += 3e6
    s.z[2] -= 3e8
    s.z[4, 2999] = 3e38
    s.scores[0] -= 1e5
    torch.cuda.synchronize()
    s.call().check()


@pytest.mark.parametrize("cus", [64, 128, 256])
def test_budgets_streams_and_repeats(env, cus):
    torch, b, ctx = env
    s = Beams(env, 2, 4, 50001, 8, "bf16", pad=5, seed=9, end=2, finished=True)
    s.call(cus).check()
    first = {n: t.clone() for n, t in s.out.items()}
    if cus < 256:   # the downstream stream of the complementary level, same results on any budget's split of rows
        down = b.hs_context_stream(ctx, cus, b.HS_ROLE_DOWN)
        s.call(256 - cus, down).check()
    for _ in range(3):
        s.call(cus)
        torch.cuda.synchronize()
        for n, t in first.items():
            assert torch.equal(t, s.out[n]), n


def test_two_selections_at_once(env):
    torch, b, ctx = env
    one, two = Beams(env, 1, 4, 90000, 8, "f32", seed=10), Beams(env, 3, 2, 50001, 5, "f16", pad=1, seed=11)
    up, down = b.hs_context_stream(ctx, 128), b.hs_context_stream(ctx, 128, b.HS_ROLE_DOWN)
    for _ in range(6):
        one.call(128, up)
        two.call(128, down)
    one.check()
    two.check()


# ---------------------------------------------------------------------------- copies

def _cache(torch, layers, slots, hkv, page, dh, seed, nan=False):
    gen = _gen(torch, seed)

    def new(*shape):
        t = torch.randn(shape, generator=gen, device="cuda", dtype=torch.float16)
        return torch.where(torch.rand(shape, generator=gen, device="cuda") < 0.01, float("nan"), t) if nan else t
    return ([new(slots, hkv, page, dh) for _ in range(layers)],
            [new(slots, hkv, page // 32, dh, 32) for _ in range(layers)])


def _copied(k, v, src, dst, positions):
    """The cache after the copies, on the host."""
    out = [t.cpu().view(t.dtype).clone() for t in k], [t.cpu().clone() for t in v]
    for kl, vl in zip(*out):
        for s, d, n in zip(src, dst, positions):
            n = -(-n // 32)
            kl[d, :, :32 * n] = kl[s, :, :32 * n]
            vl[d, :, :n] = vl[s, :, :n]
    return out


@pytest.mark.parametrize("layers,slots,hkv,page,dh,n", [
    (1, 2, 1, 64, 64, 1), (4, 9, 4, 512, 128, 3), (33, 5, 2, 64, 64, 2), (2, 40, 16, 128, 64, 17),
    (1, 800, 1, 64, 64, 390), (1, 6, 2, 4096, 128, 3), (65, 3, 1, 64, 128, 1)])
@pytest.mark.parametrize("fill", ["one", "ragged", "whole"])
def test_copies(env, layers, slots, hkv, page, dh, n, fill):
    torch, b, ctx = env
    log(f"[copy] {layers} layers, {slots} slots of {page}, {hkv} heads of {dh}, {n} copies, {fill}")
    rng = np.random.default_rng(layers + slots + n)
    order = rng.permutation(slots)
    dst = order[:n].tolist()
    src = [int(order[n + rng.integers(0, slots - n)]) for _ in range(n)]
    positions = {"one": [1] * n, "ragged": rng.integers(0, page + 1, n).tolist(), "whole": [page] * n}[fill]
    k, v = _cache(torch, layers, slots, hkv, page, dh, 3, nan=True)
    want_k, want_v = _copied(k, v, src, dst, positions)
    torch.cuda.synchronize()
    kv = (k, v, slots, page)
    b.hs_cache_copy(ctx, kv, src, dst, None if fill == "whole" else positions)
    torch.cuda.synchronize()
    for got, want in list(zip(k, want_k)) + list(zip(v, want_v)):
        assert torch.equal(got.cpu().view(torch.int16), want.view(torch.int16))


def test_a_captured_copy_keeps_its_list(env):
    torch, b, ctx = env
    k, v = _cache(torch, 2, 6, 2, 128, 64, 4)
    src, dst, positions = [0, 0, 3], [1, 2, 4], [100, 5, 128]
    stream = torch.cuda.Stream()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=stream):
        b.hs_cache_copy(ctx, (k, v, 6, 128), src, dst, positions, stream=stream.cuda_stream)
    src[0], dst[0], positions[0] = 5, 3, 1   # the call's own lists are its caller's again
    for i in range(3):
        for t in k + v:
            t.normal_(generator=_gen(torch, 40 + i))
        torch.cuda.synchronize()
        want_k, want_v = _copied(k, v, [0, 0, 3], [1, 2, 4], [100, 5, 128])
        graph.replay()
        torch.cuda.synchronize()
        for got, want in list(zip(k, want_k)) + list(zip(v, want_v)):
            assert torch.equal(got.cpu(), want)


# ---------------------------------------------------------------------------- attention

class Prefix:
    """Groups of `rows` sequences with `prefix` shared positions and `rest` keys of each sequence to itself."""

    def __init__(self, env, rows, prefix, rest, heads=(4, 2, 64), page=64, dtype="f16", pad=0, seed=1, spare=2,
                 scale=1.0, poison=True, grouped=True):
        self.torch, self.b, self.ctx = env
        torch = self.torch
        hq, hkv, dh = heads
        self.heads, self.page, self.dtype = heads, page, dtype
        self.prefix = list(prefix)
        self.offsets = np.concatenate([[0], np.cumsum(rows)]).astype(np.int64).tolist()
        n = self.offsets[-1]
        self.n = n
        rng = np.random.default_rng(seed)
        group = [g for g in range(len(rows)) for _ in range(rows[g])]
        self.lens = [self.prefix[group[i]] + rest[i] for i in range(n)]
        need = [-(-m // page) for m in self.lens]
        pps = max(need + [1]) + 1
        whole = [p // page for p in self.prefix]
        slots = sum(w for g, w in enumerate(whole) if rows[g]) + sum(need[i] - whole[group[i]] for i in range(n)) + spare
        order = rng.permutation(slots).tolist()
        self.table = np.full((n, pps), -1, np.int64)   # unreached entries name no slot
        for g in range(len(rows)):
            shared = [order.pop() for _ in range(whole[g])] if rows[g] else []
            for i in range(self.offsets[g], self.offsets[g + 1]):
                self.table[i, :need[i]] = shared + [order.pop() for _ in range(need[i] - whole[g])]
        (self.k,), (self.v,) = _cache(torch, 1, slots, hkv, page, dh, seed + 1)
        if poison:   # what no row may see is NaN
            seen = np.zeros((slots, page), bool)
            for i in range(n):
                first = i == self.offsets[group[i]]
                for p in range(0 if first else self.prefix[group[i]], self.lens[i]):
                    seen[self.table[i, p // page], p % page] = True
            hide = torch.from_numpy(~seen).cuda()
            self.k.masked_fill_(hide[:, None, :, None], float("nan"))
            self.v.masked_fill_(hide.view(slots, 1, page // 32, 1, 32), float("nan"))
        gen = _gen(torch, seed + 2)
        t = _type(torch, dtype)
        self.q = torch.empty((n, hq * dh + pad), dtype=t, device="cuda")[:, :hq * dh]
        self.q.copy_(scale * torch.randn((n, hq * dh), generator=gen, device="cuda"))
        self.store = torch.full((n, hq * dh + pad + 1), 7.0, dtype=t, device="cuda")
        self.out = self.store[:, :hq * dh]
        self.max_prefix, self.max_rest = max(self.prefix + [0]), max(rest + [0])
        self.grouped = grouped
        self.upload()

    def upload(self):
        def ints(x):
            return self.torch.as_tensor(np.asarray(x), dtype=self.torch.int32).cuda()
        self.d = dict(table=ints(self.table), lens=ints(self.lens), offsets=ints(self.offsets), prefix=ints(self.prefix))
        size = self.b.hs_prefix_attention_workspace_size(*self.heads, self.n, self.max_prefix, self.max_rest)
        self.ws = self.torch.full((max(1, size),), 255, dtype=self.torch.uint8, device="cuda")
        self.torch.cuda.synchronize()

    def call(self, cus=256, stream=None):
        d = self.d
        self.b.hs_prefix_attention(self.ctx, self.q, self.out, self.k, self.v, d["table"], d["lens"],
                                   d["offsets"] if self.grouped else None, d["prefix"] if self.grouped else None,
                                   self.max_prefix, self.max_rest, cu_budget=cus, stream=stream, workspace=self.ws)
        return self

    def check(self, rows=None):
        torch = self.torch
        torch.cuda.synchronize()
        hq, hkv, dh = self.heads
        q = self.q.double().cpu().numpy().reshape(self.n, hq, dh)
        k, v = self.k.double().cpu().numpy(), self.v.double().cpu().numpy()
        o, a, slack = ref.prefix_attention(q, k, v, self.table, self.lens, self.offsets, self.prefix)
        got = self.out.double().cpu().numpy().reshape(self.n, hq, dh)
        kmax = np.sqrt(np.nanmax((np.nan_to_num(k) ** 2).sum(-1)))
        score = 2.0 ** -24 * dh * np.sqrt((q ** 2).sum(-1)) * kmax / math.sqrt(dh)
        keys = np.asarray(self.lens, np.float64)[:, None, None]
        tol = (np.abs(o) * HALF[self.dtype] + a * (2.0 ** -11 + 2 * score[..., None] + 2.0 ** -20 + keys * 2.0 ** -24)
               + slack[..., None] + 2.0 ** -25)
        rows = list(range(self.n)) if rows is None else rows
        assert np.all(np.isfinite(got[rows]))
        bad = np.abs(got - o) > tol
        assert not bad[rows].any(), (np.argwhere(bad)[:3], np.abs(got - o)[bad][:3], tol[bad][:3])
        assert torch.all(self.store[:, hq * dh:] == 7.0)   # beside the rows
        return got


HEADS = {"tiny": (4, 2, 64), "talker": (16, 16, 64), "thinker": (28, 4, 128), "mixed": (32, 8, 128),
         "one": (1, 1, 64), "many": (40, 1, 128)}


@pytest.mark.parametrize("heads", sorted(HEADS))
@pytest.mark.parametrize("rows,prefix,rest,page", [
    ([1], [0], [1], 64), ([1], [1], [0], 64), ([1], [0], [0], 64), ([2], [64], [1, 64], 64), ([3], [65], [0, 5, 700], 64),
    ([1, 2, 0, 3], [31, 0, 50, 700], [1, 0, 33, 2, 64, 100], 128), ([5], [2000], [1, 2, 3, 4, 600], 512),
])
def test_attention(env, heads, rows, prefix, rest, page):
    log(f"[prefix] {heads} rows {rows} prefix {prefix} rest {rest} page {page}")
    for dtype, pad in (("f16", 0), ("bf16", 8)):
        s = Prefix(env, rows, prefix, rest, HEADS[heads], page, dtype, pad, seed=len(rest) + page)
        s.call().check()


@pytest.mark.parametrize("heads,n,prefix,rest,page", [
    ("thinker", 9, 3000, 50, 192), ("talker", 40, 1000, 130, 64), ("mixed", 33, 777, 20, 320), ("tiny", 100, 5001, 3, 64),
    ("thinker", 70, 500, 1, 64)])
def test_attention_of_large_groups(env, heads, n, prefix, rest, page):
    log(f"[prefix] {heads} {n} rows behind {prefix}")
    s = Prefix(env, [n], [prefix], [(37 * i) % (rest + 1) for i in range(n)], HEADS[heads], page, "f16", seed=n)
    s.call().check()


def test_many_groups(env):
    """More groups than a wavefront has lanes, some empty."""
    rng = np.random.default_rng(3)
    rows = rng.integers(0, 4, 150).tolist()
    prefix = rng.integers(0, 200, 150).tolist()
    s = Prefix(env, rows, prefix, rng.integers(0, 90, sum(rows)).tolist(), HEADS["tiny"], 64, "f16", seed=4)
    s.call().check()


def test_many_short_groups(env):
    rng = np.random.default_rng(5)
    rows = rng.integers(0, 5, 150).tolist()
    prefix = rng.integers(0, 65, 150).tolist()
    s = Prefix(env, rows, prefix, rng.integers(0, 30, sum(rows)).tolist(), HEADS["thinker"], 64, "bf16", seed=6)
    s.call().check()


@pytest.mark.parametrize("seed", range(24))
def test_drawn_attention(env, seed):
    """Groups, lengths, pages, heads, types and strides drawn together."""
    rng = np.random.default_rng(1000 + seed)
    heads = HEADS[sorted(HEADS)[rng.integers(len(HEADS))]]
    groups = int(rng.integers(1, 7))
    rows = rng.integers(0, 8, groups).tolist()
    rows[rng.integers(groups)] += 1
    reach = int(rng.choice((20, 100, 700, 3000)))
    prefix = rng.integers(0, reach + 1, groups).tolist()
    rest = rng.integers(0, int(rng.choice((1, 2, 40, 300))), sum(rows)).tolist()
    page, dtype = 64 * int(rng.integers(1, 9)), str(rng.choice(("f16", "bf16")))
    log(f"[prefix] drawn {seed}: {heads} rows {rows} prefix {prefix} rest {rest[:6]} page {page} {dtype}")
    Prefix(env, rows, prefix, rest, heads, page, dtype, pad=int(rng.choice((0, 8, 40))), seed=seed,
           scale=float(rng.choice((0.3, 1.0, 4.0)))).call(int(rng.choice((64, 128, 256)))).check()


@pytest.mark.parametrize("seed", range(24))
def test_drawn_selection(env, seed):
    rng = np.random.default_rng(2000 + seed)
    beams, groups = int(rng.integers(1, 13)), int(rng.integers(1, 12))
    vocab = int(np.exp(rng.uniform(np.log(2), np.log(60000))))
    select, dtype = int(rng.integers(1, min(64, 3 * beams) + 1)), str(rng.choice(("f32", "f16", "bf16")))
    end = int(rng.integers(0, vocab)) if rng.random() < 0.6 else -1
    log(f"[beam] drawn {seed}: {groups} x {beams}, {vocab}, {select}, {dtype}, end {end}")
    s = Beams(env, groups, beams, vocab, select, dtype, pad=int(rng.integers(0, 9)), first=int(rng.integers(0, 5)),
              seed=seed, end=end, finished=end >= 0 and rng.random() < 0.6, masked=float(rng.choice((0.0, 0.0, 0.7, 0.999))))
    s.call(int(rng.choice((64, 128, 256)))).check()


@pytest.mark.parametrize("heads", ["thinker", "talker", "many"])
def test_without_groups(env, heads):
    for rest in ([1, 0, 500, 64, 65, 3], [1, 0, 31, 20, 32, 3]):
        s = Prefix(env, [1] * 6, [0] * 6, rest, HEADS[heads], 128, "f16", seed=5, grouped=False)
        s.call().check()


def test_sharp_scores(env):
    """Queries whose heads look at one key: sums close to one, other weights below fp16."""
    for scale in (8.0, 60.0):
        Prefix(env, [4], [900], [3, 100, 0, 64], HEADS["thinker"], 64, "f16", seed=6, scale=scale).call().check()


# Groups whose ranges go through one block each, and longer ones that are split and joined.
SHORT = dict(rows=[3, 4], prefix=[40, 65], rest=[5, 30, 1, 9, 20, 3, 24], heads=HEADS["thinker"])
LONG = dict(rows=[3, 4], prefix=[100, 200], rest=[5, 70, 1, 9, 80, 3, 64], heads=HEADS["tiny"])


@pytest.mark.parametrize("case", [SHORT, LONG], ids=["short", "long"])
def test_wrong_lengths_and_slots_make_their_rows_nan(env, case):
    torch = env[0]
    s = Prefix(env, page=64, dtype="f16", seed=7, poison=False, **case)
    clean = s.call().check()
    table, lens, prefix = s.table.copy(), list(s.lens), list(s.prefix)
    s.table[1, (prefix[0] + case["rest"][1] - 1) // 64] = s.k.shape[0]   # beyond the cache: keys of row 1 alone
    s.table[4, (lens[4] - 1) // 64] = -5
    s.lens[2] = prefix[0] - 1                   # shorter than its prefix
    s.lens[5] = prefix[1] + s.max_rest + 1      # beyond the bound
    s.lens[6] = 64 * s.table.shape[1] + 1       # beyond the table (and the bound)
    s.upload()
    s.call()
    torch.cuda.synchronize()
    got = s.out.double().cpu().numpy()
    for i in range(7):
        if i in (1, 2, 4, 5, 6):
            assert np.isnan(got[i]).all(), i
        else:
            assert (got[i] == clean[i].reshape(-1)).all(), i
    s.table, s.lens = table, lens
    s.table[0, 0] = 10 ** 6                     # under a prefix: the whole group
    s.upload()
    s.call()
    torch.cuda.synchronize()
    got = s.out.double().cpu().numpy()
    assert np.isnan(got[:3]).all() and (got[3:] == clean[3:].reshape(4, -1)).all()
    s.table = table
    s.prefix = [max(prefix) + 1, -1]            # beyond its bound, negative
    s.max_prefix = max(prefix)
    s.upload()
    s.call()
    torch.cuda.synchronize()
    assert torch.all(torch.isnan(s.out))


@pytest.mark.parametrize("case", [SHORT, LONG], ids=["short", "long"])
def test_nan_and_infinity_stay_with_their_rows(env, case):
    """In the keys or values of one row, in its query: the rows beside it in the same products keep their bits."""
    torch = env[0]
    s = Prefix(env, page=64, dtype="f16", seed=13, poison=False, **case)
    clean = s.call().check()
    page, at = s.table[4, (s.lens[4] - 1) // 64], (s.lens[4] - 1) % 64
    s.v[page, :, at // 32, :, at % 32] = float("nan")
    page, at = s.table[1, (s.lens[1] - 1) // 64], (s.lens[1] - 1) % 64
    s.k[page, :, at, 3] = math.inf
    s.v[page, :, at // 32, :, at % 32] = math.inf
    s.q[5] = float("nan")
    torch.cuda.synchronize()
    s.call()
    torch.cuda.synchronize()
    got = s.out.double().cpu().numpy()
    for i in range(7):
        if i in (4, 5):
            assert np.isnan(got[i]).all()
        elif i != 1:
            assert (got[i] == clean[i].reshape(-1)).all(), i


def test_offsets_that_make_no_sense_touch_nothing(env):
    torch = env[0]
    for case in (SHORT, LONG):
        s = Prefix(env, page=64, dtype="f16", seed=8, poison=False, **case)
        for offsets in ([5, 2, 900], [-7, 100, 3], [0, 0, 0], [2 ** 31 - 1, -2 ** 31, 5]):
            s.offsets = offsets
            s.upload()
            s.call()
            torch.cuda.synchronize()
            assert torch.all(s.store[:, s.out.shape[1]:] == 7.0)


def test_offsets_beyond_32_bits(env):
    """A slot whose elements lie more than 2^32 bytes into the cache."""
    torch = env[0]
    s = Prefix(env, [2], [70], [3, 40], HEADS["thinker"], 64, "f16", seed=9, poison=False)
    slots = 70000                               # 70000 * 4 * 64 * 128 * 2 = 4.6 GB
    used = s.k.shape[0]
    far = list(range(slots - used, slots))
    for name in ("k", "v"):
        old = getattr(s, name)
        big = torch.zeros((slots,) + tuple(old.shape[1:]), dtype=torch.float16, device="cuda")
        big[slots - used:] = old
        setattr(s, name, big)
    s.table = np.where(s.table >= 0, s.table + slots - used, s.table)
    s.upload()
    s.call()
    torch.cuda.synchronize()
    got = s.out.clone()
    for name in ("k", "v"):
        setattr(s, name, getattr(s, name)[far].clone())
    s.table = np.where(s.table >= 0, s.table - (slots - used), s.table)
    s.upload()
    s.call().check()
    assert torch.equal(got, s.out)


@pytest.mark.parametrize("cus", [64, 128, 256])
def test_attention_on_budgets(env, cus):
    torch, b, ctx = env
    s = Prefix(env, [6, 2], [1200, 300], [5, 70, 1, 9, 80, 3, 64, 2], HEADS["thinker"], 128, "f16", seed=10)
    s.call(cus).check()
    if cus < 256:
        s.call(256 - cus, b.hs_context_stream(ctx, cus, b.HS_ROLE_DOWN)).check()
    s.call(cus)
    torch.cuda.synchronize()
    first = s.out.clone()
    for _ in range(3):
        s.call(cus)
        torch.cuda.synchronize()
        assert torch.equal(first, s.out)


def test_captured_attention_follows_its_arrays(env):
    """Lengths and tables of later steps, within the bounds, on one captured launch; another graph beside it."""
    torch, b, ctx = env
    s = Prefix(env, [3], [130], [90, 40, 64], HEADS["tiny"], 64, "f16", seed=11, poison=False)
    t = Prefix(env, [2], [64], [9, 1], HEADS["tiny"], 64, "bf16", seed=12)
    stream = torch.cuda.Stream()
    graphs = []
    for x in (s, t):
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=stream):
            x.call(stream=stream.cuda_stream)
        graphs.append(graph)
    full = list(s.lens)
    for cut in (0, 17, 40, 3):
        s.lens = [max(130, n - cut) for n in full]
        s.d["lens"].copy_(torch.as_tensor(s.lens, dtype=torch.int32))
        s.out.fill_(9.0)
        t.out.fill_(9.0)
        torch.cuda.synchronize()
        for graph in graphs:
            graph.replay()
        s.check()
        t.check()
        kept = s.out.clone()
        s.call()
        torch.cuda.synchronize()
        assert torch.equal(kept, s.out)


def test_timing_records_the_decoding_calls(env):
    torch, b, ctx = env
    s, p = Beams(env, 1, 2, 5000, 4), Prefix(env, [2], [64], [9, 1], HEADS["tiny"], 64)
    k, v = _cache(torch, 1, 3, 2, 64, 64, 5)
    torch.cuda.synchronize()
    b.hs_timing_enable(ctx, True)
    for _ in range(3):
        s.call()
        p.call()
        b.hs_cache_copy(ctx, (k, v, 3, 64), [0], [1], [5])
    for kind in ("beam_select", "cache_copy", "prefix_attn"):
        ms, n = b.hs_timing_read(ctx, kind)
        assert n == 3 and 0 < ms < 1000, (kind, ms, n)
    b.hs_timing_enable(ctx, False)


def test_binding_refusals(env):
    torch, b, ctx = env
    s = Beams(env, 2, 3, 100, 4)
    for change, text in ((dict(scores=s.scores.view(-1)), "dimensions"), (dict(scores=s.scores.cpu()), "is on cpu"),
                         (dict(scores=s.scores.double()), "type"), (dict(z=s.z[:5]), "rows"),
                         (dict(finished=torch.zeros((2, 2), dtype=torch.uint8, device="cuda")), "shape")):
        t = Beams(env, 2, 3, 100, 4, end=1)
        vars(t).update(change)
        with pytest.raises(ValueError, match=text):
            t.call()
    p = Prefix(env, [2], [64], [9, 1], HEADS["tiny"], 64)
    for change, text in ((dict(q=p.q.float()), "type"), (dict(out=p.out[:1]), "shape"), (dict(k=p.k[:1]), "shape"),
                         (dict(v=p.v.transpose(3, 4)), "shape"), (dict(k=p.k.float()), "type")):
        old = {n: getattr(p, n) for n in change}
        vars(p).update(change)
        with pytest.raises(ValueError, match=text):
            p.call()
        vars(p).update(old)
    k, v = _cache(torch, 2, 3, 2, 64, 64, 5)
    for kv, text in (((k, v[:1], 3, 64), "layers"), ((k, v, 4, 64), "shape"), (([k[0].cpu(), k[1]], v, 3, 64), "cpu")):
        with pytest.raises(ValueError, match=text):
            b.hs_cache_copy(ctx, kv, [0], [1], [5])
    with pytest.raises(ValueError, match="destinations"):
        b.hs_cache_copy(ctx, (k, v, 3, 64), [0], [1, 2], [5])
    log("refused as documented")
