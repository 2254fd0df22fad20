"""Decode steps behind shared prefixes, and the operators of decoding on a shared cache together: beam search.

The step is checked against the float64 layers of the oracle on each sequence's logical cache.  A search is checked
from its end: every beam's tokens go through a fresh prefill of prompt and continuation (no cache, no beams), whose
log probabilities must add up to the beam's score, and whose keys and values must be those of the beam's pages.
"""
import math

import numpy as np
import pytest

from oracle import layer as ref
from paper_2608_01785_amd import workloads as W
from tests.gpu_common import TOL, err_ratio, log, require_gpu
from tests.test_gpu_paged import make_table
from tests.util import f64, h64, weights_f64

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def env():
    torch = require_gpu()
    from paper_2608_01785_amd import binding
    ctx = binding.Context(0, budgets=(128, 192, 256))
    yield torch, binding, ctx
    torch.cuda.synchronize()
    ctx.close()


def _step(env, shape, n_layers, kv_lens, groups, prefix, page, seed, share_partial=False):
    """Inputs of a step whose groups (rows each) share `prefix` positions: (cache, table, weights, x, logical cache)."""
    torch, b, ctx = env
    from paper_2608_01785_amd.device_data import PagedCache, to_device, upload_weights
    rng = np.random.default_rng(seed)
    n = len(kv_lens)
    ends = [m + 1 for m in kv_lens]
    table, n_pages = make_table(rng, ends, page)
    offsets = np.concatenate([[0], np.cumsum(groups)])
    logical = W.make_cache(shape, n_layers, kv_lens, seed=seed + 1)
    for g, p in enumerate(prefix):
        for i in range(offsets[g] + 1, offsets[g + 1]):
            table[i, :p // page] = table[offsets[g], :p // page]
            for layer in range(n_layers):
                logical.k[layer][i][:p] = logical.k[layer][offsets[g]][:p]
                logical.v[layer][i][:p] = logical.v[layer][offsets[g]][:p]
    cache = PagedCache(n_layers, n_pages, page, shape.n_kv_heads, shape.head_dim, table, fill=7.0)
    for layer in range(n_layers):
        for i in range(n):
            cache.load_prefix(layer, i, logical.k[layer][i], logical.v[layer][i])
    layers = W.make_weights(shape, n_layers, seed + 2)
    batch = W.random_batch(shape.hidden, [1] * n, seed=seed + 3, ctx_lens=kv_lens)
    return cache, table, layers, batch, logical, [int(o) for o in offsets]


CASES = [
    ("tiny", 2, [100, 130, 64, 200, 64], [3, 2], [64, 64], 64),
    ("tiny", 1, [5, 0, 70], [2, 1], [0, 33], 64),
    ("tiny", 1, [700] * 9, [4, 0, 5], [650, 12, 640], 128),
    ("thinker_mixed", 1, [900, 513, 1000, 512], [4], [512], 256),
    ("tiny", 1, [300 + i for i in range(140)], [140], [256], 64),    # beyond the skinny products' rows
]


@pytest.mark.parametrize("name,n_layers,kv_lens,groups,prefix,page", CASES)
def test_step_behind_prefixes(env, name, n_layers, kv_lens, groups, prefix, page):
    torch, b, ctx = env
    from paper_2608_01785_amd.device_data import to_device, upload_weights
    shape = {"tiny": W.TINY, "thinker_mixed": W.THINKER_MIXED}[name]
    log(f"[prefix step] {name} x {n_layers}, cached {kv_lens[:6]}, groups {groups}, prefixes {prefix}, page {page}")
    cache, table, layers, batch, logical, offsets = _step(env, shape, n_layers, kv_lens, groups, prefix, page, 70)
    w = upload_weights(layers)
    x = to_device(batch.x)
    n = len(kv_lens)
    y = torch.empty((n, shape.hidden), dtype=torch.float32, device="cuda")
    rest = max(kv_lens[i] + 1 - prefix[g] for g in range(len(groups)) for i in range(offsets[g], offsets[g + 1]))
    ws = torch.full((b.hs_workspace_size_prefix(shape, n, max(kv_lens) + 1, page, max(prefix), rest),), 255,
                    dtype=torch.uint8, device="cuda")
    torch.cuda.synchronize()
    b.hs_downstream_decode_step_prefix(ctx, shape, w, x, y, cache.as_arg(), kv_lens, offsets, prefix, 128,
                                       workspace=ws)
    torch.cuda.synchronize()
    got = y.cpu().numpy().astype(np.float64)
    h = f64(batch.x)
    expect = np.zeros_like(h)
    rows64 = weights_f64(layers)
    for i in range(n):
        r = h[i:i + 1]
        for layer in range(n_layers):
            r, k_new, v_new = ref.layer_forward(r, rows64[layer], shape, [0, 1], [kv_lens[i]],
                                                [h64(logical.k[layer][i])], [h64(logical.v[layer][i])])
        expect[i] = r[0]
        # (The oracle's new rows are its own; the library's are compared below.)
    err = err_ratio(got, expect)
    log(f"  max err / rms = {err:.2e}")
    assert err <= TOL
    # The plain step on the same cache: the first layer's new keys and values are the same bits, the output the same
    # to the attention's roundings.
    kept = [t.clone() for t in cache.k + cache.v]
    z = torch.empty_like(y)
    ws2 = torch.empty(b.hs_workspace_size_paged(shape, n, n, max(kv_lens) + 1, page), dtype=torch.uint8, device="cuda")
    torch.cuda.synchronize()
    b.hs_downstream_decode_step(ctx, shape, w, x, z, cache.as_arg(), kv_lens, 128, workspace=ws2)
    torch.cuda.synchronize()
    assert torch.equal(kept[0], cache.k[0]) and torch.equal(kept[n_layers], cache.v[0])
    assert err_ratio(got, z.cpu().numpy()) <= TOL


def test_step_refusals(env):
    torch, b, ctx = env
    from paper_2608_01785_amd.device_data import to_device, upload_weights
    shape = W.TINY
    kv_lens, page = [100, 130, 64], 64
    cache, table, layers, batch, _, offsets = _step(env, shape, 1, kv_lens, [2, 1], [64, 0], page, 80)
    w, x = upload_weights(layers), to_device(batch.x)
    y = torch.full((3, shape.hidden), 5.0, device="cuda")
    size = b.hs_workspace_size_prefix(shape, 3, 131, page, 64, 131)
    ws = torch.empty(size, dtype=torch.uint8, device="cuda")
    torch.cuda.synchronize()

    def call(offsets=offsets, prefix=(64, 0), kv=cache.as_arg(), lens=kv_lens, **kw):
        b.hs_downstream_decode_step_prefix(ctx, shape, w, x, y, kv, lens, offsets, list(prefix), 128,
                                           **{"workspace": ws, **kw})
    for kw, text in ((dict(offsets=[1, 2, 3]), "run from"), (dict(offsets=[0, 2, 2]), "run from"),
                     (dict(offsets=[0, 5, 3]), "decrease"), (dict(prefix=(-1, 0)), "prefix_lens"),
                     (dict(prefix=(101, 0)), "cached rows"), (dict(prefix=(64, 65)), "cached rows"),
                     (dict(offsets=[0, 3], prefix=(64,)), "do not share"), (dict(kv=cache.as_arg()[:4]), "block table"),
                     (dict(offsets=[0], prefix=()), "groups"), (dict(ws_bytes=size // 2), "needed")):
        with pytest.raises(b.HorizonError, match=text):
            call(**kw)
    with pytest.raises(ValueError, match="prefixes"):
        call(offsets=[0, 3])
    with pytest.raises(ValueError, match="batch"):
        call(kv=(*cache.as_arg()[:4], table[:2]))
    for bad in ((0, 10, 64, 0, 1), (3, 0, 64, 0, 1), (3, 10, 65, 0, 1), (3, 10, 64, -1, 1), (3, 10, 64, 0, -1),
                (3, 10, 64, 2 ** 30, 1)):
        with pytest.raises(b.HorizonError):
            b.hs_workspace_size_prefix(shape, *bad)
    torch.cuda.synchronize()
    assert torch.all(y == 5.0)
    call()
    torch.cuda.synchronize()
    assert torch.all(torch.isfinite(y)) and not torch.any(y == 5.0)


# ---------------------------------------------------------------------------- beam search

class Search:
    def __init__(self, env, beams, groups, vocab, prompt, max_new, end=-1, seed=90, budgets=256, page=64, n_layers=2):
        self.torch, self.b, self.ctx = env
        torch = self.torch
        from paper_2608_01785_amd.answer import AnswerHead
        from paper_2608_01785_amd.beams import BeamSearch
        from paper_2608_01785_amd.device_data import prepare_f16, upload_weights
        self.shape = W.TINY
        self.w = prepare_f16(self.ctx, upload_weights(W.make_weights(self.shape, n_layers, seed)))
        gen = torch.Generator(device="cuda").manual_seed(seed)
        d = self.shape.hidden
        self.table = torch.randn((vocab, d), generator=gen, device="cuda").to(torch.bfloat16)
        gain = torch.ones(d, device="cuda", dtype=torch.bfloat16)
        weight = (0.12 * torch.randn((vocab, d), generator=gen, device="cuda")).to(torch.bfloat16)
        self.head = AnswerHead(self.ctx, gain, weight, max_rows=max(beams * groups, groups * (prompt + max_new)))
        self.end, self.budget = end, budgets
        rows = self.table
        self.search = BeamSearch(self.ctx, self.shape, self.w, self.head.sharing(),
                                 lambda tokens, out: torch.index_select(rows, 0, tokens, out=out), beams, groups, prompt,
                                 max_new, end, page, cu_budget=budgets)
        self.gen = gen

    def prompts(self, lengths):
        tokens = [self.torch.randint(0, len(self.table), (n,), generator=self.gen, device="cuda") for n in lengths]
        x = self.torch.cat([self.table[t] for t in tokens]).contiguous()
        self.torch.cuda.synchronize()
        return x, [0] + np.cumsum(lengths).tolist()

    def rescore(self, x, tokens):
        """Sum of log probabilities of `tokens` behind the prompt rows x, by a plain prefill; and the prefill's cache."""
        torch, b = self.torch, self.b
        from paper_2608_01785_amd.device_data import DeviceCache
        n, m = x.shape[0], len(tokens)
        rows = torch.cat([x, self.table[torch.tensor(tokens[:-1], dtype=torch.long, device="cuda")]]).contiguous()
        T = n + m - 1
        cache = DeviceCache(len(self.w), 1, -(-T // 64) * 64, self.shape.n_kv_heads, self.shape.head_dim)
        y = torch.empty((T, self.shape.hidden), device="cuda")
        ws = torch.empty(b.hs_workspace_size(self.shape, T, 1, T), dtype=torch.uint8, device="cuda")
        torch.cuda.synchronize()
        b.hs_shared_stage_forward(self.ctx, self.shape, self.w, rows, y, [0, T], [0], cache.as_arg(), 256, None, ws)
        out = self.head.outputs(m, 1)
        last = y[n - 1:]
        torch.cuda.synchronize()
        given = torch.tensor(tokens, dtype=torch.int32, device="cuda")[:, None]
        torch.cuda.synchronize()
        self.head(last, out, given)
        torch.cuda.synchronize()
        return float(out.token_logprobs.double().sum()), cache, T

    def check(self, x, offsets, cached=True):
        torch = self.torch
        results = self.search.results()
        n = self.search.beams
        for g, beams in enumerate(results):
            scores = [b.score for b in beams]
            assert scores == sorted(scores, reverse=True)
            live = [tuple(b.tokens) for b in beams if b.score > -math.inf]
            assert len(set(live)) == len(live)
            for j, beam in enumerate(beams):
                if beam.score == -math.inf:
                    assert beam.tokens == []
                    continue
                assert beam.finished == (self.end >= 0 and beam.tokens[-1] == self.end)
                score, cache, T = self.rescore(x[offsets[g]:offsets[g + 1]], beam.tokens)
                # The two paths' rows differ by roundings to fp16, which moves an 8-bit element by a step at most:
                # max |y| / 127, some 3 of y's deviations in 127.  If all 256 moved, with random signs, against
                # weights of 0.12, a logit would by 0.12 * 16 * 3 / 127 = 0.045.
                assert abs(score - beam.score) <= 0.05 * len(beam.tokens), (g, j, score, beam.score)
                if not cached or beam.finished:
                    continue
                table, lens = self.search.pages.table([g * n + j])
                assert int(lens[0]) == T
                at = torch.arange(T)
                slots = torch.as_tensor(table[0], dtype=torch.long)[at // 64]
                for layer in range(len(self.w)):
                    k = self.search.cache.k[layer][slots.cuda(), :, (at % 64).cuda()].float()
                    v = self.search.cache.v[layer][slots.cuda(), :, (at % 64 // 32).cuda(), :, (at % 32).cuda()].float()
                    k1 = cache.k[layer][0, :, :T].permute(1, 0, 2).float()
                    v1 = cache.v[layer][0].transpose(2, 3).reshape(k1.shape[1], -1, k1.shape[2])[:, :T]
                    assert err_ratio(k.cpu(), k1.cpu()) <= TOL
                    assert err_ratio(v.cpu(), v1.permute(1, 0, 2).float().cpu()) <= TOL
        return results


@pytest.mark.parametrize("beams,lengths,vocab,max_new,budget", [
    (4, [70, 5, 130], 500, 9, 256), (1, [64], 300, 4, 256), (8, [61, 63], 1001, 8, 128), (3, [40], 2, 5, 256)])
def test_beam_search(env, beams, lengths, vocab, max_new, budget):
    torch, b, ctx = env
    log(f"[beam search] {beams} beams, prompts {lengths}, vocabulary {vocab}, {max_new} tokens, {budget} CUs")
    s = Search(env, beams, len(lengths), vocab, max(lengths), max_new, budgets=budget)
    x, offsets = s.prompts(lengths)
    s.search.start(x, offsets)
    s.check(x, offsets, cached=False)
    steps = 1
    while s.search.step():
        steps += 1
    assert steps == max_new
    results = s.check(x, offsets)
    assert all(len(beam.tokens) == max_new for g in results for beam in g if beam.score > -math.inf)
    # Another search on the same object, a prompt less.
    if len(lengths) > 1:
        x, offsets = s.prompts(lengths[1:])
        s.search.start(x, offsets)
        s.search.step()
        s.check(x, offsets)
    assert s.search.pages.free_count() >= 0


def test_every_continuation_of_two_tokens(env):
    """With as many beams as tokens nothing is cut: the best pairs are those of all of them."""
    torch, b, ctx = env
    vocab = 12
    s = Search(env, vocab, 1, vocab, 30, 2, seed=91)
    x, offsets = s.prompts([30])
    s.search.start(x, offsets)
    s.search.step()
    got = s.check(x, offsets)[0]
    scored = sorted(((s.rescore(x, [i, j])[0], (i, j)) for i in range(vocab) for j in range(vocab)), reverse=True)
    for beam, (score, _) in zip(got, scored):
        assert abs(beam.score - score) <= 0.1
    sure = [p for v, p in scored[:vocab] if v > scored[vocab][0] + 0.2]   # no near tie with what is left out
    assert set(sure) <= {tuple(beam.tokens) for beam in got}


def test_beams_that_end(env):
    """An end token that many beams reach; ended ones keep their score and compete on."""
    torch, b, ctx = env
    s = Search(env, 5, 2, 40, 50, 12, seed=92)
    x, offsets = s.prompts([50, 33])
    s.search.start(x, offsets)
    while s.search.step():
        pass
    # The token that the plain search uses most becomes the end.
    used = [t for g in s.search.results() for beam in g for t in beam.tokens]
    end = max(set(used), key=used.count)
    t = Search(env, 5, 2, 40, 50, 12, end=end, seed=92)
    t.search.start(x, offsets)
    while t.search.step():
        pass
    results = t.check(x, offsets)
    assert any(beam.finished for g in results for beam in g)
    assert all(beam.tokens.count(end) <= 1 for g in results for beam in g)


def test_prompts_still_being_written(env):
    """Rows that torch's stream has yet to write when the search starts."""
    torch, b, ctx = env
    s = Search(env, 3, 1, 100, 60, 3, seed=93)
    x, offsets = s.prompts([60])
    s.search.start(x, offsets)
    first = s.search.results()
    late = torch.zeros_like(x)
    big = torch.randn((4096, 4096), device="cuda")
    torch.cuda.synchronize()
    for _ in range(20):
        big = torch.matmul(big, big).clamp(-1, 1)
    late.copy_(x + big[:1, :1].mul(0).to(x.dtype))
    s.search.start(late, offsets)
    again = s.search.results()
    assert [(q.tokens, q.score) for q in first[0]] == [(q.tokens, q.score) for q in again[0]]


def test_search_refusals(env):
    torch, b, ctx = env
    s = Search(env, 2, 2, 50, 20, 3)
    with pytest.raises(ValueError, match="started"):
        s.search.step()
    x, offsets = s.prompts([20, 5])
    for bad in ([0, 20, 20, 25], [0, 25], [0, 0, 20]):
        with pytest.raises(ValueError, match="prompts"):
            s.search.start(x, bad)
    with pytest.raises(ValueError, match="shape"):
        s.search.start(x[:20], offsets)
    from paper_2608_01785_amd.beams import BeamSearch
    for kw, text in ((dict(beams=0), "beams"), (dict(beams=65), "beams"), (dict(max_groups=0), "groups"),
                     (dict(max_groups=1000), "head")):
        a = dict(beams=2, max_groups=2, max_prompt=20, max_new=3)
        a.update(kw)
        with pytest.raises(ValueError, match=text):
            BeamSearch(ctx, s.shape, s.w, s.head, None, **a)


def test_search_after_a_failure(env):
    """A step that failed after it had reserved its positions is not gone on from; a new start works as before."""
    torch, b, ctx = env
    s = Search(env, 3, 2, 60, 40, 4, seed=94)
    x, offsets = s.prompts([40, 17])
    s.search.start(x, offsets)
    s.search.step()
    before = s.search.results()
    embed = s.search.embed

    def failing(tokens, out):
        raise RuntimeError("no rows")
    s.search.embed = failing
    with pytest.raises(RuntimeError, match="no rows"):
        s.search.step()
    s.search.embed = embed
    with pytest.raises(ValueError, match="failed"):
        s.search.step()
    assert s.search.results() == before
    s.search.start(x, offsets)
    s.search.step()
    assert s.search.results() == before
    s.check(x, offsets)

    # A start that fails leaves no search.
    product = s.search.head.product
    s.search.head.product = lambda *a: failing(None, None)
    with pytest.raises(RuntimeError, match="no rows"):
        s.search.start(x, offsets)
    s.search.head.product = product
    assert s.search.results() == []
    with pytest.raises(ValueError, match="started"):
        s.search.step()


def test_search_without_pages(env):
    """A step for which the cache has too few pages changes nothing."""
    torch, b, ctx = env
    from paper_2608_01785_amd.beams import BeamSearch
    s = Search(env, 2, 1, 60, 64, 4, seed=95)
    search = BeamSearch(ctx, s.shape, s.w, s.head.sharing(), s.search.embed, 2, 1, 64, 4, n_pages=2)
    x, offsets = s.prompts([64])
    search.start(x, offsets)      # the prompt's page; each beam's next token needs one of its own
    before = search.results()
    for _ in range(2):
        with pytest.raises(b.HorizonError, match="pages"):
            search.step()
    assert search.results() == before and search.pages.free_count() == 1
