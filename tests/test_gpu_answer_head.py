"""The text head over residual rows, in passes and inside the serving loop; every product kernel by its rule; long
strides; narrow and long rows.

Bounds (u = 2^-24): a row's scale is within 78 u, so a logit z, the product of an exact sum with two scales, is
within 160 u |z| of the float64 chain with the weights' scales as stored, and a log probability within twice the
largest of those, plus its own fp32 steps: (4 + 3 |d|) u for each e^d, at most 40 + vocab / 2048 additions, as
derived beside the operators' own tests; with |z| <= 64 and |d| <= 128 that is below (2 * 160 * 64 + 4 + 3 * 128 +
72 + vocab / 2048) u < 22000 u = 1.4e-3.  Entropy has the same terms weighted by p |d| <= 128 / e in all: 6e-3.
Alternatives may swap only where logits lie that close.
"""
import numpy as np
import pytest

from oracle import answer as A
from tests.gpu_common import log, require_gpu
from tests.test_gpu_answer import _check_linear, _check_quantize, _gen, _linear, _logprobs, _np, _quantize, _t, _view
from tests.test_gpu_answer import test_quantize_values as _quantize_values
from tests.test_gpu_algorithm1 import LADDER, _loop

pytestmark = pytest.mark.gpu

EPS = 1e-6
TOP = 5


@pytest.fixture(scope="module")
def env():
    torch = require_gpu()
    from paper_2608_01785_amd import binding
    ctx = binding.Context(0, budgets=(64,) + LADDER + (256,))
    yield torch, binding, ctx
    torch.cuda.synchronize()
    ctx.close()


def _new_head(env, d=256, vocab=2500, **kw):
    torch, b, ctx = env
    from paper_2608_01785_amd.answer import AnswerHead
    g = _gen(torch, d + vocab)
    gain = (1 + 0.1 * torch.randn(d, generator=g, device="cuda")).bfloat16()
    weight = (torch.randn(vocab, d, generator=g, device="cuda") * (2 / d ** 0.5)).bfloat16()
    return AnswerHead(ctx, gain, weight, **{"top_k": TOP, **kw})


def _check(head, y, out, tokens=None):
    """out: arrays of the answers to the rows y (float64)."""
    w, ws = head.w.cpu().numpy(), head.w_scale.cpu().numpy()
    q, qs = A.quantize_rows(y, _np(head.gain), EPS)
    z = (q.astype(np.float64) @ w.T.astype(np.float64)) * (qs[:, None] * ws)
    if head.bias is not None:
        z = z + _np(head.bias)
    half = {"torch.float32": 0.0, "torch.bfloat16": 2.0 ** -8, "torch.float16": 2.0 ** -11}[str(head.logits.dtype)]
    bad = np.isnan(z).any(1)
    ok = ~bad
    assert np.abs(z[ok]).max() <= 64
    tol, tol_h = 1.4e-3 + 2 * half * 64, 6e-3 + 2 * half * 64 * 128
    ref = A.logprobs(z, tokens, head.top_k)
    if tokens is not None:
        assert np.abs(out["token_logprobs"][ok] - ref["token"][ok]).max() <= tol
        assert np.isnan(out["token_logprobs"][bad]).all()
    assert np.abs(out["entropy"][ok] - ref["entropy"][ok]).max() <= tol_h
    assert np.isnan(out["entropy"][bad]).all()
    if head.top_k:
        logp = z - np.log(np.exp(z - z.max(1, keepdims=True)).sum(1, keepdims=True)) - z.max(1, keepdims=True)
        at = out["top_tokens"]
        assert (at[bad] == -1).all() and np.isnan(out["top_logprobs"][bad]).all()
        for r in np.flatnonzero(ok):
            assert len(set(at[r].tolist())) == head.top_k
            # Each listed token is within the bound of the probability that its place has.
            assert np.abs(logp[r, at[r]] - ref["top"][r]).max() <= 2 * tol
            assert np.abs(out["top_logprobs"][r] - ref["top"][r]).max() <= tol


def _host(out):
    return {k: (t.cpu().numpy() if t is not None else None) for k, t in vars(out).items()}


@pytest.mark.parametrize("rows,max_rows", [(1, 128), (7, 7), (11, 4), (300, 128)])
@pytest.mark.parametrize("logits", ["f32", "bf16"])
def test_head_in_passes(env, rows, max_rows, logits):
    torch, b, ctx = env
    head = _new_head(env, max_rows=max_rows, logits=_t(torch, logits))
    g = _gen(torch, rows)
    y = torch.randn(rows, head.hidden, generator=g, device="cuda") * 30
    if rows > 3:
        y[2] = 0.0                      # no activation at all: every token is as likely
        y[3, 5] = float("nan")
    tokens = torch.randint(0, head.vocab, (rows, 2), generator=g, device="cuda", dtype=torch.int32)
    out = head.outputs(rows, 2)
    for cus in (256, 128):
        for t in vars(out).values():
            t.fill_(-7)
        torch.cuda.synchronize()
        head(y, out, tokens, cu_budget=cus)
        torch.cuda.synchronize()
        _check(head, _np(y), _host(out), tokens.cpu().numpy())
    if rows > 3:
        assert abs(float(out.entropy[2]) - np.log(head.vocab)) < 1e-5 and out.top_tokens[2].tolist() == [0, 1, 2, 3, 4]


def test_head_without_alternatives_and_of_no_rows(env):
    torch, b, ctx = env
    head = _new_head(env, top_k=0)
    out = head.outputs(0)
    head(torch.empty(0, head.hidden, device="cuda"), out)
    y = torch.randn(9, 2 * head.hidden, device="cuda")[:, ::2].contiguous()
    wide = torch.zeros(9, head.hidden + 8, device="cuda")
    wide[:, :head.hidden] = y
    out = head.outputs(9)
    assert out.top_tokens is None and out.token_logprobs is None
    torch.cuda.synchronize()
    head(wide[:, :head.hidden], out)
    torch.cuda.synchronize()
    _check(head, _np(y), _host(out))


def test_two_heads_with_the_same_weights_at_once(env):
    torch, b, ctx = env
    one = _new_head(env, max_rows=16, vocab=9000)
    two = one.sharing(max_rows=8)
    assert two.w.data_ptr() == one.w.data_ptr() and two.logits.data_ptr() != one.logits.data_ptr()
    y1, y2 = (torch.randn(n, one.hidden, generator=_gen(torch, n), device="cuda") for n in (40, 30))
    o1, o2 = one.outputs(40), two.outputs(30)
    down = b.hs_context_stream(ctx, 128, b.HS_ROLE_DOWN)
    torch.cuda.synchronize()
    for _ in range(4):
        one(y1, o1, cu_budget=128)
        two(y2, o2, cu_budget=128, stream=down)
    torch.cuda.synchronize()
    _check(one, _np(y1), _host(o1))
    _check(two, _np(y2), _host(o2))


def test_a_captured_head_with_split_rows(env):
    """Rows long enough to be split over blocks and joined, replayed with new rows between eager passes."""
    torch, b, ctx = env
    head = _new_head(env, vocab=70001, max_rows=4)
    y, out = torch.randn(7, head.hidden, generator=_gen(torch, 1), device="cuda"), head.outputs(7, 1)
    tokens = torch.randint(0, head.vocab, (7, 1), generator=_gen(torch, 2), device="cuda", dtype=torch.int32)
    stream = torch.cuda.Stream()
    torch.cuda.synchronize()
    head(y, out, tokens, stream=stream.cuda_stream)
    stream.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=stream):
        head(y, out, tokens, stream=stream.cuda_stream)
    for i in range(4):
        y.copy_(torch.randn(y.shape, generator=_gen(torch, 10 + i), device="cuda"))
        for t in vars(out).values():
            t.fill_(-7)
        head.ws.fill_(255)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        _check(head, _np(y), _host(out), tokens.cpu().numpy())
        kept = {k: t.clone() for k, t in vars(out).items()}
        torch.cuda.synchronize()
        head(y, out, tokens)
        torch.cuda.synchronize()
        assert all(torch.equal(t, kept[k]) for k, t in vars(out).items())


def test_two_threads_on_one_context(env):
    """Calls from two host threads at once, each with its own head and stream; a refusal in one is not the other's."""
    import threading
    torch, b, ctx = env
    one = _new_head(env, max_rows=8, vocab=30000)
    two = one.sharing(max_rows=5)
    jobs = []
    for head, rows, role in ((one, 11, b.HS_ROLE_SHARED), (two, 9, b.HS_ROLE_DOWN)):
        y = torch.randn(rows, head.hidden, generator=_gen(torch, rows), device="cuda")
        jobs.append((head, y, head.outputs(rows), b.hs_context_stream(ctx, 128, role)))
    torch.cuda.synchronize()
    errors = []

    def run(i):
        try:
            head, y, out, stream = jobs[i]
            for n in range(40):
                head(y, out, cu_budget=128, stream=stream)
                if i and n % 8 == 0:
                    with pytest.raises(b.HorizonError, match="carries 128"):
                        head(y, out, cu_budget=64, stream=stream)
        except BaseException as e:   # noqa: B902 -- shown by the main thread
            errors.append(e)

    threads = [threading.Thread(target=run, args=(i,)) for i in (0, 1)]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    torch.cuda.synchronize()
    assert not errors, errors
    for head, y, out, _ in jobs:
        _check(head, _np(y), _host(out))


def test_head_refusals(env):
    torch, b, ctx = env
    head = _new_head(env)
    y, out = torch.randn(4, head.hidden, device="cuda"), head.outputs(4)
    with pytest.raises(ValueError, match="expected"):
        head(y[:, :-1], out)
    with pytest.raises(ValueError, match="4 rows, y 3"):
        head(y[:3], out)
    with pytest.raises(ValueError, match="tokens has 3 rows"):
        head(y, out, torch.zeros(3, 1, dtype=torch.int32, device="cuda"))
    with pytest.raises(ValueError, match="max_rows"):
        _new_head(env, max_rows=0)
    with pytest.raises(ValueError, match="alternatives"):
        _loop_with(env, "baseline", _new_head(env, top_k=0))


def _loop_with(env, policy, head, **kw):
    """The scheduling loop of the policies' own tests, with a head."""
    torch, b, ctx = env
    from paper_2608_01785_amd import serving
    made = serving.Algorithm1

    def with_head(*args, **kws):
        return made(*args, **kws, head=head)

    serving.Algorithm1 = with_head
    try:
        return _loop((torch, ctx), policy, **kw)
    finally:
        serving.Algorithm1 = made


@pytest.mark.parametrize("policy", ["joint", "baseline"])
def test_the_serving_loop_answers_every_request(env, policy):
    """Each batch's answers belong to the last prompt rows that its prefill left in the residual stream."""
    torch, b, ctx = env
    head = _new_head(env, max_rows=3)
    loop, reqs, _, _ = _loop_with(env, policy, head, n_req=9, seed=6)
    loop.begin()
    try:
        for _ in range(200):
            rec = loop.step()
            if rec is None:
                break
            if rec.batch:
                y = _np(loop.y[torch.tensor(rec.offsets[1:], device="cuda") - 1])
                got = [loop.answers[reqs[i].rid] for i in rec.batch]
                log(f"[answers] step {rec.k} on {rec.split['shared_cus']} CUs: {[a.tokens[0] for a in got]}")
                _check(head, y, {"entropy": np.array([a.entropy for a in got]),
                                 "top_tokens": np.array([a.tokens for a in got]),
                                 "top_logprobs": np.array([a.logprobs for a in got])})
        s = loop.summary()
    finally:
        loop.close()
    assert s["unfinished"] == 0 and sorted(loop.answers) == sorted(r.rid for r in reqs)


# ---------------------------------------------------------------------------- every product kernel

FEW32, FEW64, FEW6464, T64, T128, T256 = range(6)
# Kernel, m, n, k, CUs, and whether rows are 16-byte aligned.
KERNELS = [(FEW32, 1, 2060, 1024, 256, True), (FEW32, 32, 4100, 4112, 64, True), (FEW32, 31, 1030, 2049, 256, False),
           (FEW32, 20, 2060, 1040, 256, False), (FEW32, 300, 515, 1040, 256, True), (FEW32, 65, 515, 2049, 256, False),
           (FEW64, 33, 1030, 4112, 64, True), (FEW64, 300, 1030, 4112, 256, True), (FEW64, 100, 515, 4111, 64, False),
           (FEW64, 128, 2060, 4111, 256, False), (FEW6464, 100, 1030, 4112, 64, True),
           (FEW6464, 300, 2060, 4112, 256, True), (FEW6464, 500, 1030, 4112, 256, True),
           (T64, 300, 4100, 1024, 256, True), (T64, 200, 2060, 256, 64, True), (T64, 777, 1030, 2049, 256, False),
           (T64, 300, 4100, 1024, 256, False),
           (T128, 777, 4100, 1024, 256, True), (T128, 390, 4100, 2064, 64, True), (T128, 200, 4100, 1033, 64, False),
           (T128, 600, 4100, 2049, 64, False), (T128, 1100, 2060, 2064, 64, False),
           (T256, 600, 4100, 2064, 64, True), (T256, 1100, 2060, 2064, 64, True), (T256, 1500, 2060, 1040, 64, True)]


@pytest.mark.parametrize("case", KERNELS, ids=str)
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_every_product_kernel(env, case, dtype):
    torch, b, ctx = env
    kind, m, n, k, cus, aligned = case
    assert b.lib().hs_linear_i8_kernel(m, n, k, cus, aligned) == kind
    g = _gen(torch, m + n + k)
    a = torch.randint(-128, 128, (m, k), generator=g, device="cuda", dtype=torch.int8)
    w = torch.randint(-128, 128, (n, k), generator=g, device="cuda", dtype=torch.int8)
    sa = torch.rand(m, generator=g, device="cuda") + 0.01
    sw = torch.rand(n, generator=g, device="cuda") * 1e-3
    bias = torch.randn(n, generator=g, device="cuda").bfloat16()
    # What lies beside the operands must not count: no zeros there.
    _, a = _view(torch, a, 16 if aligned else 3, 0 if aligned else 7, fill=111)
    _, w = _view(torch, w, 32 if aligned else 5, 0 if aligned else 1, fill=-111)
    _check_linear(env, a, sa, w, sw, dtype, bias, pad=0 if aligned else 3, shift=0 if aligned else 1, cus=cus)


@pytest.mark.parametrize("k", [1, 15, 16, 17, 31, 100, 127, 128, 129, 255, 256, 257, 383, 384, 385, 511, 512, 513,
                               639, 641, 1000, 1025])
@pytest.mark.parametrize("m", [3, 70])
def test_product_lengths(env, k, m):
    """Sums that end inside a stage, and shorter than the stages that a block loads ahead."""
    torch = env[0]
    g = _gen(torch, k)
    a = torch.randint(-128, 128, (m, k), generator=g, device="cuda", dtype=torch.int8)
    w = torch.randint(-128, 128, (301, k), generator=g, device="cuda", dtype=torch.int8)
    sa, sw = torch.rand(m, generator=g, device="cuda"), torch.rand(301, generator=g, device="cuda")
    for pad, shift in ((-k % 16, 0), (-k % 16 + 1, 3)):
        _, av = _view(torch, a, pad, shift, fill=99)
        _, wv = _view(torch, w, pad, shift, fill=-99)
        _check_linear(env, av, sa, wv, sw, "f32")


# ---------------------------------------------------------------------------- long rows, many of them

@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("norm", [False, True])
@pytest.mark.parametrize("d", [8, 63, 64, 65, 100, 128, 129, 250, 256, 257, 32776, 40003])
def test_quantisation_of_narrow_and_long_rows(env, dtype, norm, d):
    """Several rows of a wavefront, and rows beyond a block's registers: ties, extremes, subnormals, zeros and rows that
    are not finite beside ordinary ones; odd strides."""
    torch, b, ctx = env
    _quantize_values((torch, b, ctx), dtype, norm, d)
    g = _gen(torch, d)
    x = torch.randn(5 if d > 1000 else 5003, d, generator=g, device="cuda").to(_t(torch, dtype))
    gain = (1 + 0.2 * torch.randn(d, generator=g, device="cuda")).bfloat16() if norm else None
    _check_quantize((torch, b, ctx), _view(torch, x, 3, 1, fill=7)[1], gain, pad=1, shift=5)



@pytest.mark.parametrize("rows,vocab,cus", [(64, 160001, 64), (512, 40000, 64), (3, 700001, 64)])
@pytest.mark.parametrize("top", [1, 20, 64])
def test_alternatives_of_more_chunks_than_a_block_keeps_apart(env, rows, vocab, cus, top):
    """Rows whole in a block of four wavefronts, in one, and split: maxima of several chunks in one place."""
    torch, b, ctx = env
    g = _gen(torch, vocab + top)
    z = torch.randn(rows, vocab, generator=g, device="cuda") * 3
    z[1] = 1.25                                              # every logit the same
    z[2] = torch.randint(0, 3, (vocab,), generator=g, device="cuda").float()   # a third of them the largest
    if rows > 3:
        z[3] = -float("inf")
        z[3, vocab - 40:] = 2.0                              # fewer than 64 unmasked, all at the end
        z[4, ::7] = 25.0                                     # ties above all others, spread out
    got = _logprobs((torch, b, ctx), z, None, top, cus=cus)
    rows_checked = list(range(min(rows, 8))) + ([rows - 1] if rows > 8 else [])
    ref = A.logprobs(_np(z[rows_checked]), None, top)
    np.testing.assert_array_equal(got["top_tokens"][rows_checked].cpu().numpy(), ref["top_tokens"])
    # Every row against a sort by value and then token.
    lo = torch.sort(z, dim=1, descending=True, stable=True)
    want = torch.where(lo.values[:, :top].isinf(), -1, lo.indices[:, :top]).int()
    assert torch.equal(got["top_tokens"], want)


# ---------------------------------------------------------------------------- offsets beyond 32 bits

def test_rows_further_apart_than_32_bits_reach(env):
    """Strides that put the last rows beyond 2^32 bytes give what the same rows side by side give."""
    torch, b, ctx = env
    g = _gen(torch, 31)
    far = torch.empty(2 ** 32 + 2 ** 28, dtype=torch.uint8, device="cuda")

    def spread(t, stride):
        v = far.view(t.dtype)[:t.shape[0] * stride].view(t.shape[0], stride)[:, :t.shape[1]]
        v.copy_(t)
        return v

    # Quantisation: 70 fp32 rows of 2^24 elements.
    x = torch.randn(67, 1000, generator=g, device="cuda")
    q, s = _quantize((torch, b, ctx), x, None)
    q2, s2 = _quantize((torch, b, ctx), spread(x, 2 ** 24), None)
    assert torch.equal(q, q2) and torch.equal(s, s2)
    # Products: 1027 rows of the largest stride.
    w = torch.randint(-128, 128, (1027, 500), generator=g, device="cuda", dtype=torch.int8)
    sw = torch.rand(1027, generator=g, device="cuda")
    for m in (5, 200):
        a = torch.randint(-128, 128, (m, 500), generator=g, device="cuda", dtype=torch.int8)
        sa = torch.rand(m, generator=g, device="cuda")
        near = _linear(env, a, sa, w, sw, "f32")
        assert torch.equal(_linear(env, a, sa, spread(w, 2 ** 22), sw, "f32"), near)
        assert torch.equal(_linear(env, w, sw, a, sa, "f32"), _linear(env, spread(w, 2 ** 22), sw, a, sa, "f32"))
        ldo = (2 ** 30 + 2 ** 26) // m
        out = far.view(torch.float32)[:m * ldo].view(m, ldo)[:, :1027]
        b.hs_linear_i8(ctx, a, sa, w, sw, out)
        torch.cuda.synchronize()
        assert torch.equal(out, near)
    # Log probabilities: 67 bf16 rows of 2^25 elements.
    z = torch.randn(67, 5000, generator=g, device="cuda").bfloat16()
    ws = torch.empty(b.hs_logprobs_workspace_size(67, 5000, 4), dtype=torch.uint8, device="cuda")
    got = []
    for v in (z, spread(z, 2 ** 25)):
        ent, lp = torch.empty(67, device="cuda"), torch.empty(67, 4, device="cuda")
        at = torch.empty(67, 4, dtype=torch.int32, device="cuda")
        torch.cuda.synchronize()
        b.hs_logprobs(ctx, v, entropy=ent, top_logprobs=lp, top_tokens=at, workspace=ws)
        torch.cuda.synchronize()
        got.append((ent, lp, at))
    assert all(torch.equal(p, r) for p, r in zip(*got))
