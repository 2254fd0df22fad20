"""The answering operators where values, counts and layouts leave the ordinary range, against the float64 reference.

Bounds are those derived beside the operators' own tests.
"""
import numpy as np
import pytest

from oracle import answer as A
from tests.gpu_common import require_gpu
from tests.test_gpu_algorithm1 import LADDER
from tests.test_gpu_answer import EPS, U, _check_logprobs, _close, _gen, _linear, _np, _quantize, _t
from tests.test_gpu_answer_head import KERNELS, _check, _loop_with, _new_head

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def env():
    torch = require_gpu()
    from paper_2608_01785_amd import binding
    ctx = binding.Context(0, budgets=(64, 256))
    yield torch, binding, ctx
    torch.cuda.synchronize()
    ctx.close()


# Rows, vocab, CUs: rows whole in a block of four wavefronts, whole in one, and split, with several 4 KB chunks a
# wavefront in each.
LAYOUTS = {"four": (40, 20011, 64), "one": (520, 9001, 64), "split": (8, 131072, 64)}


def _check_layout(b, name, dtype):
    rows, vocab, cus = LAYOUTS[name]
    splits = b.lib().hs_logprobs_splits(rows, vocab, 4 if dtype == "f32" else 2, cus)
    assert (splits > 1) == (name == "split") and (rows >= 8 * cus) == (name == "one")
    return rows, vocab, cus


@pytest.mark.parametrize("layout", LAYOUTS)
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_large_maxima_before_lower_chunks(env, layout, dtype):
    """Finite logits of any size: a first chunk that holds the maximum, and chunks far below it or masked."""
    torch, b, ctx = env
    rows, vocab, cus = _check_layout(b, layout, dtype)
    tops = [s * v for v in (2.0 ** 20, 2.0 ** 20 + 2.0 ** 15, 1e7, 5e9, 1e10, 2e10, 1e12, 1e15, 1e30, 1.5e30)
            for s in (1, -1)]
    g = _gen(torch, rows)
    z = torch.randn(rows, vocab, generator=g, device="cuda") * 3
    for r in range(rows):
        # Rows in turn over the maxima; eight rows take eight of them, from the fifth on.
        m = tops[(r + (6 if rows < len(tops) else 0)) % len(tops)]
        if m < 0:
            z[r] = -float("inf") if r % 4 < 2 else 4 * m      # masked, or far below
        z[r, 5] = m
        z[r, 9::vocab // 3] = m                               # and ties in later chunks
        z[r, 11] = m - 2 * abs(m) * 2.0 ** -20                # a near value, where the type has one
    tokens = torch.randint(0, vocab, (rows, 4), generator=g, device="cuda", dtype=torch.int32)
    tokens[:, 0], tokens[:, 1] = 5, 11
    _check_logprobs(env, z.to(_t(torch, dtype)), tokens, 20, cus=cus)
    # The maximum alone.
    for r in range(rows):
        m = float(z[r, 5])
        z[r, 9::vocab // 3] = 2 * m if m < 0 else 0.0
    _check_logprobs(env, z.to(_t(torch, dtype)), tokens, 20, cus=cus)


@pytest.mark.parametrize("case", [c for c in KERNELS if c[5]], ids=str)
def test_aligned_operands_of_the_largest_stride(env, case):
    """Rows 4 MB apart, the last ones in a tile that they do not fill, against the same rows side by side."""
    torch, b, ctx = env
    kind, m, n, k, cus, _ = case
    assert b.lib().hs_linear_i8_kernel(m, n, k, cus, True) == kind
    g = _gen(torch, m + n + k)
    a = torch.randint(-128, 128, (m, k), generator=g, device="cuda", dtype=torch.int8)
    w = torch.randint(-128, 128, (n, k), generator=g, device="cuda", dtype=torch.int8)
    sa, sw = torch.rand(m, generator=g, device="cuda"), torch.rand(n, generator=g, device="cuda")
    near = _linear(env, a, sa, w, sw, "f32", cus=cus)

    def spread(t):
        v = torch.empty((t.shape[0] - 1) * 2 ** 22 + t.shape[1], dtype=torch.int8, device="cuda")
        v = v.as_strided(t.shape, (2 ** 22, 1))
        v.copy_(t)
        return v

    assert torch.equal(_linear(env, spread(a), sa, spread(w), sw, "f32", cus=cus), near)
    torch.cuda.empty_cache()


def test_workspaces_elsewhere_are_refused(env):
    torch, b, ctx = env
    z, e = torch.randn(2, 70000, device="cuda"), torch.empty(2, device="cuda")
    need = b.hs_logprobs_workspace_size(2, 70000, 0)
    ws = torch.empty(need, dtype=torch.uint8, device="cuda")
    for bad, text in ((ws.cpu(), "workspace is on cpu"), (ws[:1].expand(need), "not contiguous")):
        with pytest.raises(ValueError, match=text):
            b.hs_logprobs(ctx, z, entropy=e, workspace=bad)


def test_the_serving_loop_takes_a_head_of_another_context(env):
    """The head's work belongs on the batch's stream, whatever levels and streams the head's own context has."""
    torch, b, ctx = env
    loop_ctx = b.Context(0, budgets=LADDER + (256,))
    head = _new_head(env, max_rows=3)            # a context without the ladder
    loop, reqs, _, _ = _loop_with((torch, b, loop_ctx), "joint", head, n_req=6, seed=6)
    loop.begin()
    try:
        for _ in range(200):
            rec = loop.step()
            if rec is None:
                break
            if rec.batch:
                y = _np(loop.y[torch.tensor(rec.offsets[1:], device="cuda") - 1])
                got = [loop.answers[reqs[i].rid] for i in rec.batch]
                _check(head, y, {"entropy": np.array([a.entropy for a in got]),
                                 "top_tokens": np.array([a.tokens for a in got]),
                                 "top_logprobs": np.array([a.logprobs for a in got])})
    finally:
        loop.close()
    assert sorted(loop.answers) == sorted(r.rid for r in reqs)
    torch.cuda.synchronize()
    loop_ctx.close()


# ---------------------------------------------------------------------------- paths of the head and of long lists

def _check_answers(got, z, tokens, top):
    """Log probabilities of exactly these logits, within the bounds of the operators' own tests."""
    ref = A.logprobs(z, tokens, top)
    np.testing.assert_array_equal(got["top_tokens"].cpu().numpy(), ref["top_tokens"])
    n = 32 + -(-z.shape[1] // 2048) + 40
    s, t1, t2 = ref["s"], ref["t1"], ref["t2"]
    log_s = ((n + 4) * s / (1 + s) + 3 * t1 + 2 * np.log1p(s)) * U
    for name, key in (("token_logprobs", "token"), ("top_logprobs", "top")):
        size = np.where(np.isfinite(ref[key]), np.abs(ref[key]), 0)
        _close(name, got[name], ref[key], log_s[:, None] + 4 * U * size + z.shape[1] * 2.0 ** -126)
    _close("entropy", got["entropy"], ref["entropy"],
           ((n + 8) * (t1 + s / (1 + s)) + 3 * t2 + 4 * ref["entropy"]) * U + 128 * z.shape[1] * 2.0 ** -126)


@pytest.mark.parametrize("with_bias", [False, True])
@pytest.mark.parametrize("logits", ["f32", "bf16", "f16"])
def test_head_steps_one_after_another(env, logits, with_bias):
    """Each step of a pass against the reference of the step before it, so 16-bit logits hide nothing of what follows."""
    torch, b, ctx = env
    vocab, rows = 2501, 13
    g = _gen(torch, 77)
    bias = torch.randn(vocab, generator=g, device="cuda").bfloat16() if with_bias else None
    head = _new_head(env, vocab=vocab, max_rows=16, bias=bias, logits=_t(torch, logits))
    assert (head.bias is not None) == with_bias
    y = torch.randn(rows, head.hidden, generator=g, device="cuda") * 30
    y[2] = 0.0
    y[3, 5] = float("nan")
    tokens = torch.randint(-1, vocab, (rows, 3), generator=g, device="cuda", dtype=torch.int32)
    out = head.outputs(rows, 3)
    torch.cuda.synchronize()
    head(y, out, tokens)
    torch.cuda.synchronize()
    q, _ = A.quantize_rows(_np(y), _np(head.gain), 1e-6)
    np.testing.assert_array_equal(head.q[:rows].cpu().numpy(), q)
    z = A.linear_i8(q, head.q_scale[:rows].cpu().numpy(), head.w.cpu().numpy(), head.w_scale.cpu().numpy(),
                    None if bias is None else bias.float().cpu().numpy())
    z = torch.from_numpy(z).to(head.logits.dtype)
    same = (head.logits[:rows].cpu() == z) | (head.logits[:rows].cpu().isnan() & z.isnan())
    assert bool(same.all())
    _check_answers(vars(out), z.double().numpy(), tokens.cpu().numpy(), head.top_k)


@pytest.mark.parametrize("layout", LAYOUTS)
@pytest.mark.parametrize("dtype", ["f32", "f16"])
@pytest.mark.parametrize("given", [64, 65, 130])
def test_more_given_tokens_than_lanes(env, layout, dtype, given):
    """Lists of given tokens beyond a wavefront's lanes, with -1 and tokens outside the vocabulary among the later ones."""
    torch, b, ctx = env
    rows, vocab, cus = _check_layout(b, layout, dtype)
    g = _gen(torch, given)
    z = (torch.randn(rows, vocab, generator=g, device="cuda") * 3).to(_t(torch, dtype))
    z[1] = -float("inf")
    z[2, 7] = float("nan")
    tokens = torch.randint(0, vocab, (rows, given), generator=g, device="cuda", dtype=torch.int32)
    tokens[:, -1], tokens[:, given // 2] = -1, -1
    tokens[::2, -2], tokens[1::2, -2] = vocab, -7
    if given > 65:
        tokens[:, 64], tokens[:, 127], tokens[:, 128] = vocab + 5, 0, -1
    _check_logprobs(env, z, tokens, 20, cus=cus)
    _check_logprobs(env, z, tokens, 0, cus=cus)


# ---------------------------------------------------------------------------- how near the scales are

def _scale_bound(d, dtype, norm):
    """Half steps of fp32 that a row's scale may be off by.

    Without a gain: the last rounding.  With one: that, the rounding of an fp32 row's largest product, and half of what
    the sum of squares is off by, since its root is taken.  A square passes the additions of its lane (8 a group and
    the rest's product), 3 to 6 levels of lanes and the other wavefronts; beyond 32768 columns sums are 64 bits but
    for a group's 8."""
    if not norm:
        return 1
    product = 1 if dtype == "f32" else 0
    if d > 32768 + 7:
        return 1 + 8 / 2
    if d <= 256:
        return 1 + product + (8 + 1 + (3 if d <= 64 else 4 if d <= 128 else 5)) / 2
    per_wave = -(-(d // 8) // 64)
    w, ng = next(v for most, v in ((1, (1, 1)), (2, (1, 2)), (4, (2, 2)), (8, (4, 2)), (16, (4, 4)), (32, (8, 4)),
                                   (40, (8, 5)), (64, (16, 4))) if per_wave <= most)
    return 1 + product + (8 * ng + 1 + 6 + w - 1) / 2


@pytest.mark.parametrize("d", [64, 100, 256, 500, 1024, 1500, 3584, 8192, 16384, 18944, 30001, 40000])
@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("norm", [False, True])
def test_scales_are_as_near_as_their_roundings(env, d, dtype, norm):
    """Ordinary rows, rows of one value (whose sums are all off to the same side) and rows of a few large ones."""
    torch, b, ctx = env
    g = _gen(torch, d)
    x = torch.randn(48, d, generator=g, device="cuda")
    x[16:32] = torch.rand(16, 1, generator=g, device="cuda") + 0.1
    x[32:] *= 1 + 30 * (torch.rand(d, generator=g, device="cuda") < 0.003)
    x = x.to(_t(torch, dtype))
    gain = (1 + 0.3 * torch.randn(d, generator=g, device="cuda")).bfloat16() if norm else None
    q, s = _quantize(env, x, gain)
    _, ref = A.quantize_rows(_np(x), None if gain is None else _np(gain), float(np.float32(EPS)))
    off = np.abs(s.double().cpu().numpy() / ref - 1) / U
    assert off.max() <= _scale_bound(d, dtype, norm) * (1 + 1e-5), off.max()


@pytest.mark.parametrize("layout", LAYOUTS)
@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
def test_signalling_nans(env, layout, dtype):
    """A NaN of either kind and sign anywhere in a row, beside ordinary logits and in a masked row."""
    torch, b, ctx = env
    rows, vocab, cus = _check_layout(b, layout, dtype)
    t = _t(torch, dtype)
    word = torch.int32 if dtype == "f32" else torch.int16
    quiet, signalling = {"f32": (0x7fc00000, 0x7f800001), "bf16": (0x7fc0, 0x7f81), "f16": (0x7e00, 0x7c01)}[dtype]
    sign = torch.iinfo(word).min
    z = (torch.randn(rows, vocab, generator=_gen(torch, 3), device="cuda") * 3).to(t)
    bits = z.view(word)
    for r in range(7):
        if r >= 4:
            z[r] = -float("inf")
        bits[r, (0, vocab - 1, vocab // 2, 4999)[r % 4]] = (signalling, signalling + sign, quiet + sign, signalling)[r % 4]
    tokens = torch.randint(0, vocab, (rows, 2), generator=_gen(torch, 4), device="cuda", dtype=torch.int32)
    got = _check_logprobs(env, z, tokens, 20, cus=cus)
    assert bool(got["entropy"][:7].isnan().all()) and not bool(got["entropy"][7:].isnan().any())
    q, s = _quantize(env, z[:, :5003], None)
    at = torch.isnan(z[:, :5003]).any(1) | torch.isinf(z[:, :5003]).any(1)
    assert torch.equal(torch.isnan(s), at) and not bool(q[at].any()) and int(at.sum()) >= 5
