"""Row quantisation, 8-bit products and log probabilities on the GPU against the float64 reference.

Integers (the quantised rows, the exact sums, the alternatives' tokens) are compared for equality.
Bounds of the floats, from the roundings that the formulas take (u = 2^-24, fp32's half step):

* scale: a sum of d squares over at most 128 additions in one accumulator and 16 levels of joins, halved by
  the square root, and a few roundings: ((128 + 16) / 2 + 6) u.
* products: the documented fp32 steps, bit by bit, so no bound.
* log probabilities: S = 1 + s, where s sums what all but one largest token have.  Each e^d has a relative
  error of (4 + 3 |d|) u (the difference and its product with log2 e are rounded, the hardware's
  exponential is within an ulp; below 2^-126 it is zero, so `vocab` 2^-126 in all), and s passes at most N = 32 + ceil(vocab / 2048) + 40 additions and joins.  So
  |d log S| <= ((N + 4) s / S + 3 t1) u with t1 = sum p |d|, and a log probability adds a few roundings of
  its own size; entropy sums p d with p's errors: ((N + 8) (t1 + s / S) + 3 t2 + 4 H) u, t2 = sum p d^2.
"""
import numpy as np
import pytest

from oracle import answer as A
from tests.gpu_common import log, require_gpu

pytestmark = pytest.mark.gpu

U = 2.0 ** -24
EPS = 1e-5
TYPES = ("f32", "bf16", "f16")


def _t(torch, name):
    return {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}[name]


@pytest.fixture(scope="module")
def env():
    torch = require_gpu()
    from paper_2608_01785_amd import binding
    ctx = binding.Context(0, budgets=(64, 128, 256))
    yield torch, binding, ctx
    torch.cuda.synchronize()
    ctx.close()


def _gen(torch, seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def _view(torch, values, pad=0, shift=0, fill=None):
    """The values in a wider, shifted buffer: (buffer, view of the values' shape)."""
    rows, cols = values.shape
    buf = torch.empty(rows * (cols + pad) + shift + 32, dtype=values.dtype, device="cuda")
    if fill is not None:
        buf.fill_(fill)
    v = buf[shift:shift + rows * (cols + pad)].view(rows, cols + pad)[:, :cols]
    v.copy_(values)
    return buf, v


def _outside(torch, buf, view):
    """The buffer's elements that the view does not hold."""
    keep = torch.ones_like(buf, dtype=torch.bool)
    off = view.storage_offset()
    r, c = view.shape
    idx = off + torch.arange(r, device="cuda")[:, None] * view.stride(0) + torch.arange(c, device="cuda")
    keep[idx.reshape(-1)] = False
    return buf[keep]


def _np(t):
    return t.double().cpu().numpy()


# ---------------------------------------------------------------------------- quantise

def _quantize(env, x, gain, pad=0, shift=0, eps=EPS, cus=256, stream=None):
    torch, b, ctx = env
    rows, d = x.shape
    buf, q = _view(torch, torch.zeros(rows, d, dtype=torch.int8, device="cuda"), pad, shift, fill=99)
    q.fill_(77)
    s = torch.full((rows + 3,), 5.0, device="cuda")
    torch.cuda.synchronize()
    b.hs_quantize_rows(ctx, x, q, s[:rows], gain=gain, eps=eps, cu_budget=cus, stream=stream)
    torch.cuda.synchronize()
    assert bool((_outside(torch, buf, q) == 99).all()), "bytes outside the rows were written"
    assert bool((s[rows:] == 5).all())
    return q, s[:rows]


def _check_quantize(env, x, gain, **kw):
    q, s = _quantize(env, x, gain, **kw)
    rq, rs = A.quantize_rows(_np(x), None if gain is None else _np(gain), float(np.float32(kw.get("eps", EPS))))
    np.testing.assert_array_equal(q.cpu().numpy(), rq)
    s = s.double().cpu().numpy()
    np.testing.assert_array_equal(np.isnan(s), np.isnan(rs))
    ok = ~np.isnan(rs)
    with np.errstate(over="ignore"):
        big = np.abs(rs[ok].astype(np.float32).astype(np.float64)) == np.inf
    np.testing.assert_array_equal(s[ok][big], np.inf)
    assert np.all(np.abs(s[ok] - rs[ok])[~big] <= 78 * U * rs[ok][~big] + 2.0 ** -149)


QUANT_SHAPES = [(1, 1, 0, 0), (3, 7, 0, 0), (5, 64, 0, 0), (2, 1000, 0, 0), (33, 1024, 0, 0), (257, 512, 8, 0),
                (9, 3584, 0, 0), (4, 3585, 3, 1), (3, 4097, 0, 0), (6, 4096, 24, 8), (2, 14336, 0, 0),
                (3, 18944, 8, 0), (2, 18943, 1, 0), (7, 2000, 0, 0), (5, 1537, 1, 1), (3, 8190, 2, 2),
                (2, 30001, 0, 0), (2, 32775, 1, 0), (1, 70001, 0, 0), (2, 131072, 16, 16), (1500, 300, 4, 4)]


@pytest.mark.parametrize("shape", QUANT_SHAPES, ids=str)
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("norm", [False, True])
def test_quantize_shapes(env, shape, dtype, norm):
    torch = env[0]
    rows, d, pad, shift = shape
    g = _gen(torch, rows + d)
    x = torch.randn(rows, d, generator=g, device="cuda") * torch.exp(2 * torch.randn(rows, 1, generator=g, device="cuda"))
    gain = (1 + 0.3 * torch.randn(d, generator=g, device="cuda")).bfloat16() if norm else None
    _, xv = _view(torch, x.to(_t(torch, dtype)), pad, shift)
    _check_quantize(env, xv, gain, pad=pad, shift=shift)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("norm", [False, True])
@pytest.mark.parametrize("d", [40, 1024, 4100])
def test_quantize_values(env, dtype, norm, d):
    """Ties, extremes, subnormals, zeros, rows that are not finite."""
    torch = env[0]
    t = _t(torch, dtype)
    big = torch.finfo(t).max
    tiny = torch.finfo(t).smallest_normal
    g = _gen(torch, d)
    base = torch.randn(14, d, generator=g, device="cuda").to(t)
    # Halves of steps: with a largest value of 127 every (k + 1/2) is a tie.
    base[0] = (torch.randint(-127, 127, (d,), generator=g, device="cuda") + 0.5).to(t)
    base[0, d // 2] = 127
    base[1] = (torch.randint(-63, 63, (d,), generator=g, device="cuda") * 0.5).to(t)
    base[1, 0] = -254 / 4
    base[2] = 0
    base[3] = base[3] * 0 + big
    base[4, 1], base[4, 2] = big, -big
    base[5] = base[5].sign() * tiny / 4
    base[6, 3] = float("nan")
    base[7, d - 1] = float("inf")
    base[8, 0] = -float("inf")
    base[9] = base[9] * tiny
    base[10] = 0
    base[10, d - 1] = -tiny
    base[11] = -0.0
    base[12] = base[12].sign()          # every value at the maximum
    base[13] = base[13] * 2.0 ** 10
    gain = (1 + 0.3 * torch.randn(d, generator=g, device="cuda")).bfloat16() if norm else None
    _check_quantize(env, base, gain, eps=1e-6)
    _check_quantize(env, base, gain, eps=1e-30)
    if norm:
        gain[5] = 0
        gain[7] = -gain[7] * 64
        _check_quantize(env, base, gain)
        gain[6] = float("inf")
        _, s = _quantize(env, base, gain)
        assert bool(torch.isnan(s).all())


def test_quantize_fp32_ties_next_to_borders(env):
    """Products 24 x 8 bits wide, one step of fp32 on each side of a border."""
    torch = env[0]
    d = 2048
    x = np.zeros((4, d), np.float32)
    rng = np.random.default_rng(0)
    x[:, 0] = [127.0, 254.0, 1.0, 0.7]
    for r in range(4):
        k = rng.integers(-126, 126, d - 1) + 0.5
        v = (k * float(x[r, 0]) / 127.0).astype(np.float32)
        step = rng.integers(-2, 3, d - 1, dtype=np.int32)
        x[r, 1:] = (v.view(np.int32) + step).view(np.float32)
    g = torch.ones(d, device="cuda").bfloat16()
    for gain in (None, g, g * 1.0078125):
        _check_quantize(env, torch.from_numpy(x).cuda(), gain)


def test_quantize_no_rows_and_budgets(env):
    torch, b, ctx = env
    x = torch.randn(70, 640, generator=_gen(torch, 3), device="cuda")
    full = _quantize(env, x, None)
    for cus in (64, 128):
        part = _quantize(env, x, None, cus=cus)
        down = _quantize(env, x, None, cus=256 - cus, stream=b.hs_context_stream(ctx, cus, b.HS_ROLE_DOWN))
        for p in (part, down):
            assert torch.equal(p[0], full[0]) and torch.equal(p[1], full[1])
    _quantize(env, x[:0], None)
    with pytest.raises(b.HorizonError) as e:
        _quantize(env, x, None, cus=64, stream=b.hs_context_stream(ctx, 128))
    assert e.value.status == b.HS_ERR_BUDGET


# ---------------------------------------------------------------------------- products

def _linear(env, a, sa, w, sw, dtype, bias=None, pad=0, shift=0, cus=256, stream=None):
    torch, b, ctx = env
    m, n = a.shape[0], w.shape[0]
    buf, out = _view(torch, torch.zeros(m, n, dtype=_t(torch, dtype), device="cuda"), pad, shift, fill=99)
    out.fill_(float("nan"))
    torch.cuda.synchronize()
    b.hs_linear_i8(ctx, a, sa, w, sw, out, bias=bias, cu_budget=cus, stream=stream)
    torch.cuda.synchronize()
    assert bool((_outside(torch, buf, out) == 99).all()), "elements outside the rows were written"
    return out


def _check_linear(env, a, sa, w, sw, dtype, bias=None, **kw):
    torch = env[0]
    out = _linear(env, a, sa, w, sw, dtype, bias, **kw)
    ref = A.linear_i8(a.cpu().numpy(), sa.cpu().numpy(), w.cpu().numpy(), sw.cpu().numpy(),
                      None if bias is None else bias.float().cpu().numpy())
    ref = torch.from_numpy(ref).to(_t(torch, dtype))
    got = out.cpu()
    same = (got == ref) | (got.isnan() & ref.isnan())
    assert bool(same.all()), f"{int((~same).sum())} of {same.numel()} differ, first at {(~same).nonzero()[0].tolist()}"


LINEAR_SHAPES = [(1, 1, 1, 0), (1, 16, 16, 0), (3, 5, 7, 0), (1, 1000, 4096, 0), (2, 257, 1024, 16), (15, 48, 192, 0),
                 (16, 64, 64, 0), (17, 33, 65, 0), (32, 4096, 1024, 0), (33, 300, 640, 0), (64, 64, 64, 0),
                 (64, 1030, 2048, 0), (65, 130, 129, 0), (100, 515, 2047, 2), (128, 256, 512, 0), (129, 640, 1000, 8),
                 (200, 200, 16, 0), (256, 512, 128, 0), (300, 700, 900, 4), (777, 501, 255, 1), (1100, 2060, 384, 0),
                 (40, 100, 18944, 0), (5, 72, 18943, 1)]


@pytest.mark.parametrize("shape", LINEAR_SHAPES, ids=str)
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("with_bias", [False, True])
def test_linear_shapes(env, shape, dtype, with_bias):
    torch = env[0]
    m, n, k, pad = shape
    g = _gen(torch, m * 7 + n * 3 + k)
    a = torch.randint(-128, 128, (m, k), generator=g, device="cuda", dtype=torch.int8)
    w = torch.randint(-128, 128, (n, k), generator=g, device="cuda", dtype=torch.int8)
    sa = torch.rand(m, generator=g, device="cuda") + 0.01
    sw = (torch.rand(n, generator=g, device="cuda") + 0.01) * 1e-3
    bias = torch.randn(n, generator=g, device="cuda").bfloat16() if with_bias else None
    _, a = _view(torch, a, pad, pad)
    _, w = _view(torch, w, pad, 3 * pad)
    _check_linear(env, a, sa, w, sw, dtype, bias, pad=pad % 5, shift=pad % 3)


@pytest.mark.parametrize("m", [1, 20, 70, 300])
@pytest.mark.parametrize("dtype", TYPES)
def test_linear_extremes(env, m, dtype):
    """The largest sums, scales of zero, infinity and NaN, results beyond the type's range."""
    torch = env[0]
    n, k = 130, 131071
    a = torch.full((m, k), -128, dtype=torch.int8, device="cuda")
    w = torch.full((n, k), -128, dtype=torch.int8, device="cuda")
    w[1::2] = 127
    w[5, :-1] = 0
    sa = torch.linspace(0.0, 2.0, m, device="cuda")
    sw = torch.linspace(1e-6, 1.0, n, device="cuda")
    sw[3], sw[4], sw[7], sw[8] = float("nan"), float("inf"), 0.0, 3e38
    if m > 1:
        sa[1] = float("nan")
    _check_linear(env, a, sa, w, sw, dtype)


def test_linear_budgets_rows_and_streams(env):
    """The bits do not depend on the budget, nor a row's on the rows beside it."""
    torch, b, ctx = env
    g = _gen(torch, 11)
    a = torch.randint(-127, 128, (300, 1024), generator=g, device="cuda", dtype=torch.int8)
    w = torch.randint(-127, 128, (777, 1024), generator=g, device="cuda", dtype=torch.int8)
    sa, sw = torch.rand(300, generator=g, device="cuda"), torch.rand(777, generator=g, device="cuda")
    full = _linear(env, a, sa, w, sw, "bf16")
    for cus in (64, 128):
        assert torch.equal(_linear(env, a, sa, w, sw, "bf16", cus=cus), full)
        down = b.hs_context_stream(ctx, cus, b.HS_ROLE_DOWN)
        assert torch.equal(_linear(env, a, sa, w, sw, "bf16", cus=256 - cus, stream=down), full)
    for rows in (1, 2, 16, 33, 64, 65, 128, 299):
        assert torch.equal(_linear(env, a[:rows], sa[:rows], w, sw, "bf16"), full[:rows]), rows
    _linear(env, a[:0], sa[:0], w, sw, "bf16")
    _linear(env, a, sa, w[:0], sw[:0], "bf16")


# ---------------------------------------------------------------------------- log probabilities

def _logprobs(env, z, tokens, top, entropy=True, cus=256, stream=None, ws=None):
    torch, b, ctx = env
    rows = z.shape[0]
    n = 0 if tokens is None else tokens.shape[1]

    def new(cols, dtype=torch.float32):
        return torch.full((rows + 2, cols), 77, dtype=dtype, device="cuda")

    tok, ent, lp, at = new(n), new(1), new(top), new(top, torch.int32)
    if ws is None:
        ws = torch.full((b.hs_logprobs_workspace_size(rows, z.shape[1], top) + 1,), 255, dtype=torch.uint8, device="cuda")
    torch.cuda.synchronize()
    b.hs_logprobs(ctx, z, tokens=tokens, token_logprobs=tok[:rows] if n else None,
                  entropy=ent[:rows, 0] if entropy else None, top_logprobs=lp[:rows] if top else None,
                  top_tokens=at[:rows] if top else None, cu_budget=cus, stream=stream, workspace=ws)
    torch.cuda.synchronize()
    for t in (tok, ent, lp, at):
        assert bool((t[rows:] == 77).all()), "rows behind the last one were written"
    if not entropy:
        assert bool((ent == 77).all())
    return {"token": tok[:rows], "entropy": ent[:rows, 0], "top": lp[:rows], "top_tokens": at[:rows]}


def _close(name, got, ref, bound):
    got = got.double().cpu().numpy()
    with np.errstate(over="ignore"):   # a difference of logits beyond fp32's range rounds to infinity
        ref = np.where(np.isinf(ref.astype(np.float32)), ref.astype(np.float32), ref)
    fin = np.isfinite(ref)
    np.testing.assert_array_equal(np.isnan(got), np.isnan(ref), err_msg=name)
    np.testing.assert_array_equal(got[~fin & ~np.isnan(ref)], ref[~fin & ~np.isnan(ref)], err_msg=name)
    err = np.abs(got[fin] - ref[fin]) - np.broadcast_to(bound, ref.shape)[fin]
    assert err.size == 0 or err.max() <= 0, (name, float(err.max()))


def _check_logprobs(env, z, tokens, top, **kw):
    got = _logprobs(env, z, tokens, top, **kw)
    ref = A.logprobs(_np(z), None if tokens is None else tokens.cpu().numpy(), top)
    np.testing.assert_array_equal(got["top_tokens"].cpu().numpy(), ref["top_tokens"])
    n = 32 + -(-z.shape[1] // 2048) + 40
    s, t1, t2 = ref["s"], ref["t1"], ref["t2"]
    log_s = ((n + 4) * s / (1 + s) + 3 * t1 + 2 * np.log1p(s)) * U
    for name in ("token", "top"):
        size = np.where(np.isfinite(ref[name]), np.abs(ref[name]), 0)
        _close(name, got[name], ref[name], log_s[:, None] + 4 * U * size + z.shape[1] * 2.0 ** -126)
    if kw.get("entropy", True):
        _close("entropy", got["entropy"], ref["entropy"],
               ((n + 8) * (t1 + s / (1 + s)) + 3 * t2 + 4 * ref["entropy"]) * U + 128 * z.shape[1] * 2.0 ** -126)
    return got


LP_SHAPES = [(1, 1, 1, 0, 0), (2, 2, 5, 0, 0), (3, 63, 64, 0, 0), (5, 64, 64, 1, 1), (4, 65, 20, 0, 0),
             (7, 1000, 20, 0, 3), (2, 2047, 5, 1, 0), (2, 2048, 64, 0, 0), (3, 2049, 1, 2, 1), (300, 4099, 20, 0, 0),
             (33, 8192, 0, 8, 8), (1, 50001, 33, 1, 1), (17, 50001, 20, 0, 0), (1, 131072, 64, 0, 0),
             (3, 160001, 20, 0, 0), (2100, 2500, 5, 4, 0), (600, 9000, 40, 0, 0)]


@pytest.mark.parametrize("shape", LP_SHAPES, ids=str)
@pytest.mark.parametrize("dtype", TYPES)
def test_logprobs_shapes(env, shape, dtype):
    torch = env[0]
    rows, vocab, top, pad, shift = shape
    g = _gen(torch, rows + vocab)
    z = torch.randn(rows, vocab, generator=g, device="cuda") * 3
    z[: rows // 2, vocab // 3] += 20          # rows that are sure of one token
    _, z = _view(torch, z.to(_t(torch, dtype)), pad, shift, fill=50)
    tokens = torch.randint(0, vocab, (rows, 3), generator=g, device="cuda", dtype=torch.int32)
    tokens[:, 0] = vocab // 3
    _check_logprobs(env, z, tokens, top)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("vocab", [50, 3000, 20011, 131072])
def test_logprobs_values(env, dtype, vocab):
    """Masks, ties, orders and rows that have no distribution."""
    torch = env[0]
    t = _t(torch, dtype)
    inf, low, big = float("inf"), torch.finfo(t).min, torch.finfo(t).max
    g = _gen(torch, vocab)
    z = (torch.randn(22, vocab, generator=g, device="cuda") * 4).to(t)
    mid, end = vocab // 2, vocab - 1
    z[0] = -inf                                    # nothing left
    z[1] = -inf
    z[1, mid] = 3.0                                # one token left
    z[2] = -inf
    z[2, end] = low                                # one, at the type's lowest value
    z[3] = low
    z[4] = low
    z[4, mid:] = z[5, mid:]                        # masked by the lowest value
    z[5] = 0.0                                     # all equal
    z[6, : mid] = -inf
    z[7] = torch.arange(vocab, device="cuda").to(t) / 64            # ascending, with ties
    z[8] = -(torch.arange(vocab, device="cuda").to(t) / 64)         # descending
    z[9] = 0.0
    z[9, ::2] = -0.0                               # equal values of either sign
    z[10, mid] = float("nan")
    z[11, end] = inf
    z[12, 0] = inf
    z[12, end] = inf
    z[13] = -inf
    z[13, 0] = float("nan")
    z[14] = big
    z[15] = low
    z[15, 7] = big                                 # differences beyond fp32's range
    z[16] = z[16].round()                          # many ties
    z[17] = -100.0
    z[17, mid] = 0.0                               # certain: the rest is below 2^-24
    z[18] = -18.0
    z[18, 1] = 0.0
    z[19, torch.rand(vocab, generator=g, device="cuda") < 0.99] = -inf
    z[20] = -inf
    z[20, ::7] = 1.0
    z[21] = (torch.arange(vocab, device="cuda") % 5).to(t)
    tokens = torch.randint(0, vocab, (22, 6), generator=g, device="cuda", dtype=torch.int32)
    tokens[:, 0], tokens[:, 1], tokens[:, 2], tokens[:, 3] = mid, -1, vocab, -2
    tokens[:, 4] = end
    for top in (0, 1, 20, 64):
        _check_logprobs(env, z, tokens, top)
    _check_logprobs(env, z, None, 5, entropy=False)
    # As many rows as fill the chip: each row's work is laid out otherwise, the answers are the same.
    many = z.repeat(120, 1) if vocab <= 20011 else z.repeat(30, 1)
    one = _logprobs(env, z, tokens, 20)
    rep = _logprobs(env, many, tokens.repeat(many.shape[0] // 22, 1), 20)
    for name in ("top_tokens",):
        assert torch.equal(rep[name].view(-1, 22, 20), one[name].expand(many.shape[0] // 22, 22, 20))
    _check_logprobs(env, many[22 * 5:22 * 6], tokens, 20)


@pytest.mark.parametrize("dtype", TYPES)
def test_logprobs_many_rows_of_each_value(env, dtype):
    """Rows enough that none is split over work-groups."""
    torch = env[0]
    g = _gen(torch, 5)
    z = (torch.randn(2304, 6001, generator=g, device="cuda") * 2)
    z[::3] = z[::3].round()
    z[1::7, 100:] = -float("inf")
    z[4::11] = -float("inf")
    z[5::13, 5] = float("nan")
    z = z.to(_t(torch, dtype))
    tokens = torch.randint(-1, 6001, (2304, 2), generator=g, device="cuda", dtype=torch.int32)
    _check_logprobs(env, z, tokens, 20)


def test_logprobs_budgets(env):
    torch, b, ctx = env
    g = _gen(torch, 6)
    z = torch.randn(9, 70000, generator=g, device="cuda").bfloat16()
    tokens = torch.randint(0, 70000, (9, 2), generator=g, device="cuda", dtype=torch.int32)
    for cus in (64, 128):
        _check_logprobs(env, z, tokens, 7, cus=cus)
        _check_logprobs(env, z, tokens, 7, cus=256 - cus, stream=b.hs_context_stream(ctx, cus, b.HS_ROLE_DOWN))
    _logprobs(env, z[:0], tokens[:0], 7)


# ---------------------------------------------------------------------------- together

def _head(env, rows=12, d=512, vocab=9001):
    torch, b, ctx = env
    g = _gen(torch, 21)
    s = dict(x=torch.randn(rows, d, generator=g, device="cuda"), gain=(1 + 0.1 * torch.randn(d, generator=g, device="cuda")).bfloat16(),
             w=(0.1 * torch.randn(vocab, d, generator=g, device="cuda")).bfloat16(),
             wq=torch.empty(vocab, d, dtype=torch.int8, device="cuda"), ws=torch.empty(vocab, device="cuda"),
             q=torch.empty(rows, d, dtype=torch.int8, device="cuda"), qs=torch.empty(rows, device="cuda"),
             z=torch.empty(rows, vocab, device="cuda"),
             tokens=torch.randint(0, vocab, (rows, 1), generator=g, device="cuda", dtype=torch.int32),
             lp=torch.empty(rows, 1, device="cuda"), ent=torch.empty(rows, device="cuda"),
             top=torch.empty(rows, 8, device="cuda"), at=torch.empty(rows, 8, dtype=torch.int32, device="cuda"),
             work=torch.empty(max(1, b.hs_logprobs_workspace_size(rows, vocab, 8)), dtype=torch.uint8, device="cuda"))
    torch.cuda.synchronize()
    b.hs_quantize_rows(ctx, s["w"], s["wq"], s["ws"])
    torch.cuda.synchronize()
    return s


def _score(env, s, stream=None):
    torch, b, ctx = env
    b.hs_quantize_rows(ctx, s["x"], s["q"], s["qs"], gain=s["gain"], eps=EPS, stream=stream)
    b.hs_linear_i8(ctx, s["q"], s["qs"], s["wq"], s["ws"], s["z"], stream=stream)
    b.hs_logprobs(ctx, s["z"], tokens=s["tokens"], token_logprobs=s["lp"], entropy=s["ent"], top_logprobs=s["top"],
                  top_tokens=s["at"], stream=stream, workspace=s["work"])


def _check_score(s):
    q, qs = A.quantize_rows(_np(s["x"]), _np(s["gain"]), float(np.float32(EPS)))
    np.testing.assert_array_equal(s["q"].cpu().numpy(), q)
    z = A.linear_i8(q, s["qs"].cpu().numpy(), s["wq"].cpu().numpy(), s["ws"].cpu().numpy(), None)
    np.testing.assert_array_equal(s["z"].cpu().numpy(), z)
    ref = A.logprobs(z, s["tokens"].cpu().numpy(), 8)
    np.testing.assert_array_equal(s["at"].cpu().numpy(), ref["top_tokens"])
    np.testing.assert_allclose(s["lp"].cpu().numpy(), ref["token"], rtol=0, atol=2e-5)
    # 8-bit operands against the 16-bit head: each side is off by half a step of its row's largest value,
    # sqrt(d) / 127-ish of a logit in all; what the head is for survives.
    x = _np(s["x"])
    h = x / np.sqrt((x * x).mean(1, keepdims=True) + EPS) * _np(s["gain"])
    full = h @ _np(s["w"]).T
    assert np.abs(full - z).max() <= 0.06 * np.abs(full).max()


def test_from_residual_rows_to_log_probabilities(env):
    torch = env[0]
    s = _head(env)
    _score(env, s)
    torch.cuda.synchronize()
    _check_score(s)


def test_captured_and_replayed_with_new_rows(env):
    torch, b, ctx = env
    s = _head(env)
    stream = torch.cuda.Stream()
    _score(env, s, stream.cuda_stream)
    stream.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=stream):
        _score(env, s, stream.cuda_stream)
    for i in range(4):
        s["x"].copy_(torch.randn(s["x"].shape, generator=_gen(torch, 100 + i), device="cuda"))
        for n in ("z", "lp", "ent", "top"):
            s[n].fill_(float("nan"))
        s["at"].fill_(-5)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        _check_score(s)
        kept = {n: s[n].clone() for n in ("lp", "ent", "top", "at")}
        _score(env, s)
        torch.cuda.synchronize()
        for n, t in kept.items():
            assert torch.equal(t, s[n]), (i, n)


def test_two_calls_at_once_on_two_streams(env):
    torch, b, ctx = env
    one, two = _head(env, rows=3, vocab=40000), _head(env, rows=5, vocab=50001)
    up, down = b.hs_context_stream(ctx, 128), b.hs_context_stream(ctx, 128, b.HS_ROLE_DOWN)
    for s, stream in ((one, up), (two, down)) * 5:
        b.hs_quantize_rows(ctx, s["x"], s["q"], s["qs"], gain=s["gain"], eps=EPS, cu_budget=128, stream=stream)
        b.hs_linear_i8(ctx, s["q"], s["qs"], s["wq"], s["ws"], s["z"], cu_budget=128, stream=stream)
        b.hs_logprobs(ctx, s["z"], tokens=s["tokens"], token_logprobs=s["lp"], entropy=s["ent"],
                      top_logprobs=s["top"], top_tokens=s["at"], cu_budget=128, stream=stream, workspace=s["work"])
    torch.cuda.synchronize()
    _check_score(one)
    _check_score(two)


def test_timing_records_the_calls(env):
    torch, b, ctx = env
    s = _head(env)
    b.hs_timing_enable(ctx, True)
    for _ in range(3):
        _score(env, s)
    for kind in ("quantize", "linear_i8", "logprobs"):
        ms, n = b.hs_timing_read(ctx, kind)
        assert n == 3 and 0 < ms < 1000, (kind, ms, n)
    b.hs_timing_enable(ctx, False)


def test_binding_refusals_on_the_device(env):
    torch, b, ctx = env
    x = torch.randn(4, 64, device="cuda")
    q, s = torch.empty(4, 64, dtype=torch.int8, device="cuda"), torch.empty(4, device="cuda")
    for bad, text in ((dict(x=x.t()), "contiguous"), (dict(q=q[:, :60]), "shape"), (dict(scale=s[:3]), "shape"),
                      (dict(gain=torch.ones(64, device="cuda")), "type"), (dict(scale=s.cpu()), "is on cpu")):
        a = dict(x=x, q=q, scale=s, gain=None)
        a.update(bad)
        with pytest.raises(ValueError, match=text):
            b.hs_quantize_rows(ctx, a["x"], a["q"], a["scale"], gain=a["gain"])
    with pytest.raises(ValueError, match="fit"):
        b.hs_linear_i8(ctx, q, s, q[:, :32], s, x)
    with pytest.raises(ValueError, match="together"):
        b.hs_logprobs(ctx, x, top_logprobs=x)
    with pytest.raises(b.HorizonError, match="stride"):   # one row shown four times
        b.hs_logprobs(ctx, x[:1].expand(4, 64), entropy=s)
    log("refused as documented")
