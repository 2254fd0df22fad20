"""Refusals of the answering calls: everything invalid fails before any GPU work (no context, fake pointers)."""
import ctypes

import numpy as np
import pytest

P = 0x100000   # fake device addresses, far apart and never dereferenced


@pytest.fixture(scope="module")
def b():
    from paper_2608_01785_amd import binding
    binding.lib()
    return binding


def quantize(b, **kw):
    a = dict(x=P, t=0, ldx=64, gain=None, eps=1e-6, rows=4, d=64, q=2 * P, ldq=64, scale=3 * P, cus=256)
    a.update(kw)
    st = b.lib().hs_quantize_rows(None, a["x"], a["t"], a["ldx"], a["gain"], a["eps"], a["rows"], a["d"], a["q"],
                                  a["ldq"], a["scale"], a["cus"], None)
    return st, b.hs_last_error()


def linear(b, **kw):
    a = dict(a=P, lda=64, sa=2 * P, w=3 * P, ldw=64, sw=4 * P, bias=None, out=5 * P, t=0, ldo=32, m=4, n=32, k=64)
    a.update(kw)
    st = b.lib().hs_linear_i8(None, a["a"], a["lda"], a["sa"], a["w"], a["ldw"], a["sw"], a["bias"], a["out"], a["t"],
                              a["ldo"], a["m"], a["n"], a["k"], 256, None)
    return st, b.hs_last_error()


def logprobs(b, **kw):
    a = dict(z=P, t=0, ld=64, rows=4, vocab=64, tok=2 * P, nt=1, tlp=3 * P, ent=4 * P, k=5, top=5 * P, tt=6 * P,
             ws=7 * P, wsb=1 << 30)
    a.update(kw)
    st = b.lib().hs_logprobs(None, a["z"], a["t"], a["ld"], a["rows"], a["vocab"], a["tok"], a["nt"], a["tlp"],
                             a["ent"], a["k"], a["top"], a["tt"], 256, None, a["ws"], a["wsb"])
    return st, b.hs_last_error()


INVALID, UNSUPPORTED = 1, 2
REFUSED = [
    (quantize, dict(t=3), INVALID, "type"),
    (quantize, dict(rows=-1), INVALID, "shape"),
    (quantize, dict(d=0, ldx=1), INVALID, "shape"),
    (quantize, dict(x=None), INVALID, "x is null"),
    (quantize, dict(q=None), INVALID, "q is null"),
    (quantize, dict(scale=None), INVALID, "scale is null"),
    (quantize, dict(ldx=63), INVALID, "stride"),
    (quantize, dict(ldq=63), INVALID, "stride"),
    (quantize, dict(ldx=(1 << 30) + 1), INVALID, "stride"),
    (quantize, dict(x=P + 2), INVALID, "aligned"),
    (quantize, dict(x=P + 1, t=1), INVALID, "aligned"),
    (quantize, dict(scale=3 * P + 2), INVALID, "aligned"),
    (quantize, dict(gain=4 * P + 1), INVALID, "aligned"),
    (quantize, dict(gain=4 * P, eps=0.0), INVALID, "eps"),
    (quantize, dict(gain=4 * P, eps=float("nan")), INVALID, "eps"),
    (quantize, dict(gain=4 * P, eps=float("inf")), INVALID, "eps"),
    (quantize, dict(q=P + 4 * 64 * 4 - 1), INVALID, "overlap"),
    (quantize, dict(scale=P), INVALID, "overlap"),
    (quantize, dict(scale=2 * P), INVALID, "overlap"),
    (quantize, dict(gain=2 * P), INVALID, "overlap"),
    (linear, dict(t=-1), INVALID, "type"),
    (linear, dict(m=-1), INVALID, "m -1"),
    (linear, dict(n=-1), INVALID, "n -1"),
    (linear, dict(k=0), INVALID, "k 0"),
    (linear, dict(k=131072, lda=131072, ldw=131072), UNSUPPORTED, "32-bit sums"),
    (linear, dict(lda=(1 << 22) + 1), UNSUPPORTED, "strides"),
    (linear, dict(ldw=(1 << 22) + 1), UNSUPPORTED, "strides"),
    (linear, dict(a=None), INVALID, "a is null"),
    (linear, dict(sa=None), INVALID, "a_scale is null"),
    (linear, dict(w=None), INVALID, "w is null"),
    (linear, dict(sw=None), INVALID, "w_scale is null"),
    (linear, dict(out=None), INVALID, "out is null"),
    (linear, dict(lda=63), INVALID, "stride"),
    (linear, dict(ldw=63), INVALID, "stride"),
    (linear, dict(ldo=31), INVALID, "stride"),
    (linear, dict(sa=2 * P + 1), INVALID, "aligned"),
    (linear, dict(bias=6 * P + 1), INVALID, "aligned"),
    (linear, dict(out=5 * P + 2), INVALID, "aligned"),
    (linear, dict(out=P), INVALID, "overlap"),
    (linear, dict(out=4 * P + 124), INVALID, "overlap"),
    (linear, dict(bias=5 * P), INVALID, "overlap"),
    (logprobs, dict(t=5), INVALID, "type"),
    (logprobs, dict(vocab=0), INVALID, "shape"),
    (logprobs, dict(rows=-2), INVALID, "shape"),
    (logprobs, dict(k=65), UNSUPPORTED, "top_k"),
    (logprobs, dict(k=-1), UNSUPPORTED, "top_k"),
    (logprobs, dict(nt=-1), INVALID, "n_tokens"),
    (logprobs, dict(ld=63), INVALID, "stride"),
    (logprobs, dict(z=None), INVALID, "logits is null"),
    (logprobs, dict(z=P + 1, t=1), INVALID, "aligned"),
    (logprobs, dict(tok=None), INVALID, "tokens is null"),
    (logprobs, dict(tlp=None), INVALID, "token_logprobs is null"),
    (logprobs, dict(top=None), INVALID, "top_logprobs is null"),
    (logprobs, dict(tt=None), INVALID, "top_tokens is null"),
    (logprobs, dict(tlp=P), INVALID, "overlap"),
    (logprobs, dict(ent=3 * P), INVALID, "overlap"),
    (logprobs, dict(tt=5 * P + 76), INVALID, "overlap"),
]


@pytest.mark.parametrize("i", range(len(REFUSED)))
def test_refused(b, i):
    call, kw, status, text = REFUSED[i]
    st, msg = call(b, **kw)
    assert st == status and text in msg, (kw, st, msg)


@pytest.mark.parametrize("call,kw", [
    (quantize, {}), (quantize, dict(gain=4 * P)), (quantize, dict(eps=0.0)), (quantize, dict(rows=0, x=None, q=None)),
    (quantize, dict(x=P + 2, t=2, ldx=65, ldq=67, q=2 * P + 1)), (linear, {}), (linear, dict(bias=6 * P, t=1)),
    (linear, dict(m=0, a=None, out=None, sa=None)), (linear, dict(n=0, w=None, sw=None, out=None)),
    (linear, dict(k=131071, lda=131071, ldw=131071, a=100 * P, w=200 * P)),
    (logprobs, {}), (logprobs, dict(nt=0, tok=None, tlp=None)), (logprobs, dict(k=0, top=None, tt=None)),
    (logprobs, dict(ent=None)), (logprobs, dict(rows=0, z=None)),
])
def test_valid_arguments_reach_the_context(b, call, kw):
    st, msg = call(b, **kw)
    assert st == INVALID and msg == "context is null", (st, msg)


def test_logprobs_workspace(b):
    sizes = [b.hs_logprobs_workspace_size(r, 131072, 20) for r in (0, 1, 32, 256, 4096)]
    assert sizes[0] == 0
    # A size serves every smaller call.
    for rows in (1, 7, 32, 100, 256, 1000, 4096):
        for k in (0, 1, 20, 64):
            need = b.hs_logprobs_workspace_size(rows, 131072, k)
            if need == 0:
                continue
            st, msg = logprobs(b, rows=rows, vocab=131072, ld=131072, k=k, tok=1 << 40, tlp=2 << 40, ent=3 << 40,
                               top=4 << 40, tt=5 << 40, ws=6 << 40, wsb=need - 1)
            assert st == b.HS_ERR_WORKSPACE and "needed" in msg, (rows, k, msg)
            st, msg = logprobs(b, rows=rows, vocab=131072, ld=131072, k=k, tok=1 << 40, tlp=2 << 40, ent=3 << 40,
                               top=4 << 40, tt=5 << 40, ws=None, wsb=0)
            assert st == b.HS_ERR_WORKSPACE and "null" in msg, (rows, k, msg)
            for fewer in (1, rows // 2, rows - 1):
                assert b.hs_logprobs_workspace_size(fewer, 131072, k) <= need
    for bad in ((-1, 10, 0), (1, 0, 0)):
        with pytest.raises(b.HorizonError):
            b.hs_logprobs_workspace_size(*bad)
    assert b.lib().hs_logprobs_workspace_size(1, 1, 0, None) == INVALID


def test_binding_refuses_tensors_that_do_not_fit(b):
    import torch

    class Ctx:
        handle, device = None, 0

    x = torch.zeros(4, 8)
    with pytest.raises(ValueError, match="is on cpu"):
        b.hs_quantize_rows(Ctx, x, x.to(torch.int8), torch.zeros(4))
    with pytest.raises(ValueError, match="type"):
        b.hs_quantize_rows(Ctx, x.double(), x.to(torch.int8), torch.zeros(4))
    with pytest.raises(ValueError, match="dimensions"):
        b.hs_logprobs(Ctx, x[0])


def test_linear_kernel_rule(b):
    """Few rows, then larger tiles as there is more to do; what every kernel's GPU test relies on."""
    def kernel(m, n, k, cus=256, aligned=True):
        return b.lib().hs_linear_i8_kernel(m, n, k, cus, aligned)
    few32, few64, few6464, t64, t128, t256 = range(6)
    assert kernel(1, 4608, 3584) == few32 and kernel(32, 3584, 18944) == few32
    assert kernel(64, 3584, 18944) == few32 and kernel(128, 3584, 18944) == few64
    assert kernel(64, 4608, 3584) == few64
    assert kernel(192, 3584, 18944) == few6464 and kernel(192, 3584, 18943, aligned=False) == t64
    assert kernel(128, 14336, 4096) == t64
    assert kernel(777, 4096, 4096) == t128
    assert kernel(4096, 8192, 8192) == t256 and kernel(10515, 37888, 3584) == t256
    assert kernel(4096, 8192, 8192, aligned=False) == t128
    assert kernel(777, 5120, 2047) == t128 and kernel(777, 1030, 2049, aligned=False) == t64
    for m, n, k in ((1, 1, 1), (1, 1, 131071), (2 ** 20, 2 ** 20, 1), (2 ** 31 - 1, 1, 16), (1, 2 ** 31 - 1, 16)):
        for cus in (1, 64, 256):
            for aligned in (False, True):
                assert few32 <= kernel(m, n, k, cus, aligned) <= (t256 if aligned else t128)
    assert kernel(1, 2 ** 30, 16) >= t64   # more blocks than a grid of the few rows' kernel holds
    # The few rows' groups are a grid's second dimension, which ends at 65535.
    assert kernel(2 ** 23, 32, 8192) >= t64 and kernel(2 ** 23, 32, 8192, aligned=False) >= t64


def test_too_many_rows(b):
    """Refused before anything is read: row counts beyond what the grids hold."""
    lib, one = b.lib(), 4096
    for rows, calls in ((2 ** 30 + 1, ("q", "m", "n")), (2 ** 25 + 1, ("l", "w"))):
        for call in calls:
            if call == "q":
                st = lib.hs_quantize_rows(None, one, b.HS_TYPE_F32, 4, None, 1e-6, rows, 4, one, 4, one, 256, None)
            elif call in "mn":
                m, n = (rows, 4) if call == "m" else (4, rows)
                st = lib.hs_linear_i8(None, one, 16, one, one, 16, one, None, one, b.HS_TYPE_F32, 2 ** 30, m, n, 16, 256,
                                      None)
            elif call == "l":
                st = lib.hs_logprobs(None, one, b.HS_TYPE_F32, 4, rows, 4, None, 0, None, one, 0, None, None, 256, None,
                                     None, 0)
            else:
                st = lib.hs_logprobs_workspace_size(rows, 4, 0, ctypes.byref(ctypes.c_size_t(0)))
            assert st == b.HS_ERR_UNSUPPORTED, (call, st)
            assert b"rows" in lib.hs_last_error()


def test_workspace_covers_every_split(b):
    """A block's 16 bytes of sums and its keys fit the size given for these rows or more, whatever the budget and type."""
    rng = np.random.default_rng(5)
    seen = 0
    for _ in range(4000):
        rows = int(rng.integers(1, rng.choice([4, 40, 300, 3000])))
        vocab, top = int(2 ** rng.uniform(0, 20)), int(rng.integers(0, 65))
        splits = b.lib().hs_logprobs_splits(rows, vocab, int(rng.choice([2, 4])), int(rng.integers(1, 257)))
        assert 1 <= splits <= 64
        if splits > 1:
            seen += 1
            need = rows * splits * (16 + 8 * top)
            assert need <= b.hs_logprobs_workspace_size(rows, vocab, top)
            assert need <= b.hs_logprobs_workspace_size(rows + int(rng.integers(0, 500)), vocab, top)
    assert seen > 300


def test_split_rule(b):
    """Rows are split where they leave compute units idle and are long enough for a second kernel."""
    def splits(rows, vocab, bytes_, cus=256):
        return b.lib().hs_logprobs_splits(rows, vocab, bytes_, cus)
    assert splits(1, 131072, 2) > 8 and splits(64, 131072, 2) == 4 and splits(64, 131072, 2, 64) == 1
    assert splits(257, 131072, 2) == 1 and splits(1, 1000, 4) == 1 and splits(128, 32000, 4) == 1


@pytest.mark.parametrize("ld,k", [(16, 16), (128, 128), (160, 144), (1040, 1040), (4096, 2064), (1 << 22, 512),
                                  (1 << 22, 131056)])
def test_aligned_product_loads_stay_in_the_operand(b, ld, k):
    """Every 16-byte load either lies in a row's k bytes, or its vector offset alone is past the resource's end: what a
    scalar offset counts for in that check does not matter."""
    out = (ctypes.c_uint32 * 3)()
    load = b.lib().hs_linear_i8_load
    load.argtypes = [ctypes.c_int32] * 4 + [ctypes.c_int64, ctypes.c_int32, ctypes.POINTER(ctypes.c_uint32)]
    load.restype = None
    last = (k - 1) // 128
    stages = sorted({0, 1, 2, last // 2, last - 1, last, last + 1, last + 9} & set(range(last + 10)))
    for span in (1, 2, 7, 8, 9, 31, 63, 64):
        for stage in stages:
            for lane in range(64):
                for l in range(8):
                    load(lane, l, stage, span, ld, k, out)
                    vector, scalar, records = out
                    row, at = 8 * l + lane // 8, 128 * stage + 16 * (lane % 8)
                    assert records == (span - 1) * ld + k and scalar < k
                    if row < span and at < k:
                        assert vector + scalar == row * ld + at and vector + scalar + 16 <= records
                    else:
                        assert vector >= records, (span, stage, lane, l)


def test_binding_refuses_workspaces_that_do_not_fit(b):
    """Before the library sees a pointer: on the host or another device, with gaps, of fewer bytes than claimed."""
    import torch

    class Host:
        handle, device = None, -1   # CPU tensors report device -1

    class Gpu:
        handle, device = None, 0

    z, e = torch.zeros(2, 70000), torch.zeros(2)
    need = b.hs_logprobs_workspace_size(2, 70000, 0)
    ws = torch.zeros(need, dtype=torch.uint8)
    with pytest.raises(ValueError, match="workspace is on cpu"):
        b._workspace(Gpu, ws, None)
    for bad, n, text in ((ws[::2], None, "not contiguous"), (ws[:1].expand(need), None, "not contiguous"),
                         (ws, need + 1, "ws_bytes is"), (0x1000, None, "needs ws_bytes")):
        with pytest.raises(ValueError, match=text):
            b.hs_logprobs(Host, z, entropy=e, workspace=bad, ws_bytes=n)
    for good, n in ((ws, None), (ws, need), (ws.view(torch.int32) if need % 4 == 0 else ws, None), (0x1000, need)):
        with pytest.raises(b.HorizonError, match="context is null"):
            b.hs_logprobs(Host, z, entropy=e, workspace=good, ws_bytes=n)
    for short, n in ((ws[:need - 1], None), (ws, need - 1), (None, None)):
        with pytest.raises(b.HorizonError) as err:
            b.hs_logprobs(Host, z, entropy=e, workspace=short, ws_bytes=n)
        assert err.value.status == b.HS_ERR_WORKSPACE


def test_binding_refuses_counts_beyond_32_bits(b):
    """2^32 rows (columns, tokens, alternatives) and some are not passed as some.  Meta tensors: no memory."""
    import torch

    class Ctx:
        handle, device = None, -1   # as CPU and meta tensors report

    def meta(*shape, dtype=torch.float32):
        return torch.empty(shape, dtype=dtype, device="meta")

    n, i8, i32 = 2 ** 32 + 4, torch.int8, torch.int32
    with pytest.raises(b.HorizonError, match="rows: at most"):
        b.hs_quantize_rows(Ctx, meta(n, 8), meta(n, 8, dtype=i8), meta(n))
    with pytest.raises(b.HorizonError, match="rows: at most"):
        b.hs_logprobs(Ctx, meta(n, 8), entropy=meta(n))
    for m, w, k in ((n, 8, 16), (8, n, 16), (8, 8, n)):
        with pytest.raises(b.HorizonError, match="rows: at most|32-bit sums|row strides"):
            b.hs_linear_i8(Ctx, meta(m, k, dtype=i8), meta(m), meta(w, k, dtype=i8), meta(w), meta(m, w))
    with pytest.raises(b.HorizonError, match="top_k"):
        b.hs_logprobs(Ctx, meta(2, 8), top_logprobs=meta(2, n), top_tokens=meta(2, n, dtype=i32))
    for counts in ((n, 8, 0), (8, n, 0), (8, 8, n)):
        if counts[1] == n:
            assert b.hs_logprobs_workspace_size(*counts) >= b.hs_logprobs_workspace_size(8, 2 ** 30, 0)
        else:
            with pytest.raises(b.HorizonError, match="rows: at most|top_k"):
                b.hs_logprobs_workspace_size(*counts)
    st, msg = logprobs(b, nt=2 ** 31 - 1)   # what 2^31 given tokens a row and more are passed as
    assert st == INVALID and "tokens: row stride" in msg


def test_binding_refuses_tensors_without_dimensions(b):
    import torch

    class Ctx:
        handle, device = None, -1

    z, one = torch.zeros(2, 8), torch.tensor(3, dtype=torch.int32)
    with pytest.raises(ValueError, match="tokens has 0 dimensions"):
        b.hs_logprobs(Ctx, z, tokens=one, token_logprobs=torch.zeros(2, 1))
    with pytest.raises(ValueError, match="top_tokens has 0 dimensions|top_logprobs has shape"):
        b.hs_logprobs(Ctx, z, top_tokens=one, top_logprobs=torch.zeros(2, 1))
    for bad in (torch.tensor(1.0), torch.zeros(2)):
        with pytest.raises(ValueError, match="dimensions"):
            b.hs_logprobs(Ctx, bad)
