"""Performance cases of the stand-alone operators that answer from the residual stream.

``quantize``  rows to 8-bit integers with one scale each, RMS-normalised on the way
              when a gain is given (``binding.hs_quantize_rows``);
``linear``    the product of such rows with 8-bit weight channels
              (``binding.hs_linear_i8``);
``logprobs``  log probabilities of given tokens, entropy and top alternatives of
              rows of logits (``binding.hs_logprobs``).

With ``own`` false, ``run`` computes them in elementary torch operations.
"""
from __future__ import annotations

import math

import torch

own = False

TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
SIZE = {"f32": 4, "bf16": 2, "f16": 2}
EPS = 1e-6


def _quantize(name, rows, d, dtype, gain, pad=0):
    return dict(name=name, op="quantize", rows=rows, d=d, dtype=dtype, gain=gain, pad=pad)


def _linear(name, m, n, k, dtype, bias, pad=0):
    return dict(name=name, op="linear", m=m, n=n, k=k, dtype=dtype, bias=bias, pad=pad)


def _logprobs(name, rows, vocab, dtype, given, top, masked=0.0, pad=0):
    return dict(name=name, op="logprobs", rows=rows, vocab=vocab, dtype=dtype, given=given, top=top, masked=masked,
                pad=pad)


def listed():
    return [
        # The downstream stage's decode batch on its way to the head: the smallest call.
        _quantize("quantize_norm_decode", 32, 1024, "f32", True),
        # The residual stream of the shared stage's prefill batch (8 requests), final norm included.
        _quantize("quantize_norm_prefill", 10515, 3584, "f32", True),
        # A head's weight channels, prepared once per model; an odd vocabulary, cut out of a wider matrix.
        _quantize("quantize_channels", 50001, 3584, "bf16", False, pad=24),
        # A projection of the downstream decode batch.
        _linear("linear_decode", 32, 4096, 1024, "f16", False),
        # The head for one request's next token.
        _linear("linear_head_one", 1, 65536, 3584, "f32", False),
        # The head for a full decode batch.
        _linear("linear_head_batch", 128, 65536, 4096, "bf16", False),
        # The widest projection of the prefill batch.
        _linear("linear_prefill", 10515, 37888, 3584, "bf16", True),
        # Sizes and strides that fit no tile, bytes that fit no word.
        _linear("linear_ragged", 777, 5001, 2047, "f16", True, pad=2),
        # One request's next token.
        _logprobs("logprobs_one", 1, 131072, "bf16", 1, 20),
        # A decode batch, logits as the head leaves them.
        _logprobs("logprobs_decode", 32, 65536, "f32", 1, 20),
        # Scoring whole prompts: every row's own next token and a few alternatives.
        _logprobs("logprobs_prompt", 2048, 131072, "bf16", 1, 5),
        # Constrained decoding: most of an odd vocabulary masked, several candidates a row, odd row starts.
        _logprobs("logprobs_masked", 257, 50001, "f16", 3, 33, masked=0.9, pad=2),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    """One more case of the same ranges: sizes over their logarithm, every type, aligned and odd strides."""
    op = rng.choice(("quantize", "linear", "logprobs"))
    dtype, pad = rng.choice(("f32", "bf16", "f16")), rng.choice((0, 0, 0, 1, 8, 24, 64))
    if op == "quantize":
        d = _log(rng, 64, 20000)
        if rng.random() < 0.6:
            d = max(64, d // 64 * 64)
        c = _quantize("", _log(rng, 1, min(50000, 150_000_000 // d)), d, dtype, rng.random() < 0.6, pad)
    elif op == "linear":
        n, k = _log(rng, 100, 70000), _log(rng, 64, 19000)
        if rng.random() < 0.6:
            n, k = max(128, n // 128 * 128), max(64, k // 64 * 64)
        k = min(k, 250_000_000 // n)
        m = _log(rng, 1, max(1, min(8192, 1_000_000_000_000 // (n * k), 380_000_000 // n)))
        c = _linear("", m, n, k, dtype, rng.random() < 0.5, pad)
    else:
        v = _log(rng, 1000, 160000)
        if rng.random() < 0.5:
            v = v // 8 * 8
        c = _logprobs("", _log(rng, 1, min(4096, 250_000_000 // v)), v, dtype, rng.choice((1, 1, 1, 4)),
                      rng.choice((0, 1, 5, 20, 64)), rng.choice((0.0, 0.0, 0.5, 0.99)), pad)
    del c["name"]
    return c


def work(case):
    if case["op"] == "quantize":
        n, rows = case["rows"] * case["d"], case["rows"]
        return {"bytes": n * (SIZE[case["dtype"]] + 1) + 4 * rows + (2 * case["d"] if case["gain"] else 0),
                "flops": n * (7 if case["gain"] else 4)}
    if case["op"] == "linear":
        m, n, k = case["m"], case["n"], case["k"]
        return {"bytes": (m + n) * (k + 4) + m * n * SIZE[case["dtype"]] + (2 * n if case["bias"] else 0),
                "flops": 2 * m * n * k}
    n, rows = case["rows"] * case["vocab"], case["rows"]
    return {"bytes": n * SIZE[case["dtype"]] + rows * (4 + 8 * case["given"] + 8 * case["top"]), "flops": 6 * n}


# ---------------------------------------------------------------------------- inputs

def _wide(rows, cols, pad, dtype):
    """[rows, cols] view of a matrix with `pad` more columns."""
    return torch.empty((rows, cols + pad), dtype=dtype, device="cuda")[:, :cols]


def prepare(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)

    def normal(*shape):
        return torch.randn(shape, generator=gen, device="cuda")

    st = dict(case=case)
    if case["op"] == "quantize":
        rows, d, t = case["rows"], case["d"], TYPES[case["dtype"]]
        x = normal(rows, d)
        if case["gain"]:
            # A residual stream: a few channels are far larger than the rest, and rows differ in size.
            x *= torch.exp(normal(rows, 1)) * (1 + 30 * (torch.rand(d, generator=gen, device="cuda") < 0.003))
            st["gain"] = (1 + 0.1 * normal(d)).to(torch.bfloat16)
        else:
            x *= 0.02
            st["gain"] = None
        st["x"] = _wide(rows, d, case["pad"], t)
        st["x"].copy_(x)
    elif case["op"] == "linear":
        m, n, k = case["m"], case["n"], case["k"]
        st["a"], st["w"] = _wide(m, k, case["pad"], torch.int8), _wide(n, k, case["pad"], torch.int8)
        st["a"].copy_((28 * normal(m, k)).round_().clamp_(-127, 127))
        st["w"].copy_((28 * normal(n, k)).round_().clamp_(-127, 127))
        st["a_scale"] = 0.03 * torch.exp(0.3 * normal(m))
        st["w_scale"] = 0.0007 * torch.exp(0.3 * normal(n))
        st["bias"] = (0.1 * normal(n)).to(torch.bfloat16) if case["bias"] else None
    else:
        rows, v = case["rows"], case["vocab"]
        z = normal(rows, v).mul_(2.5)
        # What a model is sure of: one token stands out, by little in some rows and far in others.
        at = torch.randint(0, v, (rows, 1), generator=gen, device="cuda")
        z.scatter_add_(1, at, 12 * torch.rand((rows, 1), generator=gen, device="cuda"))
        if case["masked"]:
            z.masked_fill_(torch.rand((rows, v), generator=gen, device="cuda") < case["masked"], -math.inf)
        st["logits"] = _wide(rows, v, case["pad"], TYPES[case["dtype"]])
        st["logits"].copy_(z)
        tokens = torch.randint(0, v, (rows, case["given"]), generator=gen, device="cuda", dtype=torch.int32)
        tokens[:, 0] = at[:, 0].to(torch.int32)
        st["tokens"] = tokens
    return st


# ---------------------------------------------------------------------------- plain forms

def _plain_quantize(x, gain):
    # Integers next to a border (127 y / max |y| halfway between two) need 64 bits; the row's
    # reciprocal root mean square scales y and its maximum alike and cancels in them.
    y = x.double()
    r = torch.ones_like(y[:, :1])
    if gain is not None:
        r = 1 / torch.sqrt((y * y).mean(-1, keepdim=True) + EPS)
        y = y * gain.double()
    a = y.abs().amax(-1, keepdim=True)
    q = torch.where(a > 0, 127 * y / a, 0).round().to(torch.int8)
    return {"q": q, "scale": (a * r / 127)[:, 0].float()}


def _plain_linear(a, a_scale, w, w_scale, bias, dtype):
    y = (a.float() @ w.float().T) * (a_scale[:, None] * w_scale)
    if bias is not None:
        y = y + bias.float()
    return {"out": y.to(dtype)}


def _plain_logprobs(logits, tokens, top):
    z = logits.float() + 0.0
    rows, v = z.shape
    m = z.amax(-1, keepdim=True)
    d = z - m
    e = torch.exp(d)
    s = e.sum(-1, keepdim=True)
    log_s = torch.log(s)
    entropy = log_s - torch.where(e > 0, e * d, 0).sum(-1, keepdim=True) / s
    out = {"token": z.gather(1, tokens.long()) - m - log_s, "entropy": entropy[:, 0]}
    if top:
        # One whole number per token, larger where it goes first: the value's order, then the lower index.
        bits = z.view(torch.int32)
        order = (bits ^ ((bits >> 31) & 0x7FFFFFFF)).long() << 32
        best = (order + torch.arange(v - 1, -1, -1, device=z.device)).topk(top, -1).values
        at = v - 1 - (best & 0xFFFFFFFF)
        values = z.gather(1, at)
        out["top"] = values - m - log_s
        out["top_tokens"] = torch.where(values > -math.inf, at, -1).to(torch.int32)
    return out


# ---------------------------------------------------------------------------- one pass

_context = None


def _ctx():
    """The program's one context."""
    global _context
    if _context is None:
        from paper_2608_01785_amd import binding
        _context = binding.hs_context_create(0, (256,))
    return _context


def _buffers(st):
    """The outputs and the workspace that a program keeps from call to call."""
    if "out" in st:
        return st["out"]
    from paper_2608_01785_amd import binding
    case = st["case"]

    def new(shape, dtype):
        return torch.empty(shape, dtype=dtype, device="cuda")

    if case["op"] == "quantize":
        st["out"] = {"q": new((case["rows"], case["d"]), torch.int8), "scale": new(case["rows"], torch.float32)}
    elif case["op"] == "linear":
        st["out"] = {"out": new((case["m"], case["n"]), TYPES[case["dtype"]])}
    else:
        rows, top = case["rows"], case["top"]
        st["out"] = {"token": new((rows, case["given"]), torch.float32), "entropy": new(rows, torch.float32)}
        if top:
            st["out"].update(top=new((rows, top), torch.float32), top_tokens=new((rows, top), torch.int32))
        st["ws"] = new(max(1, binding.hs_logprobs_workspace_size(rows, case["vocab"], top)), torch.uint8)
    torch.cuda.synchronize()
    return st["out"]


def run(st):
    case = st["case"]
    if own:
        from paper_2608_01785_amd import binding
        out = _buffers(st)
        if case["op"] == "quantize":
            binding.hs_quantize_rows(_ctx(), st["x"], out["q"], out["scale"], gain=st["gain"], eps=EPS)
        elif case["op"] == "linear":
            binding.hs_linear_i8(_ctx(), st["a"], st["a_scale"], st["w"], st["w_scale"], out["out"], bias=st["bias"])
        else:
            binding.hs_logprobs(_ctx(), st["logits"], tokens=st["tokens"], token_logprobs=out["token"],
                                entropy=out["entropy"], top_logprobs=out.get("top"),
                                top_tokens=out.get("top_tokens"), workspace=st["ws"])
        return out
    if case["op"] == "quantize":
        return _plain_quantize(st["x"], st["gain"])
    if case["op"] == "linear":
        return _plain_linear(st["a"], st["a_scale"], st["w"], st["w_scale"], st["bias"], TYPES[case["dtype"]])
    return _plain_logprobs(st["logits"], st["tokens"], case["top"])


# ---------------------------------------------------------------------------- 64 bits

def exact(case, seed):
    st = prepare(case, seed)
    if case["op"] == "quantize":
        # RMSNorm as it is defined, then its scale; the integers are compared between the two forms.
        x = st["x"].to(torch.float64)
        if st["gain"] is not None:
            x = x * torch.rsqrt(torch.linalg.vecdot(x, x) / case["d"] + EPS)[:, None] * st["gain"].to(torch.float64)
        return {"q": None, "scale": torch.linalg.vector_norm(x, math.inf, dim=-1) / 127}
    if case["op"] == "linear":
        out = torch.empty((case["m"], case["n"]), dtype=torch.float64, device="cuda")
        a = st["a"].to(torch.float64) * st["a_scale"].to(torch.float64)[:, None]
        for lo in range(0, case["n"], 8192):
            w = st["w"][lo:lo + 8192].to(torch.float64) * st["w_scale"][lo:lo + 8192].to(torch.float64)[:, None]
            out[:, lo:lo + 8192] = torch.nn.functional.linear(a, w)
        return {"out": out if st["bias"] is None else out.add_(st["bias"].to(torch.float64))}
    lp = torch.log_softmax(st["logits"].to(torch.float64), -1)
    p = lp.exp()
    out = {"token": torch.gather(lp, 1, st["tokens"].to(torch.int64)),
           "entropy": -torch.nan_to_num(torch.xlogy(p, p), nan=0.0).sum(-1)}
    if case["top"]:
        out["top"] = torch.topk(lp, case["top"], dim=-1).values
        out["top_tokens"] = None
    return out
