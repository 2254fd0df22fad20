"""The text head's bookkeeping without a GPU: buffers, passes and refusals (no kernel runs)."""
import pytest
import torch

from paper_2608_01785_amd import answer, binding


class Ctx:
    handle, device = None, -1   # CPU tensors report device -1


def _head(**kw):
    w = torch.zeros(50, 8, dtype=torch.int8), torch.zeros(50)
    return answer.AnswerHead(Ctx, torch.ones(8, dtype=torch.bfloat16), w, **kw)


def test_buffers_and_sharing():
    head = _head(max_rows=3, top_k=4, logits=torch.bfloat16)
    assert (head.vocab, head.hidden) == (50, 8) and head.logits.shape == (3, 50)
    out = head.outputs(7, 2)
    assert out.token_logprobs.shape == (7, 2) and out.entropy.shape == (7,)
    assert out.top_logprobs.shape == out.top_tokens.shape == (7, 4) and out.top_tokens.dtype == torch.int32
    assert head.outputs(7).token_logprobs is None
    other = head.sharing(max_rows=5, top_k=0)
    assert other.w is head.w and other.w_scale is head.w_scale and other.logits.dtype == torch.bfloat16
    assert other.logits.shape == (5, 50) and other.outputs(1).top_tokens is None


def test_passes_cover_every_row_once(monkeypatch):
    calls = []
    monkeypatch.setattr(binding, "hs_quantize_rows", lambda ctx, x, q, s, g, eps, cus, st: calls.append(
        ("q", tuple(x[:, 0].tolist()), q.shape, s.shape, cus, st)))
    monkeypatch.setattr(binding, "hs_linear_i8", lambda ctx, a, sa, w, sw, out, bias, cus, st: calls.append(
        ("l", a.shape, out.shape)))
    monkeypatch.setattr(binding, "hs_logprobs", lambda ctx, z, tokens, **kw: calls.append(
        ("p", z.shape, None if tokens is None else tuple(tokens[:, 0].tolist()), sorted(kw), kw["entropy"].shape)))
    head = _head(max_rows=3, top_k=2)
    y, tokens = torch.arange(7.0)[:, None].repeat(1, 8), torch.arange(7, dtype=torch.int32)[:, None]
    out = head.outputs(7, 1)
    head(y, out, tokens, cu_budget=128, stream=5)
    assert [c[1] for c in calls if c[0] == "q"] == [(0, 1, 2), (3, 4, 5), (6,)]
    assert all(c[4:] == (128, 5) for c in calls if c[0] == "q")
    assert [c[2] for c in calls if c[0] == "p"] == [(0, 1, 2), (3, 4, 5), (6,)]
    assert [tuple(c[4]) for c in calls if c[0] == "p"] == [(3,), (3,), (1,)]
    assert calls[2][3] == ["cu_budget", "entropy", "stream", "token_logprobs", "top_logprobs", "top_tokens", "workspace"]
    calls.clear()
    head(y[:0], head.outputs(0))
    assert not calls


def test_refusals():
    head = _head(max_rows=3, top_k=2)
    y, out = torch.zeros(4, 8), head.outputs(4)
    with pytest.raises(ValueError, match="expected"):
        head(y[0], out)
    with pytest.raises(ValueError, match="expected"):
        head(torch.zeros(4, 9), out)
    with pytest.raises(ValueError, match="rows"):
        head(y[:2], out)
    with pytest.raises(ValueError, match="tokens has 3 rows"):
        head(y, out, torch.zeros(3, 1, dtype=torch.int32))
    with pytest.raises(ValueError, match="max_rows"):
        _head(max_rows=0)
    with pytest.raises(binding.HorizonError, match="top_k 65"):
        _head(top_k=65)
    with pytest.raises(binding.HorizonError, match="context is null"):
        head(y, out)


def test_tensors_without_rows_are_refused():
    head = _head(max_rows=3, top_k=2)
    y, out = torch.zeros(4, 8), head.outputs(4)
    with pytest.raises(ValueError, match="tokens has no rows, y 4"):
        head(y, out, torch.tensor(1, dtype=torch.int32))
    out.entropy = torch.tensor(0.0)
    with pytest.raises(ValueError, match="entropy has no rows, y 4"):
        head(y, out)
