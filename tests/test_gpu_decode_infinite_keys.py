"""Decode steps on a cache that holds keys whose score is -inf: their weight is zero.

A bias of the queries in the dimension that rotates least makes them positive there, so that a key of -inf in it has a
score of -inf with every query.  Such keys fill whole tiles, ranges and all but the last positions of a sequence.
"""
import math

import numpy as np
import pytest

from oracle import layer as ref
from paper_2608_01785_amd import workloads as W
from tests.gpu_common import TOL, err_ratio, log, require_gpu
from tests.util import f64, h64, weights_f64

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def env():
    torch = require_gpu()
    from paper_2608_01785_amd import binding
    ctx = binding.Context(0, budgets=(128,))
    yield torch, binding, ctx
    torch.cuda.synchronize()
    ctx.close()


KV_LENS = [40, 200, 700, 2100, 3000, 64]
HIDDEN = [(0, 33), (0, 190), (100, 600), (0, 1100), (0, 2995), (0, 64)]


@pytest.mark.parametrize("call", ["slots", "pages", "noalloc", "prefixes"])
@pytest.mark.parametrize("shape", [W.TALKER, W.THINKER_MIXED], ids=["64", "128"])
def test_decode_step_with_keys_at_minus_infinity(env, shape, call):
    torch, b, ctx = env
    from paper_2608_01785_amd.device_data import DeviceCache, PagedCache, to_device, upload_weights
    log(f"[infinite keys] head size {shape.head_dim}, {call}")
    n, top, page, dh = len(KV_LENS), 3328, 256, shape.head_dim
    kv_lens, d = np.array(KV_LENS, np.int32), dh // 2 - 1
    layers = W.make_weights(shape, 1, 51)
    bias = np.zeros((shape.n_q_heads + 2 * shape.n_kv_heads, dh), np.float32)
    bias[:shape.n_q_heads, d] = 20.0
    layers[0]["b_qkv"] = W.bf16_bits(bias.reshape(-1))
    x = W.token_rows(52, n, shape.hidden)
    prefix = W.make_cache(shape, 1, kv_lens, seed=53)
    for k, (first, last) in zip(prefix.k[0], HIDDEN):
        k[first:last, :, d] = W.f16_bits(np.full(1, -math.inf, np.float32))[0]
    expect, _ = ref.decode_step(f64(x), weights_f64(layers), shape, kv_lens, [[h64(k) for k in prefix.k[0]]],
                                [[h64(v) for v in prefix.v[0]]])
    assert np.all(np.isfinite(expect))
    dims = dict(n_kv_heads=shape.n_kv_heads, head_dim=dh, fill=float("nan"))
    if call in ("pages", "prefixes"):
        table = np.random.default_rng(54).permutation(n * top // page).reshape(n, -1)
        cache = PagedCache(1, n * top // page, page, table=table, **dims)
    else:
        cache = DeviceCache(1, n, top, **dims)
    for i in range(n):
        cache.load_prefix(0, i, prefix.k[0][i], prefix.v[0][i])
    w, xd = upload_weights(layers), to_device(x)
    y = torch.full(xd.shape, float("nan"), dtype=torch.float32, device="cuda")
    size = b.hs_workspace_size_prefix(shape, n, top, page, 3000, 3000) if call == "prefixes" else \
        b.hs_workspace_size_paged(shape, n, n, top, page if call == "pages" else 0)
    ws = torch.empty(size, dtype=torch.uint8, device="cuda")
    torch.cuda.synchronize()
    if call == "noalloc":
        b.hs_downstream_decode_step_noalloc(ctx, shape, w, xd, y, cache.as_arg(), kv_lens, 128)
    elif call == "prefixes":
        b.hs_downstream_decode_step_prefix(ctx, shape, w, xd, y, cache.as_arg(), kv_lens, list(range(n + 1)),
                                           [0, 150, 512, 1000, 2990, 64], 128, None, ws)
    else:
        b.hs_downstream_decode_step(ctx, shape, w, xd, y, cache.as_arg(), kv_lens, 128, None, ws)
    torch.cuda.synchronize()
    err = err_ratio(y.cpu().numpy(), expect)
    log(f"  max err / rms = {err:.2e}")
    assert err <= TOL
