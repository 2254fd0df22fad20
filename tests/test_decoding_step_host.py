"""The decode step behind shared prefixes, without a GPU: what is refused before a context is looked at."""
import ctypes

import numpy as np
import pytest

from tests.test_decoding_host import INVALID, P, UNSUPPORTED, _i32


@pytest.fixture(scope="module")
def b():
    from paper_2608_01785_amd import binding
    binding.lib()
    return binding


def test_a_step_of_more_blocks_than_a_launch_has(b):
    """Refused before any launch, like the attention alone."""
    from paper_2608_01785_amd.workloads import LayerShape
    n = 1 << 22
    shape = LayerShape(hidden=256, n_q_heads=4, n_kv_heads=4, head_dim=64, ffn=128)
    cfg = b.LayerCfg.of(shape)
    w = (b.LayerWeights * 1)()
    for name, kind in b.LayerWeights._fields_:
        if kind is ctypes.c_void_p:
            setattr(w[0], name, P)
    layer = (ctypes.c_void_p * 1)(P)
    table = np.arange(n, dtype=np.int32)
    i32p = ctypes.POINTER(ctypes.c_int32)
    kv = b.KvCache(*(ctypes.cast(layer, ctypes.POINTER(ctypes.c_void_p)),) * 2, n, 64, table.ctypes.data_as(i32p), 1)
    lens = np.zeros(n, np.int32)

    def call(rows):
        st = b.lib().hs_downstream_decode_step_prefix(
            None, ctypes.byref(cfg), w, 1, P, 2 * P, ctypes.byref(kv), lens.ctypes.data_as(i32p), rows, _i32([0, rows]),
            _i32([0]), 1, 128, None, 3 * P, 1 << 40)
        return st, b.hs_last_error()
    st, msg = call(n)
    assert st == UNSUPPORTED and "blocks" in msg, (st, msg)
    st, msg = call(n - 1)
    assert st == INVALID and "context is null" in msg, (st, msg)
