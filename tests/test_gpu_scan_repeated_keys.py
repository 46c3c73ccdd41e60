"""kvb_scan and kvb_scan_backward where tokens repeat a key with beta = 1 and nothing decays: each token then takes back all that
the one before has put there, and terms of the key's gradient cancel.  Bounds are those of the other tests: the products that only
dK depends on keep 2^-16 of a term, and the terms stay within some two times the sum (fp64 terms of the same inputs, one chunk at a time)."""
import numpy as np
import pytest

from test_gpu_scan_backward import Grads

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("in_dtype, out_dtype", [("f16", "f16"), ("f16", "f32"), ("bf16", "bf16"), ("bf16", "f32"), ("f32", "f32")])
@pytest.mark.parametrize("keys, queries_too", [(1, False), (1, True), (2, False)])
@pytest.mark.parametrize("d", [128, 32])
def test_against_the_recurrence(d, keys, queries_too, in_dtype, out_dtype):
    t = Grads([200, 64], 1, 2, d, in_dtype, seed=20 + keys, g_lo=0.0, out_dtype=out_dtype)
    for i in range(keys):
        t.x["k"][:, i::keys] = t.x["k"][:, i:i + 1]
    if queries_too:
        t.x["q"] = t.x["k"].copy()
    t.x["beta"][:] = 1.0
    t.q, t.k, t.beta = t.pack(t.x["q"]), t.pack(t.x["k"]), t.pack(np.float32(t.x["beta"]), False)
    t.check(*t.scan(out_dtype), *t.expected(), out_dtype)
    t.check_backward()
