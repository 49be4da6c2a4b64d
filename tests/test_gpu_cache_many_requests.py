"""Attention of so many requests that a workgroup has several items, many groups of 64 requests apart."""
import numpy as np
import pytest

from tests.test_gpu_cache import _attend, _check, _step

pytestmark = pytest.mark.gpu


# top: what max_new says, and with it the kernel: few rows, tiles of 64, tiles of 128
@pytest.mark.parametrize("hq,hk,top", [(4, 2, 3), (4, 2, 20), (16, 2, 40), (16, 16, 3)])
def test_items_of_many_requests(hq, hk, top):
    rng = np.random.default_rng(hq + top)
    n = 2500
    ctx, new = rng.integers(0, 40, n), rng.integers(0, 3, n)
    new[rng.choice(n, 400, replace=False)] = 0
    new[700:900] = 0                                     # whole groups of 64 without a token
    for r in (5, 640, 1500, n - 1):                      # requests of several chunks among them
        ctx[r], new[r] = 1200, 2
    s = _step(ctx.tolist(), new.tolist(), hq, hk, 64, 16, 1, hq + top)
    print(f"[attn] {n} requests, {hq}/{hk}, max_new {top}", flush=True)
    got = _attend(s, top=top)
    _check(s, got, 64)
