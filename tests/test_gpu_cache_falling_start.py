"""Attention where tok_start falls: requests are looked up 64 at a time, and those before the group of the fall are as ever."""
import numpy as np
import pytest

from tests.test_gpu_cache import _attend, _i32, _step

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("hq,new", [(2, 1), (2, 12)])
@pytest.mark.parametrize("falls", [64, 65, 100, 127, 129])
def test_requests_before_the_group_of_a_fall(hq, new, falls):
    import torch
    import paper_2505_19578_amd as sp
    n, d = 130, 64
    rng = np.random.default_rng(falls)
    ctx = rng.integers(0, 60, n)
    ctx[3] = 1500                                        # one of several chunks
    s = _step(ctx.tolist(), [new] * n, hq, 1, d, 16, 0, falls)
    want = _attend(s)
    start = s["start"].copy()
    start[falls + 1] = start[falls] - 1                  # request `falls` has fewer than no tokens
    q, k, v, table = s["q"].cuda(), s["k"].cuda(), s["v"].cuda(), _i32(s["table"])
    o = torch.full((n * new + 1, hq, d), 5.0, dtype=torch.bfloat16, device="cuda")
    shape, cache = sp.step_shape_of(q, o[:-1], table, new), sp.cache_shape_of(k)
    ws = torch.empty(sp.sp_cache_attn_workspace_bytes(shape, cache) + 256, dtype=torch.uint8, device="cuda")
    print(f"[attn] falls at {falls}", flush=True)
    sp.sp_cache_attn(shape, cache, q, k, v, table, _i32(s["seq"]), _i32(start), None, o[:-1], None, ws)
    torch.cuda.synchronize()
    fine = falls // 64 * 64 * new                        # rows of the requests before the group
    assert np.array_equal(o[:fine].float().cpu().numpy(), want[0][:fine])
    assert (o[-1] == 5).all()
