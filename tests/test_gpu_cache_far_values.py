"""Values that are not finite at keys that a row sees, far below its largest weight: e^x is small and not zero, so they come out as the
sum says, wherever in the split of the work the key lies."""
import numpy as np
import pytest

from tests.test_gpu_cache import _attend, _check, _step

pytestmark = pytest.mark.gpu


# query rows per KV head: 1 and 8 the kernel for few rows, 40 and 100 tiles of 64, 240 tiles of 128
@pytest.mark.parametrize("hq,new", [(1, 1), (2, 4), (4, 10), (4, 25), (4, 60)])
@pytest.mark.parametrize("value", [float("inf"), -float("inf"), float("nan")])
@pytest.mark.parametrize("ctx", [100, 1500])
def test_an_infinite_value_far_below_the_largest_weight(hq, new, value, ctx):
    """Keys of one score but for one, which is 110 higher: 2^-159 of it is below what 32 bits hold and above what 64 do.  The high
    one lies before and behind the infinite value: in the same run of keys, in another wavefront's, in another chunk's."""
    import torch
    d, page = 64, 16
    s = _step([ctx], [new], hq, 1, d, page, 0, 5)
    s["q"][:] = 1.0

    def put(pos, key=None, val=None, at=None):
        e = int(s["table"][0, pos // page]), pos % page, 0
        if key is not None:
            s["k"][e] = key
        if val is not None:
            s["v"][e][at] = val

    for low, high in ((3, 40), (3, 5), (40, 3), (3, 99), (90, 2), (ctx // 2, ctx - 1), (5, ctx - 1), (ctx - 3, 7), (ctx - 40, ctx - 2)):
        s["k"][:], s["v"][:] = 0.25, torch.randn(s["v"].shape, generator=torch.Generator().manual_seed(7)).to(torch.bfloat16)
        put(high, key=0.25 + 110 / 8)        # 64 products of 1 x that, times 1 / 8
        put(low, val=value, at=11)
        print(f"[far] rows {hq * new}, value {value}, low {low}, high {high}", flush=True)
        got = _attend(s)
        _check(s, got, d)
        assert (got[0][:, :, 11] == value).all() if value == value else np.isnan(got[0][:, :, 11]).all()
        assert np.isfinite(np.delete(got[0], 11, axis=2)).all()


@pytest.mark.parametrize("hq,new", [(2, 1), (4, 10), (4, 60)])
def test_a_row_of_scores_of_minus_infinity_alone(hq, new):
    """An infinite query against keys of the other sign: every weight is e^-inf, and the row is as one that sees no key."""
    s = _step([1500], [new], hq, 1, 64, 16, 0, 5)
    s["k"][..., 3] = -s["k"][..., 3].abs() - 1
    clean = _attend(s)
    s["q"][0, 1, 3] = float("inf")
    got = _attend(s)
    assert (got[0][0, 1] == 0).all() and np.isneginf(got[1][0, 1])
    for a, b in zip(got, clean):
        a[0, 1] = b[0, 1]
        assert np.array_equal(a, b)
