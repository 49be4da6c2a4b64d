"""One element of one value that is not finite, at every place of a head: rows that do not see its key keep their bits, rows that
see it get it in that element alone."""
import numpy as np
import pytest

from tests.test_gpu_cache import _attend, _step

pytestmark = pytest.mark.gpu


# query rows per KV head: 6 the kernel for few rows, 42 and 120 tiles of 64, 210 tiles of 128
@pytest.mark.parametrize("d,hq,new", [(64, 2, 3), (128, 2, 3), (64, 6, 7), (128, 6, 20), (64, 5, 42), (128, 5, 42)])
@pytest.mark.parametrize("value", [float("inf"), -float("inf"), float("nan")])
def test_every_element_of_a_value(d, hq, new, value):
    s = _step([40], [new], hq, 1, d, 16, 1, new)
    s["mask"] = np.array([[1 << i | (1 if i % 2 else 0)] for i in range(new)], dtype=np.uint64)   # odd tokens also see the first one
    clean = _attend(s)
    page, at = int(s["table"][0, 40 // 16]), 40 % 16
    v = s["v"].clone()
    for e in list(range(8)) + [d // 2 + 1, d - 2, d - 1]:
        print(f"[odd] d {d}, rows {hq * new}, {value} in element {e}", flush=True)
        s["v"] = v.clone()
        s["v"][page, at, 0, e] = value
        o, lse = _attend(s)
        assert np.array_equal(lse, clean[1])
        for t in range(new):
            if t == 0 or t % 2:
                assert (o[t, :, e] == value).all() if value == value else np.isnan(o[t, :, e]).all(), t
                assert np.array_equal(np.delete(o[t], e, axis=1), np.delete(clean[0][t], e, axis=1)), t
            else:
                assert np.array_equal(o[t], clean[0][t]), t
