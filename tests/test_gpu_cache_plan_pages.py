"""sp_cache_plan where the lists hold pages that are none: the slot is -1, positions and masks are those of the token's place."""
import pytest

from tests.test_gpu_cache import _plan_on_gpu

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("in_place", [False, True])
def test_tokens_on_pages_that_are_none(in_place):
    # a request on held pages 3 and -7, one whose fresh page is -2, one that is refused, and a row behind the last token
    got = _plan_on_gpu([14, 16, 99], [4, 2, 1], [2, 1, 1], [[3, -7, 0], [5, 0, 0], [1, 0, 0]], [-2], 1, 16, 8, [-1, 0, 0, 2, -1, -1, -1, -1], 1,
                       in_place)
    assert got["status"].tolist() == [0, 0, 1] and got["seq_len"].tolist() == [18, 18, 0]
    assert got["slots"].tolist() == [62, 63, -1, -1, -1, -1, -1, -1]
    assert got["positions"].tolist() == [14, 15, 15, 16, 16, 16, 0, 0]
    assert got["mask"][:, 0].tolist() == [0b1, 0b11, 0b101, 0b1101, 0b1, 0b10, 0, 0]
    assert got["table"].tolist() == [[3, -7, 0], [5, -2, 0], [1, 0, 0]] and got["n_free"] == 0
