"""The largest numbers of heads that the weights and the eviction take, as the header names them, without a GPU."""
import pytest

from tests.test_cache_refusals import NO, OK, call, checks, evict, weights  # noqa: F401  (a fixture)


@pytest.mark.parametrize("kv,count,n,code", [
    (1, 2 ** 24 - 1, 1, OK), (1, 2 ** 24, 1, NO), (1, 2 ** 24 - 1, 64, OK), (1, 2 ** 24 - 1, 65, NO), (2, 2 ** 20, 7 * 64, OK), (2, 2 ** 20, 7 * 64 + 1, NO), (2 ** 14, 1023, 64, OK),
    (2 ** 14, 1024, 64, NO), (1, 1, 1000, OK)])
def test_weights(checks, kv, count, n, code):  # noqa: F811
    a = dict(weights(checks), ctx=checks.made(kv, 1, 1, 1000, 0))
    assert (-(-n // 64) * count * kv < 2 ** 24) == (code == OK)
    assert call(checks, "attend_weights", a, count=count, m=1, n=n, stride=n, mass_stride=n) == (code, int(code == OK))


@pytest.mark.parametrize("kv,count,code", [(1, 2 ** 20, OK), (1, 2 ** 20 + 1, NO), (2, 2 ** 19, OK), (2, 2 ** 19 + 1, NO), (2 ** 14, 64, OK), (2 ** 14, 65, NO), (3, 349525, OK), (3, 349526, NO)])
def test_evict(checks, kv, count, code):  # noqa: F811
    assert call(checks, "evict", dict(evict(checks), ctx=checks.made(kv, 1, 1, 1000, 0)), count=count) == (code, int(code == OK))
