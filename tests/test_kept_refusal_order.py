"""Which error a call of attention over kept rows ends with where more than one thing is wrong: arguments that are no call at all before sizes that are too large, without a GPU."""
import pytest

from paper_2509_15038_amd import binding as B
from tests.test_cache_refusals import BAD, NO, P, call, checks, shared  # noqa: F401  (a fixture)


def kept(L, mx=False):
    a = shared(L, mx)
    a.pop("share")
    return a


@pytest.mark.parametrize("mx", [False, True])
@pytest.mark.parametrize("count", [2 ** 31, 2 ** 40, 2 ** 62])
@pytest.mark.parametrize("wrong", [{"ctx": None}, {"Q": None}, {"out": None}, {"m": 0}, {"tail_n": -1}, {"scale": -1.0}, {"scratch_bytes": -1}, {"out": P + 4}])
def test_wrong_and_too_large(checks, mx, count, wrong):  # noqa: F811
    assert call(checks, "attend_kept_mx" if mx else "attend_kept", kept(checks, mx), count=count, **wrong) == (BAD, 0)
    assert call(checks, "attend_shared_mx" if mx else "attend_shared", shared(checks, mx), count=count, share=2, **wrong) == (BAD, 0)
    assert call(checks, "attend_shared_mx" if mx else "attend_shared", shared(checks, mx), count=3, share=count, **wrong) == (BAD, 0)


@pytest.mark.parametrize("count,share", [(2 ** 31, 1), (2 ** 40, 2 ** 40), (2 ** 62, 4), (1, 2 ** 31), (2 ** 31 - 1, 2)])
def test_too_large_alone(checks, count, share):  # noqa: F811
    assert call(checks, "attend_shared", shared(checks), count=count, share=share) == (NO, 0)
    if share == 1:
        assert call(checks, "attend_kept", kept(checks), count=count) == (NO, 0)


def test_codes_are_the_library_s():
    assert (BAD, NO) == (B.ERR_INVALID_ARG, B.ERR_UNSUPPORTED)
