"""A token whose lse is -infinity gives nothing to any key (curdkv_attend_weights), whatever its queries and the keys hold, in every kernel."""
import math

import pytest
import torch

from tests.test_gpu_weights import check

pytestmark = pytest.mark.gpu

# few rows, of one and of two tiles; up to 128 rows; many, by shares of the products and by tiles of keys; fp32
SIZES = [("bf16", 1, 500), ("bf16", 2, 65), ("bf16", 8, 3000), ("bf16", 32, 9001), ("bf16", 300, 300), ("bf16", 1000, 1000), ("bf16", 100, 5000), ("bf16", 700, 3001), ("fp32", 1, 500), ("fp32", 8, 900),
         ("fp32", 150, 700), ("fp32", 700, 701)]


def some(m):
    """The first token, the last, and a few between, of which some stages of 128 rows have one and some none."""
    return sorted({t for t in (0, m - 1, m // 2, m // 2 + 1, m // 3, (m * 9) // 10) if t < m})


@pytest.mark.parametrize("dtype,m,n", SIZES)
@pytest.mark.parametrize("value", [math.nan, math.inf])
@pytest.mark.parametrize("window,sinks", [(0, 0), (300, 5)])
def test_tokens_left_out(dtype, m, n, value, window, sinks):
    # tokens that a program leaves out, as the padding of a batch: their queries may be anything
    def spoil(Q, K, lse):
        for t in some(m):
            Q[0, t] = value
            lse[0, :, t] = -math.inf
    got = check(dtype, 2, 2, 4, m, n, window, sinks, decay=0.5, lengths=[n, n], seed=m, spoil=spoil)
    assert not bool(got.isnan().any())


@pytest.mark.parametrize("dtype,m,n", SIZES)
def test_keys_that_only_such_tokens_see(dtype, m, n):
    def spoil(Q, K, lse):
        K[0, 0, [0, n // 4, n - 1]] = math.nan
        K[0, 1, n // 3, 5] = math.inf
        lse[0] = -math.inf
    got = check(dtype, 1, 2, 4, m, n, lengths=[n], seed=n, spoil=spoil)
    assert not bool(got.isnan().any())


@pytest.mark.parametrize("group", [1, 3, 40])
def test_one_query_head_of_a_token(group):
    def spoil(Q, K, lse):
        for t in (0, 257, 600, 799):
            Q[0, t, group - 1] = math.nan
            lse[0, group - 1, t] = -math.inf
    got = check("bf16", 1, 2, group, 800, 800, decay=0.0, lengths=[800], seed=group, spoil=spoil)
    assert not bool(got.isnan().any())


def test_nothing_is_hidden_of_others():
    # a NaN in a token that does count still reaches the keys that it sees, beside one that does not
    def spoil(Q, K, lse):
        Q[0, 500, 0, 7] = math.nan
        Q[0, 501] = math.nan
        lse[0, :, 501] = -math.inf
    got = check("bf16", 1, 2, 4, 800, 800, lengths=[800], seed=9, spoil=spoil)
    assert int(got[0, 0].isnan().sum()) == 501 and not bool(got[0, 1].isnan().any())


def test_by_tiles_of_keys_without_scratch():
    def spoil(Q, K, lse):
        Q[0, [40, 900]] = math.nan
        lse[0, :, [40, 900]] = -math.inf
    got = check("bf16", 2, 2, 4, 1000, 1000, lengths=[1000, 1000], seed=11, spoil=spoil, scratch=torch.zeros((0,), dtype=torch.uint8, device="cuda"))
    assert not bool(got.isnan().any())
