"""Eviction from heads whose bitmaps, with the kernel's other arrays, take more LDS than a launch has by itself (64 KB), and from ones right below (curdkv_evict)."""
import pytest

from tests.test_gpu_evict import check

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("n", [160001, 163840, 190656, 190657, 193000, 196608, 196609])
@pytest.mark.parametrize("place", [True, False])
def test_heads_around_64_kb(n, place):
    check("bf16", 1, 1, n, n // 3, 4, 64, place=place, seed=n)
