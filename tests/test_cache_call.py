"""The argument marshalling of the calls that keep a cache at its size, without a GPU (as test_attend_call.py for those around it)."""
import numpy as np
import pytest
import torch

from paper_2509_15038_amd import binding as B
from tests.test_attend_call import calls, context  # noqa: F401  (a fixture)


def test_every_argument_arrives(calls):  # noqa: F811
    t = [torch.zeros(8) for _ in range(13)]
    p = [x.data_ptr() for x in t]
    table, positions, axis = torch.zeros((5, 2, 64)), torch.zeros((3, 6), dtype=torch.int32), np.zeros(64, dtype=np.uint8)
    a, tb, at = axis.__array_interface__["data"][0], table.data_ptr(), positions.data_ptr()
    ctx = context()
    ctx.rotate_axes(t[0], 3, 2, table, positions, axis, t[1], t[2], t[3], 64, starts=t[4], q_weight=t[5], k_weight=t[6], eps=0.5, pairs=True, row_stride=2000, stream=5)
    ctx.rotate_axes(t[0], 3, 2, table, positions, axis, t[1], t[2], t[3], 64)
    ctx.attend_weights(t[0], t[1], t[2], 3, 2, 50, 64, t[3], mass_stride=70, lengths=t[4], window=7, n_sink=4, scale=0.5, decay=0.75, scratch=t[5], stream=5)
    ctx.attend_weights(t[0], t[1], t[2], 3, 2, 50, 64, t[3])
    ctx.evict(t[0], t[1], t[2], 3, 50, 64, 40, t[3])
    ctx.evict(t[0], t[1], t[2], 3, 50, 64, 40, t[3], positions=t[4], lengths=t[5], n_sink=4, recent=8, stream=5)
    ctx.evict(t[0], t[1], t[2], 3, 50, 64, 40, t[3], positions=t[4], mass_out=t[5], positions_out=t[6])
    ctx.evict(t[0], t[1], t[2], 3, 50, 64, 40, t[3], positions=t[4], K_out=t[5], V_out=t[6], out_stride=48)
    ctx.attend_shared(t[0], t[1], t[2], t[3], 1, 4, 2, 30, t[4], K_tail=t[5], V_tail=t[6], tail_n=9, tail_stride=10, tail_lengths=t[7], rows=20, scale=2, lse=t[8])
    ctx.attend_shared(t[0], t[1], t[2], t[3], 1, 4, 2, 30, t[4])
    ctx.attend_shared_mx(t[0], t[1], t[2], t[3], t[4], t[5], 1, 4, 2, 30, t[6], scratch=t[7], stream=5)
    assert calls == [
        ("rotate_axes", [4321, p[0], 3, 2, 2000, p[4], at, 3, a, tb, 5, p[5], p[6], 0.5, 1, p[1], p[2], p[3], 64, 5]),
        ("rotate_axes", [4321, p[0], 3, 2, 1536, 0, at, 3, a, tb, 5, 0, 0, pytest.approx(1e-5), 0, p[1], p[2], p[3], 64, 77]),
        ("attend_weights", [4321, p[0], p[1], p[2], 3, 2, 50, 64, p[4], 7, 4, 0.5, 0.75, p[3], 70, p[5], 32, 5]),
        ("attend_weights", [4321, p[0], p[1], p[2], 3, 2, 50, 64, 0, 0, 0, 0.25, 1.0, p[3], 64, 999, 888, 77]),
        ("evict", [4321, p[0], p[1], p[2], 0, 3, 50, 64, 0, 40, 0, 0, p[0], p[1], p[2], 0, 64, p[3], 77]),
        ("evict", [4321, p[0], p[1], p[2], p[4], 3, 50, 64, p[5], 40, 4, 8, p[0], p[1], p[2], p[4], 64, p[3], 5]),
        ("evict", [4321, p[0], p[1], p[2], p[4], 3, 50, 64, 0, 40, 0, 0, p[0], p[1], p[5], p[6], 64, p[3], 77]),
        ("evict", [4321, p[0], p[1], p[2], p[4], 3, 50, 64, 0, 40, 0, 0, p[5], p[6], 0, 0, 48, p[3], 77]),
        ("attend_shared", [4321, p[0], p[1], p[2], p[3], 30, 20, p[5], p[6], 9, 10, p[7], 1, 4, 2, 2.0, p[4], p[8], 999, 888, 77]),
        ("attend_shared", [4321, p[0], p[1], p[2], p[3], 30, 30, 0, 0, 0, 0, 0, 1, 4, 2, 0.25, p[4], 0, 999, 888, 77]),
        ("attend_shared_mx", [4321, p[0], p[1], p[2], p[3], p[4], p[5], 30, 30, 0, 0, 0, 0, 0, 1, 4, 2, 0.25, p[6], 0, p[7], 32, 5])]


@pytest.mark.parametrize("axis", [np.zeros(63, dtype=np.uint8), np.zeros(64, dtype=np.int32), np.zeros(128, dtype=np.uint8)[::2], [0] * 64])
def test_what_is_no_list_of_axes(calls, axis):  # noqa: F811
    t = torch.zeros(8)
    with pytest.raises(AssertionError):
        context().rotate_axes(t, 1, 1, torch.zeros((5, 2, 64)), torch.zeros((3, 1), dtype=torch.int32), axis, t, t, t, 64)
    assert not calls


def test_no_context():
    B.lib()
    z = [None] * 20
    assert B._attend.rotate_axes(0, None, 1, 1, 1, None, None, 1, *z[:2], 1, None, None, 0.0, 0, *z[:3], 1, 0) == B.ERR_INVALID_ARG
    assert B._attend.attend_weights(0, *z[:3], 1, 1, 1, 1, None, 0, 0, 1.0, 1.0, None, 1, None, 0, 0) == B.ERR_INVALID_ARG
    assert B._attend.evict(0, *z[:4], 1, 1, 1, None, 1, 0, 0, *z[:4], 1, None, 0) == B.ERR_INVALID_ARG
    assert B._attend.attend_shared(0, *z[:4], 0, 0, None, None, 0, 0, None, 1, 1, 1, 1.0, None, None, None, 0, 0) == B.ERR_INVALID_ARG
    assert B._attend.attend_shared_mx(0, *z[:6], 0, 0, None, None, 0, 0, None, 1, 1, 1, 1.0, None, None, None, 0, 0) == B.ERR_INVALID_ARG
