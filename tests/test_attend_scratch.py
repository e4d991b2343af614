"""How much scratch the attention calls say they use, and which device a context's own is on, without a GPU."""
import os
import re
import types

import pytest
import torch

from paper_2509_15038_amd import binding as B


def test_the_constant_covers_every_call():
    header = open(os.path.join(os.path.dirname(os.path.dirname(B.__file__)), "include", "curdkv.h")).read()
    stated = int(re.search(r"#define CURDKV_ATTEND_SCRATCH_BYTES (\d+)", header).group(1))
    assert stated == B.ATTEND_SCRATCH_BYTES
    units, row, counters = 256, 128 * 4 + 2 * 4, 16384
    # prompts: two workgroups of 128 rows a unit; few tokens: two workgroups a unit, and as many items of 16 rows as there are counters
    assert stated >= counters + 2 * units * 128 * row
    assert stated >= counters + (2 * units + counters // 4) * 16 * row
    assert stated >= counters + (2 * units + 2 * 64) * 16 * row        # (up to 64 items, with workgroups of their own)


def test_a_first_call_on_another_device_leaves_no_scratch_behind(monkeypatch):
    # the current device is in `current`; the entry points refuse a context of device 0 elsewhere
    B.lib()                                                             # (binds the module that is replaced below)
    current, made, seen = [1], [], []

    def entry(*a):
        seen.append(a)
        return B.OK if current[0] == 0 else B.ERR_INVALID_ARG

    def zeros(shape, dtype, device):
        made.append(current[0])
        return types.SimpleNamespace(data_ptr=lambda: 1000 + current[0])

    monkeypatch.setattr(B, "_attend", types.SimpleNamespace(expand_mx=entry, attend=entry))
    monkeypatch.setattr(torch, "zeros", zeros)
    monkeypatch.setattr(torch.cuda, "is_current_stream_capturing", lambda: False)
    monkeypatch.setattr(torch.cuda, "current_stream", lambda: types.SimpleNamespace(synchronize=lambda: None))
    ctx = object.__new__(B.Context)
    ctx._address, ctx._h, ctx._own_scratch, ctx._scale = 4321, None, None, 0.25
    call = lambda: ctx.attend(1, 2, 3, 1, 1, 10, 10, 4, stream=0)
    with pytest.raises(B.CurdkvError) as e:
        call()
    assert e.value.code == B.ERR_INVALID_ARG and not made and ctx._own_scratch is None
    current[0] = 0
    call()
    call()
    assert made == [0] and seen[-1][-3:] == (1000, B.ATTEND_SCRATCH_BYTES, 0)
