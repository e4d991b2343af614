"""How much scratch the attention calls say they use, without a GPU."""
import os
import re

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
