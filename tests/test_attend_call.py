"""The argument marshalling of the module _attend, and of ctypes where that has not been built, without a GPU: entry points written in Python are
bound in the library's place and record what they are given."""
import ctypes as C
import os
import types

import pytest
import torch

from paper_2509_15038_amd import binding as B

VP = C.c_void_p
TYPES = {}


@pytest.fixture(params=["module", "ctypes"])
def calls(request, monkeypatch):
    L = B.lib()
    seen, kept = [], {}
    for name in B._ATTEND:
        types_of = getattr(L, "curdkv_" + name).argtypes

        def f(*a, name=name, types_of=types_of):
            seen.append((name, [x or 0 if t is VP else x for x, t in zip(a, types_of)]))
            return -1 if name == "expand_mx" else 0
        kept[name] = C.CFUNCTYPE(C.c_int, *types_of)(f)
        kept[name].argtypes = types_of
    by_default = lambda s, usual=B._stream: 77 if s is None else usual(s)
    monkeypatch.setattr(B, "_stream", by_default)
    if request.param == "module":
        if not os.path.exists(B.ATTEND_PATH):
            pytest.skip("not built for this interpreter")
        B._attend.bind(*[C.cast(kept[n], VP).value for n in B._ATTEND], B._ptr, by_default)
    else:
        monkeypatch.setattr(B, "_attend", B._AttendByCtypes(types.SimpleNamespace(**{"curdkv_" + n: f for n, f in kept.items()})))
    yield seen
    monkeypatch.undo()
    B._bind_attend(L)


def context():
    ctx = object.__new__(B.Context)
    ctx.cfg = B.make_config(1, 2, 4, 128, 32, "bf16", 64, 1)
    ctx._address, ctx._h, ctx._own_scratch, ctx._scale, ctx._row = 4321, None, (999, 888), 0.25, 1536
    return ctx


def test_every_argument_arrives(calls):
    t = [torch.zeros(8) for _ in range(12)]
    p = [x.data_ptr() for x in t]
    table = torch.zeros((5, 2, 64))
    ctx = context()
    ctx.rotate(t[0], 3, 2, table, t[1], t[2], t[3], 64, starts=t[4], positions=t[5], q_weight=t[6], k_weight=None, eps=0.5, pairs=True, row_stride=2000, stream=5)
    ctx.rotate(t[0], 3, 2, table, t[1], t[2], t[3], 64)
    ctx.attend(t[0], t[1], t[2], 3, 2, 50, 64, t[3], lengths=t[4], window=7, n_sink=4, scale=0.5, lse=t[5], scratch=t[6], stream=5)
    ctx.attend(t[0], t[1], t[2], 3, 2, 50, 64, t[3])
    ctx.compact_mx(t[0], t[1], 50, t[2], t[3], 2 ** 40, t[4], t[5], t[6], t[7])
    ctx.attend_kept(t[0], t[1], t[2], t[3], 1, 2, 30, t[4], K_tail=t[5], V_tail=t[6], tail_n=9, tail_stride=10, tail_lengths=t[7], rows=20, scale=2, lse=t[8])
    ctx.attend_kept_mx(t[0], t[1], t[2], t[3], t[4], t[5], 1, 2, 30, t[6])
    with pytest.raises(B.CurdkvError):
        ctx.expand_mx(t[0], t[1], 6, t[2], stream=p[3])
    tb = table.data_ptr()
    assert calls == [
        ("rotate", [4321, p[0], 3, 2, 2000, p[4], p[5], tb, 5, p[6], 0, 0.5, 1, p[1], p[2], p[3], 64, 5]),
        ("rotate", [4321, p[0], 3, 2, 1536, 0, 0, tb, 5, 0, 0, pytest.approx(1e-5), 0, p[1], p[2], p[3], 64, 77]),
        ("attend", [4321, p[0], p[1], p[2], 3, 2, 50, 64, p[4], 7, 4, 0.5, p[3], p[5], p[6], 32, 5]),
        ("attend", [4321, p[0], p[1], p[2], 3, 2, 50, 64, 0, 0, 0, 0.25, p[3], 0, 999, 888, 77]),
        ("compact_mx", [4321, p[0], p[1], 50, p[2], p[3], 2 ** 40, p[4], p[5], p[6], p[7], 77]),
        ("attend_kept", [4321, p[0], p[1], p[2], p[3], 30, 20, p[5], p[6], 9, 10, p[7], 1, 2, 2.0, p[4], p[8], 999, 888, 77]),
        ("attend_kept_mx", [4321, p[0], p[1], p[2], p[3], p[4], p[5], 30, 30, 0, 0, 0, 0, 0, 1, 2, 0.25, p[6], 0, 999, 888, 77]),
        ("expand_mx", [4321, p[0], p[1], 6, p[2], p[3]])]


def test_what_is_no_argument(calls):
    t = torch.zeros(8)
    for bad in ("x", [1], 1.5j):
        with pytest.raises((TypeError, ValueError)):
            context().expand_mx(t, t, bad, t)
    with pytest.raises((TypeError, AttributeError)):
        context().expand_mx("x", t, 1, t)
    with pytest.raises(TypeError):
        B._attend.expand_mx(1, 2)
    assert not calls


def test_without_the_module(monkeypatch, tmp_path):
    monkeypatch.setattr(B, "ATTEND_PATH", str(tmp_path / "_attend.none.so"))
    monkeypatch.setattr(B, "_lib", None)
    monkeypatch.setattr(B, "_attend", None)
    B.lib()
    assert isinstance(B._attend, B._AttendByCtypes)
    assert B._attend.expand_mx(0, None, None, 1, None, 0) == B.ERR_INVALID_ARG       # (no context: refused before anything is launched)


def test_no_context():
    B.lib()
    z = [None] * 20
    assert B._attend.rotate(0, None, 1, 1, 1, *z[:3], 1, None, None, 0.0, 0, *z[:3], 1, 0) == B.ERR_INVALID_ARG
    assert B._attend.attend(0, *z[:3], 1, 1, 1, 1, None, 0, 0, 1.0, None, None, None, 0, 0) == B.ERR_INVALID_ARG
    assert B._attend.compact_mx(0, None, None, 1, None, None, 0, *z[:4], 0) == B.ERR_INVALID_ARG
    assert B._attend.attend_kept(0, *z[:4], 0, 0, None, None, 0, 0, None, 1, 1, 1.0, None, None, None, 0, 0) == B.ERR_INVALID_ARG
    assert B._attend.attend_kept_mx(0, *z[:6], 0, 0, None, None, 0, 0, None, 1, 1, 1.0, None, None, None, 0, 0) == B.ERR_INVALID_ARG
