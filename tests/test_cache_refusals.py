"""What the operators that keep a cache at its size refuse, and what reaches their kernels, without a GPU: the checks of arguments (attention/cache_api.hip,
attention/attend_api.hip) built for the CPU alone, with launchers that only count."""
import ctypes as C
import os
import shutil
import subprocess

import numpy as np
import pytest

from paper_2509_15038_amd import binding as B

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
STUBS = r"""
#include "attend_internal.h"
static int current, launches;
extern "C" hipError_t hipGetDevice(int* d) { *d = current; return hipSuccess; }
extern "C" curdkv_ctx* made(int kv, int group, int dtype, long long most, int device) {
    curdkv_ctx* c = new curdkv_ctx();
    c->cfg.kv_heads = kv, c->cfg.group_size = group, c->cfg.dtype = dtype, c->cfg.max_tokens = most, c->device = device, c->num_cu = 256, c->heads = kv;
    return c;
}
extern "C" int launched() { int n = launches; launches = 0; return n; }
namespace curdkv {
hipError_t launch_attend_split(const curdkv_ctx*, const AttendCall&, hipStream_t) { ++launches; return hipSuccess; }
hipError_t launch_attend_prompt(const curdkv_ctx*, const AttendCall&, hipStream_t) { ++launches; return hipSuccess; }
hipError_t launch_attend_prompt_f32(const curdkv_ctx*, const AttendCall&, hipStream_t) { ++launches; return hipSuccess; }
hipError_t launch_rotate(const curdkv_ctx*, const void*, int64_t, int64_t, int64_t, const int32_t*, const int32_t*, const uint8_t*, const float*, int64_t,
                         const void*, const void*, float, bool, void*, void*, void*, int64_t, hipStream_t) { ++launches; return hipSuccess; }
hipError_t launch_compact_mx(const curdkv_ctx*, const void*, const void*, int64_t, const int32_t*, const int64_t*, int64_t, int, uint8_t*, uint8_t*, uint8_t*, uint8_t*,
                             hipStream_t) { ++launches; return hipSuccess; }
hipError_t launch_expand_mx(int, const uint8_t*, const uint8_t*, int64_t, void*, hipStream_t) { ++launches; return hipSuccess; }
hipError_t launch_weights(const curdkv_ctx*, const WeightsCall&, hipStream_t) { ++launches; return hipSuccess; }
hipError_t launch_evict(const curdkv_ctx*, const EvictCall&, hipStream_t) { ++launches; return hipSuccess; }
hipError_t launch_attend_shared(const curdkv_ctx*, const AttendCall&, int, hipStream_t) { ++launches; return hipSuccess; }
}
"""
BAD, NO, OK = B.ERR_INVALID_ARG, B.ERR_UNSUPPORTED, B.OK


@pytest.fixture(scope="module")
def checks(tmp_path_factory):
    gxx = shutil.which("g++")
    if gxx is None or not os.path.isdir("/opt/rocm/include"):
        pytest.skip("needs g++ and the HIP headers")
    at = tmp_path_factory.mktemp("checks")
    (at / "stubs.cpp").write_text(STUBS)
    pkg = os.path.join(ROOT, "paper_2509_15038_amd")
    subprocess.run([gxx, "-std=c++17", "-O1", "-shared", "-fPIC", "-w", "-D__HIP_PLATFORM_AMD__", "-I", os.path.join(ROOT, "include"), "-I", os.path.join(pkg, "csrc"),
                    "-I", os.path.join(pkg, "attention"), "-I", "/opt/rocm/include", "-x", "c++", str(at / "stubs.cpp"), os.path.join(pkg, "attention", "cache_api.hip"),
                    os.path.join(pkg, "attention", "attend_api.hip"), "-o", str(at / "checks.so")], check=True)
    L = C.CDLL(str(at / "checks.so"))
    L.made.restype, L.made.argtypes = C.c_void_p, [C.c_int] * 3 + [C.c_longlong, C.c_int]
    for name in B._ATTEND:
        getattr(L, "curdkv_" + name).argtypes = getattr(B.lib(), "curdkv_" + name).argtypes
    return L


def call(L, name, given, **changed):
    a = dict(given, **changed)
    return getattr(L, "curdkv_" + name)(*a.values()), L.launched()


P = 0x10000                                         # an address that nothing is read from
AXIS = np.arange(64, dtype=np.uint8) % 3


def axes(L, dtype=1):
    return dict(ctx=L.made(2, 4, dtype, 1000, 0), qkv=P, count=2, m=3, row_stride=12 * 128, starts=None, positions=P, axes=3, axis_of=AXIS.ctypes.data, table=P, table_rows=10,
                q_weight=None, k_weight=None, eps=1e-5, pairs=0, Q=P, K=P, V=P, stride=50, stream=None)


def weights(L):
    return dict(ctx=L.made(2, 4, 1, 1000, 0), Q=P, K=P, lse=P, count=2, m=3, n=40, stride=50, lengths=None, window=0, n_sink=0, scale=0.1, decay=1.0, mass=P, mass_stride=40,
                scratch=None, scratch_bytes=0, stream=None)


def evict(L):
    return dict(ctx=L.made(2, 4, 1, 1000, 0), K=P, V=2 * P, mass=3 * P, positions=4 * P, count=2, n=40, stride=50, lengths=None, keep=30, n_sink=4, recent=8, K_out=P, V_out=2 * P,
                mass_out=3 * P, positions_out=4 * P, out_stride=50, rows=5 * P, stream=None)


def shared(L, mx=False):
    kept = dict(K=P, Ks=P, V=P, Vs=P) if mx else dict(K=P, V=P)
    return dict(ctx=L.made(2, 4, 1, 1000, 0), Q=P, **kept, offsets=P, total=100, rows=100, K_tail=P, V_tail=P, tail_n=40, tail_stride=50, tail_lengths=None, count=2, share=3, m=1,
                scale=0.1, out=P, lse=None, scratch=P, scratch_bytes=B.ATTEND_SCRATCH_BYTES, stream=None)


@pytest.mark.parametrize("change,code", [
    ({}, OK), ({"axes": 4}, OK), ({"q_weight": P, "eps": 0.0}, OK), ({"table_rows": 1}, OK),
    ({"ctx": None}, BAD), ({"qkv": None}, BAD), ({"positions": None}, BAD), ({"axis_of": None}, BAD), ({"table": None}, BAD), ({"Q": None}, BAD), ({"K": None}, BAD), ({"V": None}, BAD),
    ({"axes": 0}, BAD), ({"axes": 2}, BAD), ({"axes": 5}, BAD), ({"axes": -1}, BAD), ({"count": 0}, BAD), ({"m": 0}, BAD), ({"row_stride": 12 * 128 - 8}, BAD),
    ({"row_stride": 12 * 128 + 4}, BAD), ({"stride": 0}, BAD), ({"stride": 1001}, BAD), ({"table_rows": 0}, BAD), ({"pairs": 2}, BAD), ({"k_weight": P, "eps": -1.0}, BAD),
    ({"k_weight": P, "eps": float("nan")}, BAD), ({"K": P + 8}, BAD), ({"table": P + 4}, BAD), ({"m": 2 ** 30}, NO)])
def test_axes(checks, change, code):
    assert call(checks, "rotate_axes", axes(checks), **change) == (code, int(code == OK))


@pytest.mark.parametrize("change,code", [
    ({}, OK), ({"decay": 0.0}, OK), ({"window": 7, "n_sink": 100}, OK), ({"m": 41}, OK), ({"mass_stride": 2 ** 40}, OK), ({"count": 1, "stride": 2 ** 40}, OK),
    ({"ctx": None}, BAD), ({"Q": None}, BAD), ({"K": None}, BAD), ({"lse": None}, BAD), ({"mass": None}, BAD), ({"count": 0}, BAD), ({"m": 0}, BAD), ({"m": 1001}, BAD), ({"n": 0}, BAD),
    ({"n": 1001, "stride": 1001, "mass_stride": 1001}, BAD), ({"stride": 39}, BAD), ({"mass_stride": 39}, BAD), ({"window": -1}, BAD), ({"n_sink": -1}, BAD), ({"scale": 0.0}, BAD),
    ({"scale": float("inf")}, BAD), ({"decay": -0.5}, BAD), ({"decay": float("nan")}, BAD), ({"decay": float("inf")}, BAD), ({"Q": P + 8}, BAD), ({"K": P + 8}, BAD),
    ({"scratch_bytes": -1}, BAD), ({"scratch": P + 4}, BAD), ({"count": 2 ** 28}, NO), ({"count": 2 ** 24, "m": 1}, NO)])
def test_weights(checks, change, code):
    assert call(checks, "attend_weights", weights(checks), **change) == (code, int(code == OK))


@pytest.mark.parametrize("change,code", [
    ({}, OK), ({"positions": None, "positions_out": None}, OK), ({"mass_out": None, "positions_out": None}, OK), ({"mass_out": 6 * P, "positions_out": 7 * P}, OK),
    ({"K_out": 6 * P, "V_out": 7 * P, "mass_out": None, "positions_out": None, "out_stride": 30}, OK), ({"keep": 1, "n_sink": 0, "recent": 1}, OK),
    ({"keep": 60, "K_out": 6 * P, "V_out": 7 * P, "mass_out": None, "positions_out": None, "out_stride": 40}, OK), ({"n_sink": 15, "recent": 15}, OK),
    ({"ctx": None}, BAD), ({"K": None}, BAD), ({"V": None}, BAD), ({"mass": None}, BAD), ({"K_out": None}, BAD), ({"V_out": None}, BAD), ({"rows": None}, BAD), ({"count": 0}, BAD),
    ({"n": 0}, BAD), ({"n": 51}, BAD), ({"n": 1001, "stride": 1001, "out_stride": 1001}, BAD), ({"keep": 0, "n_sink": 0, "recent": 0}, BAD), ({"n_sink": -1}, BAD), ({"recent": -1}, BAD),
    ({"n_sink": 23}, BAD), ({"recent": 31, "n_sink": 0}, BAD), ({"out_stride": 60}, BAD), ({"K_out": 6 * P}, BAD), ({"V_out": 6 * P}, BAD), ({"K_out": 2 * P, "V_out": P}, BAD),
    ({"K_out": 6 * P, "V_out": 6 * P, "mass_out": None, "positions_out": None}, BAD), ({"K_out": 6 * P, "V_out": 7 * P, "out_stride": 60}, BAD),
    ({"K_out": 6 * P, "V_out": 7 * P, "mass_out": None, "out_stride": 60}, BAD), ({"K_out": 6 * P, "V_out": 7 * P, "mass_out": None, "positions_out": None, "out_stride": 29}, BAD),
    ({"K_out": 6 * P + 8, "V_out": 7 * P, "mass_out": None, "positions_out": None}, BAD), ({"count": 2 ** 21}, NO)])
def test_evict(checks, change, code):
    assert call(checks, "evict", evict(checks), **change) == (code, int(code == OK))


def test_evict_of_long_heads(checks):
    a = evict(checks)
    a["ctx"] = checks.made(2, 4, 1, 2 ** 21, 0)
    assert call(checks, "evict", a, n=2 ** 19, stride=2 ** 20, out_stride=2 ** 20) == (OK, 1)
    assert call(checks, "evict", a, n=2 ** 19 + 1, stride=2 ** 20, out_stride=2 ** 20) == (NO, 0)


@pytest.mark.parametrize("mx", [False, True])
@pytest.mark.parametrize("change,code", [
    ({}, OK), ({"share": 1}, OK), ({"total": 0, "rows": 0, "K": None, "V": None}, OK), ({"tail_n": 0, "tail_stride": 0, "K_tail": None, "V_tail": None}, OK), ({"m": 5000}, OK), ({"lse": P}, OK),
    ({"ctx": None}, BAD), ({"Q": None}, BAD), ({"out": None}, BAD), ({"K": None}, BAD), ({"V": None}, BAD), ({"offsets": None}, BAD), ({"K_tail": None}, BAD), ({"V_tail": None}, BAD),
    ({"count": 0}, BAD), ({"share": 0}, BAD), ({"share": -1}, BAD), ({"m": 0}, BAD), ({"total": -1, "rows": -1}, BAD), ({"rows": 101}, BAD), ({"rows": -1}, BAD), ({"tail_n": -1}, BAD), ({"tail_n": 51}, BAD),
    ({"tail_n": 1001, "tail_stride": 2000}, BAD), ({"scale": -1.0}, BAD), ({"scratch": None}, BAD), ({"scratch_bytes": B.ATTEND_SCRATCH_BYTES - 1}, BAD), ({"scratch": P + 8}, BAD),
    ({"K": P + 8}, BAD), ({"V_tail": P + 8}, BAD), ({"total": 2 ** 31}, NO), ({"share": 2 ** 31}, NO), ({"m": 2 ** 29}, NO), ({"share": 2 ** 27}, NO)])
def test_shared(checks, mx, change, code):
    assert call(checks, "attend_shared_mx" if mx else "attend_shared", shared(checks, mx), **change) == (code, int(code == OK))


def test_shared_scales_and_heads(checks):
    a = shared(checks, True)
    assert call(checks, "attend_shared_mx", a, Ks=None) == (BAD, 0) and call(checks, "attend_shared_mx", a, Vs=None) == (BAD, 0)
    assert call(checks, "attend_shared_mx", a, Ks=None, Vs=None, total=0, rows=0) == (OK, 1)
    for kv, group, code in ((128, 128, OK), (128, 129, NO), (1024, 16, OK), (1025, 1, NO), (1, 2 ** 14, OK), (1, 2 ** 14 + 1, NO)):
        assert call(checks, "attend_shared", dict(shared(checks), ctx=checks.made(kv, group, 1, 1000, 0))) == (code, int(code == OK)), (kv, group)


def test_numbers_of_heads_and_rows_at_their_ends(checks):
    for kv, group, code in ((1, 2 ** 20, OK), (1, 2 ** 20 + 1, NO), (2 ** 14, 64, OK), (2 ** 14, 65, NO), (2 ** 14 + 1, 1, NO)):
        assert call(checks, "attend_weights", dict(weights(checks), ctx=checks.made(kv, group, 1, 1000, 0)), count=1, m=1) == (code, int(code == OK)), (kv, group)
    place = dict(K_out=6 * P, V_out=7 * P, mass_out=None, positions_out=None)
    assert call(checks, "evict", evict(checks), keep=2 ** 30, **place) == (OK, 1)
    assert call(checks, "evict", evict(checks), keep=2 ** 30 + 1, **place) == (NO, 0)


def test_another_device_than_the_current_one(checks):
    for name, given in (("rotate_axes", axes(checks)), ("attend_weights", weights(checks)), ("evict", evict(checks)), ("attend_shared", shared(checks)), ("attend_shared_mx", shared(checks, True))):
        assert call(checks, name, given, ctx=checks.made(2, 4, 1, 1000, 1)) == (BAD, 0), name
