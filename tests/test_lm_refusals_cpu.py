"""Argument errors of the gated linear recurrence, the gated feed-forward
product and the 4-bit product: reported before any CUDA call, so they need no
GPU."""
import ctypes

import pytest

from paper_1810_09958_gb300 import build, isam

BAD, NO = isam.ISAM_ERR_INVALID_ARG, isam.ISAM_ERR_UNSUPPORTED
P = ctypes.c_void_p(256)
BIG = 2 ** 31 - 1


def off(n):
    return ctypes.c_void_p(256 + n)


@pytest.fixture(scope="module")
def lib():
    build.build()
    return isam.load()


@pytest.mark.parametrize("change,code", [
    (dict(T=0), BAD), (dict(batch=0), BAD), (dict(hidden=-1), BAD), (dict(g_type=2), BAD), (dict(h_type=-1), BAD),
    (dict(g=None), BAD), (dict(h=None), BAD), (dict(g=off(2)), NO), (dict(h=off(1)), NO), (dict(h0=off(2)), NO),
    (dict(lengths=off(2)), NO), (dict(last=off(2)), NO), (dict(T=BIG, batch=BIG, hidden=BIG), NO),
    (dict(T=2 ** 20, batch=2 ** 10, hidden=2 ** 10), NO),
])
def test_glr_forward(lib, change, code):
    a = dict(T=4, batch=2, hidden=8, g_type=0, g=P, h0=P, lengths=P, h_type=1, h=P, last=P) | change
    assert lib.isam_glr_forward(a["T"], a["batch"], a["hidden"], a["g_type"], a["g"], a["h0"], a["lengths"],
                                a["h_type"], a["h"], a["last"]) == code
    assert b"isam_glr_forward" in lib.isam_last_error_string()


@pytest.mark.parametrize("change,code", [
    (dict(T=0), BAD), (dict(g=None), BAD), (dict(h=None), BAD), (dict(dg=None), BAD), (dict(g_type=7), BAD),
    (dict(dg=off(2)), NO), (dict(dh=off(1)), NO), (dict(dlast=off(1)), NO), (dict(dh0=off(3)), NO),
])
def test_glr_backward(lib, change, code):
    a = dict(T=4, batch=2, hidden=8, g_type=0, g=P, h0=P, lengths=None, h_type=1, h=P, dh=P, dlast=P, dg=P,
             dh0=P) | change
    assert lib.isam_glr_backward(a["T"], a["batch"], a["hidden"], a["g_type"], a["g"], a["h0"], a["lengths"],
                                 a["h_type"], a["h"], a["dh"], a["dlast"], a["dg"], a["dh0"]) == code
    assert b"isam_glr_backward" in lib.isam_last_error_string()


@pytest.mark.parametrize("change,code", [
    (dict(batch=0), BAD), (dict(slots=0), BAD), (dict(state=None), BAD), (dict(new=None), BAD), (dict(g=None), BAD),
    (dict(h=None), BAD), (dict(ids=None, slots=2), BAD), (dict(ids=off(2)), NO), (dict(state=off(2)), NO),
    (dict(new=off(2)), NO),
])
def test_glr_step(lib, change, code):
    a = dict(batch=3, hidden=8, slots=4, g_type=1, g=P, ids=P, state=P, new=P, h_type=0, h=P) | change
    assert lib.isam_glr_step(a["batch"], a["hidden"], a["slots"], a["g_type"], a["g"], a["ids"], a["state"], a["new"],
                             a["h_type"], a["h"]) == code
    assert b"isam_glr_step" in lib.isam_last_error_string()


@pytest.mark.parametrize("change,code", [
    (dict(T=0), BAD), (dict(D=0), BAD), (dict(F=0), BAD), (dict(act=4), BAD), (dict(act=-1), BAD), (dict(x=None), BAD),
    (dict(W=None), BAD), (dict(h=None), BAD), (dict(D=12), NO), (dict(x=off(8)), NO), (dict(W=off(2)), NO),
    (dict(h=off(1)), NO), (dict(F=2 ** 30), NO),
])
def test_glu_forward(lib, change, code):
    a = dict(T=4, D=16, F=8, act=0, x=P, W=P, h=P) | change
    assert lib.isam_glu_forward(a["T"], a["D"], a["F"], a["act"], a["x"], a["W"], a["h"]) == code
    assert b"isam_glu_forward" in lib.isam_last_error_string()


@pytest.mark.parametrize("change,code", [
    (dict(T=0), BAD), (dict(act=9), BAD), (dict(dh=None), BAD), (dict(ws=None), BAD), (dict(x=None), BAD),
    (dict(D=4), NO), (dict(F=4), NO), (dict(dh=off(2)), NO), (dict(ws=off(8)), NO), (dict(dx=off(2)), NO),
    (dict(dW=off(8)), NO),
])
def test_glu_backward(lib, change, code):
    a = dict(T=4, D=16, F=8, act=0, x=P, W=P, dh=P, ws=P, dx=P, dW=P) | change
    assert lib.isam_glu_backward(a["T"], a["D"], a["F"], a["act"], a["x"], a["W"], a["dh"], a["ws"], a["dx"],
                                 a["dW"]) == code
    assert b"isam_glu_backward" in lib.isam_last_error_string()


def test_glu_workspace(lib):
    n = ctypes.c_size_t()
    assert lib.isam_glu_backward_workspace(0, 8, 8, ctypes.byref(n)) == BAD
    assert lib.isam_glu_backward_workspace(8, 8, 8, None) == BAD
    assert isam.glu_backward_workspace(100_000, 4096, 16384) >= 100_000 * 16384 * 4  # past 32 bits
    assert isam.glu_backward_workspace(1, 8, 8) >= 32


@pytest.mark.parametrize("change,code", [
    (dict(M=0), BAD), (dict(N=0), BAD), (dict(K=0), BAD), (dict(group=16), BAD), (dict(group=0), BAD),
    (dict(x=None), BAD), (dict(t=None), BAD), (dict(s=None), BAD), (dict(y=None), BAD), (dict(M=33), NO),
    (dict(K=12), NO), (dict(x=off(8)), NO), (dict(t=off(4)), NO), (dict(s=off(2)), NO), (dict(y=off(2)), NO),
    (dict(N=BIG, K=2 ** 30), NO),
])
def test_gemv_w4(lib, change, code):
    a = dict(M=2, N=16, K=64, group=32, x=P, t=P, s=P, y=P) | change
    assert lib.isam_gemv_w4(a["M"], a["N"], a["K"], a["group"], a["x"], a["t"], a["s"], a["y"]) == code
    assert b"isam_gemv_w4" in lib.isam_last_error_string()


@pytest.mark.parametrize("change,code", [
    (dict(N=0), BAD), (dict(K=-8), BAD), (dict(group=256), BAD), (dict(c=None), BAD), (dict(s=None), BAD),
    (dict(t=None), BAD), (dict(ts=None), BAD), (dict(K=20), NO), (dict(t=off(4)), NO), (dict(ts=off(8)), NO),
    (dict(s=off(1)), NO),
])
def test_w4_pack(lib, change, code):
    a = dict(N=16, K=64, group=32, c=P, s=P, t=P, ts=P) | change
    assert lib.isam_w4_pack(a["N"], a["K"], a["group"], a["c"], a["s"], a["t"], a["ts"]) == code
    assert b"isam_w4_pack" in lib.isam_last_error_string()


def test_binding_refuses_what_it_can_see():
    """Python-side checks need no library call: types and devices."""
    import torch
    g = torch.zeros(4, 2, 16)
    with pytest.raises(ValueError, match="CUDA"):
        isam.glr_forward(4, 2, 8, g, None, None, torch.zeros(4, 2, 8))
    with pytest.raises(ValueError, match="float32 or torch.bfloat16"):
        isam.glr_forward(4, 2, 8, g.half(), None, None, torch.zeros(4, 2, 8))
    with pytest.raises(ValueError, match="act"):
        isam.glu_forward(4, 8, 8, "tanh", g, g, g)
    with pytest.raises(ValueError, match="group"):
        isam.gemv_w4(1, 16, 64, 48, g, g, g, g)
    assert isam.w4_tiled_bytes(17, 129) == 2 * 2 * 1024
    assert isam.w4_tiled_scales(17, 129, 32) == 2 * 2 * 16 * 4


@pytest.mark.parametrize("N", [2 ** 31 - 15, BIG])
def test_w4_rows_beyond_whole_tiles(lib, N):
    """Rows are counted in whole tiles of 16: the last 15 numbers of 31 bits are refused."""
    assert lib.isam_w4_pack(N, 8, 32, P, P, P, P) == NO
    assert b"isam_w4_pack: N" in lib.isam_last_error_string()
    assert lib.isam_gemv_w4(1, N, 8, 32, P, P, P, P) == NO
    assert b"isam_gemv_w4: N" in lib.isam_last_error_string()


@pytest.mark.parametrize("T", [1, 32, 200])
@pytest.mark.parametrize("D", [2 ** 29 + 8, 2 ** 30 - 8, 2 ** 30, 2 ** 31 - 8])
def test_glu_depths_beyond_the_limit(lib, T, D):
    assert lib.isam_glu_forward(T, D, 8, 0, P, P, P) == NO
    assert b"isam_glu_forward: D" in lib.isam_last_error_string()
    assert lib.isam_glu_backward(T, D, 8, 0, P, P, P, P, P, P) == NO
    assert b"isam_glu_backward: D" in lib.isam_last_error_string()
