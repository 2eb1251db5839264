"""Argument errors of the root-mean-square norm, the causal convolution, the
selective scan and beam search: reported before any CUDA call, so they need no GPU."""
import ctypes

import pytest

from paper_1810_09958_gb300 import build, isam

BAD, NO = isam.ISAM_ERR_INVALID_ARG, isam.ISAM_ERR_UNSUPPORTED
P = ctypes.c_void_p(256)
BIG = 2 ** 31 - 1
NAN, INF = float("nan"), float("inf")


def off(n):
    return ctypes.c_void_p(256 + n)


@pytest.fixture(scope="module")
def lib():
    build.build()
    return isam.load()


def refused(lib, name, args, change, code):
    assert set(change) <= set(args)
    assert getattr(lib, name)(*(args | change).values()) == code
    assert name.encode() in lib.isam_last_error_string()


@pytest.mark.parametrize("change,code", [
    (dict(T=0), BAD), (dict(D=-1), BAD), (dict(xt=2), BAD), (dict(rt=-1), BAD), (dict(yt=9), BAD), (dict(x=None), BAD),
    (dict(w=None), BAD), (dict(y=None), BAD), (dict(y8=P), BAD), (dict(y8=P, s=P), BAD), (dict(y=None, y8=P), BAD),
    (dict(y=None, s=P), BAD), (dict(s=P), BAD), (dict(eps=-1e-6), BAD), (dict(eps=NAN), BAD), (dict(eps=INF), BAD),
    (dict(D=32769), NO), (dict(x=off(2)), NO), (dict(res=off(1)), NO), (dict(out=off(1)), NO), (dict(w=off(2)), NO),
    (dict(y=off(1)), NO), (dict(y=None, y8=P, s=off(2)), NO),
])
def test_norm_forward(lib, change, code):
    refused(lib, "isam_rms_norm_forward", dict(T=4, D=8, xt=0, x=P, rt=1, res=P, out=P, w=P, eps=1e-5, yt=1, y=P, y8=None,
                                               s=None), change, code)


@pytest.mark.parametrize("change,code", [
    (dict(T=0), BAD), (dict(D=0), BAD), (dict(rt=2), BAD), (dict(gt=2), BAD), (dict(r=None), BAD), (dict(w=None), BAD),
    (dict(dy=None), BAD), (dict(ws=None), BAD), (dict(eps=-1.0), BAD), (dict(D=40000), NO), (dict(r=off(1)), NO),
    (dict(dy=off(2)), NO), (dict(dres=off(2)), NO), (dict(dx=off(1)), NO), (dict(dw=off(2)), NO), (dict(ws=off(8)), NO),
])
def test_norm_backward(lib, change, code):
    refused(lib, "isam_rms_norm_backward", dict(T=4, D=8, rt=1, r=P, w=P, eps=1e-5, gt=0, dy=P, dres=P, ws=P, dx=P, dw=P),
            change, code)


CONV = dict(T=4, batch=2, C=8, width=4, xt=1, x=P, stride=8, w=P, bias=P, silu=1)


@pytest.mark.parametrize("change,code", [
    (dict(T=0), BAD), (dict(batch=0), BAD), (dict(C=0), BAD), (dict(width=0), BAD), (dict(xt=3), BAD), (dict(yt=3), BAD),
    (dict(x=None), BAD), (dict(w=None), BAD), (dict(y=None), BAD), (dict(silu=2), BAD), (dict(stride=7), BAD),
    (dict(stride=-8), BAD), (dict(width=1), NO), (dict(width=9), NO), (dict(x=off(1)), NO), (dict(state=off(1)), NO),
    (dict(new=off(1)), NO), (dict(w=off(2)), NO), (dict(bias=off(2)), NO), (dict(lengths=off(1)), NO), (dict(y=off(2)), NO),
    (dict(T=BIG, batch=BIG), NO), (dict(T=2 ** 20, C=2 ** 21, stride=2 ** 21), NO), (dict(stride=2 ** 62), NO),
    (dict(batch=65536), NO), (dict(C=BIG, stride=BIG), NO), (dict(C=BIG - 510, stride=BIG), NO),
])
def test_conv_forward(lib, change, code):
    refused(lib, "isam_conv1d_forward", CONV | dict(state=P, lengths=P, yt=0, y=P, new=P), change, code)


@pytest.mark.parametrize("change,code", [
    (dict(batch=0), BAD), (dict(slots=0), BAD), (dict(state=None), BAD), (dict(new=None), BAD), (dict(ids=None), BAD),
    (dict(x=None), BAD), (dict(stride=3), BAD), (dict(width=12), NO), (dict(ids=off(2)), NO), (dict(state=off(1)), NO),
])
def test_conv_step(lib, change, code):
    refused(lib, "isam_conv1d_step", dict(batch=3, C=8, width=4, slots=2, xt=1, x=P, stride=8, w=P, bias=P, silu=0, ids=P,
                                          state=P, new=P, yt=0, y=P), change, code)


SSM = dict(ut=1, u=P, pt=0, dt=P, bias=P, A=P, B=P, Cm=P, bc=32, D=P, z=P, zs=16)


@pytest.mark.parametrize("change,code", [
    (dict(T=0), BAD), (dict(batch=0), BAD), (dict(C=0), BAD), (dict(N=0), BAD), (dict(ut=2), BAD), (dict(pt=2), BAD),
    (dict(u=None), BAD), (dict(dt=None), BAD), (dict(A=None), BAD), (dict(B=None), BAD), (dict(Cm=None), BAD),
    (dict(y=None), BAD), (dict(bc=15), BAD), (dict(zs=7), BAD), (dict(N=129, bc=129), NO), (dict(u=off(1)), NO),
    (dict(dt=off(2)), NO), (dict(bias=off(1)), NO), (dict(A=off(2)), NO), (dict(B=off(2)), NO), (dict(Cm=off(2)), NO),
    (dict(D=off(2)), NO), (dict(z=off(2)), NO), (dict(h0=off(2)), NO), (dict(lengths=off(2)), NO), (dict(y=off(1)), NO),
    (dict(last=off(2)), NO), (dict(T=BIG, batch=BIG), NO), (dict(bc=2 ** 50), NO), (dict(zs=2 ** 50), NO),
    (dict(batch=65536), NO),
])
def test_ssm_forward(lib, change, code):
    refused(lib, "isam_ssm_forward", dict(T=4, batch=2, C=8, N=16) | SSM | dict(h0=P, lengths=P, y=P, last=P), change, code)


@pytest.mark.parametrize("change,code", [
    (dict(batch=0), BAD), (dict(slots=0), BAD), (dict(state=None), BAD), (dict(new=None), BAD), (dict(ids=None), BAD),
    (dict(A=None), BAD), (dict(bc=1), BAD), (dict(N=200, bc=200), NO), (dict(ids=off(2)), NO), (dict(new=off(2)), NO),
])
def test_ssm_step(lib, change, code):
    refused(lib, "isam_ssm_step", dict(batch=3, C=8, N=16, slots=2) | SSM | dict(ids=P, state=P, new=P, y=P), change, code)


@pytest.mark.parametrize("change,code", [
    (dict(batch=0), BAD), (dict(beams=0), BAD), (dict(V=0), BAD), (dict(count=0), BAD), (dict(lt=2), BAD),
    (dict(logits=None), BAD), (dict(scores=None), BAD), (dict(ws=None), BAD), (dict(new=None), BAD),
    (dict(parents=None), BAD), (dict(tokens=None), BAD), (dict(eos=-2), BAD), (dict(eos=100), BAD), (dict(eos=-1), BAD),
    (dict(beams=65), NO), (dict(count=65), NO), (dict(batch=2 ** 20), NO), (dict(V=2 ** 28 + 1), NO),
    (dict(logits=off(2)), NO), (dict(scores=off(2)), NO), (dict(ws=off(8)), NO), (dict(new=off(2)), NO),
    (dict(parents=off(2)), NO), (dict(tokens=off(1)), NO),
])
def test_beam_select(lib, change, code):
    refused(lib, "isam_beam_select", dict(batch=2, beams=4, V=100, count=4, lt=0, logits=P, scores=P, eos=3, fin=P, ws=P,
                                          new=P, parents=P, tokens=P, nf=P), change, code)


@pytest.mark.parametrize("change,code", [
    (dict(layers=0), BAD), (dict(batch=0), BAD), (dict(beams=0), BAD), (dict(slots=0), BAD), (dict(row=0), BAD),
    (dict(parents=None), BAD), (dict(state=None), BAD), (dict(new=None), BAD), (dict(ids=None, slots=7), BAD),
    (dict(beams=65), NO), (dict(batch=2 ** 19), NO), (dict(layers=BIG, slots=2), NO), (dict(row=2 ** 31), NO),
    (dict(parents=off(2)), NO), (dict(ids=off(2)), NO),
])
def test_beam_reorder(lib, change, code):
    refused(lib, "isam_beam_reorder", dict(layers=2, batch=2, beams=4, slots=9, row=64, parents=P, ids=P, state=P, new=P),
            change, code)


def test_workspaces(lib):
    n = ctypes.c_size_t()
    assert lib.isam_rms_norm_backward_workspace(0, 8, ctypes.byref(n)) == BAD
    assert lib.isam_rms_norm_backward_workspace(8, 8, None) == BAD
    assert isam.rms_norm_backward_workspace(8, 100) >= 400
    assert lib.isam_beam_select_workspace(1, 1, 0, 1, ctypes.byref(n)) == BAD
    assert lib.isam_beam_select_workspace(1, 1, 8, 1, None) == BAD
    assert lib.isam_beam_select_workspace(1, 65, 8, 1, ctypes.byref(n)) == NO
    assert isam.beam_select_workspace(2 ** 14, 64, 2 ** 28, 64) >= 2 ** 20 * 64 * 8


def test_binding_refuses_what_it_can_see():
    """Python-side checks need no library call: types, devices and rows."""
    import torch
    f, b = torch.zeros(4, 8), torch.zeros(4, 8, dtype=torch.bfloat16)
    with pytest.raises(ValueError, match="CUDA"):
        isam.rms_norm_forward(4, 8, f, None, None, f[0], 1e-5, f)
    with pytest.raises(ValueError, match="float32 or torch.bfloat16"):
        isam.rms_norm_forward(4, 8, f.half(), None, None, f[0], 1e-5, f)
    with pytest.raises(ValueError, match="CUDA"):
        isam.conv1d_step(4, 4, 2, 4, b[:, :4], f, None, True, None, b, b, f)
    with pytest.raises(ValueError, match="bool or torch.uint8"):
        isam.beam_select(1, 1, 8, 1, f, f, 0, f, f, f, f)
    with pytest.raises(ValueError, match="rows"):
        isam.beam_reorder(3, 1, 1, 1, f, None, f, f)
