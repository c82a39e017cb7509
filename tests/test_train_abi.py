"""Refusals of the checkpoint and cross-entropy calls: every one is made on
the host before anything is enqueued (the pointers are fake)."""
import ctypes

import pytest

from paper_2606_05484_amd import mapl

FAKE = 0x7f0000000000
P = [FAKE + 0x100000000 * i for i in range(12)]


def pack(T=64, d=64, dt=1, X=P[0], q=P[1], e=P[2]):
    return mapl.lib().mapl_ckpt_pack(T, d, dt, X, q, e, None)


def unpack(T=64, d=64, dt=1, q=P[1], e=P[2], X=P[0]):
    return mapl.lib().mapl_ckpt_unpack(T, d, dt, q, e, X, None)


@pytest.mark.parametrize("call", [pack, unpack])
@pytest.mark.parametrize("kw,status", [
    (dict(T=-1), -2), (dict(T=1 << 31), -2), (dict(d=32), -2), (dict(d=100), -2), (dict(d=16448), -2), (dict(dt=2), -3),
    (dict(X=None), -1), (dict(q=None), -1), (dict(e=None), -1), (dict(X=P[0] + 8), -5), (dict(q=P[1] + 4), -5),
    (dict(q=P[0]), -6), (dict(e=P[0] + 16), -6),
])
def test_checkpoint_refusals(call, kw, status):
    assert call(**kw) == status
    assert mapl.last_error() != ""


def test_pack_outputs_may_not_overlap():
    assert pack(e=P[1] + 1024) == -6


def test_checkpoint_of_nothing_is_nothing():
    assert pack(T=0) == 0 and unpack(T=0) == 0


def bwd(D, **kw):
    a = dict(dZ=P[0], q=P[1], e=P[2], ids=P[3], U=P[4], A=P[5], B=P[6], dX=P[7], dU=P[8], ws=P[9], ws_bytes=1 << 30)
    a.update(kw)
    return mapl.lib().mapl_ckpt_encode_bwd(ctypes.byref(D), a["dZ"], a["q"], a["e"], a["ids"], a["U"], a["A"], a["B"],
                                           a["dX"], a["dU"], 0, a["ws"], a["ws_bytes"], None)


@pytest.mark.parametrize("kw,status", [
    (dict(dZ=None), -1), (dict(q=None), -1), (dict(e=None), -1), (dict(ids=None), -1), (dict(U=None), -1),
    (dict(A=None), -1), (dict(B=None), -1), (dict(dX=None), -1), (dict(dU=None), -1), (dict(ws=None), -7),
    (dict(ws_bytes=64), -7), (dict(ws=P[9] + 16), -5), (dict(q=P[1] + 1), -5), (dict(dX=P[1]), -6), (dict(dU=P[2]), -6),
    (dict(dX=P[8]), -6), (dict(dU=P[0]), -6),
])
def test_checkpoint_backward_refusals(kw, status):
    D = mapl.desc(T=64, d=256, r=64, V=100, k=16)
    assert bwd(D, **kw) == status
    assert mapl.last_error() != ""


def test_checkpoint_backward_refuses_what_encode_bwd_refuses():
    D = mapl.desc(T=64, d=256, r=96, V=100, k=16)
    assert bwd(D) == -8 and mapl.lib().mapl_ckpt_encode_bwd_workspace_bytes(ctypes.byref(D)) == 0
    with pytest.raises(mapl.MaplError):
        mapl.ckpt_encode_bwd_workspace_bytes(D)


def fwd_x(D, **kw):
    a = dict(H=P[0], W=P[1], y=P[2], loss=P[3], lse=P[4], ws=P[5], ws_bytes=1 << 31)
    a.update(kw)
    return mapl.lib().mapl_xent_fwd(ctypes.byref(D), a["H"], a["W"], a["y"], a["loss"], a["lse"], a["ws"], a["ws_bytes"], None)


def bwd_x(D, **kw):
    a = dict(H=P[0], W=P[1], y=P[2], lse=P[3], weight=P[4], dH=P[5], dW=P[6], ws=P[7], ws_bytes=1 << 31)
    a.update(kw)
    return mapl.lib().mapl_xent_bwd(ctypes.byref(D), a["H"], a["W"], a["y"], a["lse"], a["weight"], 1.0, a["dH"], a["dW"], 0,
                                    a["ws"], a["ws_bytes"], None)


@pytest.mark.parametrize("kw,status", [
    (dict(T=-1), -2), (dict(T=(1 << 22) + 1), -2), (dict(V=0), -2), (dict(V=(1 << 22) + 1), -2), (dict(d=96), -2),
    (dict(d=0), -2), (dict(d=16448), -2), (dict(x_dtype=2), -3), (dict(dw_dtype=3), -3), (dict(x_dtype=0, dw_dtype=1), -3),
])
def test_cross_entropy_descriptor_refusals(kw, status):
    D = mapl.xent_desc(64, 128, 100)
    for f, v in kw.items():
        setattr(D, f, v)
    for call in (fwd_x, bwd_x):
        assert call(D) == status
        assert mapl.last_error() != ""
    assert mapl.lib().mapl_xent_workspace_bytes(ctypes.byref(D), 0) == 0
    with pytest.raises(mapl.MaplError):
        mapl.xent_workspace_bytes(D, mapl.XENT_BWD)


@pytest.mark.parametrize("kw,status", [
    (dict(H=None), -1), (dict(W=None), -1), (dict(y=None), -1), (dict(loss=None), -1), (dict(lse=None), -1),
    (dict(H=P[0] + 2), -5), (dict(lse=P[4] + 4), -5), (dict(loss=P[0]), -6), (dict(lse=P[2]), -6), (dict(loss=P[4]), -6),
    (dict(ws=P[0]), -7), (dict(ws=None), -7), (dict(ws_bytes=256), -7), (dict(ws=P[5] + 128), -5),
])
def test_cross_entropy_forward_refusals(kw, status):
    D = mapl.xent_desc(64, 128, 100)
    if kw == dict(ws=P[0]):
        kw, status = dict(loss=P[5] + 4096), -6  # an output inside the workspace
    assert fwd_x(D, **kw) == status
    assert mapl.last_error() != ""


@pytest.mark.parametrize("kw,status", [
    (dict(H=None), -1), (dict(W=None), -1), (dict(y=None), -1), (dict(lse=None), -1), (dict(dH=None, dW=None), -1),
    (dict(weight=P[4] + 4), -5), (dict(dH=P[5] + 8), -5), (dict(dH=P[0]), -6), (dict(dW=P[1]), -6), (dict(dW=P[5]), -6),
    (dict(dW=P[4]), -6), (dict(dH=P[7] + 4096), -6), (dict(ws=None), -7), (dict(ws_bytes=4096), -7),
])
def test_cross_entropy_backward_refusals(kw, status):
    D = mapl.xent_desc(64, 128, 100)
    assert bwd_x(D, **kw) == status
    assert mapl.last_error() != ""


def test_cross_entropy_unknown_call_has_no_workspace():
    D = mapl.xent_desc(64, 128, 100)
    assert mapl.lib().mapl_xent_workspace_bytes(ctypes.byref(D), 2) == 0
    assert mapl.lib().mapl_xent_workspace_bytes(None, 0) == 0


def test_descriptor_layout_matches_header():
    assert ctypes.sizeof(mapl.XentDesc) == 32
