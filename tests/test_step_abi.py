"""Refusals of the norms around a block, the gradients' norm and AdamW: every one
is made on the host before anything is enqueued (the pointers are fake)."""
import ctypes

import pytest

from paper_2606_05484_amd import mapl

FAKE = 0x7f0000000000
P = [FAKE + 0x100000000 * i for i in range(20)]
WHOLE = dict(branch=True, post=True, pre=True, gate="silu")


def fwd(D, **kw):
    a = dict(x=P[0], h=P[1], gate=P[2], w_post=P[3], scale=P[4], w_pre=P[5], xo=P[6], y=P[7])
    a.update(kw)
    return mapl.lib().mapl_norm_fwd(ctypes.byref(D), a["x"], a["h"], a["gate"], a["w_post"], a["scale"], a["w_pre"],
                                    a["xo"], a["y"], None)


def bwd(D, **kw):
    a = dict(dy=P[0], dxo=P[1], xo=P[2], h=P[3], gate=P[4], w_post=P[5], scale=P[6], w_pre=P[7], dx=P[8], dh=P[9],
             dgate=P[10], dw_post=P[11], dscale=P[12], dw_pre=P[13], ws=P[14], ws_bytes=1 << 30)
    a.update(kw)
    return mapl.lib().mapl_norm_bwd(ctypes.byref(D), a["dy"], a["dxo"], a["xo"], a["h"], a["gate"], a["w_post"], a["scale"],
                                    a["w_pre"], a["dx"], a["dh"], a["dgate"], a["dw_post"], a["dscale"], a["dw_pre"], 0,
                                    a["ws"], a["ws_bytes"], None)


@pytest.mark.parametrize("kw,status", [
    (dict(T=-1), -2), (dict(T=1 << 31), -2), (dict(d=32), -2), (dict(d=100), -2), (dict(d=16448), -2),
    (dict(x_dtype=2), -3), (dict(h_dtype=0), -3), (dict(h_dtype=3), -3), (dict(ld_h=64), -2), (dict(ld_h=132), -2),
    (dict(ld_gate=100), -2), (dict(ld_gate=(1 << 20) + 8), -2), (dict(parts=0), -2), (dict(parts=4), -2),
    (dict(parts=5), -2), (dict(parts=8), -2), (dict(gate=3), -2), (dict(gate=-1), -2), (dict(parts=1), -2),
    (dict(eps=0.0), -2), (dict(eps=2.0), -2), (dict(eps=float("nan")), -2), (dict(alpha=float("inf")), -2),
    (dict(alpha=float("nan")), -2),
])
def test_norm_descriptor_refusals(kw, status):
    D = mapl.norm_desc(64, 128, **WHOLE)
    for f, v in kw.items():
        setattr(D, f, v)
    for call in (fwd, bwd):
        assert call(D) == status
        assert mapl.last_error() != ""
    assert mapl.lib().mapl_norm_workspace_bytes(ctypes.byref(D)) == 0
    with pytest.raises(mapl.MaplError):
        mapl.norm_workspace_bytes(D)


@pytest.mark.parametrize("kw,status", [
    (dict(x=None), -1), (dict(h=None), -1), (dict(gate=None), -1), (dict(xo=None), -1), (dict(y=None), -1),
    (dict(x=P[0] + 8), -5), (dict(h=P[1] + 2), -5), (dict(w_pre=P[5] + 4), -5), (dict(y=P[7] + 8), -5),
    (dict(xo=P[0]), -6), (dict(y=P[1]), -6), (dict(y=P[6] + 16), -6), (dict(xo=P[4]), -6), (dict(y=P[2] + 1024), -6),
])
def test_norm_forward_refusals(kw, status):
    assert fwd(mapl.norm_desc(64, 128, **WHOLE), **kw) == status
    assert mapl.last_error() != ""


@pytest.mark.parametrize("kw,status", [
    (dict(dy=None), -1), (dict(xo=None), -1), (dict(h=None), -1), (dict(gate=None), -1), (dict(dx=None), -1),
    (dict(dh=None), -1), (dict(dgate=None), -1), (dict(dy=P[0] + 8), -5), (dict(dw_pre=P[13] + 4), -5),
    (dict(dx=P[1]), -6), (dict(dh=P[3]), -6), (dict(dgate=P[9]), -6), (dict(dgate=P[9] + 128), -6), (dict(dw_post=P[8] + 64), -6),
    (dict(dscale=P[11] + 16), -6), (dict(dw_pre=P[12]), -6), (dict(dw_pre=P[7]), -6), (dict(dx=P[14] + 4096), -6),
    (dict(ws=None), -7), (dict(ws_bytes=256), -7), (dict(ws=P[14] + 16), -5),
])
def test_norm_backward_refusals(kw, status):
    assert bwd(mapl.norm_desc(64, 128, **WHOLE), **kw) == status
    assert mapl.last_error() != ""


@pytest.mark.parametrize("given", range(8))
def test_norm_backward_refuses_a_workspace_over_what_it_reads(given):
    assert bwd(mapl.norm_desc(64, 128, **WHOLE), ws=P[given] + 256) == -6
    assert "workspace" in mapl.last_error()


@pytest.mark.parametrize("parts,extra", [
    (dict(pre=True), ("h",)), (dict(pre=True), ("scale",)), (dict(pre=True), ("w_post",)), (dict(pre=True), ("xo",)),
    (dict(pre=True), ("gate",)), (dict(pre=False, branch=True), ("y",)), (dict(pre=False, branch=True), ("w_pre",)),
    (dict(pre=True, branch=True), ("w_post",)), (dict(pre=True, branch=True), ("gate",)),
])
def test_norm_forward_refuses_what_its_parts_leave_out(parts, extra):
    D = mapl.norm_desc(64, 128, **parts)
    a = dict(h=None, gate=None, w_post=None, scale=None, w_pre=None, xo=None, y=None)
    if D.parts & 2:
        a.update(h=P[1], xo=P[6])
    if D.parts & 1:
        a.update(y=P[7])
    a.update({k: P[8] for k in extra})
    assert fwd(D, **a) == -2 and mapl.last_error() != ""


@pytest.mark.parametrize("parts,extra", [
    (dict(pre=True), "h"), (dict(pre=True), "dh"), (dict(pre=True), "dscale"), (dict(pre=True), "dw_post"),
    (dict(pre=False, branch=True), "dy"), (dict(pre=False, branch=True), "xo"), (dict(pre=False, branch=True), "dx"),
    (dict(pre=False, branch=True), "dw_pre"), (dict(pre=False, branch=True), "dgate"),
])
def test_norm_backward_refuses_what_its_parts_leave_out(parts, extra):
    D = mapl.norm_desc(64, 128, **parts)
    a = {k: None for k in ("dy", "xo", "h", "gate", "w_post", "scale", "w_pre", "dx", "dh", "dgate", "dw_post", "dscale", "dw_pre")}
    a.update(dxo=P[1])
    if D.parts & 2:
        a.update(h=P[3], dh=P[9])
    if D.parts & 1:
        a.update(dy=P[0], xo=P[2], dx=P[8])
    a[extra] = P[15]
    assert bwd(D, **a) == -2 and mapl.last_error() != ""


def test_norm_without_y_needs_the_streams_gradient():
    D = mapl.norm_desc(64, 128, branch=True, pre=False)
    none = {k: None for k in ("dy", "xo", "gate", "w_post", "w_pre", "dx", "dgate", "dw_post", "dw_pre")}
    assert bwd(D, dxo=None, **none) == -1


def test_halves_of_one_product_do_not_overlap_but_their_mixtures_do():
    D = mapl.norm_desc(64, 128, ld_h=256, ld_gate=256, **WHOLE)
    ok = dict(ws=None)  # the workspace is looked at last
    assert bwd(D, dh=P[9], dgate=P[9] + 256, **ok) == -7
    assert bwd(D, dh=P[9] + 256, dgate=P[9], **ok) == -7
    assert bwd(D, dh=P[9], dgate=P[9] + 128, **ok) == -6
    assert bwd(D, dh=P[9] + 512, dgate=P[9], **ok) == -6
    D.ld_gate = 512
    assert bwd(D, dh=P[9], dgate=P[9] + 256, **ok) == -6


def test_norm_of_nothing_is_nothing():
    D = mapl.norm_desc(0, 128, **WHOLE)
    assert fwd(D) == 0
    assert bwd(D, dw_post=None, dscale=None, dw_pre=None) == 0


# ------------------------------------------------------------------ optimizer
def params(count=2, n=1000, **kw):
    a = (mapl.Param * count)()
    for i in range(count):
        for j, f in enumerate(("g", "p", "m", "v", "e", "p16")):
            setattr(a[i], f, P[j] + i * 0x1000000)
        a[i].n, a[i].lr_scale = n, 1.0
    for f, v in kw.items():
        setattr(a[1], f, v)
    return a


def norm(a, count=2, g=0, scale=1.0, most=1.0, stats=P[10], step=P[11], ws=P[12], ws_bytes=1 << 20):
    return mapl.lib().mapl_grad_norm(a, count, g, scale, most, stats, step, ws, ws_bytes, None)


@pytest.mark.parametrize("kw,status", [
    (dict(count=-1), -2), (dict(count=(1 << 20) + 1), -2), (dict(g=2), -3), (dict(scale=float("nan")), -2),
    (dict(most=0.0), -2), (dict(most=-1.0), -2), (dict(most=float("nan")), -2), (dict(stats=None), -1),
    (dict(stats=P[10] + 4), -5), (dict(step=P[11] + 4), -5), (dict(step=P[10]), -6), (dict(stats=P[0] + 16), -6),
    (dict(ws=None), -7), (dict(ws_bytes=64), -7), (dict(ws=P[12] + 16), -5), (dict(ws=P[0] + 0x1000000), -6),
])
def test_gradient_norm_refusals(kw, status):
    assert norm(params(), **kw) == status
    assert mapl.last_error() != ""


@pytest.mark.parametrize("kw,status", [(dict(g=None), -1), (dict(g=P[0] + 8), -5), (dict(n=-1), -2), (dict(n=(1 << 34) + 1), -2)])
def test_gradient_norm_refuses_a_tensor(kw, status):
    assert norm(params(**kw)) == status
    assert mapl.last_error() != ""


def test_gradient_norm_workspace():
    a = params()
    assert mapl.lib().mapl_grad_norm_workspace_bytes(a, 2, 0) >= 16
    assert mapl.lib().mapl_grad_norm_workspace_bytes(a, -1, 0) == 0
    assert mapl.lib().mapl_grad_norm_workspace_bytes(a, 2, 3) == 0
    assert mapl.lib().mapl_grad_norm_workspace_bytes(None, 2, 0) == 0
    with pytest.raises(mapl.MaplError):
        mapl.grad_norm_workspace_bytes(mapl.OptimParams(a, -1, None))
    assert norm(None) == -1


def adamw(a, count=2, stats=P[10], step=None, lr=None, states="8bit", **kw):
    D = mapl.adamw_desc(1e-3, g_dtype="f32", states=states, step=1)
    for f, v in kw.items():
        setattr(D, f, v)
    return mapl.lib().mapl_adamw_step(ctypes.byref(D), a, count, stats, step, lr, None)


@pytest.mark.parametrize("kw,status", [
    (dict(count=-1), -2), (dict(beta1=1.0), -2), (dict(beta1=-0.1), -2), (dict(beta2=1.0), -2), (dict(beta2=float("nan")), -2),
    (dict(eps=0.0), -2), (dict(eps=float("inf")), -2), (dict(lr=float("nan")), -2), (dict(step=P[11] + 4), -5),
    (dict(g_dtype=2), -3), (dict(states=5), -3), (dict(stats=P[10] + 8), -5), (dict(lr=P[11] + 8), -5), (dict(stats=P[1]), -6),
    (dict(step=P[2]), -6), (dict(lr=P[3]), -6),
])
def test_adamw_refusals(kw, status):
    if "states" in kw:
        D = mapl.adamw_desc(1e-3, step=1)
        D.states = kw["states"]
        assert mapl.lib().mapl_adamw_step(ctypes.byref(D), params(), 2, None, None, None, None) == status
    elif "lr" in kw and isinstance(kw["lr"], float):
        D = mapl.adamw_desc(kw["lr"], step=1)
        assert mapl.lib().mapl_adamw_step(ctypes.byref(D), params(), 2, None, None, None, None) == status
    else:
        assert adamw(params(), **kw) == status
    assert mapl.last_error() != ""


def test_adamw_without_a_step_on_the_device_needs_its_number():
    D = mapl.adamw_desc(1e-3, states="8bit")
    assert mapl.lib().mapl_adamw_step(ctypes.byref(D), params(), 2, None, None, None, None) == -2
    assert mapl.lib().mapl_adamw_step(None, params(), 2, None, None, None, None) == -1


B = 0x1000000  # where the second tensor's arrays lie
@pytest.mark.parametrize("kw,status", [
    (dict(g=None), -1), (dict(p=None), -1), (dict(m=None), -1), (dict(v=None), -1), (dict(e=None), -1),
    (dict(p=P[1] + B + 4), -5), (dict(m=P[2] + B + 8), -5), (dict(p16=P[5] + B + 2), -5),
    (dict(p=P[1]), -6), (dict(g=P[1] + 16), -6), (dict(m=P[3] + B), -6), (dict(v=P[3] + 992), -6), (dict(e=P[2] + B + 16), -6),
    (dict(p16=P[0] + B), -6), (dict(p16=P[5] + 1984), -6), (dict(n=-5), -2), (dict(weight_decay=float("inf")), -2),
    (dict(lr_scale=float("nan")), -2),
])
def test_adamw_refuses_a_tensor(kw, status):
    assert adamw(params(**kw)) == status
    assert mapl.last_error() != ""


def test_the_same_tensor_twice_is_refused():
    a = params()
    a[1] = a[0]
    assert adamw(a) == -6


@pytest.mark.parametrize("pack", [0, 1])
@pytest.mark.parametrize("kw,other,status", [
    (dict(m=None), {}, -1), (dict(e=None), {}, -1), ({}, dict(v=None), -1), ({}, dict(m=P[7] + B + 4), -5), (dict(n=999), {}, -2),
    (dict(n=-1), dict(n=-1), -2), (dict(m=P[8] + B), {}, -6), ({}, dict(v=P[3] + B), -6),
])
def test_conversion_refusals(pack, kw, other, status):
    q, u = params(**kw), params()
    for i in range(2):
        u[i].m, u[i].v = P[7] + i * B, P[8] + i * B
    for f, v in other.items():
        setattr(u[1], f, v)
    L = mapl.lib()
    assert (L.mapl_adamw_pack(u, q, 2, None) if pack else L.mapl_adamw_unpack(q, u, 2, None)) == status
    assert mapl.last_error() != ""


def test_the_binding_refuses_lists_that_do_not_match():
    import torch
    z = lambda n, dt=torch.float32: torch.zeros(n, dtype=dt)
    with pytest.raises(ValueError):
        mapl.optim_params([z(4)], p=[z(4), z(4)])
    with pytest.raises(ValueError):
        mapl.optim_params([z(4)], p=[z(5)])
    with pytest.raises(ValueError):
        mapl.optim_params([z(300)], e=[z(4, torch.uint8)])
    with pytest.raises(ValueError):
        mapl.optim_params([z(4)], weight_decay=[0.1, 0.1])
    with pytest.raises(ValueError):
        mapl.optim_params([z(8)[::2]])
    a = mapl.optim_params([z(300)], e=[z(6, torch.uint8)])
    with pytest.raises(ValueError):
        mapl.adamw_unpack(a, mapl.optim_params([]))
    with pytest.raises(ValueError):
        mapl.adamw_pack(mapl.optim_params([]), a)


def test_the_binding_refuses_types_that_a_call_does_not_take():
    import torch
    z = lambda dt: torch.zeros(300, dtype=dt)
    f32, bf, u8 = torch.float32, torch.bfloat16, torch.uint8
    with pytest.raises(ValueError):
        mapl.optim_params([z(f32), z(bf)])
    good = dict(g=[z(f32)], p=[z(f32)], m=[z(u8)], v=[z(u8)], e=[z(u8)], p16=[z(bf)])
    step = lambda a, **kw: mapl.adamw_step(mapl.adamw_desc(1e-3, step=1, **kw), a, stream=0)
    for name, dt in (("g", bf), ("p", bf), ("m", f32), ("v", f32), ("e", f32), ("p16", f32)):
        with pytest.raises(ValueError):
            step(mapl.optim_params(**dict(good, **{name: [z(dt)]})), states="8bit")
    with pytest.raises(ValueError):
        step(mapl.optim_params(**good))  # fp32 states asked for
    with pytest.raises(ValueError):
        mapl.grad_norm(mapl.optim_params([z(f32)]), None, None, g_dtype="bf16")
    with pytest.raises(ValueError):
        mapl.adamw_unpack(mapl.optim_params(**good), mapl.optim_params([z(f32)], m=[z(u8)], v=[z(u8)]))
    with pytest.raises(ValueError):
        mapl.adamw_pack(mapl.optim_params([z(f32)], m=[z(f32)], v=[z(f32)]), mapl.optim_params([z(f32)], m=[z(f32)], v=[z(f32)], e=[z(u8)]))


def test_descriptor_layouts_match_the_header():
    assert ctypes.sizeof(mapl.NormDesc) == 56 and ctypes.sizeof(mapl.Param) == 64 and ctypes.sizeof(mapl.AdamwDesc) == 32
