"""The norms around a block against their 64-bit forms, element by element
within the bounds of fp32 arithmetic and each result's rounding."""
import pytest
import torch

import _step_helpers as sh
from paper_2606_05484_amd import mapl

pytestmark = pytest.mark.gpu
DT = {"bf16": torch.bfloat16, "f32": torch.float32}


class Case:
    """Inputs, outputs and calls of one shape; halves: h and its gate are the halves of one [T, 2d]."""

    def __init__(self, T, d, x="bf16", h=None, branch=True, post=True, pre=True, gate="sigmoid", halves=False, seed=0, size=1.0,
                 alpha=0.5, eps=1e-5, weights=True, dxo=True):
        h = x if h is None else h
        g = torch.Generator(device="cuda").manual_seed(1000 * T + d + seed)
        rn = lambda *s: torch.randn(*s, generator=g, device="cuda")
        xt, ht = DT[x], DT[h]
        self.ht, self.kind, self.post, self.alpha, self.eps = ht, gate, post, alpha, eps
        self.halves, self.T, self.d = halves, T, d
        vec = lambda on: (1.0 + 0.3 * rn(d)) if on and weights else None
        rows = (0.3 + rn(T, 1).abs()) * size
        self.x = (rows * rn(T, d)).to(xt)
        self.h, self.G = self.pair(ht, branch, gate != "none")
        if branch:
            self.h.copy_((rows * rn(T, d)).to(ht))
            if T > 2:
                self.h[1] = 0.0
        if self.G is not None:
            self.G.copy_((3.0 * rn(T, d)).to(ht))
        if T > 2:
            self.x[2] = 0.0
        self.w_post, self.scale, self.w_pre = vec(post), vec(branch), vec(pre)
        new = lambda dt, on: torch.full((T, d), 7.0, dtype=dt, device="cuda") if on else None
        self.xo, self.y = new(xt, branch), new(ht, pre)
        self.dy = rn(T, d).to(ht) if pre else None
        self.dxo = rn(T, d).to(xt) if dxo else None
        self.dx = new(xt, pre)
        self.dh, self.dG = self.pair(ht, branch, gate != "none")
        z = lambda on: torch.full((d,), 3.0, device="cuda") if on else None
        self.dw_post, self.dscale, self.dw_pre = z(post), z(branch), z(pre)
        ld = 2 * d if halves else 0
        self.D = mapl.norm_desc(T, d, x, h, branch=branch, post=post, pre=pre, gate=gate, alpha=alpha, eps=eps, ld_h=ld, ld_gate=ld)
        self.ws = mapl.workspace(mapl.norm_workspace_bytes(self.D))
        self.branch, self.pre = branch, pre

    def pair(self, ht, one, two):
        if self.halves:
            t = torch.zeros(self.T, 2 * self.d, dtype=ht, device="cuda")
            return t[:, :self.d], t[:, self.d:] if two else None
        z = lambda on: torch.zeros(self.T, self.d, dtype=ht, device="cuda") if on else None
        return z(one), z(two)

    def fwd(self, **kw):
        mapl.norm_fwd(self.D, self.x, self.h, self.G, self.w_post, self.scale, self.w_pre, self.xo, self.y, **kw)

    def at(self):  # what the backward takes as x'
        return None if not self.pre else self.xo if self.branch else self.x

    def bwd(self, accumulate=0, **kw):
        mapl.norm_bwd(self.D, self.dy, self.dxo, self.at(), self.h, self.G, self.w_post, self.scale, self.w_pre, self.dx,
                      self.dh, self.dG, self.dw_post, self.dscale, self.dw_pre, accumulate, self.ws, **kw)

    def outputs(self):
        o = dict(xo=self.xo, y=self.y, dx=self.dx, dh=self.dh, dG=self.dG, dw_post=self.dw_post, dscale=self.dscale, dw_pre=self.dw_pre)
        return {k: v.clone() for k, v in o.items() if v is not None}

    def check(self, base=0.0):
        """Every output against the forms (base: what the vectors' gradients held before)."""
        xo = self.x
        if self.branch:
            ref, t = sh.norm_fwd(self.x, self.h, self.G, self.w_post, self.scale, self.kind, self.post, self.alpha, self.eps)
            within(self.xo, ref, sh.norm_fwd_errors(self.x, ref, t, None, None, self.G)[0], "xo")
            xo = self.xo
        if self.pre:
            y = sh.norm_y(xo, self.w_pre, self.eps)
            within(self.y, y, sh.norm_fwd_errors(self.x, y, y.abs(), y, self.ht)[1], "y")
        o = sh.norm_bwd(self.dy, self.dxo, self.at(), self.h, self.G, self.w_post, self.scale, self.w_pre, self.kind, self.post,
                        self.alpha, self.eps)
        for name, got in (("dx", self.dx), ("dh", self.dh), ("dgate", self.dG), ("dw_post", self.dw_post), ("dscale", self.dscale),
                          ("dw_pre", self.dw_pre)):
            if got is None:
                continue
            ref = o[name] + (base if got.dim() == 1 else 0.0)
            within(got, ref, o["e_" + name] + 1.01 * sh.half_step(got.dtype) * ref.abs() + 1e-38, name)


def within(got, want, tol, name):
    off = (got.double() - want).abs()
    bad = ~(off <= tol)
    assert not bad.any(), "%s: %d values off, the worst %.3g of the bound" % (name, int(bad.sum()), float((off / tol).max()))


SIZES = [(1, 64), (1000, 64), (3, 128), (5, 192), (17, 256), (37, 320), (9, 512), (33, 576), (70, 1024), (1021, 1024), (11, 1088), (300, 1536), (9, 1600), (4, 2048),
         (1, 2048), (530, 2048), (7, 2112), (600, 2560), (3, 2624), (5, 4096), (3, 4160), (300, 5120), (2, 5184), (3, 8192), (2, 8256), (300, 8704), (2, 12288), (300, 12352), (3, 16384), (1, 16384)]


@pytest.mark.parametrize("T,d", SIZES)
@pytest.mark.parametrize("x,h", [("bf16", "bf16"), ("f32", "bf16"), ("f32", "f32")])
def test_whole(T, d, x, h):
    print("norm whole", T, d, x, h, flush=True)
    c = Case(T, d, x, h, gate="silu" if d % 128 else "sigmoid")
    c.fwd()
    c.bwd()
    torch.cuda.synchronize()
    c.check()


PARTS = [dict(branch=False, post=False, gate="none"), dict(pre=False), dict(post=False), dict(gate="none"),
         dict(pre=False, post=False, gate="none"), dict(post=False, gate="silu", halves=True), dict(gate="silu", halves=True),
         dict(gate="none", halves=True), dict(weights=False), dict(dxo=False), dict(branch=False, post=False, gate="none", dxo=False),
         dict(branch=False, post=False, gate="none", weights=False), dict(alpha=-2.0), dict(alpha=0.0)]


@pytest.mark.parametrize("kw", PARTS, ids=lambda k: "-".join("%s=%s" % i for i in k.items()))
@pytest.mark.parametrize("T,d,x,h", [(6, 64, "f32", "f32"), (45, 256, "bf16", "bf16"), (129, 1024, "f32", "bf16"), (21, 2048, "bf16", "bf16"),
                                     (3, 8192, "f32", "f32"), (2, 16384, "bf16", "bf16")])
def test_parts(T, d, x, h, kw):
    print("norm parts", T, d, x, h, kw, flush=True)
    c = Case(T, d, x, h, **kw)
    c.fwd()
    c.bwd()
    torch.cuda.synchronize()
    c.check()


@pytest.mark.parametrize("T,d,x,h", [(40, 256, "f32", "f32"), (40, 2048, "bf16", "bf16"), (3, 16384, "f32", "bf16")])
@pytest.mark.parametrize("size", [1e-15, 1e15, 3e18, 1e30])
def test_rows_of_any_size(T, d, x, h, size):
    """Squares that overflow fp32 (3e18 and up, 1e30 past all doubt), and rows far below eps's root."""
    c = Case(T, d, x, h, size=size)
    c.fwd()
    c.bwd()
    torch.cuda.synchronize()
    assert all(bool(v.isfinite().all()) for v in c.outputs().values())
    c.check()


def test_a_large_eps_counts_and_a_small_one_does_too():
    for eps in (1.0, 1e-30):
        c = Case(9, 256, "f32", size=1e-14, eps=eps)
        c.fwd()
        c.bwd()
        torch.cuda.synchronize()
        c.check()


def test_zero_rows_stay_zero():
    c = Case(4, 256, gate="none")
    c.x.zero_(), c.h.zero_()
    c.fwd()
    torch.cuda.synchronize()
    assert (c.xo == 0).all() and (c.y == 0).all()


@pytest.mark.parametrize("d", [256, 1024, 2048])
def test_nan_and_infinity_stay_in_their_rows(d):
    T = 70
    c, clean = Case(T, d, "f32"), Case(T, d, "f32")
    c.x[5, 3], c.h[9, 60], c.G[20, 1] = float("nan"), float("inf"), float("nan")
    for k in (c, clean):
        k.fwd()
        k.bwd()
    torch.cuda.synchronize()
    rest = torch.ones(T, dtype=torch.bool, device="cuda")
    rest[[5, 9, 20]] = False
    a, b = c.outputs(), clean.outputs()
    for k in ("xo", "y", "dx", "dh", "dG"):
        assert torch.equal(a[k][rest], b[k][rest])
    assert c.y[5].isnan().all() and c.y[20].isnan().any() and c.y[9].isnan().any()


def test_gates_at_both_ends():
    for kind in ("sigmoid", "silu"):
        c = Case(8, 64, "f32", gate=kind)
        c.G.copy_(torch.linspace(-110, 110, 8 * 64, device="cuda").view(8, 64))
        c.G[0, 0], c.G[0, 1] = -3e38, 3e38
        c.fwd()
        c.bwd()
        torch.cuda.synchronize()
        # far out the form's own derivative underflows: compare where fp32 holds it
        assert all(bool(v[1:].isfinite().all()) for k, v in c.outputs().items() if v.dim() == 2)
        ref, t = sh.norm_fwd(c.x, c.h, c.G, c.w_post, c.scale, kind, True, c.alpha, c.eps)
        within(c.xo[1:], ref[1:], sh.norm_fwd_errors(c.x, ref, t, None, None)[0][1:], "xo")
        o = sh.norm_bwd(c.dy, c.dxo, c.at(), c.h, c.G, c.w_post, c.scale, c.w_pre, kind, True, c.alpha, c.eps)
        within(c.dG[1:], o["dgate"][1:], (o["e_dgate"] + sh.U24 * o["dgate"].abs() + 1e-37)[1:], "dgate")


@pytest.mark.parametrize("T", [5, 700])
def test_accumulate_and_left_out(T):
    c = Case(T, 320)
    c.fwd()
    c.bwd(accumulate=1)
    torch.cuda.synchronize()
    c.check(base=3.0)
    before = c.outputs()
    full = c.dw_pre.clone()
    c.dw_post = c.dscale = None
    c.dw_pre.fill_(3.0)
    c.bwd(accumulate=1)
    torch.cuda.synchronize()
    assert torch.equal(c.dw_pre, full)
    c.dw_pre = None
    c.bwd()
    torch.cuda.synchronize()
    assert all(torch.equal(v, before[k]) for k, v in c.outputs().items())


def test_nothing():
    c = Case(0, 128)
    c.fwd()
    c.bwd(accumulate=1)
    torch.cuda.synchronize()
    assert (c.dw_pre == 3.0).all()
    c.bwd()
    torch.cuda.synchronize()
    assert (c.dw_pre == 0).all() and (c.dscale == 0).all() and (c.dw_post == 0).all()


def test_rows_between_the_halves_are_left_alone():
    T, d = 19, 256
    c = Case(T, d)
    wide = torch.full((T, d + 64), 5.0, dtype=torch.bfloat16, device="cuda")
    dwide = wide.clone()
    wide[:, :d] = c.h
    c.D.ld_h = d + 64
    c.h, c.dh = wide[:, :d], dwide[:, :d]
    c.fwd()
    c.bwd()
    torch.cuda.synchronize()
    c.check()
    assert (wide[:, d:] == 5.0).all() and (dwide[:, d:] == 5.0).all()


def test_repeats_bit_for_bit_on_another_stream_and_in_a_replayed_graph():
    c = Case(777, 1024, gate="silu", halves=True)
    c.fwd()
    c.bwd()
    torch.cuda.synchronize()
    want = c.outputs()
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    for v in (c.xo, c.y, c.dx, c.dw_post, c.dscale, c.dw_pre):
        v.fill_(9.0)
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        c.fwd()
        c.bwd()
    s.synchronize()
    assert all(torch.equal(v, want[k]) for k, v in c.outputs().items())
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        c.fwd()
        c.bwd()
    x2 = (c.x.float() * 0.5 + 1.0).to(c.x.dtype)
    x1 = c.x.clone()
    for k in range(4):
        c.x.copy_(x2 if k % 2 else x1)
        g.replay()
        torch.cuda.synchronize()
        got = c.outputs()
        c.fwd()
        c.bwd()
        torch.cuda.synchronize()
        assert all(torch.equal(v, got[n]) for n, v in c.outputs().items())
    assert all(torch.equal(v, want[k]) for k, v in c.outputs().items()) is False  # x2's, not x1's


def test_against_differences():
    """The gradient along a random direction against the change of the outputs' weighted sum, in
    fp32: steps of 2^-6 both ways, whose third-order term and the outputs' rounding are below 2e-3 of it."""
    c = Case(3, 64, "f32", gate="silu", eps=1e-2)
    wx, wy = c.dxo.double(), c.dy.double()

    def value():
        c.fwd()
        torch.cuda.synchronize()
        return float((c.xo.double() * wx).sum() + (c.y.double() * wy).sum())

    value()
    c.bwd()
    torch.cuda.synchronize()
    grads = dict(x=c.dx, h=c.dh, G=c.dG, w_post=c.dw_post, scale=c.dscale, w_pre=c.dw_pre)
    grads = {k: v.clone() for k, v in grads.items()}
    for name, grad in grads.items():
        t = getattr(c, name)
        base = t.clone()
        direction = grad / grad.norm()
        step = 2.0 ** -6
        t.copy_(base + step * direction)
        up = value()
        t.copy_(base - step * direction)
        down = value()
        t.copy_(base)
        assert abs((up - down) / (2 * step) / float(grad.norm()) - 1) < 5e-3, name


@pytest.mark.parametrize("T,d,x,h,kw", [
    (33000, 256, "bf16", "bf16", {}), (9000, 1024, "f32", "bf16", dict(gate="silu")), (8200, 2048, "bf16", "bf16", dict(halves=True)),
    (3001, 8192, "bf16", "bf16", dict(gate="none")), (2001, 16384, "bf16", "bf16", {}), (17001, 2048, "f32", "f32", dict(branch=False, post=False, gate="none")),
    (4100, 4096, "f32", "f32", dict(post=False)), (70001, 512, "bf16", "bf16", dict(pre=False, gate="silu"))])
def test_calls_past_the_caches(T, d, x, h, kw):
    """More than 128 MiB of rows: the variants whose loads and stores bypass the last-level cache."""
    print("norm large", T, d, x, h, kw, flush=True)
    c = Case(T, d, x, h, **kw)
    c.fwd()
    c.bwd()
    torch.cuda.synchronize()
    c.check()


@pytest.mark.parametrize("T,d", [((1 << 21) + 3, 1088), ((1 << 23) + 5, 512)])
def test_more_rows_than_a_launch_takes(T, d):
    D = mapl.norm_desc(T, d)
    x = torch.zeros(T, d, dtype=torch.bfloat16, device="cuda")
    y = torch.full((T, d), 7.0, dtype=torch.bfloat16, device="cuda")
    g = torch.Generator(device="cuda").manual_seed(2)
    rows = [0, 1, (1 << 21) - 1, 1 << 21, T - 2, T - 1]
    few = torch.randn(len(rows), d, generator=g, device="cuda").to(torch.bfloat16)
    x[rows] = few
    mapl.norm_fwd(D, x, None, None, None, None, None, None, y)
    torch.cuda.synchronize()
    ref = sh.norm_y(few, None, 1e-5)
    within(y[rows], ref, sh.norm_fwd_errors(few, ref, ref.abs(), ref, torch.bfloat16)[1], "y")
    y[rows] = 0.0
    assert not bool(y.any())


def test_past_two_gib():
    """Offsets past 2^32 bytes and 2^31 values."""
    T, d = 131080, 16384
    if torch.cuda.mem_get_info()[0] < 40 << 30:
        pytest.skip("needs 40 GiB")
    D = mapl.norm_desc(T, d, branch=False, pre=True)
    x = torch.zeros(T, d, dtype=torch.bfloat16, device="cuda")
    y = torch.zeros_like(x)
    g = torch.Generator(device="cuda").manual_seed(1)
    rows = [0, 1, 65535, 65536, 131071, T - 1]
    few = torch.randn(len(rows), d, generator=g, device="cuda").to(torch.bfloat16)
    x[rows] = few
    w = torch.randn(d, generator=g, device="cuda")
    mapl.norm_fwd(D, x, None, None, None, None, w, None, y)
    torch.cuda.synchronize()
    ref = sh.norm_y(few, w, 1e-5)
    within(y[rows], ref, sh.norm_fwd_errors(few, ref, ref.abs(), ref, torch.bfloat16)[1], "y")
    assert int((y[2:65535] != 0).any()) == 0
    dx, dw = torch.empty_like(x), torch.empty(d, device="cuda")
    ws = mapl.workspace(mapl.norm_workspace_bytes(D))
    mapl.norm_bwd(D, y, None, x, None, None, None, None, w, dx, None, None, None, None, dw, 0, ws)
    torch.cuda.synchronize()
    o = sh.norm_bwd(y[rows], None, few, None, None, None, None, w, "none", False, 1.0, 1e-5)
    within(dx[rows], o["dx"], o["e_dx"] + 1.01 * sh.UB * o["dx"].abs() + 1e-38, "dx")
    within(dw, o["dw_pre"], o["e_dw_pre"] * (1 + T / 256 / 500) + 1e-38, "dw_pre")


@pytest.mark.parametrize("d", [64, 128, 256, 512, 1024, 1536, 2048, 2560, 4096, 5120, 8192, 12288, 16384])
@pytest.mark.parametrize("T", [1, 5, 1030])
def test_rows_behind_the_last_one_and_bytes_behind_the_workspace(T, d):
    """Arrays of more rows than the call has: those hold NaNs, are not read and not written; a
    workspace of just the bytes that are asked for."""
    if T * d > 1 << 22:
        T = 70
    c, more = Case(T, d, gate="silu"), 9
    names = ("x", "h", "G", "dy", "dxo", "xo", "y", "dx", "dh", "dG")
    whole = {}
    for name in names:
        part = getattr(c, name)
        whole[name] = torch.full((T + more, d), float("nan"), dtype=part.dtype, device="cuda")
        whole[name][:T] = part
        setattr(c, name, whole[name][:T])
    need = mapl.norm_workspace_bytes(c.D)
    c.ws = torch.full((need + 65536,), 90, dtype=torch.uint8, device="cuda")
    c.fwd()
    c.bwd(ws_bytes=need)
    torch.cuda.synchronize()
    assert all(t[T:].isnan().all() for t in whole.values()) and (c.ws[need:] == 90).all()
    c.check()


def test_two_calls_at_once():
    """Two streams side by side, each with its own arrays and workspace."""
    cases = [Case(3000, 1024, gate="silu", seed=1), Case(2000, 2048, "f32", "bf16", seed=2)]
    want = []
    for c in cases:
        c.fwd()
        c.bwd()
        torch.cuda.synchronize()
        want.append(c.outputs())
    streams = [torch.cuda.Stream() for _ in cases]
    for _ in range(10):
        for c, s in zip(cases, streams):
            with torch.cuda.stream(s):
                c.fwd()
                c.bwd()
    torch.cuda.synchronize()
    for c, w in zip(cases, want):
        assert all(torch.equal(v, w[k]) for k, v in c.outputs().items())
