"""The 64-bit forms that the norms and the optimizer are held to, pinned to
numbers worked out by hand, to torch's autograd and to torch's own AdamW."""
import math

import pytest
import torch

import _step_helpers as sh

f64 = torch.float64


def test_norm_by_hand():
    x = torch.tensor([[3.0, 4.0]], dtype=f64)  # mean of squares 12.5
    y = sh.norm_y(x, torch.tensor([2.0, 1.0]), 0.0)
    assert torch.allclose(y, torch.tensor([[6.0, 4.0]], dtype=f64) / math.sqrt(12.5))
    xo, t = sh.norm_fwd(x, torch.tensor([[1.0, -1.0]]), torch.tensor([[0.0, 0.0]]), None, torch.tensor([1.0, 4.0]), "sigmoid", True, 0.5, 0.0)
    assert torch.allclose(xo, torch.tensor([[3.25, 3.0]], dtype=f64)) and torch.allclose(t, torch.tensor([[0.25, 1.0]], dtype=f64))


@pytest.mark.parametrize("kind", ["none", "sigmoid", "silu"])
@pytest.mark.parametrize("post,pre,branch", [(True, True, True), (False, True, True), (True, False, True), (False, True, False)])
def test_norm_gradients_against_autograd(kind, post, pre, branch):
    if not branch and kind != "none":
        pytest.skip("a gate needs a branch")
    g = torch.Generator().manual_seed(3)
    rn = lambda *s: torch.randn(*s, generator=g, dtype=f64)
    T, d, alpha, eps = 5, 8, 0.7, 1e-3
    x, h, G, wp, s, w, dy, dxo = rn(T, d), rn(T, d), rn(T, d), rn(d), rn(d), rn(d), rn(T, d), rn(T, d)
    leaves = [t.requires_grad_() for t in (x, h, G, wp, s, w)]
    xo = sh.norm_fwd(x, h, G, wp, s, kind, post, alpha, eps)[0] if branch else x
    out = (xo * dxo).sum() + ((sh.norm_y(xo, w, eps) * dy).sum() if pre else 0.0)
    want = torch.autograd.grad(out, leaves, allow_unused=True)
    D = lambda t: t.detach()
    with torch.no_grad():
        o = sh.norm_bwd(dy if pre else None, dxo, D(xo), h if branch else None, G, wp, s, w, kind, post, alpha, eps)
    got = [o.get("dx", dxo if branch else None), o.get("dh"), o.get("dgate"), o.get("dw_post"), o.get("dscale"), o.get("dw_pre")]
    for a, b in zip(got, want):
        assert (a is None) == (b is None)
        assert a is None or torch.allclose(a, b, rtol=1e-12, atol=1e-13)


def test_bounds_hold_for_fp32_and_tell_a_mistake():
    # the forms evaluated in fp32 lie inside the bounds; a gradient without its mean term does not
    g = torch.Generator().manual_seed(4)
    rn = lambda *s: torch.randn(*s, generator=g)
    T, d = 6, 64
    x, dy, dxo, w = rn(T, d), rn(T, d), rn(T, d), rn(d)
    o = sh.norm_bwd(dy, dxo, x, None, None, None, None, w, "none", False, 1.0, 1e-5)
    r = torch.rsqrt(x.square().mean(1, keepdim=True) + 1e-5)
    q = dy * w
    dx = dxo + r * (q - x * r * r * (q * x).mean(1, keepdim=True))
    tol = o["e_dx"] + sh.U24 * o["dx"].abs()
    assert ((dx.double() - o["dx"]).abs() <= tol).all()
    assert (((dxo + r * q).double() - o["dx"]).abs() > tol).any()


def test_adamw_against_torchs_own():
    g = torch.Generator().manual_seed(5)
    p = torch.randn(50, generator=g, dtype=f64)
    q = p.clone().requires_grad_()
    opt = torch.optim.AdamW([q], lr=0.0625, betas=(0.875, 0.96875), eps=2.0 ** -20, weight_decay=0.125)
    m = v = torch.zeros(50, dtype=f64)
    for t in range(1, 6):
        gr = torch.randn(50, generator=g).double()
        q.grad = gr.clone()
        opt.step()
        m, v, root = sh.new_states(m, v, gr, 0.875, 0.96875)
        p, _ = sh.new_p(p, m, root, t, 0.0625, 0.875, 0.96875, 2.0 ** -20, 0.125)
    assert torch.allclose(p, q.detach(), rtol=1e-6, atol=1e-7)  # (the states here are fp32)


def test_hash_by_hand():
    assert int(sh.hash32(0)) == 0
    x = (1 * 2654435769) % 2 ** 32
    x = ((x ^ (x >> 15)) * 1779033703) % 2 ** 32
    assert int(sh.hash32(1)) == x ^ (x >> 16)


def test_noise_is_even_and_does_not_repeat():
    # 2^18 draws: the mean of a uniform number is off by 1 / sqrt(12 n) = 5.6e-4 (5 of it allowed)
    for seed, t, i in ((0, 1, 0), (7, 2, 3)):
        r = sh.noise(seed, t, i, 1 << 18, "cpu")
        for u in ((r % 65536) / 65536.0, (r >> 16) / 65536.0):
            assert abs(float(u.mean()) + 2.0 ** -17 - 0.5) < 2.9e-3
            c = torch.corrcoef(torch.stack([u[:-1], u[1:]]))[0, 1]
            assert abs(float(c)) < 5 / 512
    a, b = sh.noise(0, 1, 0, 4096, "cpu"), sh.noise(0, 2, 0, 4096, "cpu")
    assert int((a == b).sum()) < 3


def test_codes_by_hand():
    e = torch.tensor([[135, 127]], dtype=torch.uint8)  # units: m code x 1, s code x 1
    qm = torch.tensor([0, 1, 8, 0x38, 0x7e, 0xb8], dtype=torch.uint8)
    qs = torch.tensor([0, 1, 15, 16, 240, 255], dtype=torch.uint8)
    m, s = sh.decode(qm, qs, e)
    assert m.tolist() == [0.0, 2.0 ** -9, 2.0 ** -6, 1.0, 448.0, -1.0]
    assert s.tolist() == [0.0, 2.0 ** -18, 15 * 2.0 ** -18, 2.0 ** -14, 1.0, 1.9375]
    assert torch.equal(qm[:5].view(torch.float8_e4m3fn).double(), m[:5])


def test_every_code_comes_back():
    c = torch.arange(256)
    for scale in (0, 60, -90):
        m, s = sh.decode(c % 127 + 128 * (c > 127), c, torch.tensor([[135 + scale, 127 + scale]] * 2))
        qm, qs, e = sh.encode(m, s, 0x80008000)
        assert torch.equal(sh.decode(qm, qs, e)[0], m) and torch.equal(sh.decode(qm, qs, e)[1], s)
        assert torch.equal(sh.encode(m, s, 0)[1], qs) and torch.equal(sh.encode(m, s, 0xffffffff)[1], qs)  # no noise moves a code


def test_rounding_up_has_the_share_of_the_way():
    # 1 + 3/32 lies half-way of 1 + 1/16 and 1 + 1/8 (s), 3/4 of the way of 1 and 1 + 1/8 (m)
    n = 1 << 16
    x = torch.full((n,), 1 + 3 / 32, dtype=f64)
    x[::128] = 1.5  # the blocks' largest: a scale of 1
    r = torch.arange(n) * 65537 % 2 ** 32  # every 16 bits once, in both halves
    qm, qs, e = sh.encode(x, x, r)
    m, s = sh.decode(qm, qs, e)
    live = torch.arange(n) % 128 != 0
    assert set(s[live].tolist()) == {1 + 1 / 16, 1 + 1 / 8} and set(m[live].tolist()) == {1.0, 1 + 1 / 8}
    assert abs(float((s[live] > 1.1).double().mean()) - 0.5) < 1e-3 and abs(float((m[live] > 1.0).double().mean()) - 0.75) < 1e-3


def test_blocks_of_nan_zero_and_tiny_values():
    m = torch.zeros(384, dtype=f64)
    s = torch.zeros(384, dtype=f64)
    m[5], s[130], s[260] = float("nan"), float("inf"), 1e-45
    qm, qs, e = sh.encode(m, s, 0)
    assert e.tolist() == [[255, 24], [24, 255], [24, 24]]
    a, b = sh.decode(qm, qs, e)
    assert a[:128].isnan().all() and (a[128:] == 0).all() and b[128:256].isnan().all()
    assert float(b[260]) == 2.0 ** -121 and int((b[256:] != 0).sum()) == 1  # above 0 stays above 0
    assert (sh.decode(qm * 0, qs * 0, e * 0)[0] == 0).all()


def test_kept_to_nearest_the_second_moment_stands_still_and_at_random_it_follows():
    """What the random rounding is for: v decaying by 1 % a step.  Its steps are below half a
    code's distance, so that rounding to nearest keeps it where it was; at random its mean
    follows.  (A value's spread then is half the root of the codes' distance, 0.09 to 0.13 of s; the mean of 1280
    values is off by 0.13 / 36 of s, five of that and the mean's own excess (0.13^2 / 2 of s) allowed.)"""
    n = 1280
    start = torch.full((n,), 1.0, dtype=f64)
    start[::128] = 1.9375
    last = {}
    for kind in ("nearest", "random"):
        s = start.clone()
        for t in range(1, 61):
            v = torch.where(torch.arange(n) % 128 == 0, s * s, 0.99 * s * s)
            root = sh.rounded(sh.rounded(v).sqrt())
            r = 0x80008000 if kind == "nearest" else sh.noise(1, t, 0, n, "cpu")
            qm, qs, e = sh.encode(0 * root, root, r)
            s = sh.decode(qm, qs, e)[1]
        last[kind] = s[torch.arange(n) % 128 != 0]
    assert (last["nearest"] == 1.0).all()
    want = 0.99 ** 30
    assert abs(float(last["random"].mean()) / want - 1) < 5 * 0.13 / 36 + 0.13 ** 2 / 2
