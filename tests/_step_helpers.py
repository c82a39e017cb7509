"""Plain 64-bit forms of the norms around a block, of the gradients' norm and of
AdamW with fp32 and 8-bit states (torch, on whatever device their inputs live),
written from the formulas in include/mapl.h, with the element-by-element error
bounds that the kernels' arithmetic allows."""
import math

import torch

U24 = 2.0 ** -24  # fp32 unit roundoff
UB = 2.0 ** -8    # bf16 unit roundoff (8 significant bits)


def half_step(dt):
    return UB if dt == torch.bfloat16 else U24


# ------------------------------------------------------------------- norms
def act(G, kind):
    """act(G), its derivative, and the derivative's terms taken by their size."""
    if kind == "none":
        one = torch.ones((), dtype=torch.float64, device=G.device if G is not None else "cpu")
        return one, 0.0 * one, 0.0 * one
    G = G.double()
    a, b = torch.sigmoid(G), torch.sigmoid(-G)
    if kind == "sigmoid":
        return a, a * b, a * b
    return G * a, a * (1 + G * b), a * (1 + G.abs() * b)


def rms(z, eps):
    return 1.0 / torch.sqrt(z.square().mean(1, keepdim=True) + eps)


def _vec(w):
    return 1.0 if w is None else w.double()


def norm_fwd(x, h, G, w_post, scale, kind, post, alpha, eps):
    """x' (not rounded) and the size of what is added, both float64."""
    t = h.double()
    if post:
        t = t * rms(t, eps) * _vec(w_post)
    if kind != "none":
        t = t * act(G, kind)[0]
    t = alpha * _vec(scale) * t
    return x.double() + t, t.abs()


def norm_y(xo, w_pre, eps):
    xo = xo.double()
    return xo * rms(xo, eps) * _vec(w_pre)


# A row's sum of squares: at most 16 products in a lane, 6 steps over a wave and 16
# waves, each rounded: 64 u of it; the root, the division and eps's fma: 34 u of r.
R = 36 * U24


def norm_fwd_errors(x, xo, t, y, pre_dt, G=None):
    """Bounds of |x' - form| and |y - norm_y(x')|: t has r, three products, act (8 u, and a
    bf16 gate's exponent is off by 1.3 |G| u) and the sum's rounding; y r and two products; each
    its type's rounding."""
    gate = 1.3 * U24 * G.double().abs() if G is not None and G.dtype == torch.bfloat16 else 0.0
    e_x = (R + 16 * U24 + gate) * t + U24 * (x.double().abs() + t) + 1.01 * half_step(x.dtype) * xo.abs()
    e_y = None if y is None else (R + 4 * U24 + 1.01 * half_step(pre_dt)) * y.abs() + 1e-40
    return e_x + 1e-40, e_y


def norm_bwd(dy, dxo, xo, h, G, w_post, scale, w_pre, kind, post, alpha, eps):
    """dict of the gradients in float64 and, in "e_" + name, of the bounds without the
    results' own rounding (dx as the kernel goes on with it).  Sizes: A is the sum
    of the sizes of dx's terms, Q of what dh is made of.  r enters dx three times
    (3 R), the row's sums are off by 64 u of their terms' sizes."""
    o, n_t = {}, (h if h is not None else xo).shape[0]
    chain = (500 + n_t / 256) * U24  # a term's error, and the sum over a lane's, a workgroup's and all parts
    dx = None if dxo is None else dxo.double()
    A = None if dxo is None else dx.abs()
    if dy is not None:
        x = xo.double()
        d = x.shape[1]
        r, q = rms(x, eps), dy.double() * _vec(w_pre)
        own = r * (q - x * r * (r * (q * x).sum(1, keepdim=True) / d))
        size = r * (q.abs() + x.abs() * r * (r * (q * x).abs().sum(1, keepdim=True) / d))
        dx, A = (own, size) if dx is None else (dx + own, A + size)
        o["dw_pre"] = (dy.double() * x * r).sum(0)
        o["e_dw_pre"] = chain * (dy.double() * x * r).abs().sum(0)
        e = (3 * R + 64 * U24 + 8 * U24) * A
        o["dx"], o["e_dx"] = dx, e
    if h is not None:
        h = h.double()
        d = h.shape[1]
        f, df, dfa = act(G, kind)
        r = rms(h, eps) if post else torch.ones((), dtype=torch.float64, device=h.device)
        w = _vec(w_post) if post else 1.0
        n = h * r * w
        by = alpha * _vec(scale)
        o["dscale"] = (alpha * dx * n * f).sum(0)
        o["e_dscale"] = chain * (abs(alpha) * A * (n * f).abs()).sum(0)
        gate = 2.6 * U24 * G.double().abs() if kind != "none" and G.dtype == torch.bfloat16 else 0.0  # (act and 1 - sigmoid)
        if kind != "none":
            o["dgate"] = by * dx * n * df
            o["e_dgate"] = (4 * R + 120 * U24 + gate) * A * (by * n * dfa).abs()
        dn = by * dx * f
        if post:
            o["dw_post"] = (dn * h * r).sum(0)
            o["e_dw_post"] = chain * ((by * f).abs() * A * (h * r).abs()).sum(0)
            q, Q = dn * w, (by * f * w).abs() * A
            o["dh"] = r * (q - h * r * (r * (q * h).sum(1, keepdim=True) / d))
            o["e_dh"] = (6 * R + 220 * U24) * r * (Q + h.abs() * r * (r * (Q * h.abs()).sum(1, keepdim=True) / d))
        else:
            o["dh"], o["e_dh"] = dn, (3 * R + 100 * U24) * (by * f).abs() * A
    return o


# --------------------------------------------------------------- optimizer
def f32(v):
    """A number as fp32 has it."""
    return float(torch.tensor(v, dtype=torch.float32))


def rounded(x):
    """float64 to the nearest fp32, as float64."""
    return x.to(torch.float32).double()


def two_to(n):
    """2^n of whole numbers (exact: built from the bits)."""
    return ((n.long() + 1023) << 52).view(torch.float64)


def new_states(m, v, g, b1, b2):
    """m and v after a step, and sqrt(v), fp32 values as float64: every operation rounded."""
    c1, c2 = f32(1.0 - f32(b1)), f32(1.0 - f32(b2))
    m, v, g = m.double(), v.double(), g.double()
    m = rounded(m + rounded(rounded(g - m) * c1))
    v = rounded(v + rounded(rounded(rounded(g * g) - v) * c2))
    return m, v, rounded(v.sqrt())


def new_p(p, m, root, t, lr, b1, b2, eps, wd):
    """p after a step (float64) and the bound of the kernel's error: the corrections,
    root, quotient and products are each off by a few u (24 in all)."""
    b1, b2, lr, eps, wd = (f32(x) for x in (b1, b2, lr, eps, wd))
    up = lr / (1 - b1 ** t) * (m / (root / math.sqrt(1 - b2 ** t) + eps))
    p = p.double()
    q = p - (lr * wd * p + up)
    return q, U24 * (q.abs() + 24 * up.abs() + 4 * (lr * wd * p).abs()) + 1e-42


def hash32(x):
    """The 32 bits of a 32-bit number (int64 tensors)."""
    M = 2 ** 32
    x = torch.as_tensor(x) % M
    x = ((x ^ (x >> 16)) * 2654435769) % M
    x = ((x ^ (x >> 15)) * 1779033703) % M
    return x ^ (x >> 16)


def noise(seed, t, index, n, device):
    key = hash32(hash32(hash32(torch.tensor(seed, device=device)) + t) ^ index)
    return hash32(key + torch.arange(n, device=device))


def decode(qm, qs, e):
    """m and s of codes [n] and exponent bytes [ceil(n/128), 2], float64."""
    n = qm.numel()
    e = e.long().view(-1, 2).repeat_interleave(128, 0)[:n]
    c = qm.long()
    a, neg = c % 128, c >= 128
    E, f = torch.div(a, 8, rounding_mode="floor"), a % 8
    m = torch.where(E > 0, (8 + f) * two_to(E - 10), f * two_to(E * 0 - 9))
    m = torch.where(neg, -m, m) * two_to(e[:, 0] - 135)
    c = qs.long()
    E, f = torch.div(c, 16, rounding_mode="floor"), c % 16
    s = torch.where(E > 0, (16 + f) * two_to(E - 19), f * two_to(E * 0 - 18)) * two_to(e[:, 1] - 127)
    empty, bad = e < 24, e == 255
    nan = torch.full_like(m, float("nan"))
    m = torch.where(bad[:, 0], nan, torch.where(empty[:, 0], 0 * s, m))
    return m, torch.where(bad[:, 1], nan, torch.where(empty[:, 1], torch.zeros_like(s), s))


def encode(m, s, r):
    """Codes and bytes of fp32 values m and s (float64 tensors) with the 32-bit noise r
    (a number or a tensor): a grid point's share of the way to the next decides."""
    n = m.numel()
    nb = -(-n // 128)
    r = torch.zeros(n, dtype=torch.int64, device=m.device) + r
    pad = lambda x: torch.cat([x, torch.zeros(nb * 128 - n, dtype=x.dtype, device=x.device)]).view(nb, 128)
    out = []
    for x, top, bits, low, peak, u in ((m, 1.75, 3, -6, 8, r % 65536), (s, 1.9375, 4, -14, 0, r >> 16)):
        y, u = pad(x.abs()), pad(u).double() / 65536
        bad = ~torch.isfinite(y).all(1)
        a = torch.where(bad[:, None], torch.zeros_like(y), y).amax(1)
        frac, k = torch.frexp(a)
        k = k.long() - 1 + (2 * frac > top).long()
        k = torch.where(a > 0, k, torch.full_like(k, -103)).clamp(min=-103)
        bad |= k > 127
        y = torch.where(bad[:, None], torch.zeros_like(y), y) * two_to(peak - k)[:, None]
        E = torch.frexp(y)[1].long() - 1
        E = torch.where(y > 0, E, torch.full_like(E, low)).clamp(min=low)  # the binade, or that of the equal steps
        whole = torch.floor(y / two_to(E - bits) + u).long()  # in steps of the binade
        code = torch.where(y >= 2.0 ** low, (E - low) * 2 ** bits + whole, whole)
        if peak == 0:
            code = torch.maximum(code, (y > 0).long())
        out += [code, torch.where(bad, torch.full_like(k, 255), k + 127)]
    cm, em, cs, es = out
    cm = cm + 128 * pad(torch.signbit(m).long())
    return cm.view(-1)[:n], cs.view(-1)[:n], torch.stack([em, es], 1)
