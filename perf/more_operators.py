"""What a training step does around its matrix products, as measurable cases.

A case is a dict of plain values; "op" names what one pass does:

  norm        x' = x + alpha s (rms(h) w_post) act(G), y = rms(x') w_pre: what follows a block
              and precedes the next, in one pass ("branch": the sum, "post": the norm of h,
              "pre": y; a final norm is "pre" alone)
  norm_bwd    its gradient with respect to x, h, G and the three vectors
  grad_norm   the norm of all gradients of a step and the factor that clips it
  adamw       a step of AdamW over all of a stage's tensors, states in fp32 or in 8 bits; the
              states come back as the values they stand for

Activations have outlier channels and a few all-zero tokens (padding); gradients have a size
of their own for every tensor.  8-bit states: blocks of 128 values of a tensor with a power of
two each for m (sign, 4 exponent and 3 mantissa bits) and for sqrt(v) (4 and 4 bits),
stochastically rounded by 16 bits of a hash of seed, step, tensor and place.  What is rounded to
8 bits is an fp32 number, every operation of m + (1 - b1)(g - m), v + (1 - b2)(g g - v) and the
root rounded to nearest, by definition: else a value next to a border would have no one result.
"""
import math

import torch

own = False
DEV = "cuda"
BLOCK = 128  # values of a tensor that share a scale
PIECE = 1024  # tensors begin at multiples of this in the flat arrays that hold them
EPS = 1e-5


def _norm(op, T, d, x="bf16", h="bf16", branch=True, post=True, pre=True, gate="sigmoid", halves=False, name=None):
    c = dict(op=op, T=T, d=d, x=x, h=h, branch=branch, post=post, pre=pre, gate=gate, halves=halves)
    return dict(c, name=name) if name else c


def _step(op, d, f, layers, V, matrices=True, g="bf16", states="f32", t=1000, name=None):
    c = dict(op=op, d=d, f=f, layers=layers, V=V, matrices=matrices, g=g)
    if op == "adamw":
        c.update(states=states, t=t)
    else:
        c.update(clip=1.0)
    return dict(c, name=name) if name else c


def listed():
    return [
        # one token through the last norm before the head (a decoded token): latency
        _norm("norm", 1, 2048, branch=False, post=False, gate="none", name="norm_one_token"),
        # 150M model, micro-batch 4 x 2048: after a gated block and before the next
        _norm("norm", 8192, 1024, name="norm_150m"),
        # 1B model, micro-batch 16 x 2048: h and its gate are the halves of one product's output
        _norm("norm", 32768, 2048, gate="silu", halves=True, name="norm_1b_halves"),
        # the smallest configuration's activations, fp32: the norm before the head
        _norm("norm_bwd", 512, 256, x="f32", h="f32", branch=False, post=False, gate="none", name="norm_bwd_f32_small"),
        # a short, odd micro-batch (a sequence's tail), residual stream in fp32, block in bf16
        _norm("norm_bwd", 1021, 1024, x="f32", gate="silu", name="norm_bwd_tail"),
        # 1B model, micro-batch 16 x 2048
        _norm("norm_bwd", 32768, 2048, name="norm_bwd_1b"),
        # a small stage's gradients in fp32, tensors of odd lengths among them
        _step("grad_norm", 256, 704, 1, 1003, g="f32", name="grad_norm_small"),
        # a 1B model's last stage (four layers and the head), gradients in bf16
        _step("grad_norm", 2048, 5440, 4, 32000, name="grad_norm_1b"),
        # the norms' weights alone (another optimizer has the matrices): many tensors, little work
        _step("adamw", 2048, 5440, 20, 0, matrices=False, g="f32", name="adamw_vectors"),
        # a 150M model's last stage, gradients accumulated in fp32, a vocabulary of odd size
        _step("adamw", 1024, 2688, 3, 32003, g="f32", states="8bit", name="adamw_8bit_150m"),
        # a 1B model's last stage, states in fp32
        _step("adamw", 2048, 5440, 4, 32000, name="adamw_f32_1b"),
        # the same with states in 8 bits
        _step("adamw", 2048, 5440, 4, 32000, states="8bit", name="adamw_8bit_1b"),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["norm", "norm", "norm_bwd", "norm_bwd", "grad_norm", "adamw", "adamw"])
    if op in ("norm", "norm_bwd"):
        d = 64 * _log(rng, 1, 256)
        x, h = rng.choice([("bf16", "bf16"), ("bf16", "bf16"), ("f32", "bf16"), ("f32", "f32")])
        T = _log(rng, 1, max(1, (32768 if x == "bf16" else 16384 if h == "bf16" else 8192) * 2048 // d))
        branch = rng.random() < 0.7
        return _norm(op, T, d, x, h, branch, branch and rng.random() < 0.6, not branch or rng.random() < 0.7,
                     rng.choice(["none", "sigmoid", "silu"]) if branch else "none", branch and rng.random() < 0.4)
    d = 64 * rng.randint(1, 32)
    layers, V = rng.randint(1, 20), _log(rng, 2, 40000)
    matrices = rng.random() < 0.8
    most = 6 if op == "grad_norm" else 4
    while matrices and layers > 1 and layers * 12 * d * d + V * d > most * 40 * 1024 * 1024:
        layers -= 1
    return _step(op, d, 8 * (d // 3), layers, V, matrices, rng.choice(["f32", "bf16"]) if op == "grad_norm" else
                 rng.choice(["bf16", "f32"]), rng.choice(["f32", "8bit"]), _log(rng, 1, 100000))


# ------------------------------------------------------------------- inputs
def _gen(seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(int(seed))
    return g


def _rn(g, *shape):
    return torch.randn(*shape, generator=g, device=DEV)


def _dt(name):
    return torch.bfloat16 if name == "bf16" else torch.float32


def _rows(g, T, d, dt):
    x = _rn(g, T, d) * (0.5 + torch.rand(T, 1, generator=g, device=DEV))
    x[:, torch.randperm(d, generator=g, device=DEV)[:max(1, d // 128)]] *= 20.0
    if T > 1:
        x[torch.rand(T, generator=g, device=DEV) < 0.01] = 0.0
    return x.to(dt)


def _tensors(c):
    """(values, decayed) of every tensor of the stage: matrices first."""
    d, f, V = c["d"], c["f"], c["V"]
    big = ([V * d] + c["layers"] * (4 * [d * d] + 3 * [d * f])) if c["matrices"] else []
    small = c["layers"] * [d, d] + [d, 1] + ([V] if V else [])
    return [(n, True) for n in big] + [(n, False) for n in small]


def _places(c):
    """Where each tensor begins in the flat arrays, their length, and the decayed values' end."""
    at, here, end = [], 0, 0
    for n, decayed in _tensors(c):
        at.append(here)
        here += -(-n // PIECE) * PIECE
        end = here if decayed else end
    return at, here, end


def _cut(a, c):
    """The tensors of a flat array."""
    return [a[i:i + n] for i, (n, _) in zip(_places(c)[0], _tensors(c))]


def _pow2(e):
    """2^e of whole numbers, exact (a library's exp2 may be off in the last place)."""
    return ((e.to(torch.int32) + 127) << 23).view(torch.float32)


def _scale(a, room):
    """A block's exponent byte: the largest magnitude is at most 1.75 (m) or 1.9375 (sqrt v) of its power of two."""
    e = (a.view(torch.int32).amax(1) + room) >> 23
    return e.clamp(min=24)


def _codes(y, bits, low, noise):
    """Codes of y >= 0: `bits` mantissa bits, whole steps of 2^(low - bits) below 2^low."""
    drop = 23 - bits
    t = torch.where(y >= 2.0 ** low, y.view(torch.int32) - ((126 + low) << 23), (y * 2.0 ** (23 - low)).to(torch.int32))
    return (t + (noise.to(torch.int32) << (drop - 16))) >> drop


def _value(code, bits, low):
    """What a code stands for."""
    e, f = code >> bits, code & ((1 << bits) - 1)
    return torch.where(e > 0, _pow2(e - 1 + low) * (1.0 + f * 2.0 ** -bits), f * 2.0 ** (low - bits))


def _packed(m, s, noise_m, noise_s):
    """m and s = sqrt(v), [blocks, BLOCK], as codes and exponent bytes."""
    em, es = _scale(m.abs(), 0x1fffff), _scale(s, 0x7ffff)
    cm = _codes(m.abs() * _pow2(135 - em)[:, None], 3, -6, noise_m)
    cs = _codes(s * _pow2(127 - es)[:, None], 4, -14, noise_s)
    cs = torch.maximum(cs, (s > 0).to(torch.int32))
    return (cm + 128 * (m < 0)).to(torch.uint8), cs.to(torch.uint8), torch.stack([em, es], 1).to(torch.uint8)


def _unpacked(qm, qv, e):
    """m and s, [blocks, BLOCK], from codes and exponent bytes (0 at the start: all values 0)."""
    cm, cs, e = qm.to(torch.int32).view(-1, BLOCK), qv.to(torch.int32).view(-1, BLOCK), e.to(torch.int32).view(-1, 2)
    m = _value(cm & 127, 3, -6) * _pow2(e[:, 0] - 135)[:, None]
    return torch.where(cm > 127, -m, m), _value(cs, 4, -14) * _pow2(e[:, 1] - 127)[:, None]


def prepare(case, seed):
    c, g = case, _gen(seed)
    s = dict(case=c)
    if c["op"] in ("norm", "norm_bwd"):
        T, d, xt, ht = c["T"], c["d"], _dt(c["x"]), _dt(c["h"])
        new = lambda dt, on=True: torch.empty(T, d, dtype=dt, device=DEV) if on else None
        vec = lambda on, by=1.0: (by * (1.0 + 0.2 * _rn(g, d))) if on else None
        s["alpha"] = 0.5 if c["branch"] else 1.0
        gated = c["branch"] and c["gate"] != "none"
        hg = torch.empty(T, 2 * d, dtype=ht, device=DEV) if c["halves"] else None
        s["x"] = _rows(g, T, d, xt)
        s["h"] = _rows(g, T, d, ht) if c["branch"] else None
        s["G"] = (2.0 * _rn(g, T, d)).to(ht) if gated else None
        if c["halves"]:
            hg[:, :d] = s["h"]
            s["h"] = hg[:, :d]
            if gated:
                hg[:, d:] = s["G"]
                s["G"] = hg[:, d:]
        s["w_post"], s["s"], s["w_pre"] = vec(c["post"]), vec(c["branch"], 0.3), vec(c["pre"])
        if c["op"] == "norm":
            s["x1"], s["y"] = new(xt, c["branch"]), new(ht, c["pre"])
        else:
            s["dy"] = (1e-3 * _rn(g, T, d)).to(ht) if c["pre"] else None
            s["dx1"] = (1e-3 * _rn(g, T, d)).to(xt)
            dhg = torch.empty(T, 2 * d, dtype=ht, device=DEV) if c["halves"] else None
            s["dx"] = new(xt, c["pre"])
            s["dh"] = dhg[:, :d] if c["halves"] else new(ht, c["branch"])
            s["dG"] = None if not gated else dhg[:, d:] if c["halves"] else new(ht)
            for v in ("w_post", "s", "w_pre"):
                s["d" + v] = None if s[v] is None else torch.empty(d, device=DEV)
        return s
    at, n, end = _places(c)
    G = torch.zeros(n, dtype=_dt(c["g"]), device=DEV)
    adam = c["op"] == "adamw"
    if adam:
        P, m, v = (torch.zeros(n, device=DEV) for _ in range(3))
    for i, (size, _) in zip(at, _tensors(c)):
        sd = 10.0 ** float(-5.0 + 3.0 * torch.rand(1, generator=g, device=DEV))
        G[i:i + size] = sd * _rn(g, size)
        if adam:
            P[i:i + size] = 0.02 * _rn(g, size)
            m[i:i + size] = 0.25 * sd * _rn(g, size)
            v[i:i + size] = sd * sd * (0.5 + torch.rand(size, generator=g, device=DEV))
    s["G"] = G
    if not adam:
        s["stats"] = torch.empty(4, device=DEV)
        return s
    s.update(P=P, P16=torch.zeros(n, dtype=torch.bfloat16, device=DEV), end=end, lr=3e-4, b1=0.9, b2=0.95, eps=1e-8, wd=0.1, seed=int(seed) & 0xffff)
    s["stats"] = torch.tensor([2.0, 0.5, 0.0, 0.0], device=DEV)  # a norm of 2 that was clipped to 1
    if c["states"] == "f32":
        s.update(m=m, v=v)
        return s
    half = torch.full((1, 1), 1 << 15, dtype=torch.int32, device=DEV)
    s["qm"], s["qv"], s["e"] = (t.reshape(-1) for t in _packed(m.view(-1, BLOCK), v.sqrt().view(-1, BLOCK), half, half))
    s["m"], s["v"] = m, v  # where the values go
    sizes = torch.tensor([-(-k // PIECE) * PIECE // BLOCK for k, _ in _tensors(c)], device=DEV)
    s["of"] = torch.repeat_interleave(torch.arange(len(sizes), device=DEV), sizes)  # a block's tensor
    s["nth"] = torch.arange(n // BLOCK, device=DEV) - (torch.cumsum(sizes, 0) - sizes)[s["of"]]  # and its number there
    return s


# ---------------------------------------------------------------------- run
def _rms(x):
    return torch.rsqrt(x.square().mean(1, keepdim=True) + EPS)


def _act(G, kind):
    """act(G) and its derivative."""
    a = 1.0 / (1.0 + torch.exp(-G))
    return (a, a * (1.0 - a)) if kind == "sigmoid" else (G * a, a * (1.0 + G * (1.0 - a)))


def _plain_norm(s):
    c, xt, ht = s["case"], _dt(s["case"]["x"]), _dt(s["case"]["h"])
    out, x = {}, s["x"].float()
    if c["branch"]:
        t = s["h"].float()
        if c["post"]:
            t = t * _rms(t) * s["w_post"]
        if s["G"] is not None:
            t = t * _act(s["G"].float(), c["gate"])[0]
        out["x1"] = (x + s["alpha"] * s["s"] * t).to(xt)
        x = out["x1"].float()
    if c["pre"]:
        out["y"] = (x * _rms(x) * s["w_pre"]).to(ht)
    return out


def _plain_norm_bwd(s):
    c, xt, ht = s["case"], _dt(s["case"]["x"]), _dt(s["case"]["h"])
    out, dx = {}, s["dx1"].float()
    if c["pre"]:
        x, dy = s["x"].float(), s["dy"].float()
        r = _rms(x)
        out["dw_pre"] = (dy * x * r).sum(0)
        dy = dy * s["w_pre"]
        dx = dx + r * (dy - x * (r * r * (dy * x).mean(1, keepdim=True)))
        out["dx"] = dx.to(xt)
    if c["branch"]:
        h = n = s["h"].float()
        if c["post"]:
            r = _rms(h)
            n = h * r * s["w_post"]
        a, b = _act(s["G"].float(), c["gate"]) if s["G"] is not None else (None, None)
        out["ds"] = (s["alpha"] * dx * (n if a is None else n * a)).sum(0)
        dn = s["alpha"] * s["s"] * dx
        if a is not None:
            out["dG"] = (dn * n * b).to(ht)
            dn = dn * a
        if c["post"]:
            out["dw_post"] = (dn * h * r).sum(0)
            dn = dn * s["w_post"]
            dn = r * (dn - h * (r * r * (dn * h).mean(1, keepdim=True)))
        out["dh"] = dn.to(ht)
    return out


def _mix(x):
    """A hash of 32 bits (in int64): every bit of the result depends on every bit of x."""
    x = x & 0xffffffff
    x = ((x ^ (x >> 16)) * 0x9E3779B9) & 0xffffffff
    x = ((x ^ (x >> 15)) * 0x6A09E667) & 0xffffffff
    return x ^ (x >> 16)


def _noise(s):
    """32 bits for every value, [blocks, BLOCK]: of the seed, the step, the tensor and the place in it."""
    word = torch.tensor(s["seed"], device=DEV)
    key = _mix(_mix(_mix(word) + s["case"]["t"]) ^ s["of"])
    return _mix((key + s["nth"] * BLOCK)[:, None] + torch.arange(BLOCK, device=DEV))


def _plain_adamw(s):
    c, p = s["case"], s["P"]
    low = c["states"] == "8bit"
    b1, b2 = (float(torch.tensor(s[b])) for b in ("b1", "b2"))  # as fp32 has them
    g = s["G"].float() * s["stats"][1]
    m, v = s["m"], s["v"]
    if low:
        m, v = (t.reshape(-1) for t in _unpacked(s["qm"], s["qv"], s["e"]))
        v = v * v
    m = m + (g - m) * (1.0 - b1)
    v = v + (g * g - v) * (1.0 - b2)
    root = v.double().sqrt().float() if low else v.sqrt()  # (rounded to 8 bits: no value may cross a border)
    a, r = s["lr"] / (1.0 - b1 ** c["t"]), 1.0 / math.sqrt(1.0 - b2 ** c["t"])
    step = a * (m / (root * r + s["eps"]))
    step[:s["end"]] += s["lr"] * s["wd"] * p[:s["end"]]
    p -= step
    s["P16"].copy_(p)
    if low:
        noise = _noise(s)
        s["qm"], s["qv"], s["e"] = (t.reshape(-1) for t in _packed(m.view(-1, BLOCK), root.view(-1, BLOCK), noise & 0xffff, noise >> 16))
        m, v = (t.reshape(-1) for t in _unpacked(s["qm"], s["qv"], s["e"]))
        v = v * v
    s["m"], s["v"] = m, v
    return {"P": p, "P16": s["P16"], "m": m, "v": v}


def _plain(s):
    c = s["case"]
    if c["op"] == "norm":
        return _plain_norm(s)
    if c["op"] == "norm_bwd":
        return _plain_norm_bwd(s)
    if c["op"] == "adamw":
        return _plain_adamw(s)
    norm = s["G"].double().square().sum().sqrt()
    return torch.stack([norm, torch.clamp(c["clip"] / norm, max=1.0)]).float()


def run(s):
    if not own:
        return _plain(s)
    from paper_2606_05484_amd import mapl
    c = s["case"]
    if c["op"] in ("norm", "norm_bwd"):
        if "N" not in s:
            ld = 2 * c["d"] if c["halves"] else 0
            s["N"] = mapl.norm_desc(c["T"], c["d"], c["x"], c["h"], branch=c["branch"], post=c["post"], pre=c["pre"], gate=c["gate"],
                                    alpha=s["alpha"], eps=EPS, ld_h=ld, ld_gate=ld)
            s["ws"] = mapl.workspace(mapl.norm_workspace_bytes(s["N"])) if c["op"] == "norm_bwd" else None
        if c["op"] == "norm":
            mapl.norm_fwd(s["N"], s["x"], s["h"], s["G"], s["w_post"], s["s"], s["w_pre"], s["x1"], s["y"])
            return {k: s[k] for k, on in (("x1", c["branch"]), ("y", c["pre"])) if on}
        mapl.norm_bwd(s["N"], s["dy"], s["dx1"], s["x"] if c["pre"] else None, s["h"], s["G"], s["w_post"], s["s"], s["w_pre"],
                      s["dx"], s["dh"], s["dG"], s["dw_post"], s["ds"], s["dw_pre"], 0, s["ws"])
        return {k: s[k] for k in ("dx", "dh", "dG", "dw_post", "ds", "dw_pre") if s[k] is not None}
    if "params" not in s:
        cut = lambda k: _cut(s[k], c) if k in s else None
        low = c.get("states") == "8bit"
        decay = [s["wd"] if yes else 0.0 for _, yes in _tensors(c)] if c["op"] == "adamw" else 0.0
        e = [s["e"][i // BLOCK * 2:] for i in _places(c)[0]] if low else None
        s["params"] = mapl.optim_params(cut("G"), cut("P"), cut("qm" if low else "m"), cut("qv" if low else "v"), e, cut("P16"), weight_decay=decay)
        s["values"] = mapl.optim_params(cut("G"), m=cut("m"), v=cut("v")) if low else None
        if c["op"] == "grad_norm":
            s["ws"] = mapl.workspace(mapl.grad_norm_workspace_bytes(s["params"], c["g"]))
    if c["op"] == "grad_norm":
        mapl.grad_norm(s["params"], s["stats"], s["ws"], max_norm=c["clip"], g_dtype=c["g"])
        return s["stats"][:2]
    if "A" not in s:
        s["A"] = mapl.adamw_desc(s["lr"], s["b1"], s["b2"], s["eps"], g_dtype=c["g"], states=c["states"], step=c["t"], seed=s["seed"])
    mapl.adamw_step(s["A"], s["params"], stats=s["stats"])
    if c["states"] == "8bit":
        mapl.adamw_unpack(s["params"], s["values"])
    return {k: s[k] for k in ("P", "P16", "m", "v")}


# --------------------------------------------------------------------- work
def work(case):
    c = case
    if c["op"] in ("norm", "norm_bwd"):
        T, d = c["T"], c["d"]
        xe, he = (2.0 if c[k] == "bf16" else 4.0 for k in ("x", "h"))
        gated = c["branch"] and c["gate"] != "none"
        vecs = 4.0 * d * (c["pre"] + c["branch"] + c["post"])
        if c["op"] == "norm":
            value = xe * (1 + c["branch"]) + he * (c["branch"] + gated + c["pre"])
            return {"bytes": T * d * value + vecs, "flops": T * d * (4.0 * c["pre"] + 3.0 * c["branch"] + 4.0 * c["post"] + 4.0 * gated)}
        value = xe * (1 + 2 * c["pre"]) + he * (c["pre"] + 2 * c["branch"] + 2 * gated)
        return {"bytes": T * d * value + 2 * vecs, "flops": T * d * (11.0 * c["pre"] + 5.0 * c["branch"] + 11.0 * c["post"] + 8.0 * gated)}
    n, ge = float(sum(k for k, _ in _tensors(c))), 2.0 if c["g"] == "bf16" else 4.0
    if c["op"] == "grad_norm":
        return {"bytes": n * ge + 8.0, "flops": 2.0 * n}
    if c["states"] == "f32":
        return {"bytes": n * (8.0 + 2.0 + ge + 16.0), "flops": 16.0 * n}
    return {"bytes": n * (8.0 + 2.0 + ge + 4.0 + 4.0 / BLOCK + 8.0), "flops": 40.0 * n}


# -------------------------------------------------------------------- exact
def _exact_norm(c, s):
    out, x = {}, s["x"].double()
    if c["branch"]:
        t = s["h"].double()
        if c["post"]:
            t = t / (t.pow(2).sum(1, keepdim=True) / c["d"] + EPS).sqrt() * s["w_post"].double()
        if s["G"] is not None:
            u = s["G"].double()
            t = t * torch.sigmoid(u) * (u if c["gate"] == "silu" else 1.0)
        x = x + s["alpha"] * t * s["s"].double()
        out["x1"] = x
    if c["pre"]:
        out["y"] = x / (x.pow(2).sum(1, keepdim=True) / c["d"] + EPS).sqrt() * s["w_pre"].double()
    return out


def _exact_norm_bwd(c, s):
    """From the forward's 64-bit form by differentiation (x' is what the case has as x)."""
    leaf = lambda t: None if t is None else t.detach().double().clone().requires_grad_()
    unit = lambda t: t / (t.pow(2).sum(1, keepdim=True) / c["d"] + EPS).sqrt()
    x, h, G, w_post, sc, w_pre = (leaf(s[k]) for k in ("x", "h", "G", "w_post", "s", "w_pre"))
    out, dx = {}, s["dx1"].double()
    if c["pre"]:
        a, out["dw_pre"] = torch.autograd.grad(unit(x) * w_pre, (x, w_pre), s["dy"].double())
        dx = out["dx"] = dx + a
    if c["branch"]:
        t = unit(h) * w_post if c["post"] else h
        if G is not None:
            t = t * torch.sigmoid(G) * (G if c["gate"] == "silu" else 1.0)
        wanted = {k: v for k, v in (("dh", h), ("ds", sc), ("dG", G), ("dw_post", w_post)) if v is not None}
        out.update(zip(wanted, torch.autograd.grad(s["alpha"] * sc * t, list(wanted.values()), dx)))
    return out


def _exact_adamw(c, s):
    f32 = lambda v: float(torch.tensor(v, dtype=torch.float32))
    b1, b2, lr, wd, eps = (f32(s[k]) for k in ("b1", "b2", "lr", "wd", "eps"))
    g = s["G"].double() * float(s["stats"][1])
    low = c["states"] == "8bit"

    def two_to(n):  # from the bits: pow() need not be exact
        return ((n.long() + 1023) << 52).view(torch.float64)

    def grid(y, bits, low_e):  # the distance of neighbouring codes at y
        e = torch.frexp(y)[1].long() - 1
        return two_to(torch.clamp(e, min=low_e) - bits)

    def decode(q, bits, low_e):
        q = q.double()
        k = torch.clamp(torch.div(q, 2 ** bits, rounding_mode="floor") - 1, min=0)
        return (q - k * 2 ** bits) * two_to(k.long() + low_e - bits)

    def blocks(a, top):  # the smallest power of two that `top` times it holds a block's largest magnitude
        a = a.view(-1, BLOCK).abs().amax(1).float().double()
        f, k = torch.frexp(a)
        k = k.long() - 1 + (2.0 * f > top).long()
        return torch.clamp(torch.where(a > 0, k, torch.full_like(k, -103)), min=-103)

    def coded(a, k, bits, low_e, top_e, noise):
        y = a.view(-1, BLOCK).abs() * two_to(top_e - k)[:, None]
        u = grid(y, bits, low_e)
        w = torch.floor(y / u + noise.double() / 65536.0) * u
        return w * two_to(k - top_e)[:, None]

    if low:
        e = s["e"].long().view(-1, 2) - 127
        q = s["qm"].long()
        m = decode(q % 128, 3, -6) * (1.0 - 2.0 * (q >= 128).double())
        m = (m.view(-1, BLOCK) * two_to(e[:, 0] - 8)[:, None]).reshape(-1)
        v = (decode(s["qv"].long(), 4, -14).view(-1, BLOCK) * two_to(e[:, 1])[:, None]).reshape(-1) ** 2
    else:
        m, v = s["m"].double(), s["v"].double()
    if low:  # by definition fp32 numbers, rounded from the exact result of each operation
        f = lambda x: x.to(torch.float32).double()
        g = f(g)
        m = f(m + f(f(g - m) * f32(1.0 - b1)))
        v = f(f(v) + f(f(f(g * g) - f(v)) * f32(1.0 - b2)))
        root = f(v.sqrt())
    else:
        m = b1 * m + (1.0 - b1) * g
        v = b2 * v + (1.0 - b2) * g * g
        root = v.sqrt()
    up = lr * (m / (1.0 - b1 ** c["t"])) / (root / math.sqrt(1.0 - b2 ** c["t"]) + eps)
    P = s["P"].double()
    decay = torch.zeros_like(P)
    decay[:s["end"]] = lr * wd
    P = P - decay * P - up
    del up, decay, g
    def hashed(x):  # 32 bits as they are defined, by quotients and remainders
        for shift, factor in ((16, 2654435769), (15, 1779033703)):
            x = torch.bitwise_xor(x, torch.div(x, 2 ** shift, rounding_mode="floor"))
            x = (x % 65536 * factor + torch.div(x, 65536, rounding_mode="floor") * (factor % 65536) * 65536) % 2 ** 32
        return torch.bitwise_xor(x, torch.div(x, 65536, rounding_mode="floor"))

    if low:
        place = torch.arange(len(P), device=DEV)
        start = torch.tensor(_places(c)[0], device=DEV)
        which = torch.searchsorted(start, place, right=True) - 1
        key = hashed((hashed(torch.full_like(which[:1], s["seed"])) + c["t"]) % 2 ** 32)
        r = hashed((hashed(torch.bitwise_xor(key, which)) + place - start[which]) % 2 ** 32).view(-1, BLOCK)
        del place, which
        km, ks = blocks(m, 1.75), blocks(root, 1.9375)
        mq = coded(m, km, 3, -6, 8, r % 65536)
        sq = coded(root, ks, 4, -14, 0, torch.div(r, 65536, rounding_mode="floor"))
        sq = torch.where((root > 0).view(-1, BLOCK), torch.maximum(sq, two_to(ks - 18)[:, None]), sq)
        m, v = (torch.sign(m).view(-1, BLOCK) * mq).reshape(-1), (sq * sq).reshape(-1)
    return {"P": P, "P16": P, "m": m, "v": v}


def exact(case, seed):
    c, s = case, prepare(case, seed)
    if c["op"] == "norm":
        return _exact_norm(c, s)
    if c["op"] == "norm_bwd":
        return _exact_norm_bwd(c, s)
    if c["op"] == "adamw":
        return _exact_adamw(c, s)
    norm = math.sqrt(sum(float(g.double().pow(2).sum()) for g in _cut(s["G"], c)))
    return torch.tensor([norm, min(1.0, c["clip"] / norm)], dtype=torch.float64, device=DEV)
