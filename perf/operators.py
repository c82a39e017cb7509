"""The operators of a training micro-batch around a boundary, as measurable cases.

A case is a dict of plain values; "op" names what one pass does:

  ckpt        an activation kept in 8 bits between forward and backward: packed as the
              forward leaves it, unpacked as the backward wants it
  ckpt_bwd    the sender's backward (dX and dU of Eq. 1) from the 8-bit checkpoint of X
  xent        the last stage's loss: softmax cross entropy of H W^T over the vocabulary,
              loss and log-sum-exp of every token, the logits never kept
  xent_bwd    its gradient with respect to H and W, from the log-sum-exp

Activations have a decaying spectrum with outlier channels and a few all-zero tokens
(padding); hidden states lean towards their target's row of the head by a random amount,
so that some tokens are predicted well and others not; token ids are Zipf, and some
targets are masked (-1).
"""
import math

import torch

own = False
DEV = "cuda"
BLOCK = 32  # tokens of one channel that share a scale


def _ckpt(T, d, dtype="bf16", name=None):
    c = dict(op="ckpt", T=T, d=d, dtype=dtype)
    return dict(c, name=name) if name else c


def _ckpt_bwd(T, d, r, k=0, V=32000, dtype="bf16", space="ambient", name=None):
    c = dict(op="ckpt_bwd", T=T, d=d, r=r, k=k, V=V, dtype=dtype, space=space)
    return dict(c, name=name) if name else c


def _xent(op, T, d, V, dtype="bf16", masked=0.02, weight=False, name=None):
    c = dict(op=op, T=T, d=d, V=V, dtype=dtype, masked=masked)
    if op == "xent_bwd":
        c["weight"] = weight
    return dict(c, name=name) if name else c


def listed():
    return [
        # the smallest configuration's activations, fp32: two launches of a few workgroups
        _ckpt(512, 256, dtype="f32", name="ckpt_f32_small"),
        # 1B model, micro-batch 16 x 2048: a whole boundary stored and restored
        _ckpt(32768, 2048, name="ckpt_1b"),
        # a short, odd micro-batch (a sequence's tail) of a 150M model at 16x compression
        _ckpt_bwd(1021, 1024, 64, k=64, name="ckpt_bwd_tail_r64"),
        # 150M model, micro-batch 4 x 2048, rank 256
        _ckpt_bwd(8192, 1024, 256, k=64, name="ckpt_bwd_150m"),
        # 1B model, micro-batch 16 x 2048, rank 256
        _ckpt_bwd(32768, 2048, 256, k=128, name="ckpt_bwd_1b"),
        # a few tokens scored (the end of an evaluation document): the head is read once
        _xent("xent", 37, 2048, 32000, masked=0.0, name="xent_37_tokens"),
        # 150M model, micro-batch 4 x 2048
        _xent("xent", 8192, 1024, 32000, name="xent_150m"),
        # 1B model, micro-batch 16 x 2048, a vocabulary that no tile divides
        _xent("xent", 32768, 2048, 32003, name="xent_1b_odd_vocabulary"),
        # the smallest configuration, fp32 throughout
        _xent("xent_bwd", 512, 256, 1000, dtype="f32", name="xent_bwd_f32_small"),
        # a short, odd micro-batch with half of its tokens masked (prompts) and weights by token
        _xent("xent_bwd", 1021, 1024, 32000, masked=0.5, weight=True, name="xent_bwd_tail"),
        # 150M model, micro-batch 4 x 2048
        _xent("xent_bwd", 8192, 1024, 32000, name="xent_bwd_150m"),
        # 1B model, micro-batch 16 x 2048
        _xent("xent_bwd", 32768, 2048, 32000, name="xent_bwd_1b"),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["ckpt", "ckpt_bwd", "ckpt_bwd", "xent", "xent", "xent_bwd", "xent_bwd"])
    f32 = rng.random() < 0.2
    dtype = "f32" if f32 else "bf16"
    d = 64 * rng.randint(1, 16 if f32 else 32)
    if op == "ckpt":
        return _ckpt(_log(rng, 1, 16384 if f32 else 32768), d, dtype)
    if op == "ckpt_bwd":
        T = _log(rng, 1, 4096 if f32 else 32768)
        r = min(d, (32 if f32 else 64) * rng.randint(1, 4))
        return _ckpt_bwd(T, d, r, k=min(d, 16 * rng.randint(0, 8)), V=rng.choice([1000, 32000]), dtype=dtype,
                         space="coord" if rng.random() < 0.2 else "ambient")
    T = _log(rng, 1, 2048 if f32 else 32768)
    V = _log(rng, 2, 8192 if f32 else 65536)
    V = min(V, int(32768 * 32000 * 2048 / (T * d)))
    return _xent(op, T, d, V, dtype, masked=rng.choice([0.0, 0.02, 0.5]), weight=rng.random() < 0.3)


# ------------------------------------------------------------------- inputs
def _gen(seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(int(seed))
    return g


def _rn(g, *shape):
    return torch.randn(*shape, generator=g, device=DEV)


def _dt(c):
    return torch.bfloat16 if c["dtype"] == "bf16" else torch.float32


def _ids(g, T, V):
    p = torch.arange(1, V + 1, device=DEV, dtype=torch.float64) ** -1.1
    cdf = torch.cumsum(p, 0) / p.sum()
    u = torch.rand(T, generator=g, device=DEV, dtype=torch.float64)
    return torch.searchsorted(cdf, u).clamp_(max=V - 1).to(torch.int32)


def _activations(g, T, d, dt):
    x = _rn(g, T, d) * torch.arange(1, d + 1, device=DEV, dtype=torch.float32) ** -0.7
    for v in _rn(g, 2, d):  # the spectrum's axes are no channels: two reflections
        v = v / v.norm()
        x -= 2.0 * (x @ v)[:, None] * v
    x += 0.1 * _rn(g, T, d)
    x[:, torch.randperm(d, generator=g, device=DEV)[:max(1, d // 128)]] *= 20.0
    if T > 1:
        x[torch.rand(T, generator=g, device=DEV) < 0.01] = 0.0
    return x.to(dt)


def _pow2(e):
    """2^e of whole numbers, exact (a library's exp2 may be off in the last place)."""
    return ((e.to(torch.int32) + 127) << 23).view(torch.float32)


def _stored(x):
    """The checkpoint of x [T, d] as tensors: int8 values [T/32, d, 32] and, for each 32 tokens
    of a channel, the exponent of the largest magnitude plus 127 [T/32, d] (T rounded up, zeros)."""
    T, d = x.shape
    nb = -(-T // BLOCK)
    p = torch.zeros(nb * BLOCK, d, device=x.device)
    p[:T] = x
    p = p.view(nb, BLOCK, d).transpose(1, 2).contiguous()
    e = (torch.frexp(p.abs().amax(2))[1] - 1).clamp(-120, 127)
    e = torch.where(p.abs().amax(2) == 0, torch.full_like(e, -120), e)
    q = torch.round(p * _pow2(6 - e)[:, :, None]).clamp(-127, 127)
    return q.to(torch.int8), (e + 127).to(torch.uint8)


def _restored(q, e, T):
    x = q.float() * _pow2(e.to(torch.int32) - 133)[:, :, None]
    return x.transpose(1, 2).reshape(-1, q.shape[1])[:T]


def _head(g, c):
    T, d, V = c["T"], c["d"], c["V"]
    W = (0.02 * _rn(g, V, d)).to(_dt(c))
    y = _ids(g, T, V)
    wt = W[y.long()].float()
    lean = 12.0 * torch.rand(T, 1, generator=g, device=DEV)  # what the target's logit gains
    H = (_rn(g, T, d) + lean * wt / (wt * wt).sum(1, keepdim=True)).to(_dt(c))
    y[torch.rand(T, generator=g, device=DEV) < c["masked"]] = -1
    return H, W, y


def _lse(H, W):
    rows = max(1, (1 << 28) // W.shape[0])
    return torch.cat([torch.logsumexp(h.float() @ W.float().t(), 1) for h in H.split(rows)])


def prepare(case, seed):
    c, g = case, _gen(seed)
    T, d, dt = c["T"], c["d"], _dt(c)
    s = dict(case=c)
    if c["op"] == "ckpt":
        nb = -(-T // BLOCK)
        s.update(X=_activations(g, T, d, dt), q=torch.empty(nb, d, BLOCK, dtype=torch.int8, device=DEV),
                 e=torch.empty(nb, d, dtype=torch.uint8, device=DEV), Y=torch.empty(T, d, dtype=dt, device=DEV))
    elif c["op"] == "ckpt_bwd":
        r, k, V = c["r"], c["k"], c["V"]
        s["q"], s["e"] = _stored(_activations(g, T, d, dt))
        s["U"] = torch.linalg.qr(_rn(g, d, r).cpu())[0].to(DEV).contiguous()
        s["ids"] = _ids(g, T, V) if k else None
        s["A"] = (0.02 * _rn(g, V, k)).to(dt) if k else None
        s["B"] = (0.02 * _rn(g, k, d if c["space"] == "ambient" else r)).to(dt) if k else None
        s["dZ"] = (1e-2 * _rn(g, T, r)).to(dt)
        s["dX"], s["dU"] = torch.empty(T, d, dtype=dt, device=DEV), torch.empty(d, r, device=DEV)
    else:
        s["H"], s["W"], s["y"] = _head(g, c)
        if c["op"] == "xent":
            s["loss"], s["lse"] = torch.empty(T, device=DEV), torch.empty(T, device=DEV)
        else:
            s["lse"] = _lse(s["H"], s["W"])
            s["weight"] = 0.5 + torch.rand(T, generator=g, device=DEV) if c["weight"] else None
            s["scale"] = 1.0 / max(1, T)
            s["dH"], s["dW"] = torch.empty_like(s["H"]), torch.empty_like(s["W"])
    return s


# ---------------------------------------------------------------------- run
def _plain(s):
    c, dt = s["case"], _dt(s["case"])
    if c["op"] == "ckpt":
        return _restored(*_stored(s["X"]), c["T"]).to(dt)
    if c["op"] == "ckpt_bwd":
        dZ, x = s["dZ"].float(), _restored(s["q"], s["e"], c["T"])
        if c["k"] and c["space"] == "ambient":
            x = x - s["A"][s["ids"].long()].float() @ s["B"].float()
        return {"dX": (dZ @ s["U"].t()).to(dt), "dU": x.t() @ dZ}
    y, H, W = s["y"].long(), s["H"].float(), s["W"].float()
    at, live = y.clamp(min=0)[:, None], y >= 0
    logits = H @ W.t()
    if c["op"] == "xent":
        m = logits.amax(1, keepdim=True)
        lse = (m + torch.log(torch.exp(logits - m).sum(1, keepdim=True)))[:, 0]
        return {"loss": torch.where(live, lse - logits.gather(1, at)[:, 0], torch.zeros_like(lse)), "lse": lse}
    p = torch.exp(logits - s["lse"][:, None])
    p.scatter_add_(1, at, torch.full_like(p[:, :1], -1.0))
    w = live.float() if s["weight"] is None else torch.where(live, s["weight"], torch.zeros_like(s["weight"]))
    p *= (s["scale"] * w)[:, None]
    return {"dH": (p @ W).to(dt), "dW": (p.t() @ H).to(dt)}


def run(s):
    if not own:
        return _plain(s)
    from paper_2606_05484_amd import mapl
    c = s["case"]
    T, d = c["T"], c["d"]
    if c["op"] == "ckpt":
        mapl.ckpt_pack(T, d, s["X"], s["q"], s["e"], c["dtype"])
        mapl.ckpt_unpack(T, d, s["q"], s["e"], s["Y"], c["dtype"])
        return s["Y"]
    if c["op"] == "ckpt_bwd":
        D = mapl.desc(T=T, d=d, r=c["r"], V=c["V"], k=c["k"], x_dtype=c["dtype"], anchor_space=c["space"])
        if "ws" not in s:
            s["ws"] = mapl.workspace(mapl.ckpt_encode_bwd_workspace_bytes(D))
        mapl.ckpt_encode_bwd(D, s["dZ"], s["q"], s["e"], s["ids"], s["U"], s["A"], s["B"], s["dX"], s["dU"], 0,
                             s["ws"])
        return {"dX": s["dX"], "dU": s["dU"]}
    D = mapl.xent_desc(T=T, d=d, V=c["V"], x_dtype=c["dtype"], dw_dtype=c["dtype"])
    call = mapl.XENT_FWD if c["op"] == "xent" else mapl.XENT_BWD
    if "ws" not in s:
        s["ws"] = mapl.workspace(mapl.xent_workspace_bytes(D, call))
    if c["op"] == "xent":
        mapl.xent_fwd(D, s["H"], s["W"], s["y"], s["loss"], s["lse"], s["ws"])
        return {"loss": s["loss"], "lse": s["lse"]}
    mapl.xent_bwd(D, s["H"], s["W"], s["y"], s["lse"], s["weight"], s["scale"], s["dH"], s["dW"], 0, s["ws"])
    return {"dH": s["dH"], "dW": s["dW"]}


# --------------------------------------------------------------------- work
def work(case):
    c = case
    T, d, xe = c["T"], c["d"], 2.0 if c["dtype"] == "bf16" else 4.0
    q = -(-T // BLOCK) * d * (BLOCK + 1.0)  # the checkpoint
    if c["op"] == "ckpt":
        return {"bytes": 2.0 * T * d * xe + 2.0 * q, "flops": 4.0 * T * d}
    if c["op"] == "ckpt_bwd":
        r, k = c["r"], c["k"] if c["space"] == "ambient" else 0
        rows = min(T, c["V"]) * k * xe + T * 4.0 * (k > 0) + k * d * xe  # anchor rows, ids, B
        return {"bytes": q + T * r * xe + d * r * 4.0 + rows + T * d * xe + d * r * 4.0,
                "flops": 4.0 * T * d * r + 2.0 * T * k * r + 2.0 * k * d * r}
    V = c["V"]
    read, product = (T + V) * d * xe + 4.0 * T, 2.0 * T * V * d
    if c["op"] == "xent":
        return {"bytes": read + 8.0 * T, "flops": product}
    return {"bytes": read + 4.0 * T * (2 if c["weight"] else 1) + (T + V) * d * xe, "flops": 3 * product}


# -------------------------------------------------------------------- exact
def exact(case, seed):
    c, s = case, prepare(case, seed)
    T, d = c["T"], c["d"]

    def two_to(n):  # from the bits: pow() need not be exact
        return ((n.long() + 1023) << 52).view(torch.float64)

    def values(q, e):  # [T, d]: int8 times a power of two, the 64th part of what the exponent says
        return (q.double() * two_to(e.long() - 127 - 6).unsqueeze(-1)).permute(0, 2, 1).reshape(-1, d)[:T]

    if c["op"] == "ckpt":
        out = torch.empty(T, d, dtype=torch.float64, device=DEV)
        for t in range(0, T, BLOCK):
            x = s["X"][t:t + BLOCK].double()
            e = (x.abs().amax(0).view(torch.int64) >> 52) - 1023  # zero: far below -120
            unit = two_to(e.clamp(-120, 127) - 6)
            out[t:t + BLOCK] = (x / unit).round().clamp(-127, 127) * unit
        return out
    if c["op"] == "ckpt_bwd":
        dZ = s["dZ"].double()
        dU = values(s["q"], s["e"]).t() @ dZ
        if c["k"] and c["space"] == "ambient":
            dU -= s["B"].double().t() @ (s["A"].double()[s["ids"].long()].t() @ dZ)
        return {"dX": dZ @ s["U"].double().t(), "dU": dU}
    H, W, y = s["H"].double(), s["W"].double(), s["y"].long()
    some = torch.nonzero(y >= 0)[:, 0]
    if c["op"] == "xent":
        loss, lse = torch.zeros(T, dtype=torch.float64, device=DEV), []
        for h in H.split(max(1, (1 << 28) // c["V"])):
            lse.append(torch.logsumexp(h @ W.t(), 1))
        lse = torch.cat(lse)
        loss[some] = lse[some] - (H[some] * W[y[some]]).sum(1)
        return {"loss": loss, "lse": lse}
    dH, dW = torch.zeros_like(H), torch.zeros_like(W)
    for i in some.split(max(1, (1 << 28) // c["V"])):
        g = torch.softmax(H[i] @ W.t(), 1)
        g[torch.arange(len(i), device=DEV), y[i]] -= 1.0
        g *= s["scale"] * (s["weight"][i].double() if c["weight"] else torch.ones(len(i), device=DEV))[:, None]
        dH[i] = g @ W
        dW += g.t() @ H[i]
    return {"dH": dH, "dW": dW}
