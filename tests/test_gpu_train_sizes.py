"""The training step's operators where offsets pass 32 bits, and token weights
of both signs."""
import pytest
import torch

import _train_helpers as th
from paper_2606_05484_amd import mapl

pytestmark = pytest.mark.gpu
bf = torch.bfloat16


def test_checkpoint_past_32_bits():
    """More than 2^31 values: the last blocks as on their own, and the backward's last rows."""
    T, d, r = (1 << 20) + 33, 2112, 64
    assert T * d > 1 << 31
    print("ckpt", T, d, flush=True)
    g = torch.Generator(device="cuda").manual_seed(1)
    X = torch.empty(T, d, dtype=bf, device="cuda")
    X.normal_(generator=g)
    sq, se = mapl.ckpt_shapes(T, d)
    q, e = torch.empty(sq, dtype=torch.int8, device="cuda"), torch.empty(se, dtype=torch.uint8, device="cuda")
    mapl.ckpt_pack(T, d, X, q, e)
    Y = torch.zeros_like(X)
    mapl.ckpt_unpack(T, d, q, e, Y)
    for t in (0, 1 << 19, (1 << 20) - 64, 1 << 20):
        n = min(64, T - t)
        rq, re = th.ckpt(X[t:t + n])
        b = t // 32
        assert torch.equal(q[b:b + len(rq)].long(), rq) and torch.equal(e[b:b + len(re)].long(), re)
        assert torch.equal(Y[t:t + n].double(), th.ckpt_values(rq, re, n))
    del X
    # gradients that only the last 40 tokens have
    D = mapl.desc(T, d, r)
    U = torch.linalg.qr(torch.randn(d, r, generator=g, device="cuda"))[0].contiguous()
    dZ = torch.zeros(T, r, dtype=bf, device="cuda")
    dZ[-40:] = torch.randn(40, r, generator=g, device="cuda").to(bf)
    dX, dU = torch.empty_like(Y), torch.empty(d, r, device="cuda")
    mapl.ckpt_encode_bwd(D, dZ, q, e, None, U, None, None, dX, dU, 0,
                         mapl.workspace(mapl.ckpt_encode_bwd_workspace_bytes(D)))
    z, y = dZ[-40:].double(), Y[-40:].double()
    # at most 40 products of bf16 values in fp32, in any order, sums doubled exactly; zeros add nothing
    assert ((dU.double() - y.t() @ z).abs() <= 2 * 40 * th.U24 * (y.abs().t() @ z.abs())).all()
    want, mag = z @ U.to(bf).double().t(), z.abs() @ U.to(bf).double().abs().t()
    assert ((dX[-40:].double() - want).abs() <= 2 * r * th.U24 * mag + 1.01 * th.UB * want.abs()).all()
    assert not dX[:-40].any()


@pytest.mark.parametrize("T", [3, 130])
def test_vocabulary_past_32_bits(T):
    """More than 2^31 weights, and dW's bytes past 2^33."""
    d, V = 2112, 1020007
    assert V * d > 1 << 31
    print("xent", T, d, V, flush=True)
    g = torch.Generator(device="cuda").manual_seed(T)
    W = torch.empty(V, d, dtype=bf, device="cuda")
    W.normal_(std=0.02, generator=g)
    H = torch.randn(T, d, generator=g, device="cuda").to(bf)
    y = torch.randint(V, (T,), generator=g, device="cuda", dtype=torch.int32)
    y[0], y[1], y[2] = V - 1, 0, -1
    D = mapl.xent_desc(T, d, V)
    ws = mapl.workspace(max(mapl.xent_workspace_bytes(D, c) for c in (0, 1)))
    loss, lse = torch.empty(T, device="cuda"), torch.empty(T, device="cuda")
    mapl.xent_fwd(D, H, W, y, loss, lse, ws)
    l = torch.cat([H.double() @ w.double().t() for w in W.split(1 << 16)], 1)
    ref = dict(l=l, lse=torch.logsumexp(l, 1))
    top = torch.cat([th.logit_error(H, w)[None] for w in W.split(1 << 16)]).amax(0)
    err = top + th.U24 * (4 * l.abs().amax(1) + 2 * ref["lse"].abs() + 200.0)
    live = y >= 0
    at = l.gather(1, y.clamp(min=0).long()[:, None])[:, 0]
    assert ((lse.double() - ref["lse"]).abs() <= err).all()
    assert ((loss.double() - (ref["lse"] - at))[live].abs() <= 2 * err[live]).all() and (loss[~live] == 0).all()
    dH, dW = torch.empty_like(H), torch.empty(V, d, device="cuda")
    mapl.xent_bwd(D, H, W, y, lse, None, 0.5, dH, dW, 0, ws)
    p = torch.exp(l - lse.double()[:, None])
    dl = p.clone()
    dl[torch.arange(T, device="cuda"), y.clamp(min=0).long()] -= 1.0
    dl[~live], p[~live] = 0.0, 0.0
    rel = top + th.U24 * (4 * l.abs().amax(1) + 2 * lse.double().abs() + 16.0)
    ddl = p * rel[:, None] + 1.01 * th.UB * dl.abs() + 2.0 ** -133
    for v in (0, 500001, V - 300):  # dW's first, middle and last rows
        s = slice(v, v + 300)
        want = 0.5 * (dl[:, s].t() @ H.double())
        eW = 0.5 * ((ddl + 2 * T * th.U24 * dl.abs())[:, s].t() @ H.double().abs()) + 4 * th.U24 * want.abs()
        assert ((dW[s].double() - want).abs() <= eW).all()
    want = sum(0.5 * (a @ w.double()) for a, w in zip(dl.split(1 << 16, 1), W.split(1 << 16)))
    eH = sum(0.5 * (a @ w.double().abs()) for a, w in zip((ddl + 2 * V * th.U24 * dl.abs()).split(1 << 16, 1), W.split(1 << 16)))
    assert ((dH.double() - want).abs() <= eH + 1.01 * th.UB * want.abs()).all() and not dH[2].any()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_weights_of_both_signs(dtype):
    """A negative weight (a token to be made less likely) is a weight like any other."""
    T, d, V = 200, 128, 700
    dt = {"bf16": bf, "f32": torch.float32}[dtype]
    g = torch.Generator(device="cuda").manual_seed(9)
    H = torch.randn(T, d, generator=g, device="cuda").to(dt)
    W = (torch.randn(V, d, generator=g, device="cuda") / d ** 0.5).to(dt)
    y = torch.randint(V, (T,), generator=g, device="cuda", dtype=torch.int32)
    y[::7] = -3
    weight = torch.randn(T, generator=g, device="cuda")
    weight[3], weight[4], weight[5] = 0.0, -1e-30, 1e30
    r = th.xent(H, W, y, weight, 1.0)
    D = mapl.xent_desc(T, d, V, dtype, "f32")
    dH, dW = torch.empty_like(H), torch.empty(V, d, device="cuda")
    ws = mapl.workspace(mapl.xent_workspace_bytes(D, mapl.XENT_BWD))
    mapl.xent_bwd(D, H, W, y, r["lse"].float(), weight, 1.0, dH, dW, 0, ws)
    eH, _ = th.grad_errors(H, W, r, 1.0, dtype == "bf16", False)
    assert ((dH.double() - r["dH"]).abs() <= eH).all()
    weight[5] = 2.0  # (1e30 hides the rest of dW)
    r = th.xent(H, W, y, weight, 1.0)
    mapl.xent_bwd(D, H, W, y, r["lse"].float(), weight, 1.0, dH, dW, 0, ws)
    _, eW = th.grad_errors(H, W, r, 1.0, dtype == "bf16", False)
    assert ((dW.double() - r["dW"]).abs() <= eW).all()
