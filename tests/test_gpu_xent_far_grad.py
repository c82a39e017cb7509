"""The loss's gradient of tokens whose log-sum-exp lies far from zero, beside
ordinary ones and vocabulary entries masked through a channel."""
import pytest
import torch

import _train_helpers as th
from paper_2606_05484_amd import mapl

pytestmark = pytest.mark.gpu
DT = {"bf16": torch.bfloat16, "f32": torch.float32}
FAR = (3e3, -3e3, 1e6, -1e6, 1e10, -1e10, 1e20, -1e20, 1e30, -1e30, 1.6e38, -1.6e38)


def backward(H, W, y, lse, weight, dtype):
    D = mapl.xent_desc(H.shape[0], H.shape[1], W.shape[0], dtype, "f32")
    ws = torch.full((mapl.xent_workspace_bytes(D, mapl.XENT_BWD),), 255, dtype=torch.uint8, device="cuda")
    dH, dW = torch.full_like(H, float("nan")), torch.full(W.shape, float("nan"), device="cuda")
    mapl.xent_bwd(D, H, W, y, lse, weight, 1.0, dH, dW, 0, ws)
    torch.cuda.synchronize()
    return dH, dW


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("weighted", [False, True])
@pytest.mark.parametrize("T,V", [(24, 3), (70, 500), (1024, 9216)])  # (9216 x 1024: the larger tiles)
def test_dH_of_far_tokens(T, V, weighted, dtype):
    """Tokens whose logits are exact multiples of a large number and whose largest
    logit is one entry's alone: p is 1 there and 0 elsewhere, so that
    dH = weight (W[largest] - W[target])."""
    print("xent far grad", T, V, weighted, dtype, flush=True)
    d, n = 64, len(FAR)
    g = torch.Generator(device="cuda").manual_seed(V)
    W = (torch.randn(V, d, generator=g, device="cuda") / 8).to(DT[dtype])
    W[:, 0] = 1.5
    top, low = V - 1, V // 2  # the largest logit of positive and of negative multiples
    W[top, 0], W[low, 0] = 2.0, 1.0
    H = torch.randn(T, d, generator=g, device="cuda").to(DT[dtype])
    H[:n] = 0
    H[:n, 0] = torch.tensor(FAR, device="cuda").to(DT[dtype])
    y = torch.randint(V, (T,), generator=g, device="cuda", dtype=torch.int32)
    y[0], y[4], y[5] = top, top, low  # (nothing is left of these)
    y[7], y[n + 1] = -1, -1
    weight = None
    if weighted:
        weight = 2.0 ** torch.randint(-3, 1, (T,), generator=g, device="cuda") * torch.where(
            torch.rand(T, generator=g, device="cuda") < 0.5, -1.0, 1.0)
        weight[2] = 0.0
    w = torch.ones(T, dtype=torch.float64, device="cuda") if weight is None else weight.double()
    w = torch.where(y < 0, torch.zeros_like(w), w)
    s = H[:n, 0].double()
    best = torch.where(s > 0, top, low)
    lse = torch.empty(T, device="cuda")
    lse[:n] = (s * W[best, 0].double()).float()
    r = th.xent(H[n:], W, y[n:], None if weight is None else weight[n:], 1.0)
    lse[n:] = r["lse"].float()
    dH, dW = backward(H, W, y, lse, weight, dtype)
    # two exact products' sum in fp32, the result's rounding
    want = w[:n, None] * (W[best].double() - W[y[:n].clamp(min=0).long()].double())
    size = w[:n, None].abs() * (W[best].double().abs() + W[y[:n].clamp(min=0).long()].double().abs())
    tol = 2 * th.U24 * size + want.abs() * (th.UB * 1.01 if dtype == "bf16" else th.U24)
    assert ((dH[:n].double() - want).abs() <= tol).all()
    assert (dH[0] == 0).all() and (dH[4] == 0).all() and (dH[5] == 0).all() and (dH[7] == 0).all()
    eH, _ = th.grad_errors(H[n:], W, r, 1.0, dtype == "bf16", False)
    assert ((dH[n:].double() - r["dH"]).abs() <= eH).all()
    assert torch.isfinite(dW).all()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("far", [3e3, -1e6, 1e10, -1e20, 1e30])
def test_dW_of_far_tokens(far, dtype):
    """dW[largest] gains H, dW[target] loses it."""
    T, d, V = 100, 64, 300
    g = torch.Generator(device="cuda").manual_seed(5)
    W = torch.zeros(V, d, device="cuda")
    W[:, 0] = 1.5
    best = 17
    W[best, 0] = 2.0 if far > 0 else 1.0
    H = torch.zeros(T, d, device="cuda")
    H[:, 0] = far * (1.0 + torch.rand(T, generator=g, device="cuda"))
    H[:, 1:] = torch.randn(T, d - 1, generator=g, device="cuda")  # (no weight there: no part in the logits)
    H, W = H.to(DT[dtype]), W.to(DT[dtype])
    y = torch.randint(V, (T,), generator=g, device="cuda", dtype=torch.int32)
    y[::4] = best
    lse = (H[:, 0].double() * W[best, 0].double()).float()
    _, dW = backward(H, W, y, lse, None, dtype)
    dl = torch.zeros(T, V, dtype=torch.float64, device="cuda")
    dl[:, best] = 1.0
    dl[torch.arange(T, device="cuda"), y.long()] -= 1.0
    want, size = dl.t() @ H.double(), dl.abs().t() @ H.double().abs()
    assert ((dW.double() - want).abs() <= 2 * T * th.U24 * size).all()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_masked_runs_have_no_gradient(dtype):
    """Runs of vocabulary entries at the type's lowest logit, from the forward's
    log-sum-exp: no gradient there, the others' as if they were not there."""
    T, d, V = 200, 64, 1024
    g = torch.Generator(device="cuda").manual_seed(6)
    H = torch.randn(T, d, generator=g, device="cuda").to(DT[dtype])
    W = (torch.randn(V, d, generator=g, device="cuda") / 8).to(DT[dtype])
    H[:, 0], W[:, 0] = 1, 0
    gone = torch.zeros(V, dtype=torch.bool, device="cuda")
    gone[128:256] = gone[640:1024] = True
    W[gone] = 0
    W[gone, 0] = torch.finfo(DT[dtype]).min
    kept = torch.nonzero(~gone)[:, 0]
    at = torch.randint(len(kept), (T,), generator=g, device="cuda")
    r = th.xent(H, W[kept], at)
    dH, dW = backward(H, W, kept[at].int(), r["lse"].float(), None, dtype)
    eH, eW = th.grad_errors(H, W[kept], r, 1.0, dtype == "bf16", False)
    assert ((dH.double() - r["dH"]).abs() <= eH).all()
    assert ((dW[kept].double() - r["dW"]).abs() <= eW).all() and (dW[gone] == 0).all()
