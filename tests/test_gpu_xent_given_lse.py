"""The loss's gradient from a log-sum-exp that is not this vocabulary's own (a
larger vocabulary whose other entries lie elsewhere, a shifted normaliser):
dl = weight (exp(l - lse) - [target]) for every type and number of pieces."""
import pytest
import torch

import _train_helpers as th
from paper_2606_05484_amd import mapl

pytestmark = pytest.mark.gpu
DT = {"bf16": torch.bfloat16, "f32": torch.float32}


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("T,d,V", [(33, 64, 1), (60, 128, 300), (513, 256, 1000), (4100, 64, 33003)])
def test_the_given_normaliser_counts(T, d, V, dtype):
    print("xent given lse", T, d, V, dtype, flush=True)
    g = torch.Generator(device="cuda").manual_seed(T)
    H = torch.randn(T, d, generator=g, device="cuda").to(DT[dtype])
    W = (torch.randn(V, d, generator=g, device="cuda") / d ** 0.5).to(DT[dtype])
    y = torch.randint(V, (T,), generator=g, device="cuda", dtype=torch.int32)
    y[::5] = -1
    weight = torch.rand(T, generator=g, device="cuda") - 0.3
    r = th.xent(H, W, y, weight, 0.5)
    shift = torch.tensor([0.0, 0.7, -0.7, 3.0, 0.01, -0.01], device="cuda", dtype=torch.float64)
    lse = (r["lse"] + shift[torch.arange(T, device="cuda") % 6]).float()
    live, w = r["live"], r["w"]
    dl = torch.exp(r["l"][live] - lse.double()[live, None])
    dl[torch.arange(len(live), device="cuda"), y.long()[live]] -= 1.0
    r["dl"] = w[live, None] * dl
    r["dH"] = torch.zeros_like(r["dH"])
    r["dH"][live] = 0.5 * (r["dl"] @ W.double())
    r["dW"] = 0.5 * (r["dl"].t() @ H.double()[live])
    r["lse"] = lse.double()
    D = mapl.xent_desc(T, d, V, dtype, "f32")
    ws = torch.full((mapl.xent_workspace_bytes(D, mapl.XENT_BWD),), 255, dtype=torch.uint8, device="cuda")
    dH, dW = torch.full_like(H, float("nan")), torch.full((V, d), float("nan"), device="cuda")
    mapl.xent_bwd(D, H, W, y, lse, weight, 0.5, dH, dW, 0, ws)
    eH, eW = th.grad_errors(H, W, r, 0.5, dtype == "bf16", False)
    assert ((dH.double() - r["dH"]).abs() <= eH).all()
    assert ((dW.double() - r["dW"]).abs() <= eW).all()
