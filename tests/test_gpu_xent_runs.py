"""Cross entropy's gradient at vocabularies on both sides of where dH's sum over
runs of the vocabulary begins to pay."""
import pytest
import torch

import _train_helpers as th
from paper_2606_05484_amd import mapl

pytestmark = pytest.mark.gpu
bf = torch.bfloat16


@pytest.mark.parametrize("T,d,V", [(500, 64, 513), (500, 64, 1000), (300, 256, 1000), (600, 1024, 1000), (2049, 192, 1000), (2049, 192, 1537),
                                   (2049, 192, 5000), (1, 64, 513)])
def test_both_sides(T, d, V):
    print("xent runs", T, d, V, flush=True)
    g = torch.Generator(device="cuda").manual_seed(T + V)
    W = (torch.randn(V, d, generator=g, device="cuda") / d ** 0.5).to(bf)
    H = torch.randn(T, d, generator=g, device="cuda").to(bf)
    y = torch.randint(V, (T,), generator=g, device="cuda", dtype=torch.int32)
    y[1::7] = -1
    H[1::7] = float("nan")  # what a masked token's row holds has no part in anything
    weight = torch.rand(T, generator=g, device="cuda") - 0.25
    scale = 1.0 / T
    r = th.xent(torch.where(y[:, None] < 0, torch.zeros_like(H), H), W, y, weight, scale)
    D = mapl.xent_desc(T, d, V)
    ws = torch.full((mapl.xent_workspace_bytes(D, mapl.XENT_BWD),), 255, dtype=torch.uint8, device="cuda")
    dH, dW = torch.full_like(H, float("nan")), torch.full((V, d), float("nan"), device="cuda")
    mapl.xent_bwd(D, H, W, y, r["lse"].float(), weight, scale, dH, dW, 0, ws)
    eH, eW = th.grad_errors(torch.where(y[:, None] < 0, torch.zeros_like(H), H), W, r, scale, True, False)
    assert ((dH.double() - r["dH"]).abs() <= eH).all() and not dH[y < 0].any()
    assert ((dW.double() - r["dW"]).abs() <= eW).all()
