"""The loss's gradient on more values of H than a launch has threads for."""
import pytest
import torch

import _train_helpers as th
from paper_2606_05484_amd import mapl

pytestmark = pytest.mark.gpu


def test_more_than_2_to_34_values():
    T, d, V = (1 << 20) + 40, 16384, 200
    assert T * d > 1 << 34
    if torch.cuda.get_device_properties(0).total_memory < 150 << 30:
        pytest.skip("needs about 105 GB")
    print("xent wide", T, d, V, flush=True)
    g = torch.Generator(device="cuda").manual_seed(1)
    H = torch.empty(T, d, dtype=torch.bfloat16, device="cuda")
    H.zero_()
    H[-100:] = torch.randn(100, d, generator=g, device="cuda").to(torch.bfloat16)
    W = (torch.randn(V, d, generator=g, device="cuda") / 128).to(torch.bfloat16)
    y = torch.randint(V, (T,), generator=g, device="cuda", dtype=torch.int32)
    y[:-100] = -1
    y[-50] = -1
    r = th.xent(H[-100:], W, y[-100:], None, 0.5)
    lse = torch.zeros(T, device="cuda")
    lse[-100:] = r["lse"].float()
    D = mapl.xent_desc(T, d, V)
    ws = mapl.workspace(mapl.xent_workspace_bytes(D, mapl.XENT_BWD))
    dH, dW = torch.empty_like(H), torch.empty(V, d, device="cuda")
    mapl.xent_bwd(D, H, W, y, lse, None, 0.5, dH, dW, 0, ws)
    eH, eW = th.grad_errors(H[-100:], W, r, 0.5, True, False)
    assert ((dH[-100:].double() - r["dH"]).abs() <= eH).all() and not dH[-50].any() and not dH[:1000].any()
    assert ((dW.double() - r["dW"]).abs() <= eW).all()
    del H, dH, ws
    torch.cuda.empty_cache()
