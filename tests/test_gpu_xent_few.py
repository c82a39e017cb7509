"""Cross entropy of few tokens: every number of 16-token groups, chunks of d
fewer than those in flight, vocabularies that end inside a wave's rows."""
import pytest
import torch

import _train_helpers as th
from paper_2606_05484_amd import mapl

pytestmark = pytest.mark.gpu
bf = torch.bfloat16


@pytest.mark.parametrize("d", [64, 320, 1088])
@pytest.mark.parametrize("T,V", [(1, 1), (15, 31), (16, 33), (17, 128), (31, 129), (32, 1000), (33, 95), (48, 257), (49, 4099),
                                 (63, 161), (64, 2048), (65, 300)])
def test_few_tokens(T, V, d):
    print("xent few", T, V, d, flush=True)
    g = torch.Generator(device="cuda").manual_seed(T * d + V)
    H = torch.randn(T, d, generator=g, device="cuda").to(bf)
    W = (2.0 * torch.randn(V, d, generator=g, device="cuda") / d ** 0.5).to(bf)
    y = torch.randint(V, (T,), generator=g, device="cuda", dtype=torch.int32)
    y[T // 2], y[T // 3] = V - 1, -1
    r = th.xent(H, W, y)
    D = mapl.xent_desc(T, d, V)
    ws = torch.full((mapl.xent_workspace_bytes(D, mapl.XENT_FWD),), 255, dtype=torch.uint8, device="cuda")
    loss, lse = (torch.full((T,), float("nan"), device="cuda") for _ in range(2))
    mapl.xent_fwd(D, H, W, y, loss, lse, ws)
    e = th.lse_error(H, W, r)
    assert ((lse.double() - r["lse"]).abs() <= e).all()
    assert ((loss.double() - r["loss"]).abs() <= 2 * e).all() and (loss[y < 0] == 0).all()


def test_a_nan_stays_in_its_token():
    T, d, V = 20, 128, 400
    g = torch.Generator(device="cuda").manual_seed(2)
    H, W = torch.randn(T, d, generator=g, device="cuda").to(bf), torch.randn(V, d, generator=g, device="cuda").to(bf)
    y = torch.arange(T, dtype=torch.int32, device="cuda")
    D = mapl.xent_desc(T, d, V)
    ws = mapl.workspace(mapl.xent_workspace_bytes(D, mapl.XENT_FWD))
    loss, lse, bad = (torch.empty(T, device="cuda") for _ in range(3))
    mapl.xent_fwd(D, H, W, y, loss, lse, ws)
    H[7, 3] = float("nan")
    mapl.xent_fwd(D, H, W, y, bad, lse, ws)
    other = y != 7
    assert torch.isnan(bad[7]) and torch.equal(bad[other], loss[other])
