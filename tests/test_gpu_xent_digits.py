"""The fp32 gradient of tokens whose target has nearly all of the probability."""
import pytest
import torch

import _train_helpers as th
from paper_2606_05484_amd import mapl

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("T,d,V", [(1, 64, 1), (40, 64, 2), (100, 128, 37), (300, 256, 1003)])
def test_confident_targets_keep_their_digits(T, d, V):
    """dl's entries are right relative to their own size, the target's too: its
    1 - p is the others' sum, not a difference of numbers near 1."""
    print("xent digits", T, d, V, flush=True)
    g = torch.Generator(device="cuda").manual_seed(V)
    H = torch.randn(T, d, generator=g, device="cuda")
    W = torch.randn(V, d, generator=g, device="cuda") * (10.0 / d ** 0.5)
    y = (H @ W.t()).argmax(1).int()
    r = th.xent(H, W, y, None, 0.5)
    D = mapl.xent_desc(T, d, V, "f32", "f32")
    ws = mapl.workspace(mapl.xent_workspace_bytes(D, mapl.XENT_BWD))
    # a log-sum-exp with another rounding: four units in the last place away
    lse = (r["lse"] * (1 + 8 * th.U24)).float()
    dH, dW = torch.empty_like(H), torch.empty_like(W)
    mapl.xent_bwd(D, H, W, y, lse, None, 0.5, dH, dW, 0, ws)
    # of an entry: its own exponential's error and the normalising sum's, each the logit's, the argument's and its base-2
    # scaling's (4 u max |l| + 8 u |lse|), and the sums, divisions and products; then as every product of the path
    # the oracle's own 1 - p as the others' sum: float64's digits go too where p is 1 - 1e-17
    dl, at = torch.exp(r["l"] - r["lse"][:, None]), (torch.arange(T, device="cuda"), y.long())
    dl[at] = 0.0
    dl[at] = -dl.sum(1)
    r["dl"], r["dH"], r["dW"] = dl, 0.5 * (dl @ W.double()), 0.5 * (dl.t() @ H.double())
    big = r["l"].abs().amax(1) + r["lse"].abs()
    rel = 2 * (th.logit_error(H, W) + th.U24 * (12 * big + 16)) + V * th.U24
    ddl = r["dl"].abs() * rel[:, None] + 2.0 ** -126
    eH = 0.5 * ((ddl + 2 * V * th.U24 * r["dl"].abs()) @ W.double().abs()) + 4 * th.U24 * r["dH"].abs()
    eW = 0.5 * ((ddl + 2 * T * th.U24 * r["dl"].abs()).t() @ H.double().abs()) + 4 * th.U24 * r["dW"].abs()
    assert ((dH.double() - r["dH"]).abs() <= eH).all()
    assert ((dW.double() - r["dW"]).abs() <= eW).all()
