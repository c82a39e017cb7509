"""The plain 64-bit forms that the checkpoint and cross-entropy kernels are
tested against, tied to something other than themselves: hand values,
differences of the loss, torch's own cross entropy."""
import math

import pytest
import torch

import _train_helpers as th


def test_checkpoint_hand_values():
    X = torch.zeros(33, 64, dtype=torch.float64)
    X[0, 0], X[1, 0], X[2, 0] = 1.0, -0.5, 0.0234375  # a = 1: unit 2^-6; 0.0234375 = 1.5 units, ties to 2
    X[3, 1], X[4, 1] = 1.9999, 0.9  # 1.9999 * 64 = 127.99 rounds to 128, held at 127
    X[5, 2] = 2.0 ** -140            # under the smallest scale: nothing is left
    X[6, 3] = float("inf")
    X[32, 4] = -3.0
    q, e = th.ckpt(X)
    assert q.shape == (2, 64, 32) and e.shape == (2, 64)
    assert q[0, 0, :3].tolist() == [64, -32, 2] and e[0, 0] == 127
    assert q[0, 1, 3] == 127 and q[0, 1, 4] == 58 and e[0, 1] == 127
    assert q[0, 2].abs().sum() == 0 and e[0, 2] == 7
    assert e[0, 3] == 255
    assert q[1, 4, 0] == -96 and e[1, 4] == 128 and q[1, :, 1:].abs().sum() == 0
    v = th.ckpt_values(q, e, 33)
    assert v[2, 0] == 2.0 / 64 and v[32, 4] == -3.0 and torch.isnan(v[:32, 3]).all() and v[32, 3] == 0


def test_checkpoint_error_and_idempotence():
    g = torch.Generator().manual_seed(1)
    X = (torch.randn(100, 64, generator=g, dtype=torch.float64) * torch.logspace(-6, 6, 64, dtype=torch.float64)).float()
    q, e = th.ckpt(X)
    v = th.ckpt_values(q, e, 100)
    unit = th.two_to(e - 133).repeat_interleave(32, 0)[:100]
    err = (v - X.double()).abs()
    top = q.abs().transpose(1, 2).reshape(-1, 64)[:100] == 127
    assert (err <= torch.where(top, unit, unit / 2)).all()
    q2, e2 = th.ckpt(v)
    assert torch.equal(th.ckpt_values(q2, e2, 100), v)
    assert torch.equal(v.float().to(torch.bfloat16).double(), v)  # exact in bf16


def test_cross_entropy_matches_torch():
    g = torch.Generator().manual_seed(2)
    H, W = torch.randn(9, 64, generator=g, dtype=torch.float64), 0.3 * torch.randn(17, 64, generator=g, dtype=torch.float64)
    y = torch.tensor([0, 16, -1, 3, 3, 5, -1, 9, 1])
    w = torch.rand(9, generator=g, dtype=torch.float64)
    Hg, Wg = H.clone().requires_grad_(), W.clone().requires_grad_()
    loss = torch.nn.functional.cross_entropy(Hg @ Wg.t(), y, ignore_index=-1, reduction="none")
    (0.25 * (w * loss).sum()).backward()
    r = th.xent(H, W, y, w, 0.25)
    for got, ref in ((r["loss"], loss.detach()), (r["dH"], Hg.grad), (r["dW"], Wg.grad)):
        assert torch.allclose(got, ref, rtol=1e-12, atol=1e-14)


def test_cross_entropy_gradient_by_differences():
    g = torch.Generator().manual_seed(3)
    H, W = torch.randn(5, 64, generator=g, dtype=torch.float64), 0.3 * torch.randn(11, 64, generator=g, dtype=torch.float64)
    y, w = torch.tensor([1, -1, 10, 0, 4]), torch.tensor([1.0, 1.0, 0.5, 2.0, 0.0], dtype=torch.float64)
    r = th.xent(H, W, y, w, 0.5)
    total = lambda a, b: 0.5 * (w * th.xent(a, b, y)["loss"]).sum().item()
    for k in range(4):
        dh, dw = torch.randn(5, 64, generator=g, dtype=torch.float64), torch.randn(11, 64, generator=g, dtype=torch.float64)
        h = 1e-5
        num = (total(H + h * dh, W + h * dw) - total(H - h * dh, W - h * dw)) / (2 * h)
        ana = ((r["dH"] * dh).sum() + (r["dW"] * dw).sum()).item()
        assert math.isclose(num, ana, rel_tol=1e-7, abs_tol=1e-8)


@pytest.mark.parametrize("bf16", [False, True])
def test_error_bounds_hold_for_an_emulation(bf16):
    """The bounds, against the same formulas carried out with fp32 products (and
    dl rounded to bf16): wide enough for that, and not vacuous."""
    g = torch.Generator().manual_seed(4)
    H, W = torch.randn(40, 128, generator=g), 0.1 * torch.randn(300, 128, generator=g)
    if bf16:
        H, W = H.bfloat16(), W.bfloat16()
    y = torch.randint(-1, 300, (40,), generator=g)
    r = th.xent(H, W, y, None, 0.1)
    l = H.float() @ W.float().t()
    lse = torch.logsumexp(l, 1)
    assert ((lse.double() - r["lse"]).abs() <= th.lse_error(H, W, r)).all()
    assert th.lse_error(H, W, r).max() < 1e-3
    dl = torch.exp(l - lse[:, None])
    dl[torch.arange(40), y.clamp(min=0)] -= 1.0
    dl[y < 0] = 0
    if bf16:
        dl = dl.bfloat16().float()
    dH, dW = 0.1 * (dl @ W.float()), 0.1 * (dl.t() @ H.float())
    if bf16:
        dH, dW = dH.bfloat16(), dW.bfloat16()
    eH, eW = th.grad_errors(H, W, r, 0.1, bf16, bf16)
    assert ((dH.double() - r["dH"]).abs() <= eH).all() and ((dW.double() - r["dW"]).abs() <= eW).all()
    assert eH.norm() < (2e-2 if bf16 else 1e-3) * r["dH"].norm() and eW.norm() < (2e-2 if bf16 else 1e-3) * r["dW"].norm()
