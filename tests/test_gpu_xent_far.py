"""The loss where logits lie far from zero: whole runs of vocabulary entries
masked through a channel, tokens of large logits, a logit near the type's largest."""
import pytest
import torch

import _train_helpers as th
from paper_2606_05484_amd import mapl

pytestmark = pytest.mark.gpu
DT = {"bf16": torch.bfloat16, "f32": torch.float32}


def forward(H, W, y, dtype):
    D = mapl.xent_desc(H.shape[0], H.shape[1], W.shape[0], dtype, "f32")
    ws = torch.full((mapl.xent_workspace_bytes(D, mapl.XENT_FWD),), 255, dtype=torch.uint8, device="cuda")
    loss, lse = (torch.full((D.T,), float("nan"), device="cuda") for _ in range(2))
    mapl.xent_fwd(D, H, W, y, loss, lse, ws)
    torch.cuda.synchronize()
    return loss, lse


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("low", [-2e3, -1e9, -1e10, -1e15, -1e20, -1e30, "lowest"])
@pytest.mark.parametrize("T,V", [(1, 300), (70, 1024), (1024, 9216)])  # (9216 x 1024: the larger tiles)
def test_masked_runs_of_the_vocabulary(T, V, low, dtype):
    """Runs of 64, 128 and 256 entries, and the vocabulary's end, that a constant
    channel takes to a large negative logit: as if they were not there."""
    print("xent far", T, V, low, dtype, flush=True)
    d = 64
    g = torch.Generator(device="cuda").manual_seed(V)
    H = torch.randn(T, d, generator=g, device="cuda").to(DT[dtype])
    W = (torch.randn(V, d, generator=g, device="cuda") / 8).to(DT[dtype])
    H[:, 0], W[:, 0] = 1, 0
    gone = torch.zeros(V, dtype=torch.bool, device="cuda")
    for a, b in ((64, 128), (256, 384), (512, 768), (V - 130, V)):
        gone[a:b] = True
    W[gone] = 0
    W[gone, 0] = torch.finfo(DT[dtype]).min if low == "lowest" else low
    kept = torch.nonzero(~gone)[:, 0]
    at = torch.randint(len(kept), (T,), generator=g, device="cuda")
    y = kept[at].int()
    r = th.xent(H, W[kept], at)
    e = th.lse_error(H, W[kept], r)
    loss, lse = forward(H, W, y, dtype)
    assert ((lse.double() - r["lse"]).abs() <= e).all()
    assert ((loss.double() - r["loss"]).abs() <= 2 * e).all()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("V", [2, 100, 1000])
def test_tokens_far_from_zero(V, dtype):
    """Tokens whose logits are exact multiples of one large number, beside ordinary
    ones: the log-sum-exp is the largest logit, up to its rounding and the
    logarithm of how many entries have it."""
    print("xent far tokens", V, dtype, flush=True)
    T, d = 40, 64
    g = torch.Generator(device="cuda").manual_seed(V)
    W = (torch.randn(V, d, generator=g, device="cuda") / 8).to(DT[dtype])
    W[:, 0] = torch.arange(V, device="cuda") % 2 + 1.0
    H = torch.randn(T, d, generator=g, device="cuda").to(DT[dtype])
    far = torch.tensor([3e3, -3e3, 1e6, -1e6, 1e10, -1e10, 1e20, -1e20, 1e30, -1e30, 1.6e38, -1.6e38], device="cuda")
    n = 12
    H[:n] = 0
    H[:n, 0] = far.to(DT[dtype])
    y = torch.randint(V, (T,), generator=g, device="cuda", dtype=torch.int32)
    loss, lse = forward(H, W, y, dtype)
    s = H[:n, 0].double()
    count = torch.where(s > 0, V // 2, V - V // 2).double()
    big = torch.where(s > 0, 2 * s, s)
    want = big + torch.log(count)
    e = th.U24 * (2 * want.abs() + 200.0)
    assert ((lse[:n].double() - want).abs() <= e).all()
    l = s * W[y[:n].long(), 0].double()
    assert ((loss[:n].double() - (want - l)).abs() <= e + th.U24 * (want - l).abs()).all()
    r = th.xent(H[n:], W, y[n:])
    e = th.lse_error(H[n:], W, r)
    assert ((lse[n:].double() - r["lse"]).abs() <= e).all() and ((loss[n:].double() - r["loss"]).abs() <= 2 * e).all()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("T,V", [(5, 300), (1024, 9216)])
def test_one_logit_near_the_largest(T, V, dtype):
    """One entry at the type's largest value is all of the probability; with
    every entry at its lowest the log-sum-exp is that value."""
    d = 64
    for value in (torch.finfo(DT[dtype]).max, 2.4e38, -2.4e38, torch.finfo(DT[dtype]).min):
        H, W = torch.zeros(T, d, dtype=DT[dtype], device="cuda"), torch.zeros(V, d, dtype=DT[dtype], device="cuda")
        H[:, 0] = 1
        if value > 0:
            W[V // 2, 0] = value
        else:
            W[:, 0] = value
        y = torch.full((T,), V // 2, dtype=torch.int32, device="cuda")
        loss, lse = forward(H, W, y, dtype)
        assert (lse == W[V // 2, 0].float()).all() and (loss == 0).all()


def test_an_ordinary_token_does_not_depend_on_its_neighbours():
    T, d, V = 64, 64, 700
    g = torch.Generator(device="cuda").manual_seed(3)
    H = torch.randn(T, d, generator=g, device="cuda").bfloat16()
    W = torch.randn(V, d, generator=g, device="cuda").bfloat16()
    y = torch.randint(V, (T,), generator=g, device="cuda", dtype=torch.int32)
    one = forward(H, W, y, "bf16")
    H[::3] *= 1e6
    two = forward(H, W, y, "bf16")
    near = torch.arange(T, device="cuda") % 3 != 0
    assert all(torch.equal(a[near], b[near]) for a, b in zip(one, two))
