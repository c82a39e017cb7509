"""Cross entropy in fp32 where an operand passes 2 GiB, and the largest
vocabulary in both types."""
import pytest
import torch

import _train_helpers as th
from paper_2606_05484_amd import mapl

pytestmark = pytest.mark.gpu
DT = {"bf16": torch.bfloat16, "f32": torch.float32}
NAN = float("nan")


def space(D):
    return torch.full((max(mapl.xent_workspace_bytes(D, c) for c in (0, 1)),), 255, dtype=torch.uint8, device="cuda")


def test_hidden_states_past_2_gib():
    T, d, V = 32768 + 40, 16384, 103
    assert T * d * 4 > 1 << 31
    print("xent fp32", T, d, V, flush=True)
    g = torch.Generator(device="cuda").manual_seed(1)
    H = torch.randn(T, d, generator=g, device="cuda")
    W = torch.randn(V, d, generator=g, device="cuda") / 64
    y = torch.full((T,), -1, dtype=torch.int32, device="cuda")
    some = torch.cat([torch.arange(20, device="cuda"), torch.arange(T - 60, T, device="cuda")])
    y[some] = torch.randint(V, (len(some),), generator=g, device="cuda", dtype=torch.int32)
    r = th.xent(H[some], W, y[some], None, 0.5)
    D = mapl.xent_desc(T, d, V, "f32", "f32")
    ws = space(D)
    loss, lse = (torch.full((T,), NAN, device="cuda") for _ in range(2))
    mapl.xent_fwd(D, H, W, y, loss, lse, ws)
    e = th.lse_error(H[some], W, r)
    assert ((lse[some].double() - r["lse"]).abs() <= e).all() and ((loss[some].double() - r["loss"]).abs() <= 2 * e).all()
    assert not loss[20:T - 60].any() and torch.isfinite(lse).all()
    lse[some] = r["lse"].float()
    dH, dW = torch.full_like(H, NAN), torch.full_like(W, NAN)
    mapl.xent_bwd(D, H, W, y, lse, None, 0.5, dH, dW, 0, ws)
    eH, eW = th.grad_errors(H[some], W, r, 0.5, False, False)
    assert ((dH[some].double() - r["dH"]).abs() <= eH).all() and not dH[20:T - 60].any()
    # (dW's product runs over all T tokens, the masked ones as zeros: zeros round nothing)
    assert ((dW.double() - r["dW"]).abs() <= eW).all()


def test_weights_past_2_gib():
    T, d, V = 5, 4096, 131072 + 37
    assert V * d * 4 > 1 << 31
    print("xent fp32", T, d, V, flush=True)
    g = torch.Generator(device="cuda").manual_seed(2)
    H, W = torch.randn(T, d, generator=g, device="cuda"), torch.randn(V, d, generator=g, device="cuda")
    W /= 32
    y = torch.tensor([0, V - 1, -1, 131072, 77], dtype=torch.int32, device="cuda")
    D = mapl.xent_desc(T, d, V, "f32", "f32")
    ws = space(D)
    loss, lse = (torch.full((T,), NAN, device="cuda") for _ in range(2))
    mapl.xent_fwd(D, H, W, y, loss, lse, ws)
    r = th.xent(H, W, y, None, 0.5)
    e = th.lse_error(H, W, r)
    assert ((lse.double() - r["lse"]).abs() <= e).all() and ((loss.double() - r["loss"]).abs() <= 2 * e).all()
    dH, dW = torch.full_like(H, NAN), torch.full_like(W, NAN)
    mapl.xent_bwd(D, H, W, y, r["lse"].float(), None, 0.5, dH, dW, 0, ws)
    eH, eW = th.grad_errors(H, W, r, 0.5, False, False)
    assert ((dH.double() - r["dH"]).abs() <= eH).all()
    assert ((dW.double() - r["dW"]).abs() <= eW).all()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_largest_vocabulary(dtype):
    T, d, V = 3, 64, 1 << 22
    print("xent largest vocabulary", dtype, flush=True)
    g = torch.Generator(device="cuda").manual_seed(3)
    H, W = torch.randn(T, d, generator=g, device="cuda").to(DT[dtype]), torch.randn(V, d, generator=g, device="cuda").to(DT[dtype])
    y = torch.tensor([V - 1, 1 << 21, 0], dtype=torch.int32, device="cuda")
    D = mapl.xent_desc(T, d, V, dtype, "f32")
    ws = space(D)
    loss, lse = (torch.full((T,), NAN, device="cuda") for _ in range(2))
    mapl.xent_fwd(D, H, W, y, loss, lse, ws)
    r = th.xent(H, W, y, None, 0.5)
    e = th.lse_error(H, W, r)
    assert ((lse.double() - r["lse"]).abs() <= e).all() and ((loss.double() - r["loss"]).abs() <= 2 * e).all()
    dH, dW = torch.full_like(H, NAN), torch.full((V, d), NAN, device="cuda")
    mapl.xent_bwd(D, H, W, y, r["lse"].float(), None, 0.5, dH, dW, 0, ws)
    eH, eW = th.grad_errors(H, W, r, 0.5, dtype == "bf16", False)
    assert ((dH.double() - r["dH"]).abs() <= eH).all()
    assert ((dW.double() - r["dW"]).abs() <= eW).all()
