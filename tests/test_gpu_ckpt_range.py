"""The sender's backward from checkpoints at both ends of fp32's range."""
import pytest
import torch

import _train_helpers as th
from paper_2606_05484_amd import mapl

pytestmark = pytest.mark.gpu
DT = {"bf16": torch.bfloat16, "f32": torch.float32}


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("size,gain", [(2.0 ** -122, 2.0 ** 100), (2.0 ** -120, 2.0 ** 110), (2.0 ** -60, 1.0), (2.0 ** 120, 2.0 ** -100)])
def test_backward_at_the_range_s_ends(size, gain, dtype):
    """Small activations keep the digits their blocks have (units down to 2^-126),
    large ones stay finite."""
    T, d, r = 300, 128, 64
    print("ckpt range", size, gain, dtype, flush=True)
    g = torch.Generator(device="cuda").manual_seed(7)
    X = (torch.randn(T, d, generator=g, device="cuda") * size).to(DT[dtype])
    dZ = (torch.randn(T, r, generator=g, device="cuda") * gain).to(DT[dtype])
    U = torch.linalg.qr(torch.randn(d, r, generator=g, device="cuda").cpu())[0].cuda().contiguous()
    sq, se = mapl.ckpt_shapes(T, d)
    q, e = torch.empty(sq, dtype=torch.int8, device="cuda"), torch.empty(se, dtype=torch.uint8, device="cuda")
    mapl.ckpt_pack(T, d, X, q, e, dtype)
    D = mapl.desc(T=T, d=d, r=r, x_dtype=dtype)
    dX, dU = torch.empty_like(X), torch.empty(d, r, device="cuda")
    mapl.ckpt_encode_bwd(D, dZ, q, e, None, U, None, None, dX, dU, 0, mapl.workspace(mapl.ckpt_encode_bwd_workspace_bytes(D)))
    x, z = th.ckpt_values(*th.ckpt(X), T), dZ.double()
    assert ((dU.double() - x.t() @ z).abs() <= 2 * (T + 64) * th.U24 * (x.abs().t() @ z.abs()) + 2.0 ** -140).all()
