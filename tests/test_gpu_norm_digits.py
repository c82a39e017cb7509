"""The norms' gradients where rows are large and gradients small: every result within its
bound (_step_helpers), nothing lost to a product that falls below fp32 on the way."""
import pytest
import torch

from test_gpu_norm import Case

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("T,d,x,h", [(9, 64, "f32", "f32"), (40, 256, "bf16", "bf16"), (70, 1024, "f32", "bf16"), (21, 2048, "bf16", "bf16"),
                                     (5, 4096, "f32", "f32"), (3, 16384, "bf16", "bf16")])
@pytest.mark.parametrize("size,small", [(1e36, 1e-10), (1e35, 1e-6)])
@pytest.mark.parametrize("kw", [dict(branch=False, post=False, gate="none", dxo=False), dict(gate="silu"), dict(gate="none", dxo=False)],
                         ids=["y_alone", "gated", "no_dxo"])
def test_small_gradients_of_large_rows(T, d, x, h, size, small, kw):
    """dw_pre = sum dy x' r is of dy's size, x' r being about 1, while dy r (1e-46, 1e-41) is below
    fp32's normal numbers; dx and dh are too, and may be anything up to 1e-38."""
    print("norm small gradients", T, d, x, h, size, small, kw, flush=True)
    c = Case(T, d, x, h, size=size, **kw)
    c.dy.mul_(small)
    if c.dxo is not None:
        c.dxo.mul_(small)
    c.fwd()
    c.bwd()
    torch.cuda.synchronize()
    assert float(c.dw_pre.abs().max()) > 0.1 * small
    c.check()
