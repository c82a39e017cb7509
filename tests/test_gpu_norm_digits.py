"""The norms' gradients where rows are large and gradients small: every result within its
bound (_step_helpers), nothing lost to a product that falls below fp32 on the way."""
import pytest
import torch

import _step_helpers as sh
from test_gpu_norm import Case, within

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


# act(G) alone: x = 0, h = 1 and no norm leave x' = alpha s act(G) in fp32, off by act's error (8 u: the exponential's two, its
# correction, 1 + e, the reciprocal and their steps, the products), two products and the sum's rounding.
@pytest.mark.parametrize("h", ["bf16", "f32"])
@pytest.mark.parametrize("kind", ["sigmoid", "silu"])
def test_an_fp32_stream_has_the_gates_digits(h, kind):
    T, d = 5, 1024
    c = Case(T, d, "f32", h, post=False, gate=kind)
    c.x.zero_(), c.h.fill_(1.0)
    c.G.copy_(torch.linspace(-85, 85, T * d, device="cuda").view(T, d))
    c.fwd()
    torch.cuda.synchronize()
    want = c.alpha * c.scale.double() * sh.act(c.G, kind)[0]
    within(c.xo, want, 11.01 * sh.U24 * want.abs() + 1e-38, "xo")


@pytest.mark.parametrize("h", ["bf16", "f32"])
@pytest.mark.parametrize("kind", ["sigmoid", "silu"])
def test_an_fp32_streams_scale_gradient_has_the_gates_digits(h, kind):
    """One token: dscale = alpha dx' h act(G), no sum to hide in."""
    d = 4096
    c = Case(1, d, "f32", h, post=False, pre=False, gate=kind)
    c.G.copy_(torch.linspace(-85, 85, d, device="cuda").view(1, d))
    c.bwd()
    torch.cuda.synchronize()
    want = (c.alpha * c.dxo.double() * c.h.double() * sh.act(c.G, kind)[0])[0]
    within(c.dscale, want, 11.01 * sh.U24 * want.abs() + 1e-38, "dscale")
