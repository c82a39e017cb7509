"""Rows past 8192 values, whose backward reads them twice, in every set of parts and type, and in calls
past the caches.  A row's sum there is of at most 32 products in a lane, 6 steps over a wave and 12
waves, each rounded: 50 u, within the 64 u that the bounds count (_step_helpers)."""
import pytest
import torch

from test_gpu_norm import PARTS, Case

pytestmark = pytest.mark.gpu
TYPES = [("bf16", "bf16"), ("f32", "bf16"), ("f32", "f32")]


def run(T, d, x, h, **kw):
    print("norm wide", T, d, x, h, kw, flush=True)
    c = Case(T, d, x, h, **kw)
    c.fwd()
    c.bwd()
    torch.cuda.synchronize()
    c.check()


@pytest.mark.parametrize("kw", PARTS, ids=lambda k: "-".join("%s=%s" % i for i in k.items()))
@pytest.mark.parametrize("x,h", TYPES)
@pytest.mark.parametrize("T,d", [(5, 8256), (3, 12288), (4, 12352), (3, 16384)])
def test_parts(T, d, x, h, kw):
    run(T, d, x, h, **kw)


@pytest.mark.parametrize("kw", [dict(gate="silu"), dict(gate="none", halves=True), dict(pre=False), dict(pre=False, gate="none"), dict(post=False, gate="silu", dxo=False),
                                dict(branch=False, post=False, gate="none")], ids=lambda k: "-".join("%s=%s" % i for i in k.items()))
@pytest.mark.parametrize("x,h", TYPES)
@pytest.mark.parametrize("T,d", [(5200, 8256), (3300, 12352)])
def test_past_the_caches(T, d, x, h, kw):
    """More than 128 MiB of rows in both directions, whatever the types and parts."""
    run(T, d, x, h, **kw)


@pytest.mark.parametrize("x,h", TYPES)
@pytest.mark.parametrize("size", [1e-15, 3e18, 1e30])
@pytest.mark.parametrize("T,d", [(3, 8704), (2, 14336)])
def test_rows_of_any_size(T, d, x, h, size):
    run(T, d, x, h, size=size)
