"""Norms on other streams and side by side: every output and workspace holds a mark before the
calls, and every round of them leaves copies of its own."""
import pytest
import torch

from test_gpu_norm import Case

pytestmark = pytest.mark.gpu


def wanted(c):
    c.fwd()
    c.bwd()
    torch.cuda.synchronize()
    return c.outputs()


def mark(c):
    for t in (c.xo, c.y, c.dx, c.dh, c.dG, c.dw_post, c.dscale, c.dw_pre):
        if t is not None:
            t.fill_(9.0)
    c.ws.fill_(255)  # (NaNs)


@pytest.mark.parametrize("halves", [False, True])
def test_another_stream_writes_everything(halves):
    c = Case(777, 1024, gate="silu", halves=halves)
    want = wanted(c)
    mark(c)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        c.fwd()
        c.bwd()
    s.synchronize()
    assert all(torch.equal(v, want[k]) for k, v in c.outputs().items())


@pytest.mark.parametrize("shapes", [[(3000, 1024, "bf16", "bf16"), (2000, 2048, "f32", "bf16")], [(500, 8192, "bf16", "bf16"), (5000, 256, "f32", "f32")],
                                    [(300, 16384, "bf16", "bf16"), (1021, 1024, "f32", "bf16"), (4000, 64, "bf16", "bf16")]], ids=lambda s: "%d_at_once" % len(s))
def test_calls_at_once(shapes):
    """A stream each, arrays and a workspace each, ten rounds with no wait between them."""
    cases = [Case(*shape, gate="silu", seed=i) for i, shape in enumerate(shapes)]
    want = [wanted(c) for c in cases]
    for c in cases:
        mark(c)
    torch.cuda.synchronize()
    streams, got = [torch.cuda.Stream() for _ in cases], []
    for _ in range(10):
        for c, s, w in zip(cases, streams, want):
            with torch.cuda.stream(s):
                c.fwd()
                c.bwd()
                got.append((c.outputs(), w))  # copies, made in the stream's order
                mark(c)
    torch.cuda.synchronize()
    assert all(torch.equal(v, w[k]) for o, w in got for k, v in o.items())
