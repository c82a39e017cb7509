"""8-bit activation checkpoints on the GPU: the stored integers and what they
stand for bit for bit, and the sender's backward from them."""
import numpy as np
import pytest
import torch

import _train_helpers as th
from paper_2606_05484_amd import mapl

pytestmark = pytest.mark.gpu
DT = {"bf16": torch.bfloat16, "f32": torch.float32}


def acts(T, d, dtype, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    X = torch.randn(T, d, generator=g, device="cuda") * torch.logspace(-8, 4, d, device="cuda")
    X[:, ::7] = 0.0
    return X.to(DT[dtype])


def packed(X, dtype, stream=None):
    T, d = X.shape
    sq, se = mapl.ckpt_shapes(T, d)
    q = torch.full(sq, 99, dtype=torch.int8, device="cuda")
    e = torch.full(se, 99, dtype=torch.uint8, device="cuda")
    mapl.ckpt_pack(T, d, X, q, e, dtype, stream=stream)
    return q, e


def roundtrip(X, dtype):
    q, e = packed(X, dtype)
    out = {}
    for n, dt in DT.items():
        out[n] = torch.full(X.shape, 7.0, dtype=dt, device="cuda")
        mapl.ckpt_unpack(*X.shape, q, e, out[n], n)
    torch.cuda.synchronize()
    return q, e, out


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("T,d", [(1, 64), (31, 64), (32, 128), (33, 192), (1000, 320), (4097, 1024)])
def test_stored_values_are_exact(T, d, dtype):
    print("ckpt", T, d, dtype, flush=True)
    X = acts(T, d, dtype, T + d)
    q, e, out = roundtrip(X, dtype)
    rq, re = th.ckpt(X)
    assert torch.equal(q.long(), rq) and torch.equal(e.long(), re)
    v = th.ckpt_values(rq, re, T)
    for n in out:
        assert torch.equal(out[n].double(), v)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_extreme_values(dtype):
    top = torch.finfo(DT[dtype]).max
    X = torch.zeros(70, 64, device="cuda")
    X[3, 0], X[4, 0] = top, -top
    X[5, 1], X[6, 1] = 2.0 ** -126, 2.0 ** -133       # under the smallest scale, and subnormal
    X[7, 2], X[8, 3], X[40, 4] = float("nan"), float("-inf"), float("inf")
    X[9, 2] = X[9, 3] = 1.0
    X[64, 5] = -0.0
    X[10, 6], X[11, 6] = 1.9921875, 1.5 / 64          # rounds to 127.5 -> held; a tie
    X = X.to(DT[dtype])
    q, e, out = roundtrip(X, dtype)
    rq, re = th.ckpt(X)
    assert torch.equal(q.long(), rq) and torch.equal(e.long(), re)
    v = th.ckpt_values(rq, re, 70)
    for n in out:
        o = out[n].double()
        assert torch.equal(torch.isnan(o), torch.isnan(v)) and torch.equal(o.nan_to_num(0), v.nan_to_num(0))
    assert torch.isnan(v[:32, 2]).all() and not torch.isnan(v[32:, 2]).any()


def backward(D, dZ, q, e, ids, U, A, B, acc, dtype, call=None):
    dX = torch.full((D.T, D.d), float("nan"), dtype=DT[dtype], device="cuda")
    dU = torch.full((D.d, D.r), 0.5 if acc else float("nan"), device="cuda")
    n = mapl.ckpt_encode_bwd_workspace_bytes(D)
    ws = torch.full((n,), 255, dtype=torch.uint8, device="cuda")
    mapl.ckpt_encode_bwd(D, dZ, q, e, ids, U, A, B, dX, dU, acc, ws)
    torch.cuda.synchronize()
    return dX, dU


@pytest.mark.parametrize("T,d,r,k,space,dtype,acc", [
    (1, 64, 64, 16, "ambient", "bf16", 0), (33, 128, 64, 0, "ambient", "bf16", 1),
    (77, 192, 128, 32, "coord", "bf16", 0), (1021, 1024, 64, 64, "ambient", "bf16", 1),
    (2049, 512, 256, 128, "ambient", "bf16", 0), (4100, 320, 192, 48, "ambient", "bf16", 0),
    (700, 1088, 320, 16, "ambient", "bf16", 0), (8190, 2048, 256, 128, "ambient", "bf16", 1),
    (1, 64, 32, 16, "ambient", "f32", 1), (515, 256, 32, 16, "ambient", "f32", 0), (300, 192, 96, 16, "coord", "f32", 0),
])
def test_backward_from_checkpoint(T, d, r, k, space, dtype, acc):
    print("ckpt_encode_bwd", T, d, r, k, space, dtype, acc, flush=True)
    g = torch.Generator(device="cuda").manual_seed(T + r)
    rn = lambda *s: torch.randn(*s, generator=g, device="cuda")
    X = acts(T, d, dtype, T)
    U = torch.linalg.qr(rn(d, r).cpu())[0].cuda().contiguous()
    V = 300
    ids = torch.randint(V, (T,), generator=g, device="cuda", dtype=torch.int32)
    A = (0.5 * rn(V, k)).to(DT[dtype]) if k else None
    B = (0.5 * rn(k, d if space == "ambient" else r)).to(DT[dtype]) if k else None
    dZ = rn(T, r).to(DT[dtype])
    q, e = packed(X, dtype)
    D = mapl.desc(T=T, d=d, r=r, V=V, k=k, x_dtype=dtype, anchor_space=space)
    dX, dU = backward(D, dZ, q, e, ids if k else None, U, A, B, acc, dtype)
    x, dz, u = th.ckpt_values(*th.ckpt(X), T), dZ.double(), U.double()
    ut = U.bfloat16().double() if dtype == "bf16" else u  # U as the matrix units take it
    ref = dz @ ut.t()
    # r products summed in fp32 in any order (twice the unit roundoff each), the result's rounding
    tol = 2 * r * th.U24 * (dz.abs() @ ut.abs().t()) + ref.abs() * (th.UB * 1.01 if dtype == "bf16" else th.U24)
    assert ((dX.double() - ref).abs() <= tol).all()
    ref, size = x.t() @ dz + 0.5 * acc, x.abs().t() @ dz.abs() + 0.5 * acc
    if k and space == "ambient":
        a, b = A.double()[ids.long()], B.double()
        ref = ref - b.t() @ (a.t() @ dz)
        size = size + b.abs().t() @ (a.abs().t() @ dz.abs())
    tol = 2 * (T + k + 64) * th.U24 * size
    assert ((dU.double() - ref).abs() <= tol).all()


def test_backward_equals_encode_bwd_on_the_unpacked_values():
    T, d, r, k, V = 1500, 512, 128, 32, 100
    g = torch.Generator(device="cuda").manual_seed(5)
    rn = lambda *s: torch.randn(*s, generator=g, device="cuda")
    X, dZ = acts(T, d, "bf16", 6), rn(T, r).bfloat16()
    U, A, B = rn(d, r), rn(V, k).bfloat16(), rn(k, d).bfloat16()
    ids = torch.randint(V, (T,), generator=g, device="cuda", dtype=torch.int32)
    q, e = packed(X, "bf16")
    D = mapl.desc(T=T, d=d, r=r, V=V, k=k)
    dX, dU = backward(D, dZ, q, e, ids, U, A, B, 0, "bf16")
    Y = torch.empty_like(X)
    mapl.ckpt_unpack(T, d, q, e, Y)
    dX2, dU2 = torch.empty_like(dX), torch.empty_like(dU)
    mapl.encode_bwd(D, dZ, Y, ids, U, A, B, dX2, dU2, 0, mapl.workspace(mapl.workspace_bytes(D, mapl.CALL_ENCODE_BWD)))
    torch.cuda.synchronize()
    assert torch.equal(dX, dX2)
    size = Y.double().abs().t() @ dZ.double().abs()
    assert ((dU - dU2).double().abs() <= 4 * (T + k + 64) * th.U24 * (size + B.double().abs().t() @ (
        A.double()[ids.long()].abs().t() @ dZ.double().abs()))).all()


def test_non_finite_blocks_stay_in_their_rows_of_dU():
    T, d, r = 200, 128, 64
    g = torch.Generator(device="cuda").manual_seed(9)
    X = acts(T, d, "bf16", 9)
    X[77, 5] = float("inf")
    U, dZ = torch.randn(d, r, generator=g, device="cuda"), torch.randn(T, r, generator=g, device="cuda").bfloat16()
    q, e = packed(X, "bf16")
    dX, dU = backward(mapl.desc(T=T, d=d, r=r), dZ, q, e, None, U, None, None, 0, "bf16")
    assert torch.isnan(dU[5]).all() and torch.isfinite(dX).all()
    rest = torch.arange(d, device="cuda") != 5
    assert torch.isfinite(dU[rest]).all()


def test_empty_batch():
    D = mapl.desc(T=0, d=64, r=64)
    e0 = torch.empty(16, dtype=torch.uint8, device="cuda")
    dU = torch.ones(64, 64, device="cuda")
    ws = mapl.workspace(max(256, mapl.ckpt_encode_bwd_workspace_bytes(D)))
    U = torch.ones(64, 64, device="cuda")
    for acc, want in ((1, 1.0), (0, 0.0)):
        mapl.ckpt_encode_bwd(D, e0, e0, e0, None, U, None, None, e0, dU, acc, ws)
        torch.cuda.synchronize()
        assert (dU == want).all()


def test_own_stream_and_repeatability():
    T, d, r = 3000, 256, 64
    X = acts(T, d, "bf16", 3)
    g = torch.Generator(device="cuda").manual_seed(4)
    dZ, U = torch.randn(T, r, generator=g, device="cuda").bfloat16(), torch.randn(d, r, generator=g, device="cuda")
    D = mapl.desc(T=T, d=d, r=r)
    q, e = packed(X, "bf16")
    one = backward(D, dZ, q, e, None, U, None, None, 0, "bf16")
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    with torch.cuda.stream(s):
        q2, e2 = packed(X, "bf16")
        two = backward(D, dZ, q2, e2, None, U, None, None, 0, "bf16")
    s.synchronize()
    assert torch.equal(q, q2) and torch.equal(e, e2) and torch.equal(one[0], two[0]) and torch.equal(one[1], two[1])


def test_graph_replays():
    T, d, r = 515, 256, 64
    X = acts(T, d, "bf16", 3)
    g = torch.Generator(device="cuda").manual_seed(4)
    dZ, U = torch.randn(T, r, generator=g, device="cuda").bfloat16(), torch.randn(d, r, generator=g, device="cuda")
    D = mapl.desc(T=T, d=d, r=r)
    sq, se = mapl.ckpt_shapes(T, d)
    q, e = torch.empty(sq, dtype=torch.int8, device="cuda"), torch.empty(se, dtype=torch.uint8, device="cuda")
    dX, dU = torch.empty(T, d, dtype=torch.bfloat16, device="cuda"), torch.empty(d, r, device="cuda")
    ws = mapl.workspace(mapl.ckpt_encode_bwd_workspace_bytes(D))

    def step():
        mapl.ckpt_pack(T, d, X, q, e)
        mapl.ckpt_encode_bwd(D, dZ, q, e, None, U, None, None, dX, dU, 0, ws)

    step()
    torch.cuda.synchronize()
    want = [t.clone() for t in (q, e, dX, dU)]
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for _ in range(3):
        for t in (q, e):
            t.zero_()
        dX.fill_(float("nan"))
        dU.fill_(float("nan"))
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip((q, e, dX, dU), want))
