"""The gradients' norm and AdamW against their 64-bit forms: states bit for bit,
parameters within the bound of the update's arithmetic."""
import math

import pytest
import torch

import _step_helpers as sh
from paper_2606_05484_amd import mapl

pytestmark = pytest.mark.gpu
DT = {"bf16": torch.bfloat16, "f32": torch.float32}
SIZES = [1, 7, 8, 127, 128, 129, 1000, 2048, 4095, 4096, 4097, 12345, 100003]


def rn(g, *s):
    return torch.randn(*s, generator=g, device="cuda")


def grads(sizes, dt, seed=0, size=1e-3):
    g = torch.Generator(device="cuda").manual_seed(seed)
    return [(size * 10.0 ** (i % 4 - 2) * rn(g, n)).to(DT[dt]) for i, n in enumerate(sizes)]


# ------------------------------------------------------------------- norm
@pytest.mark.parametrize("dt", ["bf16", "f32"])
@pytest.mark.parametrize("sizes", [[1], SIZES, [0, 5, 0], [33] * 160, [], [3000001, 17], [0, 4097, 33] * 150], ids=lambda s: "%d_tensors_%d" % (len(s), sum(s)))
def test_norm(dt, sizes):
    print("grad norm", dt, sizes[:20], flush=True)
    G = grads(sizes, dt)
    P = mapl.optim_params(G)
    ws = mapl.workspace(mapl.grad_norm_workspace_bytes(P, dt))
    stats, step = torch.full((2,), -1.0, device="cuda"), torch.tensor([4], dtype=torch.int32, device="cuda")
    norm = math.sqrt(sum(float(g.double().square().sum()) for g in G))
    for scale, most in ((1.0, float("inf")), (0.25, 0.1 * norm + 1e-9), (-2.0, 10.0 * norm + 1e-9)):
        mapl.grad_norm(P, stats, ws, step=step, grad_scale=scale, max_norm=most, g_dtype=dt)
        want = abs(scale) * norm
        factor = scale * min(1.0, sh.f32(most) / want) if want else scale
        got = stats.tolist()
        assert abs(got[0] - want) <= 1.01 * sh.U24 * want and abs(got[1] - factor) <= 1.01 * sh.U24 * abs(factor)
    assert int(step) == 7


def test_norm_of_huge_tiny_and_not_finite_gradients():
    stats, step = torch.zeros(2, device="cuda"), torch.zeros(1, dtype=torch.int32, device="cuda")
    G = [torch.full((5000,), 2.0 ** 100, device="cuda"), torch.full((3,), 2.0 ** -140, device="cuda")]
    P = mapl.optim_params(G)
    ws = mapl.workspace(mapl.grad_norm_workspace_bytes(P))
    mapl.grad_norm(P, stats, ws, step=step, max_norm=1.0)
    assert abs(float(stats[0]) / (2.0 ** 100 * math.sqrt(5000)) - 1) < 2.0 ** -23 and int(step) == 1
    G[0].zero_()
    mapl.grad_norm(P, stats, ws, step=step, max_norm=1.0)
    assert abs(float(stats[0]) / (2.0 ** -140 * math.sqrt(3)) - 1) < 2.0 ** -8 and int(step) == 2  # (subnormal)
    for bad in (float("nan"), float("inf"), -float("inf")):
        G[0].zero_()
        G[0][4999] = bad
        mapl.grad_norm(P, stats, ws, step=step, max_norm=1.0)
        assert not math.isfinite(float(stats[0])) and int(step) == 2


# ------------------------------------------------------------------- AdamW
class Stage:
    """Tensors of the given sizes with states of a training in progress."""

    def __init__(self, sizes, dt="f32", low=False, seed=1, copy=True, b1=0.9, b2=0.95, lr=1e-2, eps=1e-8):
        g = torch.Generator(device="cuda").manual_seed(seed)
        self.sizes, self.dt, self.low = sizes, dt, low
        self.b1, self.b2, self.lr, self.eps = b1, b2, lr, eps
        self.G = grads(sizes, dt, seed + 1)
        self.P = [0.5 * rn(g, n) for n in sizes]
        size = [float(x.float().square().mean().sqrt()) if len(x) else 1.0 for x in self.G]
        self.m = [0.3 * s * rn(g, n) for s, n in zip(size, sizes)]
        self.v = [s * s * (0.2 + rn(g, n).square()) for s, n in zip(size, sizes)]
        self.e = None
        if low:
            coded = [sh.encode(m.double(), sh.rounded(v.double().sqrt()), 0x80008000) for m, v in zip(self.m, self.v)]
            self.m, self.v, self.e = ([c[i].to(torch.uint8) for c in coded] for i in range(3))
            self.e = [t.contiguous() for t in self.e]
        self.p16 = [torch.zeros(n, dtype=torch.bfloat16, device="cuda") for n in sizes] if copy else None
        self.decay = [0.1 * (i % 3) for i in range(len(sizes))]
        self.lrs = [1.0 + 0.5 * (i % 2) for i in range(len(sizes))]
        self.params = mapl.optim_params(self.G, self.P, self.m, self.v, self.e, self.p16, self.decay, self.lrs)

    def desc(self, step=0, seed=0):
        return mapl.adamw_desc(self.lr, self.b1, self.b2, self.eps, g_dtype=self.dt, states="8bit" if self.low else "f32", step=step, seed=seed)

    def everything(self):
        return [t.clone() for x in (self.P, self.m, self.v, self.e or [], self.p16 or []) for t in x]

    def expected(self, t, seed=0, factor=1.0, lr=None):
        """A list of (p, its bound, m, v, e) by the forms, from the present state."""
        out = []
        for i, n in enumerate(self.sizes):
            m, v = self.m[i].double(), self.v[i].double()
            if self.low:
                m, s = sh.decode(self.m[i], self.v[i], self.e[i])
                v = sh.rounded(s * s)
            g = sh.rounded(self.G[i].double() * sh.f32(factor))
            m, v, root = sh.new_states(m, v, g, self.b1, self.b2)
            rate = sh.f32(sh.f32(self.lr if lr is None else lr) * sh.f32(self.lrs[i]))
            p, tol = sh.new_p(self.P[i], m, root, t, rate, self.b1, self.b2, self.eps, self.decay[i])
            e = None
            if self.low and n:
                m, v, e = sh.encode(m, root, sh.noise(seed, t, i, n, "cuda"))
            out.append((p, tol, m, v, e))
        return out

    def check(self, want):
        for i, (p, tol, m, v, e) in enumerate(want):
            if self.sizes[i] == 0:
                continue
            off = (self.P[i].double() - p).abs()
            assert (off <= tol).all(), "p of tensor %d (%d values): %.3g of the bound" % (i, self.sizes[i], float((off / tol).max()))
            assert torch.equal(self.m[i].double(), m.double()) and torch.equal(self.v[i].double(), v.double()), "states of tensor %d" % i
            if e is not None:
                assert torch.equal(self.e[i].long(), e.long())
            if self.p16 is not None:
                assert torch.equal(self.p16[i], self.P[i].to(torch.bfloat16))


@pytest.mark.parametrize("low", [False, True], ids=["f32", "8bit"])
@pytest.mark.parametrize("dt", ["bf16", "f32"])
@pytest.mark.parametrize("sizes", [[1], SIZES, [0, 5, 0], [257] * 130, [1000003]], ids=lambda s: "%d_tensors_%d" % (len(s), sum(s)))
def test_step(low, dt, sizes):
    print("adamw", low, dt, sizes[:20], flush=True)
    s = Stage(sizes, dt, low)
    for t in (1, 2, 1000):
        want = s.expected(t, seed=5)
        mapl.adamw_step(s.desc(t, 5), s.params)
        torch.cuda.synchronize()
        s.check(want)


@pytest.mark.parametrize("low", [False, True], ids=["f32", "8bit"])
def test_from_nothing(low):
    """The first steps, all states zero (8 bits: all bytes), without a copy."""
    s = Stage(SIZES, low=low, copy=False)
    for x in s.m + s.v + (s.e or []):
        x.zero_()
    for t in range(1, 4):
        want = s.expected(t)
        mapl.adamw_step(s.desc(t), s.params)
        torch.cuda.synchronize()
        s.check(want)


@pytest.mark.parametrize("b1,b2,eps,lr", [(0.0, 0.0, 1e-8, 1e-2), (0.9, 0.999, 1e-15, 3.0), (0.99, 0.5, 1.0, -1e-3), (0.5, 0.9999, 1e-8, 0.0)])
def test_hyperparameters(b1, b2, eps, lr):
    for low in (False, True):
        s = Stage([5000, 3], low=low, b1=b1, b2=b2, eps=eps, lr=lr)
        for t in (1, 3, 2147483647):
            want = s.expected(t, 9)
            mapl.adamw_step(s.desc(t, 9), s.params)
            torch.cuda.synchronize()
            s.check(want)


@pytest.mark.parametrize("low", [False, True], ids=["f32", "8bit"])
def test_clipped_counted_and_skipped_on_the_device(low):
    s = Stage(SIZES, low=low)
    stats, step = torch.zeros(2, device="cuda"), torch.tensor([10], dtype=torch.int32, device="cuda")
    rate = torch.tensor([0.003], device="cuda")
    ws = mapl.workspace(mapl.grad_norm_workspace_bytes(s.params))
    norm = math.sqrt(sum(float(g.double().square().sum()) for g in s.G))
    mapl.grad_norm(s.params, stats, ws, step=step, max_norm=0.5 * norm)
    want = s.expected(11, 3, float(stats[1]), lr=0.003)
    mapl.adamw_step(s.desc(0, 3), s.params, stats=stats, step=step, lr=rate)
    torch.cuda.synchronize()
    assert abs(float(stats[1]) - 0.5) < 1e-6
    s.check(want)
    for bad in (float("nan"), float("inf")):
        keep, s.G[3][100] = float(s.G[3][100]), bad
        mapl.grad_norm(s.params, stats, ws, step=step, max_norm=0.5 * norm)
        before = s.everything()
        mapl.adamw_step(s.desc(0, 3), s.params, stats=stats, step=step, lr=rate)
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(before, s.everything())) and int(step) == 11
        s.G[3][100] = keep


def test_nan_and_infinity_without_the_norm():
    """A block of 128 holds NaNs from then on; its neighbours and other tensors go on."""
    s = Stage([1000, 300], low=True)
    s.G[0][200], s.G[0][513] = float("nan"), float("inf")
    want = s.expected(4, 2)
    mapl.adamw_step(s.desc(4, 2), s.params)
    torch.cuda.synchronize()
    for i, (p, tol, m, v, e) in enumerate(want):
        assert torch.equal(s.m[i].long(), m) and torch.equal(s.v[i].long(), v) and torch.equal(s.e[i].long(), e)
    assert int(s.e[0][1, 0]) == 255 and int(s.e[0][4, 1]) == 255 and int(s.e[0][2, 0]) < 255
    fine = torch.isfinite(want[0][0])
    assert ((s.P[0].double() - want[0][0]).abs()[fine] <= want[0][1][fine]).all()
    want = s.expected(5, 2)
    s.G[0].zero_()
    mapl.adamw_step(s.desc(5, 2), s.params)
    torch.cuda.synchronize()
    assert s.P[0][128:256].isnan().all() and s.P[0][:128].isfinite().all() and s.P[0][256:512].isfinite().all()


@pytest.mark.parametrize("size", [1e-30, 1e-18, 1e-8, 1e8, 1e16])
def test_gradients_of_any_size(size):
    for low in (False, True):
        s = Stage([3000], low=low)
        s.G[0].copy_(size * torch.randn(3000, device="cuda", generator=torch.Generator(device="cuda").manual_seed(8)))
        for t in (1, 2):
            want = s.expected(t, 1)
            mapl.adamw_step(s.desc(t, 1), s.params)
            torch.cuda.synchronize()
            s.check(want)


@pytest.mark.parametrize("size,eps", [(1e-20, 1e-24), (1e-21, 1e-21), (1e-10, 1e-24)])
def test_a_tiny_eps_beside_the_root_of_a_subnormal_number(size, eps):
    for low in (False, True):
        s = Stage([3000], low=low, eps=eps)
        for x in s.m + s.v + (s.e or []):
            x.zero_()
        s.G[0].copy_(size * torch.randn(3000, device="cuda", generator=torch.Generator(device="cuda").manual_seed(8)))
        for t in (1, 2, 3):
            want = s.expected(t, 1)
            mapl.adamw_step(s.desc(t, 1), s.params)
            torch.cuda.synchronize()
            s.check(want)


def test_states_over_many_powers_of_two_in_a_block():
    s = Stage([128 * 40], low=True)
    s.G[0].copy_(torch.randn(128 * 40, device="cuda") * 2.0 ** torch.linspace(-60, 0, 128, device="cuda").repeat(40))
    for t in range(1, 5):
        want = s.expected(t, 6)
        mapl.adamw_step(s.desc(t, 6), s.params)
        torch.cuda.synchronize()
        s.check(want)
    assert int((s.v[0] == 0).sum()) == 0  # no second moment above 0 became 0


def test_unpack_and_pack():
    s = Stage(SIZES + [0, 70000], low=True)
    M, V = ([torch.full((n,), 9.0, device="cuda") for n in s.sizes] for _ in range(2))
    U = mapl.optim_params(s.G, m=M, v=V)
    mapl.adamw_unpack(s.params, U)
    torch.cuda.synchronize()
    for i, n in enumerate(s.sizes):
        if n:
            m, r = sh.decode(s.m[i], s.v[i], s.e[i])
            assert torch.equal(M[i].double(), m) and torch.equal(V[i].double(), sh.rounded(r * r))
    for x in s.m + s.v + s.e:
        x.fill_(1)
    mapl.adamw_pack(U, s.params)
    torch.cuda.synchronize()
    for i, n in enumerate(s.sizes):  # values of the grid come back as they were (not their bytes: where a block's
        if n:  # largest was rounded down to 1.75 2^k, the next smaller power of two holds it now)
            m, r = sh.decode(s.m[i], s.v[i], s.e[i])
            assert torch.equal(M[i].double(), m) and torch.equal(V[i].double(), sh.rounded(r * r))
    g = torch.Generator(device="cuda").manual_seed(2)
    for i, n in enumerate(s.sizes):
        M[i].copy_(rn(g, n))
        V[i].copy_(rn(g, n).square() * 1e-6)
    mapl.adamw_pack(U, s.params)
    torch.cuda.synchronize()
    for i, n in enumerate(s.sizes):
        if n:
            m, v, e = sh.encode(M[i].double(), sh.rounded(V[i].double().sqrt()), 0x80008000)
            assert torch.equal(s.m[i].long(), m) and torch.equal(s.v[i].long(), v) and torch.equal(s.e[i].long(), e)


def test_nothing_behind_a_tensor_is_touched():
    n, room = 1001, 64
    wide = lambda dt, k: torch.full((k + room,), 77, dtype=dt, device="cuda")
    nb = mapl.optim_exponents(n)
    G, P, m, v, e, c = (wide(dt, k) for dt, k in ((torch.float32, n), (torch.float32, n), (torch.uint8, n), (torch.uint8, n),
                                                  (torch.uint8, nb), (torch.bfloat16, n)))
    for x in (m, v, e):
        x[:-room] = 0
    A = mapl.optim_params([G[:n]], [P[:n]], [m[:n]], [v[:n]], [e[:nb]], [c[:n]])
    mapl.adamw_step(mapl.adamw_desc(1e-3, states="8bit", step=1), A)
    torch.cuda.synchronize()
    for x in (P, m, v, e, c):
        assert (x[-room:] == 77).all()
        assert x is c or not (x[:-room] == 77).all()  # (77 - 1e-3 is 77 in bf16)


@pytest.mark.parametrize("low", [False, True], ids=["f32", "8bit"])
def test_repeats_bit_for_bit_and_in_a_replayed_graph(low):
    """The norm, the step's number and the rate live on the device: a replay is the next step."""
    sizes = [4096 * 3 + 5, 33, 700001]
    a, b = Stage(sizes, "bf16", low), Stage(sizes, "bf16", low)
    state = lambda: (torch.zeros(2, device="cuda"), torch.zeros(1, dtype=torch.int32, device="cuda"), torch.tensor([1e-2], device="cuda"))
    (sa, ta, ra), (sb, tb, rb) = state(), state()
    ws = [mapl.workspace(mapl.grad_norm_workspace_bytes(a.params, "bf16")) for _ in range(2)]

    def one(s, stats, step, rate, w):
        mapl.grad_norm(s.params, stats, w, step=step, max_norm=0.01, g_dtype="bf16")
        mapl.adamw_step(s.desc(0, 4), s.params, stats=stats, step=step, lr=rate)

    start = b.everything()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        one(b, sb, tb, rb, ws[1])
    torch.cuda.synchronize()
    assert all(torch.equal(x, y) for x, y in zip(start, b.everything()))
    for k in range(4):
        for s in (a, b):
            for x in s.G:
                x.mul_(0.9 if k != 2 else 1.0)
            if k == 2:
                s.G[1][3] = float("inf")
            if k == 3:
                s.G[1][3] = 0.001
        ra.mul_(0.7), rb.mul_(0.7)
        one(a, sa, ta, ra, ws[0])
        g.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(x, y) for x, y in zip(a.everything(), b.everything()))
        assert torch.equal(sa, sb) and int(ta) == int(tb)
    assert int(ta) == 3


def test_on_another_stream():
    a, b = Stage(SIZES, low=True), Stage(SIZES, low=True)
    mapl.adamw_step(a.desc(1), a.params)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    mapl.adamw_step(b.desc(1), b.params, stream=s)
    torch.cuda.synchronize()
    assert all(torch.equal(x, y) for x, y in zip(a.everything(), b.everything()))


@pytest.mark.parametrize("low,n", [(False, 6000001), (True, 11000003)], ids=["f32", "8bit"])
def test_calls_past_the_caches(low, n):
    """More than 128 MiB: the variants whose loads and stores bypass the last-level cache."""
    s = Stage([4097, n, 12], "bf16", low)
    want = s.expected(3, 1)
    mapl.adamw_step(s.desc(3, 1), s.params)
    torch.cuda.synchronize()
    s.check(want)
    G = grads([40000001, 5], "f32")
    P = mapl.optim_params(G)
    stats = torch.zeros(2, device="cuda")
    mapl.grad_norm(P, stats, mapl.workspace(mapl.grad_norm_workspace_bytes(P)))
    norm = math.sqrt(sum(float(g.double().square().sum()) for g in G))
    assert abs(float(stats[0]) / norm - 1) <= 1.01 * sh.U24


@pytest.mark.parametrize("low", [False, True], ids=["f32", "8bit"])
def test_tensors_between_each_other(low):
    """All arrays of all tensors out of one buffer, tensor after tensor: legal, and nothing is lost."""
    sizes = [1000, 5, 4096, 70001]
    a, b = Stage(sizes, low=low), Stage(sizes, low=low)
    buf = torch.zeros(1 << 22, dtype=torch.uint8, device="cuda")
    at = 0

    def move(t):
        nonlocal at
        at = -(-at // 16) * 16
        new = buf[at:at + t.numel() * t.element_size()].view(t.dtype)
        at += t.numel() * t.element_size()
        return new.copy_(t.reshape(-1))

    for i in range(len(sizes)):
        for x in (b.G, b.P, b.m, b.v, b.e or [None] * 9, b.p16):
            if x[i] is not None:
                x[i] = move(x[i])
    P = mapl.optim_params(b.G, b.P, b.m, b.v, b.e, b.p16, b.decay, b.lrs)
    mapl.adamw_step(a.desc(7), a.params)
    mapl.adamw_step(b.desc(7), P)
    torch.cuda.synchronize()
    assert all(torch.equal(x.view(-1), y.view(-1)) for x, y in zip(a.everything(), b.everything()))


def test_the_second_moment_in_8_bits_follows_the_gradients():
    """1000 steps of b2 = 0.99 from four times the right v: the mean over 8192 values ends at the
    gradients' variance.  A value is off by 0.13 of s at most (its spread), so the mean of v by
    0.13^2 of it and 2 * 0.13 / 90 at random, and by 3 * 0.99^1000 of the start: 5 % allows twice that."""
    n = 8192
    gen = torch.Generator(device="cuda").manual_seed(0)
    G, P = torch.zeros(n, device="cuda"), torch.zeros(n, device="cuda")
    m, v = (torch.zeros(n, device="cuda") for _ in range(2))
    v.fill_(4.0)
    qm, qv, e = (torch.zeros(k, dtype=torch.uint8, device="cuda") for k in (n, n, mapl.optim_exponents(n)))
    A, U = mapl.optim_params([G], [P], [qm], [qv], [e]), mapl.optim_params([G], m=[m], v=[v])
    mapl.adamw_pack(U, A)
    for t in range(1, 1001):
        G.normal_(generator=gen)
        mapl.adamw_step(mapl.adamw_desc(0.0, 0.9, 0.99, states="8bit", step=t), A)
    mapl.adamw_unpack(A, U)
    torch.cuda.synchronize()
    assert abs(float(v.mean()) - 1.0) < 0.05
    assert abs(float(m.mean())) < 5 * 0.23 / math.sqrt(n) + 0.01


def test_past_two_to_the_32():
    """A tensor of more than 2^32 values: every piece in its place (8 bits, bf16 gradients)."""
    n = 2 ** 32 + 5000
    if torch.cuda.mem_get_info()[0] < 60 << 30:
        pytest.skip("needs 60 GiB")
    G = torch.zeros(n, dtype=torch.bfloat16, device="cuda")
    P = torch.zeros(n, device="cuda")
    qm, qv, e = (torch.zeros(k, dtype=torch.uint8, device="cuda") for k in (n, n, mapl.optim_exponents(n)))
    at = [0, 2 ** 31 - 1, 2 ** 31 + 3, 2 ** 32 - 1, 2 ** 32, n - 1]
    G[at] = torch.tensor([1.0, -2.0, 3.0, -4.0, 5.0, -6.0], device="cuda").to(torch.bfloat16)
    A = mapl.optim_params([G], [P], [qm], [qv], [e])
    ws = mapl.workspace(mapl.grad_norm_workspace_bytes(A, "bf16"))
    stats = torch.zeros(2, device="cuda")
    mapl.grad_norm(A, stats, ws, g_dtype="bf16")
    mapl.adamw_step(mapl.adamw_desc(0.5, g_dtype="bf16", states="8bit", step=1), A, stats=stats)
    torch.cuda.synchronize()
    assert abs(float(stats[0]) - math.sqrt(91.0)) < 1e-6
    assert torch.allclose(P[at], torch.tensor([-0.5, 0.5, -0.5, 0.5, -0.5, 0.5], device="cuda"), rtol=1e-6)
    assert int((P != 0).sum()) == len(at)


@pytest.mark.parametrize("sizes", [[1], [4096 * 3000 + 1], [5000] * 60, [5000] * 360])
def test_bytes_behind_the_norms_workspace(sizes):
    G = grads(sizes, "f32", 3)
    p = mapl.optim_params(G)
    need = mapl.grad_norm_workspace_bytes(p)
    ws = torch.full((need + 65536,), 90, dtype=torch.uint8, device="cuda")
    stats = torch.full((8,), 7.0, device="cuda")
    mapl.grad_norm(p, stats, ws, ws_bytes=need)
    torch.cuda.synchronize()
    assert (ws[need:] == 90).all() and (stats[2:] == 7.0).all()
    norm = math.sqrt(sum(float(g.double().square().sum()) for g in G))
    assert abs(float(stats[0]) - norm) <= 2.0 ** -23 * norm and float(stats[1]) == 1.0


@pytest.mark.parametrize("low", [False, True], ids=["f32", "8bit"])
def test_two_steps_at_once(low):
    """Two streams side by side, each with its own tensors."""
    a, b = [Stage(SIZES, low=low, seed=k) for k in (1, 2)], [Stage(SIZES, low=low, seed=k) for k in (1, 2)]
    torch.cuda.synchronize()
    for t in range(1, 6):
        for s in a:
            mapl.adamw_step(s.desc(t, 4), s.params)
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in b]
    for t in range(1, 6):
        for s, on in zip(b, streams):
            with torch.cuda.stream(on):
                mapl.adamw_step(s.desc(t, 4), s.params)
    torch.cuda.synchronize()
    for x, y in zip(a, b):
        assert all(torch.equal(p, q) for p, q in zip(x.everything(), y.everything()))
