"""The training step with a gated block and AdamW between the boundary and the
head: norms, products, loss, gradients, clipping and update, as they run together."""
import numpy as np
import pytest
import torch

import _step_helpers as sh
from oracle import codec as oc
from paper_2606_05484_amd import head_step

pytestmark = pytest.mark.gpu
bf = torch.bfloat16


def rel(got, want):
    g, w = (np.asarray(t.double().cpu() if torch.is_tensor(t) else t, dtype=np.float64) for t in (got, want))
    return np.linalg.norm(g - w) / np.linalg.norm(w)


@pytest.mark.parametrize("T,d,r,V,rank,micro", [(300, 128, 64, 500, 64, 2), (1, 64, 64, 33, 64, 1), (777, 256, 128, 1001, 128, 2)])
def test_gradients(T, d, r, V, rank, micro):
    """Against float64 autograd through the block and the loss.  About ten bf16 roundings lie on
    the longest path, each off by 1.7e-3 (relative, rms): 5.4e-3 together; 2e-2 is allowed."""
    print("head block", T, d, r, V, rank, micro, flush=True)
    g = torch.Generator(device="cuda").manual_seed(T + d)
    rnd = lambda *s: torch.randn(*s, generator=g, device="cuda")
    U = torch.linalg.qr(rnd(d, r))[0].contiguous()
    X = [(rnd(T, r) @ U.T + 0.3 * rnd(T, d)).to(bf) for _ in range(micro)]
    y = [torch.randint(V, (T,), generator=g, device="cuda", dtype=torch.int32) for _ in range(micro)]
    for t in y:
        t[1::9] = -1
    W = (rnd(V, d) / d ** 0.5).to(bf)
    weight = [0.5 + torch.rand(T, generator=g, device="cuda") for _ in range(micro)]
    scale = 1.0 / sum(int((t >= 0).sum()) for t in y)
    step = head_step.HeadStep(T, d, r, V, micro, block=rank)
    p = {k: rnd(*s) / s[1] ** 0.5 if len(s) > 1 else 1.0 + 0.3 * rnd(*s) for k, s in step.block.shapes.items()}
    step.gradients(X, [None] * micro, y, U, None, None, None, None, W, scale, weight, block=p)
    torch.cuda.synchronize()

    h = lambda t: t.double().cpu().numpy()
    q = {k: v.double().requires_grad_() for k, v in p.items()}
    W64 = W.double().requires_grad_()
    total, heads = 0.0, []
    for m in range(micro):
        Xh = torch.from_numpy(oc.decode(oc.encode(h(X[m]), None, h(U), None, None, operand="bf16"), None, h(U), None, None,
                                        operand="bf16")).cuda().requires_grad_()
        heads.append(Xh)
        hg = (sh.norm_y(Xh, q["w_in"], 1e-5) @ q["P1"]) @ q["P2"].T
        n = hg[:, :d] * sh.rms(hg[:, :d], 1e-5) * q["w_post"]
        x = Xh + q["scale"] * n * torch.nn.functional.silu(hg[:, d:])
        l = sh.norm_y(x, q["w_out"], 1e-5) @ W64.T
        live = y[m] >= 0
        loss = torch.logsumexp(l, 1)[live] - l[live, y[m].long()[live]]
        assert ((step.loss[m][live].double() - loss).abs() <= 2e-2 * (1 + loss.abs())).all()
        total = total + scale * (weight[m].double()[live] * loss).sum()
    names = list(q)
    want = torch.autograd.grad(total, heads + [W64] + [q[k] for k in names])
    dU = 0.0
    for m in range(micro):
        Z = oc.encode(h(X[m]), None, h(U), None, None, operand="bf16")
        dZ, du = oc.decode_bwd(h(want[m]), Z, None, h(U), None, None, operand="bf16")
        dX, due = oc.encode_bwd(dZ, h(X[m]), None, h(U), None, None, operand="bf16")
        dU = dU + du + due
        assert rel(step.dX[m], dX) < 2e-2
    assert rel(step.dW, want[micro]) < 2e-2 and rel(step.dU, dU) < 2e-2
    for k, grad in zip(names, want[micro + 1:]):
        assert rel(step.block.grads[k], grad) < 2e-2, k


@pytest.mark.parametrize("states", ["f32", "8bit"])
def test_adamw_of_a_step(states):
    """Clip and update of all of a step's parameters against the forms, and a gradient that is not finite."""
    g = torch.Generator(device="cuda").manual_seed(1)
    rnd = lambda *s: torch.randn(*s, generator=g, device="cuda")
    shapes = {"W": (1001, 64), "P": (128, 64), "w": (64,)}
    params, grads = ({k: rnd(*s) for k, s in shapes.items()} for _ in range(2))
    W = params["W"].to(bf)
    opt = head_step.AdamW(params, grads, {"W": W}, lr=1e-2, states=states, clip=1.0, weight_decay=0.1, seed=3)
    norm = float(torch.cat([x.double().flatten() for x in grads.values()]).norm())
    before = {k: v.clone() for k, v in params.items()}
    opt.step()
    torch.cuda.synchronize()
    factor = sh.f32(1.0 / norm)
    assert abs(float(opt.stats[1]) / factor - 1) < 2 * sh.U24 and int(opt.count) == 1
    factor = float(opt.stats[1])
    for k in shapes:
        zero = torch.zeros_like(before[k], dtype=torch.float64)
        m, v, root = sh.new_states(zero, zero, sh.rounded(grads[k].double() * factor), 0.9, 0.95)
        p, tol = sh.new_p(before[k], m, root, 1, 1e-2, 0.9, 0.95, 1e-8, 0.1 if len(shapes[k]) > 1 else 0.0)
        assert ((params[k].double() - p).abs() <= tol).all()
    assert torch.equal(W, params["W"].to(bf))
    grads["P"][5, 5] = float("inf")
    before = {k: v.clone() for k, v in params.items()}
    opt.step()
    torch.cuda.synchronize()
    assert int(opt.count) == 1 and all(torch.equal(params[k], before[k]) for k in shapes)


@pytest.mark.parametrize("more", [["--optimizer", "adamw"], ["--optimizer", "adamw8", "--block", "64"], ["--block", "128", "--lr", "0.1"]],
                         ids=lambda m: "-".join(m))
def test_the_command_runs(more, capsys):
    head_step.main(["--tokens", "500", "--d", "128", "--r", "64", "--vocabulary", "1001", "--micro", "2", "--steps", "3"] + more)
    lines = [l for l in capsys.readouterr().out.splitlines() if l.startswith("step")]
    assert len(lines) == 3 and all(np.isfinite(float(l.split()[3])) for l in lines)
