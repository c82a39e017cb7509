"""The training step over a stage boundary and the vocabulary's loss, against
the float64 forms of every call in turn."""
import numpy as np
import pytest
import torch

import _train_helpers as th
from oracle import codec as oc
from paper_2606_05484_amd import head_step

pytestmark = pytest.mark.gpu
bf = torch.bfloat16


def rel(got, want):
    g, w = (np.asarray(t.double().cpu() if torch.is_tensor(t) else t, dtype=np.float64) for t in (got, want))
    return np.linalg.norm(g - w) / np.linalg.norm(w)


@pytest.mark.parametrize("T,d,r,V,k,micro", [(300, 128, 64, 500, 16, 3), (1, 64, 64, 33, 0, 2), (1027, 256, 128, 3001, 64, 2)])
def test_step(T, d, r, V, k, micro):
    print("head step", T, d, r, V, k, micro, flush=True)
    g = torch.Generator(device="cuda").manual_seed(T)
    rnd = lambda *s: torch.randn(*s, generator=g, device="cuda")
    n_ids = 90
    U = torch.linalg.qr(rnd(d, r))[0].contiguous()
    A_s, A_r = ((0.3 * rnd(n_ids, k)).to(bf) if k else None for _ in range(2))
    B_s, B_r = ((0.3 * rnd(k, d)).to(bf) if k else None for _ in range(2))
    X = [rnd(T, d).to(bf) for _ in range(micro)]
    ids = torch.randint(n_ids, (micro, T), generator=g, device="cuda", dtype=torch.int32) if k else [None] * micro
    y = torch.randint(V, (micro, T), generator=g, device="cuda", dtype=torch.int32)
    y[:, 1::9] = -1
    W = (0.3 * rnd(V, d) / d ** 0.5).to(bf)
    weight = 0.5 + torch.rand(micro, T, generator=g, device="cuda")
    scale = 1.0 / int((y >= 0).sum())
    y, weight = [t.clone() for t in y], [t.clone() for t in weight]  # each on its own: 16-byte aligned
    ids = [None if t is None else t.clone() for t in ids]
    step = head_step.HeadStep(T, d, r, V, micro, ids=n_ids if k else 0, k=k)
    step.gradients(X, ids, y, U, A_s, B_s, A_r, B_r, W, scale, weight)
    torch.cuda.synchronize()

    h = lambda t: None if t is None else t.double().cpu().numpy()
    gpu = lambda a: torch.from_numpy(np.ascontiguousarray(a)).cuda()
    dU, dW = 0.0, 0.0
    for m in range(micro):
        i = None if ids[m] is None else ids[m].cpu().numpy()
        Z = oc.encode(h(X[m]), i, h(U), h(A_s), h(B_s), operand="bf16")
        H = oc.decode(Z, i, h(U), h(A_r), h(B_r), operand="bf16")
        x = th.xent(gpu(H), W, y[m], weight[m], scale)
        assert ((step.loss[m].double() - x["loss"]).abs() <= 2e-2 * (1 + x["loss"].abs())).all()
        dZ, du = oc.decode_bwd(h(x["dH"]), Z, i, h(U), h(A_r), h(B_r), operand="bf16")
        dU, dW = dU + du, dW + x["dW"]
        dX, du = oc.encode_bwd(dZ, h(th.ckpt_values(*th.ckpt(X[m]), T)), i, h(U), h(A_s), h(B_s), operand="bf16")
        dU = dU + du
        assert rel(step.dX[m], dX) < 2e-2
    assert rel(step.dU, dU) < 2e-2 and rel(step.dW, dW) < 2e-2


def test_the_loss_falls(capsys):
    head_step.main(["--tokens", "1000", "--d", "256", "--r", "64", "--vocabulary", "2001", "--micro", "2", "--steps", "8"])
    lines = [l for l in capsys.readouterr().out.splitlines() if l.startswith("step")]
    losses = [float(l.split()[3]) for l in lines]
    assert len(losses) == 8 and losses[0] > 5.0 and losses[-1] < 0.9 * losses[0]
