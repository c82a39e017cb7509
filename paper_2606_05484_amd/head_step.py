"""One training step of the last two pipeline stages: the boundary between them
and the vocabulary's loss, with several micro-batches in flight.

    python -m paper_2606_05484_amd.head_step [--tokens 8192 --d 1024 --r 256 --vocabulary 32000 --micro 4 --steps 10
                                              --block 0 --optimizer sgd]

For every micro-batch the sender encodes its activations X, keeps them in 8
bits (ckpt_pack) and lets X go; the receiver decodes, and its head gives the
loss (xent_fwd), dH and the head's gradient (xent_bwd) without the logits ever
being kept; decode_bwd turns dH into the coordinates' gradient.  Then the
sender's backward of every micro-batch reads X from its 8 bits
(ckpt_encode_bwd).  Without a block the head stands directly at the boundary
(H = Xhat).  With block = b one gated residual block of rank b and the last
norm lie between the two, as a stage's own layers would:
  [h | G] = (norm(Xhat; w_in) P1) P2^T         P1 [d, b], P2 [2 d, b]
  x' = Xhat + scale norm(h; w_post) silu(G),   H = norm(x'; w_out)
its products those of the codec without anchors (encode, decode), everything
else norm_fwd and norm_bwd.

main() trains the head, the block and the projector (stiefel_step) on
synthetic tokens whose activations carry their targets, and prints the loss
and the time of every step: its gradients and the update of the head and the block.  The head and the block learn by plain SGD or by
AdamW on the gradient clipped to norm 1 (grad_norm, adamw_step), with states in
fp32 (adamw) or in 8 bits (adamw8).
"""
import argparse

import torch

from . import mapl


class Block:
    """What the gated residual block adds to a step: its parameters' names and shapes, buffers, and calls."""

    def __init__(self, T, d, rank, new):
        bf, f32 = torch.bfloat16, torch.float32
        self.d = d
        self.shapes = dict(P1=(d, rank), P2=(2 * d, rank), w_in=(d,), w_post=(d,), scale=(d,), w_out=(d,))
        self.grads = {name: new(shape, f32) for name, shape in self.shapes.items()}
        self.before = mapl.norm_desc(T, d)
        self.after = mapl.norm_desc(T, d, branch=True, post=True, gate="silu", ld_h=2 * d, ld_gate=2 * d)
        self.down, self.up = mapl.desc(T=T, d=d, r=rank), mapl.desc(T=T, d=2 * d, r=rank)
        self.y, self.x, self.H, self.dy, self.dx, self.dX = (new((T, d), bf) for _ in range(6))
        self.z, self.dz = new((T, rank), bf), new((T, rank), bf)
        self.hg, self.dhg = new((T, 2 * d), bf), new((T, 2 * d), bf)
        self.need = [mapl.workspace_bytes(self.down, mapl.CALL_ENCODE), mapl.workspace_bytes(self.up, mapl.CALL_DECODE),
                     mapl.workspace_bytes(self.up, mapl.CALL_DECODE_BWD), mapl.workspace_bytes(self.down, mapl.CALL_ENCODE_BWD),
                     mapl.norm_workspace_bytes(self.before), mapl.norm_workspace_bytes(self.after)]

    def forward(self, X, p, ws):
        """H from X = Xhat; p: a dict of the parameters (fp32)."""
        h, g = self.hg[:, :self.d], self.hg[:, self.d:]
        mapl.norm_fwd(self.before, X, None, None, None, None, p["w_in"], None, self.y)
        mapl.encode(self.down, self.y, None, p["P1"], None, None, None, self.z, ws)
        mapl.decode(self.up, self.z, None, p["P2"], None, None, None, self.hg, ws)
        mapl.norm_fwd(self.after, X, h, g, p["w_post"], p["scale"], p["w_out"], self.x, self.H)
        return self.H

    def backward(self, X, dH, p, add, ws):
        """dXhat from dH, and the parameters' gradients (added to with add)."""
        d, o = self.d, self.grads
        h, g, dh, dg = self.hg[:, :d], self.hg[:, d:], self.dhg[:, :d], self.dhg[:, d:]
        mapl.norm_bwd(self.after, dH, None, self.x, h, g, p["w_post"], p["scale"], p["w_out"], self.dx, dh, dg,
                      o["w_post"], o["scale"], o["w_out"], add, ws)
        mapl.decode_bwd(self.up, self.dhg, self.z, None, p["P2"], None, None, None, self.dz, o["P2"], add, ws)
        mapl.encode_bwd(self.down, self.dz, self.y, None, p["P1"], None, None, self.dy, o["P1"], add, ws)
        mapl.norm_bwd(self.before, self.dy, self.dx, X, None, None, None, None, p["w_in"], self.dX, None, None, None, None,
                      o["w_in"], add, ws)
        return self.dX


class HeadStep:
    """Buffers and calls of one step: `micro` micro-batches of T tokens, d
    channels, r coordinates (not quantised), a table of `ids` anchors of width
    k and `vocabulary` entries, and with `block` > 0 a block of that rank.  gradients(...)
    leaves the step's dU [d, r] and dW [vocabulary, d], both fp32, every micro-batch's
    loss [T] and dX [T, d], and the block's in block.grads."""

    def __init__(self, T, d, r, vocabulary, micro=1, ids=0, k=0, device="cuda", block=0):
        self.T, self.d, self.micro = T, d, micro
        self.D = mapl.desc(T=T, d=d, r=r, V=ids, k=k)
        self.X = mapl.xent_desc(T, d, vocabulary)
        e = lambda shape, dt: torch.empty(shape, dtype=dt, device=device)
        bf, f32 = torch.bfloat16, torch.float32
        sq, se = mapl.ckpt_shapes(T, d)
        # what a micro-batch in flight holds: 1.03 bytes a value of X, and dZ
        self.q, self.e = e((micro,) + sq, torch.int8), e((micro,) + se, torch.uint8)
        self.dZ = e((micro, T, r), bf)
        self.Z, self.H, self.dH = e((T, r), bf), e((T, d), bf), e((T, d), bf)
        self.loss = [e((T,), f32) for _ in range(micro)]  # (rows of a matrix need not be 16-byte aligned)
        self.lse, self.dX = e((T,), f32), e((micro, T, d), bf)
        self.dU, self.dW = e((d, r), f32), e((vocabulary, d), f32)
        n = [mapl.workspace_bytes(self.D, c) for c in (mapl.CALL_ENCODE, mapl.CALL_DECODE, mapl.CALL_DECODE_BWD)]
        n += [mapl.xent_workspace_bytes(self.X, c) for c in (mapl.XENT_FWD, mapl.XENT_BWD)]
        self.block = Block(T, d, block, e) if block else None
        if block:
            n += self.block.need
        self.ws = mapl.workspace(max(n + [mapl.ckpt_encode_bwd_workspace_bytes(self.D)]), device)

    def gradients(self, X, ids, targets, U, A_s, B_s, A_r, B_r, W, scale, weight=None, block=None):
        """Sequences of `micro` tensors: X [T, d], ids, targets (negative: masked) and
        weight [T].  The gradients are of scale sum_t weight loss over all of them.
        block: a dict of the block's parameters (block.shapes), fp32."""
        D, ws = self.D, self.ws
        for m in range(self.micro):
            mapl.ckpt_pack(self.T, self.d, X[m], self.q[m], self.e[m])
            mapl.encode(D, X[m], ids[m], U, A_s, B_s, None, self.Z, ws)
            mapl.decode(D, self.Z, ids[m], U, A_r, B_r, None, self.H, ws)
            H = self.H if self.block is None else self.block.forward(self.H, block, ws)
            mapl.xent_fwd(self.X, H, W, targets[m], self.loss[m], self.lse, ws)
            w = None if weight is None else weight[m]
            mapl.xent_bwd(self.X, H, W, targets[m], self.lse, w, scale, self.dH, self.dW, m > 0, ws)
            dH = self.dH if self.block is None else self.block.backward(self.H, self.dH, block, m > 0, ws)
            mapl.decode_bwd(D, dH, self.Z, ids[m], U, A_r, B_r, None, self.dZ[m], self.dU, m > 0, ws)
        for m in range(self.micro):
            mapl.ckpt_encode_bwd(D, self.dZ[m], self.q[m], self.e[m], ids[m], U, A_s, B_s, self.dX[m], self.dU, 1, ws)


class SGD:
    """Plain steps of a dict of fp32 tensors by their gradients, under the same names; copies: bf16 copies to
    keep up to date, by name."""

    def __init__(self, params, grads, copies=(), lr=1.0):
        self.params, self.grads, self.copies, self.lr = params, grads, dict(copies), lr

    def step(self):
        for name, p in self.params.items():
            p.add_(self.grads[name], alpha=-self.lr)
        for name, copy in self.copies.items():
            copy.copy_(self.params[name])


class AdamW:
    """The optimizer of a step's parameters: a dict of fp32 tensors and, under the same names, their
    gradients (fp32); copies: bf16 copies to keep up to date, by name.  What has one dimension does not decay."""

    def __init__(self, params, grads, copies=(), lr=1e-3, states="f32", clip=1.0, weight_decay=0.01, seed=0):
        names, low = list(params), states == "8bit"
        like = lambda name, n: torch.zeros(n, dtype=torch.uint8 if low else torch.float32, device=params[name].device)
        m, v = ([like(k, params[k].numel()) for k in names] for _ in range(2))
        e = [like(k, mapl.optim_exponents(params[k].numel())) for k in names] if low else None
        self.clip = clip
        self.params = mapl.optim_params([grads[k] for k in names], [params[k] for k in names], m, v, e,
                                        [dict(copies).get(k) for k in names],
                                        [weight_decay if params[k].dim() > 1 else 0.0 for k in names])
        self.desc = mapl.adamw_desc(lr, states=states, seed=seed)
        device = params[names[0]].device
        self.stats, self.count = torch.zeros(2, device=device), torch.zeros(1, dtype=torch.int32, device=device)
        self.ws = mapl.workspace(mapl.grad_norm_workspace_bytes(self.params), device)

    def step(self):
        """Clips and steps; a gradient that is not finite changes nothing (count stays too)."""
        mapl.grad_norm(self.params, self.stats, self.ws, step=self.count, max_norm=self.clip)
        mapl.adamw_step(self.desc, self.params, stats=self.stats, step=self.count)


def main(argv=None):
    ap = argparse.ArgumentParser(description="training steps over a stage boundary and the vocabulary's loss")
    ap.add_argument("--tokens", type=int, default=8192, help="tokens of a micro-batch")
    ap.add_argument("--d", type=int, default=1024)
    ap.add_argument("--r", type=int, default=256)
    ap.add_argument("--vocabulary", type=int, default=32000)
    ap.add_argument("--micro", type=int, default=4, help="micro-batches in flight")
    ap.add_argument("--steps", type=int, default=10)
    ap.add_argument("--block", type=int, default=0, help="rank of the gated block before the head (a multiple of 64; 0: none)")
    ap.add_argument("--optimizer", choices=("sgd", "adamw", "adamw8"), default="sgd", help="of the head and the block")
    ap.add_argument("--lr", type=float, default=None, help="1 (sgd) or 3e-3")
    a = ap.parse_args(argv)
    torch.manual_seed(0)
    T, d, r, V, k, bf = a.tokens, a.d, a.r, a.vocabulary, 64, torch.bfloat16
    step = HeadStep(T, d, r, V, a.micro, ids=V, k=k, block=a.block)
    rnd = lambda *s: torch.randn(*s, device="cuda")
    # activations of rank r that carry the next token, and the anchors' share of the present one
    U = torch.linalg.qr(rnd(d, r))[0].contiguous()
    meaning = rnd(V, r) @ torch.linalg.qr(rnd(d, r))[0].T
    A, B = (0.1 * rnd(V, k)).to(bf), (0.1 * rnd(k, d)).to(bf)
    W32 = 0.02 * rnd(V, d)
    learned, grads = {"W": W32}, {"W": step.dW}
    if a.block:
        for name, shape in step.block.shapes.items():
            ones = torch.ones(shape, device="cuda")
            learned[name] = rnd(*shape) / shape[1] ** 0.5 if len(shape) > 1 else 0.1 * ones if name == "scale" else ones
        grads.update(step.block.grads)
    lr = a.lr if a.lr is not None else 1.0 if a.optimizer == "sgd" else 3e-3
    W = W32.to(bf)
    if a.optimizer == "sgd":
        optimizer = SGD(learned, grads, {"W": W}, lr)
    else:
        optimizer = AdamW(learned, grads, {"W": W}, lr, "8bit" if a.optimizer == "adamw8" else "f32")
    M = torch.zeros(1, d, r, device="cuda")
    wsU = mapl.workspace(mapl.workspace_bytes(None, mapl.CALL_STIEFEL, 1, d, r))
    spent = []
    for n in range(a.steps):
        # a few hundred frequent entries, so that some steps see them often
        ids, y = ([((torch.rand(T, device="cuda") ** 4) * min(V, 400)).int() for _ in range(a.micro)] for _ in range(2))
        X = [(meaning[y[m].long()] + A[ids[m].long()].float() @ B.float() + 0.1 * rnd(T, d)).to(bf)
             for m in range(a.micro)]
        for t in y:
            t[T - T // 64:] = -1  # padding
        live = a.micro * (T - T // 64)
        t0, t1 = (torch.cuda.Event(enable_timing=True) for _ in range(2))
        t0.record()
        step.gradients(X, ids, y, U, A, B, A, B, W, 1.0 / live, block=learned)
        optimizer.step()
        t1.record()
        mapl.stiefel_step(1, d, r, U, step.dU, M, 0.02, 0.9, 5, 7, wsU)
        torch.cuda.synchronize()
        spent.append(t0.elapsed_time(t1))
        print("step %d  loss %.4f  %.2f ms" % (n, sum(float(l.sum()) for l in step.loss) / live, spent[-1]), flush=True)
    held = (step.q.numel() + step.e.numel()) / 2 ** 20
    print("%d tokens a step, %.2f ms (median); %.0f MiB hold the activations in flight (bf16: %.0f); logits kept: none"
          % (a.micro * T, sorted(spent)[len(spent) // 2], held, 2 * a.micro * T * d / 2 ** 20))


if __name__ == "__main__":
    main()
