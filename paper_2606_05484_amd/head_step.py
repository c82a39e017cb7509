"""One training step of the last two pipeline stages: the boundary between them
and the vocabulary's loss, with several micro-batches in flight.

    python -m paper_2606_05484_amd.head_step [--tokens 8192 --d 1024 --r 256 --vocabulary 32000 --micro 4 --steps 10]

For every micro-batch the sender encodes its activations X, keeps them in 8
bits (ckpt_pack) and lets X go; the receiver decodes, and its head gives the
loss (xent_fwd), dH and the head's gradient (xent_bwd) without the logits ever
being kept; decode_bwd turns dH into the coordinates' gradient.  Then the
sender's backward of every micro-batch reads X from its 8 bits
(ckpt_encode_bwd).  Here the head stands directly at the boundary (H = Xhat);
a stage's own layers would lie between the two.

main() trains the head (plain SGD) and the projector (stiefel_step) on
synthetic tokens whose activations carry their targets, and prints the loss
and the time of every step.
"""
import argparse

import torch

from . import mapl


class HeadStep:
    """Buffers and calls of one step: `micro` micro-batches of T tokens, d
    channels, r coordinates (not quantised), a table of `ids` anchors of width
    k and `vocabulary` entries.  gradients(...) leaves the step's dU [d, r] and
    dW [vocabulary, d], both fp32, and every micro-batch's loss [T] and dX [T, d]."""

    def __init__(self, T, d, r, vocabulary, micro=1, ids=0, k=0, device="cuda"):
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
        self.ws = mapl.workspace(max(n + [mapl.ckpt_encode_bwd_workspace_bytes(self.D)]), device)

    def gradients(self, X, ids, targets, U, A_s, B_s, A_r, B_r, W, scale, weight=None):
        """Sequences of `micro` tensors: X [T, d], ids, targets (negative: masked) and
        weight [T].  The gradients are of scale sum_t weight loss over all of them."""
        D, ws = self.D, self.ws
        for m in range(self.micro):
            mapl.ckpt_pack(self.T, self.d, X[m], self.q[m], self.e[m])
            mapl.encode(D, X[m], ids[m], U, A_s, B_s, None, self.Z, ws)
            mapl.decode(D, self.Z, ids[m], U, A_r, B_r, None, self.H, ws)
            mapl.xent_fwd(self.X, self.H, W, targets[m], self.loss[m], self.lse, ws)
            w = None if weight is None else weight[m]
            mapl.xent_bwd(self.X, self.H, W, targets[m], self.lse, w, scale, self.dH, self.dW, m > 0, ws)
            mapl.decode_bwd(D, self.dH, self.Z, ids[m], U, A_r, B_r, None, self.dZ[m], self.dU, m > 0, ws)
        for m in range(self.micro):
            mapl.ckpt_encode_bwd(D, self.dZ[m], self.q[m], self.e[m], ids[m], U, A_s, B_s, self.dX[m], self.dU, 1, ws)


def main(argv=None):
    ap = argparse.ArgumentParser(description="training steps over a stage boundary and the vocabulary's loss")
    ap.add_argument("--tokens", type=int, default=8192, help="tokens of a micro-batch")
    ap.add_argument("--d", type=int, default=1024)
    ap.add_argument("--r", type=int, default=256)
    ap.add_argument("--vocabulary", type=int, default=32000)
    ap.add_argument("--micro", type=int, default=4, help="micro-batches in flight")
    ap.add_argument("--steps", type=int, default=10)
    a = ap.parse_args(argv)
    torch.manual_seed(0)
    T, d, r, V, k, bf = a.tokens, a.d, a.r, a.vocabulary, 64, torch.bfloat16
    step = HeadStep(T, d, r, V, a.micro, ids=V, k=k)
    rnd = lambda *s: torch.randn(*s, device="cuda")
    # activations of rank r that carry the next token, and the anchors' share of the present one
    U = torch.linalg.qr(rnd(d, r))[0].contiguous()
    meaning = rnd(V, r) @ torch.linalg.qr(rnd(d, r))[0].T
    A, B = (0.1 * rnd(V, k)).to(bf), (0.1 * rnd(k, d)).to(bf)
    W32 = 0.02 * rnd(V, d)
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
        W = W32.to(bf)
        t0, t1 = (torch.cuda.Event(enable_timing=True) for _ in range(2))
        t0.record()
        step.gradients(X, ids, y, U, A, B, A, B, W, 1.0 / live)
        t1.record()
        W32.add_(step.dW, alpha=-1.0)
        mapl.stiefel_step(1, d, r, U, step.dU, M, 0.02, 0.9, 5, 7, wsU)
        torch.cuda.synchronize()
        spent.append(t0.elapsed_time(t1))
        print("step %d  loss %.4f  %.2f ms" % (n, sum(float(l.sum()) for l in step.loss) / live, spent[-1]), flush=True)
    held = (step.q.numel() + step.e.numel()) / 2 ** 20
    print("%d tokens a step, %.2f ms (median); %.0f MiB hold the activations in flight (bf16: %.0f); logits kept: none"
          % (a.micro * T, sorted(spent)[len(spent) // 2], held, 2 * a.micro * T * d / 2 ** 20))


if __name__ == "__main__":
    main()
