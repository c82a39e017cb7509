"""Plain 64-bit forms of the 8-bit checkpoint and of the vocabulary's cross
entropy (torch float64, on whatever device their inputs live), written from
the formulas in include/mapl.h, with the element-by-element error bounds that
the kernels' arithmetic allows."""
import torch

U24 = 2.0 ** -24  # fp32 unit roundoff
UB = 2.0 ** -8    # bf16 unit roundoff (8 significant bits)


def two_to(n):
    """2^n of whole numbers (exact: built from the bits)."""
    return ((n.long() + 1023) << 52).view(torch.float64)


def ckpt(X):
    """(q [nb, d, 32], e [nb, d]) of X [T, d], as int64."""
    T, d = X.shape
    nb = -(-T // 32)
    p = torch.zeros(nb * 32, d, dtype=torch.float64, device=X.device)
    p[:T] = X.double()
    p = p.view(nb, 32, d).transpose(1, 2).contiguous()
    a = p.abs().amax(2)
    bad = ~torch.isfinite(p).all(2)
    k = torch.where(bad | (a == 0), torch.full_like(a, -120.0).long(), ((a.view(torch.int64) >> 52) - 1023))
    k = k.clamp(min=-120)
    q = torch.where(bad[:, :, None], torch.zeros_like(p), p) / two_to(k - 6)[:, :, None]
    q = q.round().clamp(-127, 127).long()
    return q, torch.where(bad, torch.full_like(k, 255), k + 127)


def ckpt_values(q, e, T):
    """What a checkpoint stands for, [T, d] float64."""
    v = q.double() * two_to(e.long() - 133)[:, :, None]
    v = torch.where((e.long() == 255)[:, :, None], torch.full_like(v, float("nan")), v)
    return v.transpose(1, 2).reshape(-1, q.shape[1])[:T]


def xent(H, W, y, weight=None, scale=1.0):
    """dict of loss, lse, dH, dW in float64; masked tokens (y < 0, weight 0)
    have no part in anything but lse."""
    H, W, y = H.double(), W.double(), y.long()
    T = H.shape[0]
    l = H @ W.t()
    lse = torch.logsumexp(l, 1)
    at = y.clamp(min=0)[:, None]
    loss = torch.where(y < 0, torch.zeros_like(lse), lse - l.gather(1, at)[:, 0])
    w = torch.ones(T, dtype=torch.float64, device=H.device) if weight is None else weight.double()
    w = torch.where(y < 0, torch.zeros_like(w), w)
    live = torch.nonzero(w != 0)[:, 0]
    dl = torch.exp(l[live] - lse[live, None])
    dl[torch.arange(len(live), device=H.device), y[live]] -= 1.0
    dl *= w[live, None]
    dH = torch.zeros_like(H)
    dH[live] = scale * (dl @ W)
    dW = scale * (dl.t() @ H[live])
    return dict(loss=loss, lse=lse, dH=dH, dW=dW, dl=dl, live=live, l=l, w=w)


def logit_error(H, W):
    """[T] bound of a logit's error: d products summed in fp32 in any order
    (2 d u sum |h w|, the 2 for sums that the matrix units may truncate)."""
    return 2 * H.shape[1] * U24 * (H.double().abs() @ W.double().abs().t()).amax(1)


def lse_error(H, W, ref):
    """[T] bound of lse's error: the logits', each exponential's argument and
    its base-2 scaling (4 u max |l|), the sum of up to 128 numbers in a lane and then in a tree,
    and the logarithm with its result's rounding."""
    big = ref["l"].abs().amax(1)
    return logit_error(H, W) + U24 * (4 * big + 2 * ref["lse"].abs() + 200.0)


def grad_errors(H, W, ref, scale, bf16_in, bf16_dw):
    """Element bounds (dH [T, d], dW [V, d]): dl is off by the logit's and
    lse's error times exp(l - lse) and, in bf16, by its rounding; each product
    adds its fp32 sum, and the result its own rounding."""
    live, w = ref["live"], ref["w"]
    Hl, Wd = H.double()[live], W.double()
    big = ref["l"].abs().amax(1)[live]
    p_rel = logit_error(H, W)[live] + U24 * (4 * big + 2 * ref["lse"].abs()[live] + 16.0)
    p = torch.exp(ref["l"][live] - ref["lse"][live, None])  # at a target dl is p - 1, whose error is p's
    ddl = w[live, None].abs() * p * p_rel[:, None] + ref["dl"].abs() * (UB * 1.01 if bf16_in else 4 * U24) + 2.0 ** -133
    n_v, n_t = 2 * W.shape[0] * U24, 2 * max(1, len(live)) * U24
    eH = torch.zeros_like(ref["dH"])
    eH[live] = scale * ((ddl + n_v * ref["dl"].abs()) @ Wd.abs())
    eW = scale * ((ddl + n_t * ref["dl"].abs()).t() @ Hl.abs())
    eH = eH + ref["dH"].abs() * (UB * 1.01 if bf16_in else 4 * U24)
    eW = eW + ref["dW"].abs() * (UB * 1.01 if bf16_dw else 4 * U24)
    return eH, eW
