"""The operators beside the layer in 64 bits, written from their formulas, and how far a kernel that
sums in fp32 may be from them.

U is half an fp32 step: a rounding is off by at most U relative to its value.  A sum of n terms in
any order is off by at most n U times the sum of their magnitudes."""
import numpy as np
import torch

U = 2.0 ** -24


def half_step(dtype) -> float:
    return torch.finfo(dtype).eps / 2


# ------------------------------------------------------------- sorted tokens


def lists(ids: np.ndarray, n: int):
    """offset, pair and row, pair by pair."""
    T, k = ids.shape
    groups = [[] for _ in range(n)]
    for p, e in enumerate(ids.reshape(-1).tolist()):
        if 0 <= e < n:
            groups[e].append(p)
    offset = np.cumsum([0] + [len(g) for g in groups]).astype(np.int32)
    pair, row = np.full(T * k, -1, np.int32), np.full(T * k, -1, np.int32)
    for r, p in enumerate(q for g in groups for q in g):
        pair[r], row[p] = p, r
    return offset, pair, row.reshape(T, k)


def combine(row, w, ys):
    """(y, error bound before its rounding): sum over held pairs of w * ys[row]."""
    held = row >= 0
    got = ys.double()[row.long().clamp(min=0)] * held[..., None]
    wd = torch.where(held, w.double(), torch.zeros((), dtype=torch.float64, device=w.device))[..., None]
    got = torch.where(held[..., None], got, torch.zeros_like(got))
    return (wd * got).sum(1), (row.shape[1] + 1) * U * (wd * got).abs().sum(1)


def combine_backward(row, w, ys, dy):
    """(dys, rows written, dw, bound of dw): a thread's chain is at most h / 128 products, the joins 10."""
    held, h = row >= 0, dy.shape[1]
    at = row.long()[held]
    dys = torch.zeros_like(ys, dtype=torch.float64)
    dys[at] = (torch.where(held, w.double(), 0.0)[..., None] * dy.double()[:, None])[held]
    written = torch.zeros(len(ys), dtype=torch.bool, device=ys.device)
    written[at] = True
    terms = torch.where(held[..., None], ys.double()[row.long().clamp(min=0)], 0.0) * dy.double()[:, None]
    return dys, written, terms.sum(-1), (h / 128 + 20) * U * terms.abs().sum(-1)


# ------------------------------------------------------------ 4-bit products


def w4_matrix(codes, scale, group):
    q = torch.empty(*codes.shape[:-1], 2 * codes.shape[-1], dtype=torch.float64, device=codes.device)
    q[..., 0::2] = (codes % 16).double()
    q[..., 1::2] = (codes // 16).double()
    return (q - 8) * scale.double().repeat_interleave(group, -1)


def w4_product(x, codes, scale, group):
    """(x W^T, bound).  A group's sum runs from 0 over -24 x to the (16 + q) x: 2 * group additions, none
    of them past 31 * sum |x|, each off by up to a whole step; then the scale and the sum over groups."""
    w, xd = w4_matrix(codes, scale, group), x.double()
    g = xd.abs().unflatten(-1, (-1, group)).sum(-1)
    bound = 2 * group * 2 * U * 31 * (g @ scale.double().abs().T)
    bound = bound + (scale.shape[-1] + 2) * U * (xd.abs() @ w.abs().T)
    return xd @ w.T, bound


def swiglu(a, ea, b, eb):
    """SiLU(a) b and its bound from those of a and b: |SiLU'| < 1.1, a few roundings on the way."""
    s = a * torch.sigmoid(a)
    return s * b, 1.1 * ea * b.abs() + s.abs() * eb + 1.1 * ea * eb + 32 * U * (s * b).abs()


# -------------------------------------------------------------------- norms


def rms(v, eps):
    return v / torch.sqrt((v * v).mean(-1, keepdim=True) + eps)


def postnorm(x, y, w, gate, a, eps):
    return a * x + gate * (rms(y, eps) * w)


def grads(fn, inputs, cotangents):
    """Gradients of sum(cotangent * output) with respect to the inputs (float64 leaves)."""
    leaves = [t.detach().double().requires_grad_() for t in inputs]
    outs = fn(*leaves)
    loss = sum((o * c.double()).sum() for o, c in zip(outs, cotangents))
    return torch.autograd.grad(loss, leaves)
