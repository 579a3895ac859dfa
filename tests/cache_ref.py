"""Plain 64-bit forms of the cache operators, sequence by sequence and head by head, and how far a kernel may be from them."""
import math

import torch

U32 = 2.0 ** -24


def half_step(dtype) -> float:
    return torch.finfo(dtype).eps / 2


def sees(tree, b, T):
    """[T, T] truth values: row t sees column j."""
    if tree is None:
        return torch.ones((T, T), dtype=torch.bool).tril()
    w = (tree if tree.dim() == 2 else tree[b]).cpu()
    return torch.stack([(w[:, j // 64] >> (j % 64)) & 1 for j in range(T)], 1).bool()


def attn(q, kn, vn, kc, vc, cached, tree=None, drafted=None, scale=None):
    """(out, lse, tolerance of out, tolerance of lse), rows of tokens that a sequence has not drafted NaN.

    A score is a sum of D products in 32 bits: off by at most (D + 2) half steps of the sum of magnitudes S, so a weight by
    e = 2 (D + 2) U32 S + 2^-21 of itself (2: both numerator and reference value; 2^-21: the exponential and its argument's
    rounding).  For the product with V weights are rounded to 16 bits (half a step u); sums run over the keys in 32 bits.
    With A = sum p |v| / sum p:  |out - exact| <= u |out| + A (u + 2 e + (keys + 64) U32), and 1 % for the products of errors."""
    B, T, Hq, D = q.shape
    Hk = kn.shape[2]
    scale = scale or 1 / math.sqrt(D)
    u = half_step(q.dtype)
    q, kn, vn = (t.detach().cpu().double() for t in (q, kn, vn))
    kc, vc = (None, None) if kc is None else (kc.detach().cpu(), vc.detach().cpu())
    out = torch.full((B, T, Hq, D), float("nan"), dtype=torch.float64)
    lse, tol, tol_lse = out[..., 0].clone(), out.clone(), out[..., 0].clone()
    for b in range(B):
        n = 0 if kc is None else min(max(int(cached[b]), 0), kc.shape[1])
        m = T if drafted is None else min(max(int(drafted[b]), 0), T)
        if m == 0:
            continue
        see = torch.cat([torch.ones((m, n), dtype=torch.bool), sees(tree, b, T)[:m, :m]], 1)
        for h in range(Hq):
            g = h // (Hq // Hk)
            k, v = kn[b, :m, g], vn[b, :m, g]
            if n:
                k, v = torch.cat([kc[b, :n, g].double(), k]), torch.cat([vc[b, :n, g].double(), v])
            x = (q[b, :m, h] @ k.T * scale).masked_fill(~see, -math.inf)
            S = (q[b, :m, h].abs() @ k.abs().nan_to_num(0, 0, 0).T * scale).masked_fill(~see, 0).amax(1)
            top = x.amax(1, keepdim=True).clamp(min=-1e300)
            p = (x - top).exp()
            l = p.sum(1)
            v0, a0 = v.nan_to_num(0, 0, 0), v.nan_to_num(0, 0, 0).abs()
            o, A = p @ v0, p @ a0
            for j in (~v.isfinite()).any(1).nonzero().flatten().tolist():    # what is not finite reaches the rows that see it
                rows = see[:, j]
                o[rows] += p[rows, j, None] * torch.where(v[j].isfinite(), 0.0, v[j])
            some = l > 0
            e = 2 * (D + 2) * U32 * S + 2.0 ** -21
            l1 = torch.where(some, l, 1.0)[:, None]
            out[b, :m, h] = torch.where(some[:, None], o / l1, 0.0)
            A = A / l1
            tol[b, :m, h] = 1.01 * (u * out[b, :m, h].abs().nan_to_num(0, 0, 0) + A * (u + 2 * e[:, None] + (n + m + 64) * U32)) + 1e-30
            lse[b, :m, h] = torch.where(some, top[:, 0] + l.log(), -math.inf)
            tol_lse[b, :m, h] = 1.01 * (2 * e + (n + m + 64) * U32 + 4 * U32 * (lse[b, :m, h].abs().nan_to_num(0, 0, 0) + 20))
    return out, lse, tol, tol_lse


def accepted_of(accepted, n_accepted, b, T, n_max):
    n = n_max if n_accepted is None else min(max(int(n_accepted[b]), 0), n_max)
    return [i if accepted is None else min(max(int(accepted[b, i]), 0), T - 1) for i in range(n)]


def append(kn, vn, kc, vc, cached, weights, pos, start, accepted=None, n_accepted=None):
    """The tensors after the call (copies on the host) and the new lengths."""
    kn, vn = kn.cpu(), vn.cpu()
    kc, vc, w, pos = (t.cpu().clone() for t in (kc, vc, weights, pos))
    B, T = kn.shape[:2]
    cap = kc.shape[1]
    new = []
    for b in range(B):
        at = min(max(int(cached[b]), 0), cap)
        for i, t in enumerate(accepted_of(accepted, n_accepted, b, T, T if accepted is None else accepted.shape[1])):
            if at == cap:
                break
            kc[b, at], vc[b, at], w[b, :, at], pos[b, :, at] = kn[b, t], vn[b, t], 0.0, int(start[b]) + i
            at += 1
        new.append(at)
    return kc, vc, w, pos, torch.tensor(new, dtype=torch.int32)


def add_weights(q, lse, kc, cached, weights, accepted=None, n_accepted=None, scale=None):
    """(weights after the call, tolerance).  A weight is exp2 of a difference of two 32-bit numbers (see attn for the score's error S),
    rounded at 4 U32 (|score| + |lse|) at most; the sum over rows adds U32 per row and the sum onto the old value one more."""
    B, T, Hq, D = q.shape
    Hk, cap = kc.shape[2], kc.shape[1]
    scale = scale or 1 / math.sqrt(D)
    q, kc, lse = q.cpu().double(), kc.cpu(), lse.cpu().double()
    w = weights.cpu().double()
    tol = torch.zeros_like(w)
    for b in range(B):
        n = min(max(int(cached[b]), 0), cap)
        rows = accepted_of(accepted, n_accepted, b, T, T if accepted is None else accepted.shape[1])
        if not rows or not n:
            continue
        for h in range(Hq):
            g = h // (Hq // Hk)
            k = kc[b, :n, g].double()
            x = q[b, rows, h] @ k.T * scale
            S = q[b, rows, h].abs() @ k.abs().T * scale
            L = lse[b, rows, h][:, None]
            p = torch.where(L == -math.inf, 0.0, (x - L).exp()).tril(n - len(rows))
            w[b, g, :n] += p.sum(0)
            e = (D + 2) * U32 * S + 4 * U32 * (x.abs() + L.abs().nan_to_num(0, 0, 0)) + 2.0 ** -21
            tol[b, g, :n] += 1.01 * (p * (e + (len(rows) * Hq // Hk + 8) * U32)).sum(0)
    return w, tol + 2 * U32 * w.abs() + 1e-30


def kept_rows(w, pos, n, budget, recent):
    """The rows that stay, in ascending order, of one head's lists of weights and positions."""
    newest = max(pos[:n], default=0)

    def rank(r):
        if pos[r] > newest - recent:
            return (0, 0.0, r)
        return (2, 0.0, r) if w[r] != w[r] else (1, -w[r], r)
    return sorted(sorted(range(n), key=rank)[:budget])


def evict(kc, vc, weights, pos, cached, budget, recent, others=None):
    """In place (copies of the tensors after the call), or `others` = (k, v, weights, pos) after the call; and the new lengths."""
    src = [t.cpu() for t in (kc, vc, weights, pos)]
    dst = [t.clone() for t in src] if others is None else [t.cpu().clone() for t in others]
    B, Hk, cap = src[2].shape
    new = []
    for b in range(B):
        n = min(max(int(cached[b]), 0), cap)
        new.append(min(n, budget))
        for h in range(Hk):
            kept = kept_rows(src[2][b, h].tolist(), src[3][b, h].tolist(), n, budget, recent)
            if others is None:
                stay = set(kept)
                come = [r for r in kept if r >= budget]
                rows = [r if r in stay else come.pop(0) for r in range(min(n, budget))]
                assert not come
            else:
                rows = kept
            for i in (0, 1):
                dst[i][b, : len(rows), h] = src[i][b, rows, h]
            for i in (2, 3):
                dst[i][b, h, : len(rows)] = src[i][b, h, rows]
    return (*dst, torch.tensor(new, dtype=torch.int32))
