"""Plain 64-bit forms of the operators of a round of drafts over a cache of 8 bits, and how far a kernel may be from them."""
import math

import torch

import cache_ref as ref

U32 = ref.U32
E4M3 = torch.float8_e4m3fn


# ---- numbers of 8 bits, from their definition ---------------------------------------------------------------------------------------

def e4m3_value(byte: int) -> float:
    """Sign, 4 bits of exponent (bias 7), 3 of mantissa; exponent 0: multiples of 2^-9; all ones: NaN."""
    e, m = byte >> 3 & 15, byte & 7
    x = math.nan if byte & 127 == 127 else m * 2.0 ** -9 if e == 0 else (8 + m) * 2.0 ** (e - 10)
    return -x if byte & 128 else x


def scale_of(top: float) -> float:
    """The smallest power of two, 2^-126 at least, times which 448 is no less than `top`; 0 of 0."""
    if top == 0.0:
        return 0.0
    e = max(math.frexp(top)[1] - 9, -126)
    while top > 448.0 * 2.0 ** e:
        e += 1
    while e > -126 and top <= 448.0 * 2.0 ** (e - 1):
        e -= 1
    return 2.0 ** e


POSITIVE = torch.tensor([e4m3_value(i) for i in range(127)], dtype=torch.float64)   # ascending; an even place has an even mantissa


def quantise(x):
    """(numbers as float64 [rows, D], scale) of one head's block x [rows, D]."""
    x = x.double()
    s = scale_of(float(x.abs().nan_to_num(0, 0, 0).max()))
    if s == 0.0:
        y = torch.zeros_like(x)
        y[x == math.inf], y[x == -math.inf], y[x.isnan()] = 448.0, -448.0, math.nan   # (only where all else is zeros)
        return y, s
    a = (x.abs() / s).clamp(max=448.0).nan_to_num(0)
    hi = torch.searchsorted(POSITIVE, a.contiguous()).clamp(max=126)
    lo = (hi - 1).clamp(min=0)
    below, above = a - POSITIVE[lo], POSITIVE[hi] - a
    at = torch.where((below < above) | ((below == above) & (lo % 2 == 0)), lo, hi)
    y = POSITIVE[at] * x.sign()
    y[x.isnan()] = math.nan
    return y, s


def append8(kn, vn, k, v, ks, vs, kt, vt, cached, accepted=None, n_accepted=None):
    """The cache's tensors after the call (copies on the host, numbers as float64), the new lengths and the rows appended."""
    kn, vn = kn.cpu(), vn.cpu()
    k, v = k.cpu().double(), v.cpu().double()
    ks, vs, kt, vt = (t.cpu().clone() for t in (ks, vs, kt, vt))
    B, T, Hk, D = kn.shape
    block, cap = kt.shape[1], k.shape[1]
    lengths, counts = [], []
    for b in range(B):
        n = min(max(int(cached[b]), 0), cap)
        take = ref.accepted_of(accepted, n_accepted, b, T, T if accepted is None else accepted.shape[1])[: cap - n]
        lengths.append(n + len(take))
        counts.append(len(take))
        for num, scale, tail, fresh in ((k, ks, kt, kn), (v, vs, vt, vn)):
            rows = torch.cat([tail[b, : n % block], fresh[b, take]]).clone()
            full = rows.shape[0] // block
            for i in range(full):
                at = n // block + i
                for h in range(Hk):
                    num[b, at * block: (at + 1) * block, h], scale[b, h, at] = quantise(rows[i * block: (i + 1) * block, h])
            left = rows[full * block:]
            tail[b, : left.shape[0]] = left
    return k, v, ks, vs, kt, vt, torch.tensor(lengths, dtype=torch.int32), torch.tensor(counts, dtype=torch.int32)


def make_cache(g, B, cap, Hk, D, block, dtype, std=1.0):
    """(k, v, k_scale, v_scale, k_tail, v_tail) of random numbers; scales are powers of two and numbers between them."""
    def one():
        num = (torch.randn((B, cap, Hk, D), generator=g, device="cuda") * 60).clamp(-448, 448).to(E4M3)
        scale = std / 60 * torch.exp2(torch.randint(-2, 3, (B, Hk, cap // block), generator=g, device="cuda").float())
        scale = torch.where(torch.rand(scale.shape, generator=g, device="cuda") < 0.5, scale, torch.exp2(scale.log2().round()))
        return num, scale.contiguous(), (torch.randn((B, block, Hk, D), generator=g, device="cuda") * std).to(dtype)
    (k, ks, kt), (v, vs, vt) = one(), one()
    return k, v, ks, vs, kt, vt


def values(num, scale, tail, n):
    """The n rows that one sequence's cache stands for, [n, Hk, D]: num [cap, Hk, D], scale [Hk, blocks], tail [block, Hk, D]."""
    block = tail.shape[0]
    full = n // block
    x = num[: full * block].double().view(full, block, *num.shape[1:]) * scale[:, :full].double().T[:, None, :, None]
    return torch.cat([x.reshape(full * block, *num.shape[1:]), tail[: n - full * block].double()])


def attn8(q, kn, vn, cache, cached, tree=None, drafted=None, scale=None):
    """(out, lse, tolerance of out, tolerance of lse) as cache_ref.attn's, whose derivation holds with these additions: a score's factor is rounded
    once more for its block (2 U32 S), a weight is multiplied by its block's scale and the sum by its inverse, each rounded, and the exponent moved by the scale's
    logarithm, both off by U32 of a number below 2^8: 2^8 U32 and 4 U32.  A weight that carries its scale may fall out of fp16's range: it is then off by 2^-25 of
    numbers that carry 2^9 and are relative to the largest scale, of which a value is at most 448 times as large: 2^-34 of the largest value, a key."""
    B, T, Hq, D = q.shape
    k8, v8, ks, vs, kt, vt = (t.detach().cpu() for t in cache)
    cap, block, Hk = k8.shape[1], kt.shape[1], k8.shape[2]
    kc, vc = torch.zeros((B, cap, Hk, D), dtype=torch.float64), torch.zeros((B, cap, Hk, D), dtype=torch.float64)
    big = torch.zeros(B, dtype=torch.float64)
    top = 0
    for b in range(B):
        n = min(max(int(cached[b]), 0), cap)
        top = max(top, n)
        kc[b, :n], vc[b, :n] = values(k8[b], ks[b], kt[b], n), values(v8[b], vs[b], vt[b], n)
        if n // block:
            big[b] = 448 * vs[b, :, : n // block].max()
        big[b] = torch.cat([big[b, None], vc[b, :n].abs().nan_to_num(0, 0, 0).flatten(), vn[b].detach().cpu().double().abs().nan_to_num(0, 0, 0).flatten()]).max()
    out, lse, tol, tol_lse = ref.attn(q, kn, vn, kc, vc, cached, tree, drafted, scale)
    sc = scale or 1 / math.sqrt(D)
    # (S, the largest sum of magnitudes of a row's scores, as there; A <= the largest value)
    kmax = torch.cat([kc, kn.detach().cpu().double()], 1).abs().nan_to_num(0, 0, 0).amax((1, 2))      # [B, D]
    S = (q.detach().cpu().double().abs() * kmax[:, None, None]).sum(-1) * sc
    extra = 2 * (2 * U32 * S + 2 ** 8 * U32 + 4 * U32)
    keys = top + T
    return out, lse, tol + (big[:, None, None] * (extra + keys * 2.0 ** -33))[..., None], tol_lse + extra


def norm_rope(x, angles, gain=None, start=None, depth=None, eps=1e-6, norm=True, interleaved=False):
    """(y, tolerance) of x [B, T, H, D].  In 32 bits: a sum of D squares (D + 2 half steps), its root and quotient (4), products with the gain (2) move y by
    e = (D / 2 + 8) U32 of itself; cosines and sines are off by 2^-22, and two products and a sum round thrice; one rounding to the element type at the end."""
    B, T, H, D = x.shape
    u = ref.half_step(x.dtype)
    x = x.detach().cpu().double()
    y = x / (x.square().mean(-1, keepdim=True) + eps).sqrt() if norm else x.clone()
    if gain is not None:
        y = y * gain.cpu().double()
    pos = torch.zeros((B, 1), dtype=torch.float64) if start is None else start.cpu().double()[:, None]
    pos = pos + (torch.arange(T) if depth is None else depth.cpu()).double()
    pos = pos.expand(B, T)
    size = y.abs()
    if angles is not None:
        R = 2 * len(angles)
        z = pos[..., None, None] * torch.as_tensor(angles, dtype=torch.float64)
        lo, hi = (slice(0, R, 2), slice(1, R, 2)) if interleaved else (slice(0, R // 2), slice(R // 2, R))
        a, b = y[..., lo].clone(), y[..., hi].clone()
        y[..., lo], y[..., hi] = a * z.cos() - b * z.sin(), b * z.cos() + a * z.sin()
        size = size.clone()
        size[..., lo] = size[..., hi] = a.abs() + b.abs()
    tol = 1.01 * (u * y.abs() + size * ((D / 2 + 8 + 4) * U32 + 2.0 ** -22)) + (2.0 ** -25 if u == 2.0 ** -11 else 1e-37)
    return y, tol


def verify(p, ids, u, q=None, parents=None, drafted=None):
    """[(tokens that stay, next)] for each sequence, from the definition; None for a sequence without tokens."""
    def mass(x):
        x = x.detach().cpu().double()
        return torch.where((x > 0) & x.isfinite(), x, 0.0)
    B, T, V = p.shape
    ids, u = ids.cpu(), u.cpu().double()
    u = torch.where(u > 0, u.clamp(max=1.0), 0.0)
    res = []
    for b in range(B):
        m = T if drafted is None else min(max(int(drafted[b]), 0), T)
        if m == 0:
            res.append(None)
            continue
        up = [t - 1 for t in range(T)] if parents is None else (parents if parents.dim() == 1 else parents[b]).tolist()
        path, w, R = [0], mass(p[b, 0]), 1.0
        while True:
            n = path[-1]
            w, R = mass(p[b, n]), 1.0
            for c in range(n + 1, m):
                x = int(ids[b, c])
                if up[c] != n or not 0 <= x < V:
                    continue
                if q is not None:
                    qn = mass(q[b, n])
                    if float(u[b, c]) * float(qn[x]) * R < float(w[x]):
                        path.append(c)
                        break
                    w = (w - R * qn).clamp(min=0.0)
                    R = float(w.sum())
                else:
                    if float(u[b, c]) * R < float(w[x]):
                        path.append(c)
                        break
                    R = max(R - float(w[x]), 0.0)
                    w[x] = 0.0
            else:
                break
        if not float(w.sum()) > 0:
            w = mass(p[b, path[-1]])
        edges = w.cumsum(0)
        over = (edges > float(u[b, 0]) * float(edges[-1])).nonzero().flatten()
        some = (w > 0).nonzero().flatten()
        res.append((path, int(over[0]) if len(over) else int(some[-1]) if len(some) else -1))
    return res
