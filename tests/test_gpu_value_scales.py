"""GPU tests of attention over a cache of 8 bits where the values' scales are far apart or as large as they can be."""
import math

import pytest
import torch

import cache_ref
import draft_ref as ref
from test_gpu_draft_ops import BF, E4M3, FP, gen, ints, normal, run_attn

pytestmark = pytest.mark.gpu
U32 = 2.0 ** -24


def relative(q, kn, vn, cache, cached):
    """(out, tolerance) as cache_ref.attn's for the rows that the cache stands for.  The scales' roundings move a weight by `extra` of itself (draft_ref.attn8), so an output by
    extra times A = sum p |v| / sum p, of which cache_ref's tolerance holds a half step and more: A <= tolerance / u.  fp16 outputs below 2^-14 are rounded to
    multiples of 2^-24."""
    B, cap, Hk, D = cache[0].shape
    k8, v8, ks, vs, kt, vt = (t.detach().cpu() for t in cache)
    kc, vc = torch.zeros((B, cap, Hk, D), dtype=torch.float64), torch.zeros((B, cap, Hk, D), dtype=torch.float64)
    for b in range(B):
        n = int(cached[b])
        kc[b, :n], vc[b, :n] = ref.values(k8[b], ks[b], kt[b], n), ref.values(v8[b], vs[b], vt[b], n)
    out, _, tol, _ = cache_ref.attn(q, kn, vn, kc, vc, cached)
    u = cache_ref.half_step(q.dtype)
    kmax = torch.cat([kc, kn.detach().cpu().double()], 1).abs().amax((1, 2))
    S = (q.detach().cpu().double().abs() * kmax[:, None, None]).sum(-1, keepdim=True) / math.sqrt(D)
    return out, tol * (1 + 2 * (2 * U32 * S + 2 ** 8 * U32 + 4 * U32) / u) + (2.0 ** -25 if q.dtype == FP else 0.0)


def check(q, kn, vn, cache, cached):
    got, _ = run_attn(q, kn, vn, cache, cached)
    want, tol = relative(q, kn, vn, cache, cached)
    over = (got.cpu().double() - want).abs() / tol
    assert float(over.max()) <= 1.0, f"{float(over.max()):.3f} of the tolerance"


# Query rows look either at blocks with large values or at blocks with small ones: scores of the others are e^-70 and less of theirs.  up to 64 rows to a head,
# and more; the latter's weights are fp16 numbers
@pytest.mark.parametrize("dtype", [BF, FP], ids=["bf16", "fp16"])
@pytest.mark.parametrize("order", ["LS", "SL", "LSL", "SLS", "LLSSLS", "SSSSLLLL"])
@pytest.mark.parametrize("T,Hq,Hk,D,block", [(2, 4, 2, 128, 32), (20, 4, 2, 64, 32), (90, 4, 1, 128, 32), (40, 6, 2, 64, 64), (80, 2, 1, 128, 128)])
def test_rows_that_see_small_values_alone_are_as_good(T, Hq, Hk, D, block, order, dtype):
    print("small values", T, Hq, Hk, D, block, order, dtype, flush=True)
    g = gen(97)
    n = len(order) * block
    large, small = (2.0 ** 10, 2.0 ** -20) if dtype == BF else (2.0 ** 7, 2.0 ** -22)
    q, kn, vn = normal(g, (2, T, Hq, D), dtype, 0.1), normal(g, (2, T, Hk, D), dtype, 0.1), normal(g, (2, T, Hk, D), dtype)
    q[..., 0] = torch.where(torch.arange(T, device="cuda") % 2 == 0, 16.0, -16.0)[None, :, None].to(dtype)
    kn[..., 0] = 0.0
    k, v = ((8 * torch.randn((2, n, Hk, D), generator=g, device="cuda")).to(E4M3).float() for _ in range(2))
    v = 224 + 224 * torch.rand(v.shape, generator=g, device="cuda")
    ks, vs = torch.full((2, Hk, len(order)), 2.0 ** -4, device="cuda"), torch.zeros((2, Hk, len(order)), device="cuda")
    for i, c in enumerate(order):
        k[:, i * block: (i + 1) * block, :, 0] = 448.0 if c == "L" else -448.0
        vs[:, :, i] = large if c == "L" else small
    tails = torch.zeros((2, block, Hk, D), dtype=dtype, device="cuda")
    check(q, kn, vn, (k.to(E4M3), v.to(E4M3), ks, vs, tails, tails.clone()), ints([n, n]))


SHAPES = pytest.mark.parametrize("T,Hq,Hk,D,block", [(1, 4, 2, 128, 64), (9, 4, 2, 64, 32), (90, 4, 1, 128, 32), (40, 6, 2, 64, 64)])


@SHAPES
def test_scales_up_to_the_largest_finite_one(T, Hq, Hk, D, block):
    # all weights alike, and numbers so small that their sums fit 32 bits
    g = gen(98)
    n = 4 * block
    for scale in (2.0 ** 61, 2.0 ** 100, 2.0 ** 120, 2.0 ** 126, 2.0 ** 127):
        q, kn, vn = torch.zeros((1, T, Hq, D), dtype=BF, device="cuda"), normal(g, (1, T, Hk, D), BF), normal(g, (1, T, Hk, D), BF)
        k, v = (torch.randint(-3, 4, (1, n, Hk, D), generator=g, device="cuda").float() * 2.0 ** -9 for _ in range(2))
        tails = torch.zeros((1, block, Hk, D), dtype=BF, device="cuda")
        check(q, kn, vn, (k.to(E4M3), v.to(E4M3), torch.ones((1, Hk, 4), device="cuda"), torch.full((1, Hk, 4), scale, device="cuda"), tails, tails.clone()), ints([n]))


@SHAPES
def test_large_scales_and_scores_that_rise_a_little(T, Hq, Hk, D, block):
    # from the second 128 rows on weights are 2^5.9 of what the maximum was before: with their scale a sum of eight passes 2^128, and is not to
    g = gen(99)
    n = 512
    q, kn, vn = torch.zeros((1, T, Hq, D), dtype=BF, device="cuda"), torch.zeros((1, T, Hk, D), dtype=BF, device="cuda"), normal(g, (1, T, Hk, D), BF)
    q[..., 0] = 5.875 * math.log(2.0) * math.sqrt(D)
    kn[..., 0] = -8.0
    k = torch.zeros((1, n, Hk, D), device="cuda")
    k[:, 128:, :, 0] = 1.0
    v = (torch.randint(1, 8, (1, n, Hk, D), generator=g, device="cuda").float() * 2.0 ** -9).to(E4M3)
    tails = torch.zeros((1, block, Hk, D), dtype=BF, device="cuda")
    vs = torch.full((1, Hk, n // block), 2.0 ** 120, device="cuda")
    check(q, kn, vn, (k.to(E4M3), v, torch.ones_like(vs), vs, tails, tails.clone()), ints([n]))
