"""Tests that attention over a cache of 8 bits keeps the bits of its softmax weights that it says it does: two 16-bit numbers each where few rows share a head, fp16 numbers beyond."""
import math

import pytest
import torch

import cache_ref
import draft_ref as ref
from test_gpu_draft_ops import BF, E4M3, FP, gen, ints, normal, run_attn

U32 = 2.0 ** -24
BOTH = pytest.mark.parametrize("dtype", [BF, FP], ids=["bf16", "fp16"])


def halves(g, shape, device="cuda"):
    """-1, -1/2 .. 1: sums of their products are exact in 32 bits."""
    return torch.randint(-2, 3, shape, generator=g, device=device) / 2


def softmax_and_tolerance(x, seen, v, u, kept):
    """(weights, outputs, tolerance) of scores x [rows, keys].  Scores are exact up to the factor to base 2 (four roundings); the exponent's argument, with 9 for fp16 weights and
    the logarithm of a power of two for the V scale, rounds once more: a weight is off by e = U32 (8 max |x| + 12) + 2^-21, in the numerator and in the sum.
    For the product with v it is off by `kept` of itself, and fp16 ones by 2^-25 of numbers that carry 2^9 and 2^-8 at least of the block's scale: 2^-26 of the row's largest.
    The sums over keys round once a key, and the output by half a step u."""
    p = torch.softmax(x.masked_fill(~seen, -math.inf), 1)
    o, A = p @ v, p @ v.abs()
    e = U32 * (8 * float(x.abs().max()) + 12) + 2.0 ** -21
    return p, o, 1.01 * (u * o.abs() + A * (kept + 2 * e + (x.shape[1] + 64) * U32)) + x.shape[1] * 2.0 ** -26 * float(v.abs().max())


def worst(out, q, kn, vn, cache, cached, tree_seen, scale, kept):
    B, T, Hq, D = q.shape
    k8, v8, ks, vs, kt, vt = (t.cpu() for t in cache)
    q, kn, vn, out = (t.cpu().double() for t in (q, kn, vn, out))
    Hk, over = kn.shape[2], 0.0
    for b, n in enumerate(cached.tolist()):
        kc, vc = ref.values(k8[b], ks[b], kt[b], n), ref.values(v8[b], vs[b], vt[b], n)
        for h in range(Hq):
            g = h // (Hq // Hk)
            k, v = torch.cat([kc[:, g], kn[b, :, g]]), torch.cat([vc[:, g], vn[b, :, g]])
            seen = torch.cat([torch.ones((T, n), dtype=torch.bool), tree_seen], 1)
            _, o, tol = softmax_and_tolerance(q[b, :, h] @ k.T * scale, seen, v, cache_ref.half_step(kept[0]), kept[1])
            over = max(over, float(((out[b, :, h] - o).abs() / tol).max()))
    return over


def cache_of(g, B, cap, Hk, D, block, dtype, integers):
    v = torch.randint(-4, 5, (B, cap, Hk, D), generator=g, device="cuda").float() if integers else torch.randn((B, cap, Hk, D), generator=g, device="cuda") * 8
    vs = torch.exp2(torch.randint(-2, 3, (B, Hk, cap // block), generator=g, device="cuda").float())
    return (halves(g, (B, cap, Hk, D)).to(E4M3), v.to(E4M3), torch.ones_like(vs), vs, halves(g, (B, block, Hk, D)).to(dtype), normal(g, (B, block, Hk, D), dtype))


@pytest.mark.gpu
@BOTH
@pytest.mark.parametrize("T,Hq,Hk,D,block,lens", [(1, 12, 12, 128, 32, [64, 250]), (4, 8, 2, 64, 64, [64, 130, 255]), (13, 8, 4, 128, 64, [64, 200]), (32, 4, 2, 64, 32, [64, 100]),
                                                  (2, 8, 2, 128, 128, [128, 256])])
def test_weights_of_few_rows_are_two_numbers_each(T, Hq, Hk, D, block, lens, dtype):
    # less than 2^-7 of a bf16 weight is cut off, and that rounded by 2^-8 of itself; fp16 ones, of rows of 16 bits, are finer
    print("few rows", T, Hq, Hk, D, block, lens, dtype, flush=True)
    g, B = gen(111), len(lens)
    q, kn, vn = halves(g, (B, T, Hq, D)).to(dtype), halves(g, (B, T, Hk, D)).to(dtype), normal(g, (B, T, Hk, D), dtype)
    cache = cache_of(g, B, 256, Hk, D, block, dtype, False)
    out, _ = run_attn(q, kn, vn, cache, ints(lens))
    over = worst(out, q, kn, vn, cache, ints(lens), torch.ones((T, T)).tril() > 0, 1 / math.sqrt(D), (dtype, 2.0 ** -15))
    assert over <= 1.0, f"{over:.3f} of the tolerance"


@pytest.mark.gpu
@BOTH
@pytest.mark.parametrize("T,Hq,Hk,D,block,n", [(5, 16, 1, 64, 64, 64), (5, 16, 1, 128, 64, 128), (70, 4, 2, 128, 32, 256), (70, 2, 1, 64, 128, 128), (33, 4, 2, 64, 32, 96)])
def test_weights_of_many_rows_over_8_bits_are_fp16_numbers(T, Hq, Hk, D, block, n, dtype):
    # (the tokens see cached rows alone: those of 16 bits have weights of their own type)
    print("many rows", T, Hq, Hk, D, block, n, dtype, flush=True)
    g, B = gen(112), 2
    q, kn, vn = halves(g, (B, T, Hq, D)).to(dtype), halves(g, (B, T, Hk, D)).to(dtype), normal(g, (B, T, Hk, D), dtype)
    cache = cache_of(g, B, n, Hk, D, block, dtype, True)
    tree = torch.zeros((B, T, (T + 63) // 64), dtype=torch.int64, device="cuda")
    out, _ = run_attn(q, kn, vn, cache, ints([n, n]), tree=tree, scale=0.5)
    over = worst(out, q, kn, vn, cache, ints([n, n]), torch.zeros((T, T), dtype=torch.bool), 0.5, (dtype, 2.0 ** -11))
    assert over <= 1.0, f"{over:.3f} of the tolerance"


@BOTH
@pytest.mark.parametrize("D", [64, 128])
def test_the_tolerances_tell_coarser_weights(D, dtype):
    # weights rounded to bf16 once, planted in the 64-bit form: past both tolerances; and what the kernels say they keep is within them
    g = torch.Generator().manual_seed(113)
    for n, scale, kept, integers in ((64, 1 / math.sqrt(D), 2.0 ** -15, False), (256, 1 / math.sqrt(D), 2.0 ** -15, False), (64, 0.5, 2.0 ** -11, True), (128, 0.5, 2.0 ** -11, True)):
        q, k = halves(g, (80, D), "cpu").double(), halves(g, (n, D), "cpu").double()
        v = torch.randint(-4, 5, (n, D), generator=g).double() if integers else (torch.randn((n, D), generator=g) * 8).to(E4M3).double()
        x = q @ k.T * scale
        p, o, tol = softmax_and_tolerance(x, torch.ones_like(x, dtype=torch.bool), v, cache_ref.half_step(dtype), kept)
        w = p / p.amax(1, keepdim=True)
        high = (w.float().view(torch.int32) & -65536).view(torch.float32).double()               # cut off
        fine = (w * 512).half().double() / 512 if integers else high + (w - high).bfloat16().double()
        for weights, told in ((w.bfloat16().double(), True), (fine, False)):
            got = ((weights @ v) / w.sum(1, keepdim=True)).to(dtype).double()
            assert (float(((got - o).abs() / tol).max()) > 1.0) == told
