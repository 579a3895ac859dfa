"""GPU tests of a round of drafts over a cache of 8 bits where values, lengths, strides, streams or graphs are unusual, and of whole rounds."""
import math

import pytest
import torch

import draft_ref as ref
import paper_2305_13450_amd as ds
from test_gpu_draft_ops import (BF, E4M3, FP, INF, NAN, angles_of, check_append, check_attn, check_norm, check_verify, drawn_ids, gen, ints, normal, probabilities, run_attn, same,
                                spoil, tree_of)

pytestmark = pytest.mark.gpu
BOTH = pytest.mark.parametrize("dtype", [BF, FP], ids=["bf16", "fp16"])


def setup(g, B, T, Hq, Hk, D, block, lens, dtype, cap=None):
    cached = ints(lens)
    cap = cap or -(-max(max(lens), 1) // block) * block
    cache = spoil(ref.make_cache(g, B, cap, Hk, D, block, dtype), cached)
    return normal(g, (B, T, Hq, D), dtype, 2.0), normal(g, (B, T, Hk, D), dtype), normal(g, (B, T, Hk, D), dtype), cache, cached


# ---- attention -----------------------------------------------------------------------------------------------------------------------

# rows to a head of 1 to 300: every form, with the 16-bit rows inside one tile and over several
FORMS = pytest.mark.parametrize("T,Hq,Hk,D,block,lens", [(1, 4, 2, 128, 64, [150, 3]), (9, 4, 2, 64, 32, [31, 200]), (13, 8, 4, 128, 128, [127, 300]), (40, 6, 2, 64, 64, [100, 640]),
                                                         (90, 4, 1, 128, 32, [31, 333])])


@BOTH
@FORMS
def test_numbers_that_are_not_finite_reach_only_the_rows_that_see_them(T, Hq, Hk, D, block, lens, dtype):
    print("not finite", T, Hq, Hk, D, block, lens, dtype, flush=True)
    g = gen(11)
    q, kn, vn, cache, cached = setup(g, 2, T, Hq, Hk, D, block, lens, dtype)
    if T == 1:
        cache[5][1, 1, 0, 3] = INF                                    # a value of a row held in 16 bits: every token sees it
        got, _ = run_attn(q, kn, vn, cache, cached)
        assert bool((got[1, :, : Hq // Hk, 3] == INF).all()) and bool(got[0].isfinite().all()) and bool(got[1, :, : Hq // Hk, :3].isfinite().all())
        return
    parents, tree = tree_of(g, 2, T)
    vn[:, T // 2, 0, 5], vn[:, T - 1, 0, 6], vn[0, 1, Hk - 1, 7] = INF, -INF, NAN
    cache[5][:, 1, 0, 9] = -INF
    check_attn(q, kn, vn, cache, cached, tree=tree)
    # keys likewise, where nobody sees them: two sequences of which the first has drafted one token less than it seems
    kn[:, T - 1] = NAN
    vn[:, T - 1] = INF
    drafted = ints([T - 1, T - 1])
    check_attn(q, kn, vn, cache, cached, tree=tree, drafted=drafted)


@BOTH
@FORMS
def test_a_cached_number_that_is_none_reaches_its_head_alone(T, Hq, Hk, D, block, lens, dtype):
    g = gen(12)
    q, kn, vn, cache, cached = setup(g, 2, T, Hq, Hk, D, block, lens, dtype)
    clean, clean_lse = run_attn(q, kn, vn, cache, cached)
    G, last = Hq // Hk, lens[1] // block * block - 1
    if last < 0:
        return
    cache[1].view(torch.uint8)[1, last, 0, 2] = 127
    got, lse = run_attn(q, kn, vn, cache, cached)
    assert bool(got[1, :, :G, 2].isnan().all())
    got[1, :, :G, 2] = clean[1, :, :G, 2]
    assert torch.equal(got, clean) and torch.equal(lse, clean_lse)
    cache[0].view(torch.uint8)[1, last, 0, 2] = 127
    got, lse = run_attn(q, kn, vn, cache, cached)
    assert bool(got[1, :, :G].isnan().all()) and bool(lse[1, :, :G].isnan().all())
    assert torch.equal(got[0], clean[0]) and torch.equal(got[1, :, G:], clean[1, :, G:])


@BOTH
@FORMS
def test_scales_of_every_size(T, Hq, Hk, D, block, lens, dtype):
    print("scales", T, Hq, Hk, D, block, lens, dtype, flush=True)
    g = gen(13)
    lens = [6 * block + 5, 3 * block]
    for make in (lambda n: torch.tensor([2.0 ** -20, 2.0 ** -6, 0.0, 2.0 ** -3, 2.0 ** -30, 0.013])[:n], lambda n: torch.tensor([0.0, 0.0, 2.0 ** -7, 0.0, 2.0 ** -8, 0.0])[:n],
                 lambda n: torch.tensor([2.0 ** (-126 if dtype == BF else -20), 2.0 ** (-100 if dtype == BF else -18), 2.0 ** (-80 if dtype == BF else -15)] * 2)[:n],
                 lambda n: torch.zeros(n)):
        q, kn, vn, cache, cached = setup(g, 2, T, Hq, Hk, D, block, lens, dtype, cap=6 * block + block)
        cache[3][:, :, :6] = make(6).cuda()
        cache[2][:, :, 1] = 0.0
        spoil(cache, cached)
        check_attn(q, kn, vn, cache, cached)
    # all values small: the output is as good, relative to them
    q, kn, vn, cache, cached = setup(g, 2, T, Hq, Hk, D, block, [6 * block, 3 * block], dtype, cap=6 * block)
    by = 2.0 ** -70 if dtype == BF else 2.0 ** -12
    cache[3][:] *= by
    spoil(cache, cached)
    check_attn(q, kn, vn * by, cache, cached)


@BOTH
@FORMS
def test_large_values_before_rows_of_16_bits(T, Hq, Hk, D, block, lens, dtype):
    # rows of 16 bits have no scale, so theirs says nothing about their values beside those of blocks
    print("large values", T, Hq, Hk, D, block, lens, dtype, flush=True)
    g = gen(23)
    for by in (2.0 ** 70, 2.0 ** 100) if dtype == BF else (2.0 ** 9,):
        q, kn, vn, cache, cached = setup(g, 2, T, Hq, Hk, D, block, [4 * block + 11, 2 * block], dtype, cap=5 * block)
        cache[3][:] *= by
        cache[5][:] *= by
        check_attn(q, kn, vn * by, cache, cached)
        cache[3][:, :, 1] = by                                        # with the last block's scale, and one that a row of 16 bits has by itself
        cache[3][:, :, 2:] = 1.0
        check_attn(q, kn, vn * by, cache, cached)


@BOTH
@pytest.mark.parametrize("T,Hq,Hk,D", [(3, 4, 2, 64), (20, 4, 2, 128), (100, 2, 1, 128)])
def test_rows_that_see_nothing(T, Hq, Hk, D, dtype):
    g = gen(14)
    q, kn, vn, cache, cached = setup(g, 2, T, Hq, Hk, D, 32, [0, 0], dtype, cap=64)
    _, tree = tree_of(g, 2, T)
    tree[0, 1] = 0
    tree[1] = 0
    out, lse = check_attn(q, kn, vn, cache, cached, tree=tree)
    assert bool((out[1] == 0).all()) and bool((lse[1] == -INF).all()) and bool((out[0, 1] == 0).all())
    # with cached rows they see these
    cached = ints([40, 32])
    cache = spoil(ref.make_cache(g, 2, 64, Hk, D, 32, dtype), cached)
    check_attn(q, kn, vn, cache, cached, tree=tree)


@BOTH
@pytest.mark.parametrize("T,Hq,Hk,D,block", [(1, 6, 3, 64, 32), (1, 5, 5, 128, 64), (8, 14, 7, 64, 64), (70, 6, 3, 64, 128), (65, 10, 5, 128, 32)])
def test_head_counts_lengths_out_of_range_and_hints(T, Hq, Hk, D, block, dtype):
    print("lengths", T, Hq, Hk, D, block, dtype, flush=True)
    g = gen(15)
    cap = 6 * block
    lens = [cap, cap + 100, -5, cap - 1, 1]
    q, kn, vn, cache, cached = setup(g, 5, T, Hq, Hk, D, block, lens, dtype, cap=cap)
    drafted = ints([T, T + 9, T, 0, -3])
    check_attn(q, kn, vn, cache, cached, drafted=drafted)
    for hint in (1, block, cap, 10 * cap):                            # a hint changes the cut alone
        check_attn(q, kn, vn, cache, cached, drafted=drafted, got=run_attn(q, kn, vn, cache, cached, drafted=drafted, max_cached=hint))


@BOTH
@pytest.mark.parametrize("B,T,Hq,Hk,D", [(100, 1, 8, 2, 128), (66, 3, 4, 1, 64), (130, 40, 2, 1, 64)])
def test_many_sequences_of_uneven_length(B, T, Hq, Hk, D, dtype):
    g = gen(16)
    lens = [(37 * i) % 1500 for i in range(B)]
    q, kn, vn, cache, cached = setup(g, B, T, Hq, Hk, D, 64, lens, dtype)
    check_attn(q, kn, vn, cache, cached)


@BOTH
def test_strides_and_layouts(dtype):
    g = gen(17)
    for T, Hq, Hk, D, block in ((1, 8, 2, 128, 64), (5, 4, 4, 64, 32), (30, 8, 2, 64, 64), (50, 8, 2, 128, 32)):
        lens = [5 * block + 7, 2 * block]
        q, kn, vn, cache, cached = setup(g, 2, T, Hq, Hk, D, block, lens, dtype)
        want = run_attn(q, kn, vn, cache, cached)

        def heads_first(x):                                           # [B, H, rows, D] in memory
            return x.transpose(1, 2).contiguous().transpose(1, 2)

        def padded(x):                                                # rows and tokens further apart
            big = torch.zeros((x.shape[0], x.shape[1] + 3, x.shape[2] + 1, x.shape[3] + 16), dtype=x.dtype, device="cuda")
            v = big[:, : x.shape[1], : x.shape[2], : x.shape[3]]
            v.view(torch.uint8).copy_(x.view(torch.uint8)) if x.dtype == E4M3 else v.copy_(x)
            return v
        for f in (heads_first, padded):
            def e4m3(x):
                return f(x.view(torch.uint8)).view(E4M3) if f is heads_first else f(x)
            k, v, ks, vs, kt, vt = cache
            other = (e4m3(k), e4m3(v), ks, vs, f(kt), f(vt))
            got = run_attn(f(q), f(kn), f(vn), other, cached)
            assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])
            out = f(torch.zeros_like(q))
            ds.dep_tree_attn8(q, kn, vn, *cache, cached, out)
            torch.cuda.synchronize()
            assert torch.equal(out, want[0])


def far_apart(x, batch_stride):
    """x [B, ..] as 8-bit numbers whose sequences lie `batch_stride` bytes apart."""
    room = torch.empty(batch_stride * (x.shape[0] - 1) + x[0].numel(), dtype=torch.uint8, device="cuda")
    v = room.as_strided(x.shape, (batch_stride, *x.stride()[1:]))
    v.copy_(x.view(torch.uint8))
    return v.view(E4M3)


@pytest.mark.parametrize("T", [1, 80])
def test_offsets_past_32_bits(T):
    g = gen(18)
    q, kn, vn, cache, cached = setup(g, 2, T, 4, 2, 128, 64, [700, 640], BF)
    want = run_attn(q, kn, vn, cache, cached)
    k, v, ks, vs, kt, vt = cache
    other = (far_apart(k, (1 << 32) + 4096), far_apart(v, (1 << 32) + 4096), ks, vs, kt, vt)
    got = run_attn(q, kn, vn, other, cached)
    assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])
    fresh, n = normal(g, (2, 60, 2, 128), BF), ints([0, 0])
    before = [t.clone() for t in (ks, vs, kt, vt)]
    ds.dep_cache_append8(fresh, fresh, *other, cached, n)
    for t, b in zip((ks, vs, kt, vt), before):
        t_new, t_old = t.clone(), b
        t.copy_(t_old)
        b.copy_(t_new)
    near = (k, v, ks, vs, kt, vt)
    ds.dep_cache_append8(fresh, fresh, *near, cached, n)
    torch.cuda.synchronize()
    assert same(other[0], k) and same(other[1], v) and all(same(t, b) for t, b in zip((ks, vs, kt, vt), before))


def test_rows_far_apart_in_one_sequence():
    # a token stride of 8 MiB: rows of one sequence past 32 bits
    g = gen(19)
    q, kn, vn, cache, cached = setup(g, 1, 1, 2, 1, 64, 32, [640], BF)
    k, v, ks, vs, kt, vt = cache
    room = torch.empty((640 << 23) + 64, dtype=torch.uint8, device="cuda")
    far = room.as_strided(k.shape, (0, 1 << 23, 64, 1))
    far.copy_(k.view(torch.uint8))
    got = run_attn(q, kn, vn, (far.view(E4M3), far.view(E4M3), ks, vs, kt, vt), cached)
    want = run_attn(q, kn, vn, (k, k, ks, vs, kt, vt), cached)
    assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])


# ---- append ----------------------------------------------------------------------------------------------------------------------------

def test_append_lengths_out_of_range():
    g = gen(21)
    B, T, Hk, D, block, cap = 6, 9, 2, 64, 32, 96
    cache = ref.make_cache(g, B, cap, Hk, D, block, BF)
    kn, vn = normal(g, (B, T, Hk, D), BF), normal(g, (B, T, Hk, D), BF)
    accepted = torch.randint(-4, T + 5, (B, 40), generator=g, device="cuda").int()
    check_append(kn, vn, cache, ints([-3, 96, 95, 200, 70, 0]), accepted, ints([40, 5, 99, 40, 31, -2]))


def test_append_strides():
    g = gen(22)
    B, T, Hk, D, block, cap = 2, 70, 3, 128, 32, 160
    cache = ref.make_cache(g, B, cap, Hk, D, block, FP)
    qkv = normal(g, (B, T, 9 * D), FP)
    kn, vn = qkv[:, :, 3 * D: 6 * D].view(B, T, Hk, D), qkv[:, :, 6 * D:].view(B, T, Hk, D)
    k, v, ks, vs, kt, vt = cache
    flip = lambda x: x.transpose(1, 2).contiguous().transpose(1, 2)
    other = (flip(k.view(torch.uint8)).view(E4M3), flip(v.view(torch.uint8)).view(E4M3), ks.clone(), vs.clone(), flip(kt), flip(vt))
    check_append(kn, vn, cache, ints([20, 63]))
    check_append(kn, vn, other, ints([20, 63]))
    assert all(same(a, b) for a, b in zip(cache, other))


# ---- verification -----------------------------------------------------------------------------------------------------------------------

@pytest.mark.parametrize("V", [1000, 20000])
@pytest.mark.parametrize("drawn", [True, False], ids=["drawn", "likely"])
def test_verification_of_odd_numbers(V, drawn):
    print("odd numbers", V, drawn, flush=True)
    g = gen(31)
    B, T = 12, 10
    p, q = probabilities(g, B, T, V)
    p[0, :, ::3], p[0, :, 1::3] = NAN, INF                           # these count for nothing
    p[1] = -p[1]
    p[2] = 0.0
    p[3] = 0.0
    p[3, :, V - 1] = 1.0
    p[4] *= 3.0                                                      # not a distribution, but numbers all the same
    q[5], q[6, :, ::2] = 0.0, NAN
    p[7] = q[7]                                                      # nothing is ever left
    p[8] = 0.0
    p[8, :, 0] = 1e-38
    parents, _ = tree_of(g, B, T)
    ids = torch.multinomial(torch.ones((B * T, V), device="cuda"), 1, generator=g).view(B, T).int()
    ids[:, 1::2] = p.nan_to_num(0, 0, 0).argmax(-1)[torch.arange(B, device="cuda")[:, None], parents.clamp(min=0)][:, 1::2].int()
    ids[9, 1:], ids[10, 1::2], ids[10, 2::2] = 3, -1, V              # the same token again and again; tokens that there are not
    words = parents.int().contiguous()
    words[11] = torch.tensor([-1, 5, 0, 2, 4, 100, -7, 2, 2 ** 31 - 1, 3], device="cuda")
    u = torch.rand((B, T), generator=g, device="cuda")
    for value in (None, 0.0, 1 - 2.0 ** -24, 1.0, 7.0, -1.0, NAN):
        v = u if value is None else torch.full_like(u, value)
        check_verify(p, ids, v, q if drawn else None, words)
        check_verify(p, ids, v, q if drawn else None, words[4].contiguous())   # one tree for all
        check_verify(p, ids, v, q if drawn else None)


@pytest.mark.parametrize("T,V", [(400, 700), (320, 17000), (1000, 300), (4096, 16400)])
@pytest.mark.parametrize("drawn", [True, False], ids=["drawn", "likely"])
def test_verification_of_hundreds_of_children(T, V, drawn):
    g = gen(32)
    p, q = probabilities(g, 2, T, V, spread=0.5)
    parents = torch.zeros((2, T), dtype=torch.int32, device="cuda")
    parents[:, 0] = -1
    parents[1, T // 2:] = T // 2 - 1
    ids = torch.randint(0, V, (2, T), generator=g, device="cuda").int()
    for u0 in (0.1, 0.999):
        u = torch.full((2, T), 0.9999, device="cuda")
        u[:, 0] = u0
        u[1, T // 2 - 1] = 0.0
        check_verify(p, ids, u, q if drawn else None, parents)


def test_verification_of_strided_rows():
    g = gen(33)
    B, T, V = 3, 5, 33000
    p, q = probabilities(g, B, T, V + 7)
    ids = torch.randint(0, V, (B, T), generator=g, device="cuda").int()
    u = torch.rand((B, T), generator=g, device="cuda")
    check_verify(p[:, :, :V], ids, u, q[:, :, 5: V + 5])
    check_verify(p[:1, :, :V].expand(B, T, V), ids, u, q[:, :1, :V].expand(B, T, V))
    check_verify(p.transpose(0, 1).contiguous().transpose(0, 1)[:, :, :V], ids, u)


def test_verification_past_32_bits():
    T, V = 70, 1 << 24
    p = torch.zeros((1, T, V), device="cuda")                         # 4.7 GB
    p[0, :, V - 3], p[0, :, 17] = 0.75, 0.25
    ids = torch.full((1, T), V - 3, dtype=torch.int32, device="cuda")
    u = torch.full((1, T), 0.5, device="cuda")
    u[0, 69] = 0.8
    u[0, 0] = 0.3
    acc, n, nxt = ids.clone(), ints([0]), ints([0])
    ds.dep_verify_drafts(p, ids, u, acc, n, nxt)
    torch.cuda.synchronize()
    assert n.item() == 69 and nxt.item() == 17 and acc[0, :69].tolist() == list(range(69))


def test_tokens_that_stay_follow_the_targets_probabilities():
    # 40000 sequences of one distribution each: the first token behind the root, accepted or drawn, has the target's frequencies, off by 5 standard deviations at most
    g = gen(34)
    n, V = 40000, 8
    p1, q1 = probabilities(g, 1, 1, V, spread=1.0, near=1.5)
    p, q = p1.expand(n, 4, V), q1.expand(n, 4, V)
    for drawn in (True, False):
        ids = torch.multinomial(q1.view(1, V).expand(n, V), 4, replacement=True, generator=g).int() if drawn else torch.tensor([0, 5, 2, 5], dtype=torch.int32, device="cuda").expand(n, 4).contiguous()
        u = torch.rand((n, 4), generator=g, device="cuda")
        parents = ints([-1, 0, 0, 0])
        acc, cnt, nxt = torch.zeros((n, 4), dtype=torch.int32, device="cuda"), torch.zeros(n, dtype=torch.int32, device="cuda"), torch.zeros(n, dtype=torch.int32, device="cuda")
        ds.dep_verify_drafts(p, ids, u, acc, cnt, nxt, q=q if drawn else None, parents=parents)
        torch.cuda.synchronize()
        first = torch.where(cnt > 1, ids.gather(1, acc[:, 1:2].long())[:, 0], nxt)
        f = torch.bincount(first.long(), minlength=V).double().cpu() / n
        want = p1.view(V).double().cpu()
        assert bool(((f - want).abs() <= 5 * (want * (1 - want) / n).sqrt()).all()), (f, want)
        stays = float((cnt > 1).double().mean())
        if not drawn:                                                # a child of tokens 5 and 2 stays as often as the target has them
            w = float(want[5] + want[2])
            assert abs(stays - w) <= 5 * math.sqrt(w * (1 - w) / n)
        assert 0.0 < stays < 1.0


# ---- norm and rotation ---------------------------------------------------------------------------------------------------------------

def test_norm_of_rows_past_32_bits():
    g = gen(41)
    room = torch.empty((1 << 31) + (1 << 20), dtype=BF, device="cuda")
    q = room.as_strided((2, 3, 4, 64), (1 << 31, 256, 64, 1))
    x = normal(g, (2, 3, 4, 64), BF)
    q.copy_(x)
    freq, k = ds.rope_frequencies(angles_of(64), "cuda"), normal(g, (2, 3, 1, 64), BF)
    want, tol = ref.norm_rope(x, angles_of(64))
    ds.dep_qk_norm_rope(q, k, freq)
    torch.cuda.synchronize()
    check_norm(x, q, want, tol, "q")


@BOTH
def test_norm_of_many_tokens(dtype):
    # several waves to a token, the last with heads that are not there
    g = gen(42)
    for B, T, Hq, Hk, D in ((2, 2000, 39, 3, 128), (1, 5000, 34, 17, 64)):
        q, k = normal(g, (B, T, Hq, D), dtype), normal(g, (B, T, Hk, D), dtype)
        gain, start = torch.randn(D, generator=g, device="cuda"), torch.randint(0, 9000, (B,), generator=g, device="cuda").int()
        qo, ko = torch.empty_like(q), torch.empty_like(k)
        ds.dep_qk_norm_rope(q, k, ds.rope_frequencies(angles_of(D), "cuda"), gain, None, qo, ko, start=start)
        torch.cuda.synchronize()
        for x, y, w in ((q, qo, gain), (k, ko, None)):
            check_norm(x, y, *ref.norm_rope(x, angles_of(D), w, start), (B, T))


@BOTH
@pytest.mark.parametrize("interleaved", [False, True])
def test_numbers_behind_the_rotated_ones_are_no_pairs(interleaved, dtype):
    g = gen(43)
    x = normal(g, (1, 2, 3, 64), dtype)
    x[0, 1, 1, 40], x[0, 1, 2, 63], x[0, 0, 0, 33] = INF, NAN, -INF
    y, z = torch.empty_like(x), torch.empty_like(x)
    ds.dep_qk_norm_rope(x, x.clone(), ds.rope_frequencies(angles_of(32), "cuda"), q_out=y, k_out=z, norm=False, interleaved=interleaved)
    torch.cuda.synchronize()
    assert same(y[..., 32:], x[..., 32:]) and same(y, z) and bool(y[..., :32].isfinite().all())


# ---- streams, graphs, whole rounds --------------------------------------------------------------------------------------------------

class Round:
    """One round of a serving loop with buffers of its own: norm and rotation, attention, verification, append."""

    def __init__(self, seed, B, T, Hq, Hk, D, block, cap, V, lens, dtype=BF):
        g = gen(seed)
        self.T, self.sizes = T, (B, T, Hq, Hk, D)
        self.qkv = normal(g, (B, T, (Hq + 2 * Hk) * D), dtype, 2.0)
        self.q, self.k, self.v = (self.qkv[:, :, a * D: b * D].view(B, T, b - a, D) for a, b in ((0, Hq), (Hq, Hq + Hk), (Hq + Hk, Hq + 2 * Hk)))
        self.gain = 1 + 0.1 * torch.randn(D, generator=g, device="cuda")
        self.angles = angles_of(D)
        self.freq = ds.rope_frequencies(self.angles, "cuda")
        self.cached = ints(lens)
        self.cache = spoil(ref.make_cache(g, B, cap, Hk, D, block, dtype), self.cached)
        self.parents, self.tree = tree_of(g, B, T)
        self.depth = (sum((self.tree[:, :, 0] >> j) & 1 for j in range(T)) - 1).int()   # (64 tokens at most)
        self.parents = self.parents.int().contiguous()
        self.p, self.qprob = probabilities(g, B, T, V)
        self.ids = drawn_ids(g, self.qprob, self.parents.long())
        self.u = torch.rand((B, T), generator=g, device="cuda")
        self.out, self.lse = torch.zeros_like(self.q, memory_format=torch.contiguous_format), torch.zeros((B, T, Hq), device="cuda")
        self.accepted = torch.zeros((B, T), dtype=torch.int32, device="cuda")
        self.n, self.next, self.cached_out, self.n_out = (torch.zeros(B, dtype=torch.int32, device="cuda") for _ in range(4))
        normed = torch.zeros_like(self.qkv)                          # (rows as far apart as the values')
        self.q2, self.k2 = normed[:, :, : Hq * D].view(B, T, Hq, D), normed[:, :, Hq * D: (Hq + Hk) * D].view(B, T, Hk, D)
        self.work = torch.empty(ds.tree_attn8_workspace(self.q2, self.k2, self.v, *self.cache, self.cached, self.out), dtype=torch.uint8, device="cuda")
        self.vwork = torch.empty(max(16, ds.verify_drafts_workspace(self.p, self.ids, self.u, self.accepted, self.n, self.next, self.qprob, self.parents)), dtype=torch.uint8, device="cuda")

    def run(self, stream=None):
        ds.dep_qk_norm_rope(self.q, self.k, self.freq, self.gain, self.gain, self.q2, self.k2, start=self.cached, depth=self.depth, stream=stream)
        ds.dep_tree_attn8(self.q2, self.k2, self.v, *self.cache, self.cached, self.out, lse=self.lse, tree=self.tree, workspace=self.work if self.work.numel() else None, stream=stream)
        ds.dep_verify_drafts(self.p, self.ids, self.u, self.accepted, self.n, self.next, q=self.qprob, parents=self.parents, workspace=self.vwork, stream=stream)
        ds.dep_cache_append8(self.k2, self.v, *self.cache, self.cached, self.cached_out, accepted=self.accepted, n_accepted=self.n, n_out=self.n_out, stream=stream)

    def results(self):
        return [t.clone() for t in (self.q2, self.k2, self.out, self.lse, self.n, self.next, self.cached_out, self.n_out, *self.cache)]

    def check(self, cache_before, cached_before):
        """The round that has run, against the 64-bit forms; each step on what the one before gave."""
        check_norm(self.q, self.q2, *ref.norm_rope(self.q, self.angles, self.gain, cached_before, self.depth), "q")
        check_norm(self.k, self.k2, *ref.norm_rope(self.k, self.angles, self.gain, cached_before, self.depth), "k")
        check_attn(self.q2, self.k2, self.v, cache_before, cached_before, tree=self.tree, got=(self.out, self.lse))
        want = ref.verify(self.p, self.ids, self.u, self.qprob, self.parents.cpu())
        n = self.n.tolist()
        assert [(self.accepted[b, : n[b]].tolist(), self.next[b].item()) for b in range(len(n))] == want
        w = ref.append8(self.k2, self.v, *cache_before, cached_before.cpu(), self.accepted.cpu(), self.n.cpu())
        for got, x in zip(self.cache[:2], w[:2]):
            assert torch.equal(got.cpu().double().nan_to_num(9e9), x.nan_to_num(9e9))
        for got, x in zip(self.cache[2:], w[2:6]):
            assert torch.equal(got.cpu().double().nan_to_num(9e9), x.double().nan_to_num(9e9))
        assert torch.equal(self.cached_out.cpu(), w[6]) and torch.equal(self.n_out.cpu(), w[7])


SHAPES = [(3, 13, 8, 2, 128, 32, 512, 3000, [300, 31, 0]), (2, 40, 6, 2, 64, 64, 1024, 20000, [700, 63]), (4, 1, 16, 2, 128, 64, 512, 50257, [256, 255, 1, 400])]


@pytest.mark.parametrize("shape", SHAPES)
def test_rounds_one_after_another(shape):
    r = Round(51, *shape)
    for step in range(4):
        before = [t.clone() for t in r.cache]
        cached = r.cached.clone()
        r.run()
        torch.cuda.synchronize()
        r.check(before, cached)
        g = gen(100 + step)
        r.cached.copy_(r.cached_out)
        r.qkv.copy_(normal(g, r.qkv.shape, r.qkv.dtype, 2.0))
        r.u.copy_(torch.rand(r.u.shape, generator=g, device="cuda"))


@pytest.mark.parametrize("shape", SHAPES)
def test_a_captured_round_replayed(shape):
    print("graph", shape, flush=True)
    a, b = Round(52, *shape), Round(52, *shape)
    a.run()                                                          # (loads what is loaded once)
    torch.cuda.synchronize()
    a = Round(52, *shape)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        a.run()
    torch.cuda.synchronize()
    for step in range(5):
        g = gen(200 + step)
        x = normal(g, a.qkv.shape, a.qkv.dtype, 2.0)
        u = torch.rand(a.u.shape, generator=g, device="cuda")
        for r in (a, b):
            r.qkv.copy_(x)
            r.u.copy_(u)
        graph.replay()
        if step % 2:
            torch.cuda.synchronize()
        b.run()
        torch.cuda.synchronize()
        for got, want in zip(a.results(), b.results()):
            assert same(got, want), step
        for r in (a, b):                                             # lengths that the graph has not seen
            r.cached.copy_(r.cached_out)


def test_two_rounds_at_once():
    # on two streams with workspaces of their own; and two captured rounds replayed at once
    shapes = SHAPES[0], SHAPES[1]
    want = []
    for i, s in enumerate(shapes):
        r = Round(60 + i, *s)
        r.run()
        torch.cuda.synchronize()
        want.append(r.results())
    for captured in (False, True):
        rounds = [Round(60 + i, *s) for i, s in enumerate(shapes)]
        torch.cuda.synchronize()
        streams = [torch.cuda.Stream() for _ in rounds]
        graphs = []
        if captured:
            for r in rounds:
                graphs.append(torch.cuda.CUDAGraph())
                with torch.cuda.graph(graphs[-1]):
                    r.run()
            torch.cuda.synchronize()
        for i, (r, s) in enumerate(zip(rounds, streams)):
            if captured:
                with torch.cuda.stream(s):
                    graphs[i].replay()
            else:
                r.run(s)
        torch.cuda.synchronize()
        for r, w in zip(rounds, want):
            assert all(same(x, y) for x, y in zip(r.results(), w))


def test_calls_follow_torchs_current_stream():
    r = Round(70, *SHAPES[0])
    want = Round(70, *SHAPES[0])
    want.run()
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    x = r.qkv.clone()
    r.qkv.zero_()
    torch.cuda.synchronize()
    with torch.cuda.stream(s):
        torch.cuda._sleep(20_000_000)                                # (the copy below is late: a call on another stream would not see it)
        r.qkv.copy_(x)
        r.run()
    torch.cuda.synchronize()
    assert all(same(a, b) for a, b in zip(r.results(), want.results()))


# ---- refusals of the binding --------------------------------------------------------------------------------------------------------

def test_refusals_of_the_binding():
    g = gen(80)
    q, kn, vn, cache, cached = setup(g, 2, 3, 4, 2, 128, 32, [40, 50], BF, cap=64)
    k, v, ks, vs, kt, vt = cache
    out = torch.zeros_like(q)
    bad = [dict(k_cache=k.view(torch.uint8)), dict(k_cache=k.cpu()), dict(k_cache=k[:, :50], v_cache=v[:, :50]), dict(ks=ks[:, :, :1]), dict(vs=vs.double()), dict(kt=kt[:, :16], vt=vt[:, :16]),
           dict(kt=kt.half()), dict(vt=vt[:, :, :1]), dict(q=q.float()), dict(q=q.half()), dict(cached=cached.long()), dict(out=out[:, :1]), dict(v_cache=v[:1])]
    for kw in bad:
        x = dict(q=q, kn=kn, vn=vn, k_cache=k, v_cache=v, ks=ks, vs=vs, kt=kt, vt=vt, cached=cached, out=out)
        x.update(kw)
        with pytest.raises((ValueError, TypeError)):
            ds.dep_tree_attn8(x["q"], x["kn"], x["vn"], x["k_cache"], x["v_cache"], x["ks"], x["vs"], x["kt"], x["vt"], x["cached"], x["out"])
    with pytest.raises(ValueError):
        ds.dep_tree_attn8(q, kn, vn, None, None, ks, vs, kt, vt, cached, out)
    big = ref.make_cache(g, 1, 64000, 2, 128, 64, BF)
    args = (q[:1], kn[:1], vn[:1], *big, ints([60000]), out[:1])
    need = ds.tree_attn8_workspace(*args)
    assert need > 0
    for w in (torch.empty(need - 4, dtype=torch.uint8, device="cuda"), torch.empty(need + 16, dtype=torch.uint8, device="cuda")[4:]):
        with pytest.raises(ds.DepsyncError):
            ds.dep_tree_attn8(*args, workspace=w)
    with pytest.raises(ValueError):
        ds.dep_cache_append8(kn, vn, k, v, ks, vs, kt[:, :, :, :64], vt[:, :, :, :64], cached, cached.clone())
    with pytest.raises(ds.DepsyncError):
        ds.dep_cache_append8(kn, vn, k, v, ks, vs, kt, vt, cached, cached)
    freq = ds.rope_frequencies(angles_of(128), "cuda")
    for kw in (dict(freq=freq.int()), dict(freq=freq[:9]), dict(q_gain=torch.ones(64, device="cuda")), dict(k_gain=torch.ones(128, device="cuda").half()), dict(start=cached.long()),
               dict(depth=torch.zeros((2, 4), dtype=torch.int32, device="cuda")), dict(eps=-1.0), dict(q_out=out[:, :2]), dict(freq=torch.cat([freq, freq]))):
        with pytest.raises((ValueError, TypeError, ds.DepsyncError)):
            ds.dep_qk_norm_rope(q, kn, kw.pop("freq", freq), **kw)
    p, qq = probabilities(g, 2, 3, 50)
    ids, u = torch.zeros((2, 3), dtype=torch.int32, device="cuda"), torch.zeros((2, 3), device="cuda")
    acc, n, nxt = ids.clone(), ints([0, 0]), ints([0, 0])
    for x in ((p.half(), ids, u, acc, n, nxt), (p, ids.long(), u, acc, n, nxt), (p, ids, u.double(), acc, n, nxt), (p, ids, u, acc[:, :2], n, nxt), (p.cpu(), ids, u, acc, n, nxt),
              (p.transpose(1, 2), ids, u, acc, n, nxt)):
        with pytest.raises(ValueError):
            ds.dep_verify_drafts(*x)
    with pytest.raises(ValueError):
        ds.dep_verify_drafts(p, ids, u, acc, n, nxt, q=qq[:, :2])
    with pytest.raises(ds.DepsyncError):
        ds.dep_verify_drafts(p, ids, u, acc, n, n)
