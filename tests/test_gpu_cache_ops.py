"""GPU tests of dep_cache_append, dep_cache_weights and dep_cache_evict against plain 64-bit forms (tests/cache_ref.py), and of
the loop that they make with dep_tree_attn."""
import math

import pytest
import torch

import cache_ref as ref
import paper_2305_13450_amd as ds

pytestmark = pytest.mark.gpu
BF, FP = torch.bfloat16, torch.float16


def gen(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return g


def normal(g, shape, dtype, std=1.0):
    return (torch.randn(shape, generator=g, device="cuda") * std).to(dtype)


def ints(v):
    return torch.tensor(v, dtype=torch.int32, device="cuda")


def cache(B, Hk, D, cap, dtype, seed):
    g = gen(seed)
    w = torch.rand((B, Hk, cap), generator=g, device="cuda")
    pos = torch.argsort(torch.rand((B, Hk, cap), generator=g, device="cuda"), -1).int()
    return normal(g, (B, cap, Hk, D), dtype), normal(g, (B, cap, Hk, D), dtype), w, pos


def same(got, want):
    for a, b in zip(got, want):
        a, b = a.cpu(), b.cpu()
        assert torch.equal(a.nan_to_num(3), b.nan_to_num(3)) if a.is_floating_point() else torch.equal(a, b)


# ---- append ------------------------------------------------------------------------------------------------------------------

@pytest.mark.parametrize("B,T,A,Hk,D,cap,lens,counts,dtype", [
    (1, 1, 1, 1, 128, 1, [0], [1], BF), (3, 16, 5, 2, 64, 40, [0, 7, 40], [5, 1, 3], FP), (4, 33, 6, 8, 128, 50, [48, 46, 44, 10], [6, 6, 6, 0], BF),
    (2, 8, 3, 3, 128, 20, [-5, 99], [9, 2], BF), (2, 3, 12, 1, 64, 30, [4, 9], [12, 11], BF)])
def test_append_of_accepted_tokens(B, T, A, Hk, D, cap, lens, counts, dtype):
    print("append", B, T, A, Hk, D, cap, flush=True)
    g = gen(1)
    kc, vc, w, pos = cache(B, Hk, D, cap, dtype, 2)
    kn, vn = normal(g, (B, T, Hk, D), dtype), normal(g, (B, T, Hk, D), dtype)
    accepted = torch.randint(-1, T + 1, (B, A), generator=g, device="cuda").int()   # the same token twice and indices outside among them
    cached, n, start, out = ints(lens), ints(counts), ints([100 + b for b in range(B)]), ints([7] * B)
    want = ref.append(kn, vn, kc, vc, cached, w, pos, start, accepted, n)
    ds.dep_cache_append(kn, vn, kc, vc, cached, out, accepted=accepted, n_accepted=n, weights=w, pos=pos, start=start)
    torch.cuda.synchronize()
    same((kc, vc, w, pos, out), want)
    assert cached.tolist() == lens


def test_append_of_a_whole_prompt_with_strides():
    print("append prompt", flush=True)
    B, T, Hk, D, cap = 2, 301, 3, 128, 500
    g = gen(3)
    qkv = normal(g, (B, T, 3 * Hk * D), BF)
    kn, vn = (qkv[..., i * Hk * D: (i + 1) * Hk * D].view(B, T, Hk, D) for i in (1, 2))
    kv = normal(g, (2, Hk, B, cap, D + 8), BF)
    kc, vc = (kv[i, ..., :D].permute(1, 2, 0, 3) for i in (0, 1))
    before = kv.clone()
    w, pos = torch.ones((B, Hk, cap), device="cuda"), torch.zeros((B, Hk, cap), dtype=torch.int32, device="cuda")
    cached, out = ints([0, 150]), ints([0, 0])
    want = ref.append(kn, vn, kc, vc, cached, w, pos, cached)
    ds.dep_cache_append(kn, vn, kc, vc, cached, out, weights=w, pos=pos, start=cached)
    torch.cuda.synchronize()
    same((kc, vc, w, pos, out), want)
    assert torch.equal(kv[..., D:], before[..., D:])
    # neither weights nor positions kept
    kv.copy_(before)
    ds.dep_cache_append(kn, vn, kc, vc, cached, out)
    torch.cuda.synchronize()
    same((kc, vc, out), (want[0], want[1], want[4]))


# ---- weights -----------------------------------------------------------------------------------------------------------------

def near(w, want, tol):
    w = w.cpu().double()
    over = ((w - want).abs() / tol)
    assert torch.isfinite(w[torch.isfinite(want)]).all() and float(over[torch.isfinite(want)].max()) <= 1.0, f"{float(over.max()):.3f} of the tolerance"


@pytest.mark.parametrize("dtype", [BF, FP], ids=["bf16", "fp16"])
@pytest.mark.parametrize("B,T,A,Hq,Hk,D,lens,counts", [
    (1, 1, None, 1, 1, 128, [1], None), (3, 16, 5, 8, 2, 64, [31, 128, 200], [5, 1, 0]), (2, 8, 4, 16, 1, 128, [127, 129], [4, 3]),
    (4, 12, 3, 6, 6, 128, [0, 2, 700, 33], [1, 3, 2, 3]), (2, 70, None, 4, 2, 64, [70, 333], None), (1, 300, None, 3, 1, 128, [300], None),
    (2, 65, None, 1, 1, 128, [300, 64], [65, 20]), (1, 700, None, 12, 12, 128, [1500], None),
    (2, 90, 60, 4, 2, 64, [500, 61], [60, 33]), (3, 50, 40, 8, 2, 128, [40, 900, 0], [40, 7, 40]), (40, 80, None, 2, 1, 128, [2100] * 40, None)])
def test_weights(B, T, A, Hq, Hk, D, lens, counts, dtype):
    print("weights", B, T, A, Hq, Hk, D, lens, dtype, flush=True)
    g = gen(4)
    cap = max(lens) + 5
    kc, _, w, _ = cache(B, Hk, D, cap, dtype, 5)
    kc[:, max(lens):] = float("nan")
    q = normal(g, (B, T, Hq, D), dtype, 2.0)
    lse = 4.0 + torch.rand((B, T, Hq), generator=g, device="cuda")
    lse[0, 0, 0] = -math.inf                                # a row that saw nothing
    accepted = None if A is None else torch.randint(0, T, (B, A), generator=g, device="cuda").int()
    cached, n = ints(lens), None if counts is None else ints(counts)
    want, tol = ref.add_weights(q, lse, kc, cached, w, accepted, n)
    w0 = w.clone()
    ds.dep_cache_weights(q, lse, kc, cached, w, accepted=accepted, n_accepted=n)
    torch.cuda.synchronize()
    near(w, want, tol)
    for b in range(B):
        assert torch.equal(w[b, :, lens[b]:], w0[b, :, lens[b]:])
    for hint in (1, 64, 200):
        again = w0.clone()
        ds.dep_cache_weights(q, lse, kc, cached, again, accepted=accepted, n_accepted=n, max_cached=hint)
        near(again, want, tol)


def test_weights_of_more_accepted_than_cached():
    # the first of five tokens have no row of their own in a cache of three, and see nothing; the last sees row 2 and before
    g = gen(6)
    kc, _, w, _ = cache(1, 1, 128, 9, BF, 7)
    q, lse = normal(g, (1, 5, 2, 128), BF), torch.full((1, 5, 2), 2.0, device="cuda")
    want, tol = ref.add_weights(q, lse, kc, ints([3]), w)
    ds.dep_cache_weights(q, lse, kc, ints([3]), w)
    torch.cuda.synchronize()
    near(w, want, tol)


# ---- evict -------------------------------------------------------------------------------------------------------------------

CASES = [
    # B, Hk, D, cap, lens, budget, recent
    (1, 1, 128, 1, [1], 1, 0), (3, 2, 64, 70, [0, 33, 70], 32, 8), (2, 4, 128, 300, [300, 299], 298, 1), (4, 1, 128, 200, [64, 65, 1, 200], 64, 64),
    (2, 3, 64, 5000, [4999, 2100], 2048, 100), (1, 2, 128, 33000, [33000], 1500, 300), (2, 2, 128, 9000, [9000, 4097], 1, 1), (2, 2, 64, 50, [-1, 70], 20, 0),
]


@pytest.mark.parametrize("B,Hk,D,cap,lens,budget,recent", CASES)
def test_evict(B, Hk, D, cap, lens, budget, recent):
    print("evict", B, Hk, D, cap, lens, budget, recent, flush=True)
    kc, vc, w, pos = cache(B, Hk, D, cap, BF, 8)
    w[..., ::3] = 0.0                                       # many equal weights, two signs of nothing, and what orders badly
    w[..., 1::17] = -0.0
    if cap > 10:
        w[..., 3], w[..., 5], w[..., 7], w[..., 9] = float("nan"), float("inf"), float("-inf"), 1e-42
    cached, out = ints(lens), ints([9] * B)
    want = ref.evict(kc, vc, w, pos, cached, budget, recent)
    other = [torch.full((B, budget + 3, Hk, D), 2.0, dtype=BF, device="cuda") for _ in range(2)] + \
            [torch.full((B, Hk, budget + 3), 2.0, device="cuda"), torch.full((B, Hk, budget + 3), 2, dtype=torch.int32, device="cuda")]
    want_other = ref.evict(kc, vc, w, pos, cached, budget, recent, other)
    before = [t.clone() for t in (kc, vc, w, pos)]
    ds.dep_cache_evict(kc, vc, w, pos, cached, out, budget, recent, k_out=other[0], v_out=other[1], weights_out=other[2], pos_out=other[3])
    torch.cuda.synchronize()
    same((*other, out), want_other)
    same((kc, vc, w, pos), before)
    out.fill_(9)
    ds.dep_cache_evict(kc, vc, w, pos, cached, out, budget, recent, max_cached=min(cap, budget + 7))
    torch.cuda.synchronize()
    same((kc, vc, w, pos, out), want)


def test_evict_with_equal_positions_and_strides():
    B, Hk, D, cap, budget = 2, 3, 128, 90, 40
    kv = normal(gen(9), (2, Hk, B, cap, D + 8), FP)
    kc, vc = (kv[i, ..., :D].permute(1, 2, 0, 3) for i in (0, 1))
    w, pos = torch.zeros((B, Hk, cap), device="cuda"), torch.zeros((B, Hk, cap), dtype=torch.int32, device="cuda")
    pos[1, :, 50:] = 2 ** 31 - 1                             # more rows at the newest position than are kept
    cached, out = ints([90, 90]), ints([0, 0])
    want = ref.evict(kc, vc, w, pos, cached, budget, 10)
    edge = kv[..., D:].clone()
    ds.dep_cache_evict(kc, vc, w, pos, cached, out, budget, 10)
    torch.cuda.synchronize()
    same((kc, vc, w, pos, out), want)
    assert torch.equal(kv[..., D:], edge)


def test_offsets_past_32_bits():
    # rows 4 MiB apart: the last ones lie behind 4 GiB
    print("offsets past 32 bits", flush=True)
    rows, pitch, Hk, D = 1200, 1 << 21, 2, 128
    buf = torch.zeros(rows * pitch, dtype=BF, device="cuda")
    kc, vc = (buf.as_strided((1, rows, Hk, D), (0, pitch, D, 1), at) for at in (0, 4096))
    g = gen(30)
    kc.copy_(normal(g, kc.shape, BF))
    vc.copy_(normal(g, vc.shape, BF))
    w, pos = torch.rand((1, Hk, rows), generator=g, device="cuda"), torch.arange(rows, device="cuda").int().expand(1, Hk, rows).contiguous()
    kn, vn = normal(g, (1, 40, Hk, D), BF), normal(g, (1, 40, Hk, D), BF)
    cached, mid, out = ints([rows - 40]), ints([0]), ints([0])
    want = ref.append(kn, vn, kc, vc, cached, w, pos, cached)
    ds.dep_cache_append(kn, vn, kc, vc, cached, mid, weights=w, pos=pos, start=cached)
    torch.cuda.synchronize()
    same((kc, vc, w, pos, mid), want)
    for T in (3, 40):
        q, lse = normal(g, (1, T, 4, D), BF, 2.0), torch.full((1, T, 4), 8.0, device="cuda")
        want_w, tol = ref.add_weights(q, lse, kc, mid, w)
        ds.dep_cache_weights(q, lse, kc, mid, w)
        torch.cuda.synchronize()
        near(w, want_w, tol)
    for budget in (rows - 5, 600):                          # a few rows one by one, many through the list
        want = ref.evict(kc, vc, w, pos, mid, budget, 50)
        ds.dep_cache_evict(kc, vc, w, pos, mid, out, budget, 50)
        torch.cuda.synchronize()
        same((kc, vc, w, pos, out), want)


def test_calls_at_once_on_two_streams():
    print("two streams", flush=True)
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    jobs = []
    for k, (cap, lens, budget) in enumerate(((3000, [3000, 2500], 1000), (300, [300, 290], 297))):
        t = cache(2, 4, 128, cap, BF, 40 + k)
        cached = ints(lens)
        jobs.append((t, cached, budget, ref.evict(*t, cached, budget, 20), ints([0, 0])))
    torch.cuda.synchronize()
    for (t, cached, budget, _, out), s in zip(jobs, streams):
        ds.dep_cache_evict(*t, cached, out, budget, 20, stream=s)
    torch.cuda.synchronize()
    for t, _, _, want, out in jobs:
        same((*t, out), want)


# ---- the loop ----------------------------------------------------------------------------------------------------------------

def step(state, t, tree, accepted, n, budget, recent, stream=None):
    """One round of a serving program: attention, append, weights, eviction."""
    k, v, w, pos, cached, mid, start = state
    ds.dep_tree_attn(t["q"], t["k"], t["v"], k, v, cached, t["out"], lse=t["lse"], tree=tree, stream=stream)
    ds.dep_cache_append(t["k"], t["v"], k, v, cached, mid, accepted=accepted, n_accepted=n, weights=w, pos=pos, start=start, stream=stream)
    ds.dep_cache_weights(t["q"], t["lse"], k, mid, w, accepted=accepted, n_accepted=n, stream=stream)
    ds.dep_cache_evict(k, v, w, pos, mid, cached, budget, recent, stream=stream)


@pytest.mark.parametrize("graph", [False, True])
def test_rounds_of_drafting_and_eviction(graph):
    print("loop", graph, flush=True)
    B, T, A, Hq, Hk, D, budget, recent, cap = 3, 7, 3, 4, 2, 128, 40, 12, 48
    g = gen(10)
    k, v = torch.zeros((B, cap, Hk, D), dtype=BF, device="cuda"), torch.zeros((B, cap, Hk, D), dtype=BF, device="cuda")
    w, pos = torch.zeros((B, Hk, cap), device="cuda"), torch.zeros((B, Hk, cap), dtype=torch.int32, device="cuda")
    cached, mid, start = ints([0, 0, 0]), ints([0, 0, 0]), ints([0, 0, 0])
    state = (k, v, w, pos, cached, mid, start)
    tree = ds.tree_mask([-1, 0, 0, 1, 1, 3, 2]).cuda()       # paths 0-1-3-5, 0-1-4 and 0-2-6
    t = {"q": torch.empty((B, T, Hq, D), dtype=BF, device="cuda"), "k": torch.empty((B, T, Hk, D), dtype=BF, device="cuda"),
         "v": torch.empty((B, T, Hk, D), dtype=BF, device="cuda"), "out": torch.empty((B, T, Hq, D), dtype=BF, device="cuda"),
         "lse": torch.empty((B, T, Hq), device="cuda")}
    accepted, n = torch.zeros((B, A), dtype=torch.int32, device="cuda"), ints([0, 0, 0])
    cg = None
    if graph:
        cg = torch.cuda.CUDAGraph()
        with torch.cuda.graph(cg):
            step(state, t, tree, accepted, n, budget, recent, stream=torch.cuda.current_stream())
    for it in range(40):
        for name, std in (("q", 2.0), ("k", 1.0), ("v", 1.0)):
            t[name].copy_(normal(g, t[name].shape, BF, std))
        path = [[0, 1, 3], [0, 1, 4], [0, 2, 6]][it % 3]
        accepted.copy_(torch.tensor([path] * B))
        n.copy_(torch.tensor([1 + it % 3, 3, (it * 2) % 4]))
        k0, v0, w0, p0, c0 = k.clone(), v.clone(), w.clone(), pos.clone(), cached.clone()
        torch.cuda.synchronize()
        if graph:
            cg.replay()
        else:
            step(state, t, tree, accepted, n, budget, recent)
        torch.cuda.synchronize()
        # each operator's result against its plain form on what the round began with
        o, l, tol, tol_l = ref.attn(t["q"], t["k"], t["v"], k0, v0, c0, tree)
        assert ((t["out"].cpu().double() - o).abs() <= tol).all() and ((t["lse"].cpu().double() - l).abs() <= tol_l).all()
        k1, v1, w1, p1, c1 = ref.append(t["k"], t["v"], k0, v0, c0, w0, p0, start, accepted, n)
        assert torch.equal(mid.cpu(), c1)
        w2, tol_w = ref.add_weights(t["q"], t["lse"], k1, c1, w1, accepted, n)
        # what was evicted depends on the very weights: the kernel's own are taken, up to their tolerance, where rows stay
        for b in range(B):
            m = int(c1[b])
            assert int(cached[b]) == min(m, budget)
            for h in range(Hk):
                stay = {int(p): i for i, p in enumerate(pos[b, h, : int(cached[b])].tolist())}
                assert len(stay) == int(cached[b])
                rows = {int(p): i for i, p in enumerate(p1[b, h, :m].tolist())}
                for p, i in stay.items():
                    j = rows[p]
                    assert torch.equal(k[b, i, h].cpu(), k1[b, j, h]) and torch.equal(v[b, i, h].cpu(), v1[b, j, h])
                    assert abs(float(w[b, h, i]) - float(w2[b, h, j])) <= float(tol_w[b, h, j])
                gone = [(float(w2[b, h, j]), float(tol_w[b, h, j])) for p, j in rows.items() if p not in stay]
                newest = max(rows, default=0)
                assert all(p in stay for p in rows if p > newest - recent)
                old = [(float(w2[b, h, rows[p]]), float(tol_w[b, h, rows[p]])) for p in stay if p <= newest - recent]
                for x, dx in gone:                            # nothing that went outweighs anything old that stayed
                    assert all(x - dx <= y + dy for y, dy in old)
        start += n


def test_refusals_of_the_binding():
    kc, vc, w, pos = cache(2, 2, 128, 20, BF, 11)
    kn, vn = (normal(gen(12), (2, 4, 2, 128), BF) for _ in range(2))
    cached, out, start = ints([3, 4]), ints([0, 0]), ints([0, 0])
    q, lse = normal(gen(13), (2, 4, 4, 128), BF), torch.zeros((2, 4, 4), device="cuda")

    def refused(status, f, *a, **kw):
        with pytest.raises(ds.DepsyncError) as e:
            f(*a, **kw)
        assert e.value.status == status
    refused(ds.EINVAL, ds.dep_cache_append, kn, vn, kc, vc, cached, cached)                          # in and out are the same
    refused(ds.EINVAL, ds.dep_cache_append, kn, vn, kc, vc, cached, out, pos=pos)                    # positions without a start
    refused(ds.EINVAL, ds.dep_cache_evict, kc, vc, w, pos, cached, out, 0)
    refused(ds.EINVAL, ds.dep_cache_evict, kc, vc, w, pos, cached, out, 4, 5)
    refused(ds.EINVAL, ds.dep_cache_evict, kc, vc, w, pos, cached, cached, 4)
    refused(ds.EINVAL, ds.dep_cache_evict, kc, vc, w, pos, cached, out, 4, k_out=kc[:, :8].contiguous())   # one of four
    refused(ds.EINVAL, ds.dep_cache_evict, kc, vc, w, pos, cached, out, 9, k_out=kc[:, :8].contiguous(), v_out=vc[:, :8].contiguous(),
            weights_out=w[..., :8].contiguous(), pos_out=pos[..., :8].contiguous())                  # too small
    refused(ds.EINVAL, ds.dep_cache_weights, q, lse, kc, cached, w, scale=-2.0)
    refused(ds.ENOTIMPL, ds.dep_cache_append, *(x[..., :96].contiguous() for x in (kn, vn, kc, vc)), cached, out)
    for f, a in ((ds.dep_cache_append, (kn, vn, kc, vc[:, :7], cached, out)), (ds.dep_cache_append, (kn, vn.half(), kc, vc, cached, out)),
                 (ds.dep_cache_weights, (q, lse[:, :3], kc, cached, w)), (ds.dep_cache_weights, (q, lse, kc, cached, w.double())),
                 (ds.dep_cache_evict, (kc, vc, w, pos.long(), cached, out, 4)), (ds.dep_cache_evict, (kc, vc, w.transpose(0, 1), pos, cached, out, 4))):
        with pytest.raises((ValueError, TypeError)):
            f(*a)
    torch.cuda.synchronize()


@pytest.mark.parametrize("D", [64, 128])
def test_weights_of_many_sequences(D):
    print("weights of many sequences", D, flush=True)
    B, T, A, Hq, Hk = 33, 80, 70, 16, 8
    lens, counts = [(37 * i) % 141 for i in range(B)], [A - i % 3 * 30 for i in range(B)]
    g = gen(31)
    kc, _, w, _ = cache(B, Hk, D, 145, BF, 32)
    kc[:, max(lens):] = float("nan")
    q, lse = normal(g, (B, T, Hq, D), BF, 2.0), 4.0 + torch.rand((B, T, Hq), generator=g, device="cuda")
    accepted, cached, n = torch.randint(0, T, (B, A), generator=g, device="cuda").int(), ints(lens), ints(counts)
    want, tol = ref.add_weights(q, lse, kc, cached, w, accepted, n)
    w0 = w.clone()
    ds.dep_cache_weights(q, lse, kc, cached, w, accepted=accepted, n_accepted=n)
    torch.cuda.synchronize()
    near(w, want, tol)
    for b in range(B):
        assert torch.equal(w[b, :, lens[b]:], w0[b, :, lens[b]:])
