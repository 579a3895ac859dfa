"""GPU tests that nothing behind a sequence's last row is read: what lies there, NaN and infinities, changes no bit of a result."""
import pytest
import torch

import draft_ref
import paper_2305_13450_amd as ds
from test_gpu_draft_ops import BF, FP, INF, NAN, gen, ints, normal, same, tree_of

pytestmark = pytest.mark.gpu
BOTH = pytest.mark.parametrize("dtype", [BF, FP], ids=["bf16", "fp16"])


def behind(x, lens, value):
    """A copy of x [B, rows, H, D] with `value` in every row from lens[b] on."""
    y = x.clone()
    for b, n in enumerate(lens):
        y[b, n:] = value
    return y


# up to 32 rows to a head and more than 64: both forms; every number of rows in a last tile, of cached rows and of drafted tokens
@BOTH
@pytest.mark.parametrize("B,T,Hq,Hk,D", [(64, 7, 4, 2, 128), (100, 4, 4, 1, 64), (40, 40, 4, 1, 128), (36, 70, 2, 1, 64)])
def test_attention_reads_nothing_behind_the_ends(B, T, Hq, Hk, D, dtype):
    print("ends", B, T, Hq, Hk, D, dtype, flush=True)
    g = gen(91)
    lens, drafted = [1 + (5 * b) % 97 for b in range(B)], [1 + b % T for b in range(B)]
    cap = 97
    q, kn, vn = normal(g, (B, T, Hq, D), dtype, 2.0), normal(g, (B, T, Hk, D), dtype), normal(g, (B, T, Hk, D), dtype)
    kc, vc = normal(g, (B, cap, Hk, D), dtype), normal(g, (B, cap, Hk, D), dtype)
    _, tree = tree_of(g, B, T)
    for words in (None, tree):
        got = []
        for value in (0.0, NAN, INF):
            out, lse = torch.zeros_like(q), torch.zeros((B, T, Hq), device="cuda")
            ds.dep_tree_attn(q, behind(kn, drafted, value), behind(vn, drafted, value), behind(kc, lens, value), behind(vc, lens, value), ints(lens), out, lse=lse,
                             tree=words, drafted=ints(drafted))
            torch.cuda.synchronize()
            got.append((out, lse))
        assert bool(got[0][0].isfinite().all())
        for out, lse in got[1:]:
            assert same(out, got[0][0]) and same(lse, got[0][1])


# accepted paths (up to 64 rows to a head) and prompts: the keys' ends, and with rows taken in order the queries'
@BOTH
@pytest.mark.parametrize("B,T,Hq,Hk,D", [(97, 6, 4, 2, 128), (97, 9, 4, 1, 64), (3, 97, 4, 1, 128), (3, 97, 4, 2, 64), (97, 33, 8, 2, 128), (97, 70, 2, 1, 64)])
def test_weights_read_nothing_behind_the_ends(B, T, Hq, Hk, D, dtype):
    print("weights' ends", B, T, Hq, Hk, D, dtype, flush=True)
    g = gen(92)
    cap = 200
    n = [1 + (7 * b) % T for b in range(B)]
    lens = [n[b] + (11 * b) % (cap - T) for b in range(B)]
    q, kc, lse = normal(g, (B, T, Hq, D), dtype, 2.0), normal(g, (B, cap, Hk, D), dtype), 8 + torch.randn((B, T, Hq), generator=g, device="cuda")
    got = []
    for value in (0.0, NAN, INF):
        w = torch.zeros((B, Hk, cap), device="cuda")
        ds.dep_cache_weights(behind(q, n, value), behind(lse.unsqueeze(-1), n, 0.0).squeeze(-1).contiguous(), behind(kc, lens, value), ints(lens), w, n_accepted=ints(n))
        torch.cuda.synchronize()
        got.append(w)
    assert bool(got[0].isfinite().all()) and all(same(w, got[0]) for w in got[1:])
    for b in range(B):
        assert bool((got[0][b, :, lens[b]:] == 0).all()) and bool((got[0][b, :, : lens[b] - n[b] + 1] > 0).all())


@BOTH
@pytest.mark.parametrize("B,T,Hq,Hk,D,block", [(64, 7, 4, 2, 128, 32), (100, 4, 4, 1, 64, 64), (40, 40, 4, 1, 128, 128), (36, 70, 2, 1, 64, 32), (48, 14, 4, 2, 128, 64)])
def test_attention_over_8_bits_reads_nothing_behind_the_ends(B, T, Hq, Hk, D, block, dtype):
    print("8-bit ends", B, T, Hq, Hk, D, block, dtype, flush=True)
    g = gen(93)
    cap = 4 * block
    lens, drafted = [(29 * b) % (cap + 1) for b in range(B)], [1 + b % T for b in range(B)]
    full, held = [n // block * block for n in lens], [n % block for n in lens]
    q, kn, vn = normal(g, (B, T, Hq, D), dtype, 2.0), normal(g, (B, T, Hk, D), dtype), normal(g, (B, T, Hk, D), dtype)
    k, v, ks, vs, kt, vt = draft_ref.make_cache(g, B, cap, Hk, D, block, dtype)
    eight = lambda x, byte: behind(x.view(torch.uint8), full, byte).view(x.dtype)
    ends = lambda s, value: behind(s.transpose(1, 2), [n // block for n in full], value).transpose(1, 2).contiguous()   # (full blocks have scales)
    _, tree = tree_of(g, B, T)
    for words in (None, tree):
        got = []
        for value, byte in ((0.0, 0), (NAN, 127), (INF, 126)):
            out, lse = torch.zeros_like(q), torch.zeros((B, T, Hq), device="cuda")
            ds.dep_tree_attn8(q, behind(kn, drafted, value), behind(vn, drafted, value), eight(k, byte), eight(v, byte), ends(ks, value), ends(vs, value),
                              behind(kt, held, value), behind(vt, held, value), ints(lens), out, lse=lse, tree=words, drafted=ints(drafted))
            torch.cuda.synchronize()
            got.append((out, lse))
        assert bool(got[0][0].isfinite().all())
        for out, lse in got[1:]:
            assert same(out, got[0][0]) and same(lse, got[0][1])
