"""GPU tests of attention over a cache of 8 bits for whole chunks of a prompt: long stretches of rows of 16 bits behind those of 8, cut into parts and uncut."""
import pytest
import torch

import draft_ref as ref
import paper_2305_13450_amd as ds
from test_gpu_draft_ops import BF, FP, check_attn, gen, ints, normal, run_attn, spoil, tree_of

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", [BF, FP], ids=["bf16", "fp16"])
@pytest.mark.parametrize("shape", ["chain", "tree"])
@pytest.mark.parametrize("T,Hq,Hk,D,block,lens,cut", [(1024, 4, 2, 128, 32, [31, 700], True), (700, 2, 1, 64, 128, [127], True), (1500, 1, 1, 128, 64, [0], True), (640, 3, 3, 64, 64, [64, 1000, 5], True),
                                                      (330, 8, 8, 64, 32, [31, 96, 0, 33, 64, 1, 128, 65, 70, 99, 2, 127, 40, 50, 60, 95], False)])
def test_prompt_chunks(T, Hq, Hk, D, block, lens, cut, shape, dtype):
    print("prompt", T, Hq, Hk, D, block, lens, shape, dtype, flush=True)
    g, B = gen(121), len(lens)
    cap = -(-max(lens + [1]) // block) * block
    cached = ints(lens)
    cache = spoil(ref.make_cache(g, B, cap, Hk, D, block, dtype), cached)
    q, kn, vn = normal(g, (B, T, Hq, D), dtype, 2.0), normal(g, (B, T, Hk, D), dtype), normal(g, (B, T, Hk, D), dtype)
    need = ds.tree_attn8_workspace(q, kn, vn, *cache, cached, torch.empty_like(q))
    assert (need > 0) == cut                                          # (which is what this size is for)
    tree = tree_of(g, B, T)[1] if shape == "tree" else None
    drafted = ints([T - (b * 97) % (T // 2) for b in range(B)])
    out, lse = check_attn(q, kn, vn, cache, cached, tree=tree, drafted=drafted)
    # the same numbers again, and as the only sequence of a call up to rounding
    again, again_lse = run_attn(q, kn, vn, cache, cached, tree=tree, drafted=drafted)
    assert torch.equal(again.cpu().double(), out) and torch.equal(again_lse.cpu().double(), lse)
    one = lambda x: None if x is None else x[:1]
    check_attn(q[:1], kn[:1], vn[:1], tuple(t[:1] for t in cache), cached[:1], tree=one(tree), drafted=drafted[:1])
