"""GPU tests of verification without draft probabilities where one token has very many children: exact, and in a time that grows with their number."""
import pytest
import torch

import paper_2305_13450_amd as ds
from test_gpu_draft_ops import check_verify, gen, ints, probabilities

pytestmark = pytest.mark.gpu


def star(T, B=2):
    parents = torch.zeros((B, T), dtype=torch.int32, device="cuda")
    parents[:, 0] = -1
    return parents


# few different tokens again and again over many lots of 64, and many different ones: neighbours, and as far apart as the filter is long
@pytest.mark.parametrize("V", [3000, 40000, 1 << 20])
@pytest.mark.parametrize("T,numbers", [(65, 3), (513, 40), (512, 511), (2000, 2000), (4096, 900), (4096, 4096)])
def test_children_in_many_lots(T, numbers, V):
    print("children", T, numbers, V, flush=True)
    g = gen(95)
    p, _ = probabilities(g, 2, 1, V, spread=0.5)
    p = p.expand(2, T, V)
    for step in (1, 32768, 7919):
        ids = (torch.randint(0, numbers, (2, T), generator=g, device="cuda") * step % V).int()
        parents = star(T)
        parents[1, T // 2:] = T // 2 - 1                             # the second sequence goes on from a late child
        for u0 in (0.0, 0.37, 0.99999):
            u = torch.full((2, T), 0.99999, device="cuda")
            u[:, 0] = u0
            u[1, T // 2 - 1] = 0.0
            check_verify(p, ids, u, None, parents)


def test_a_star_of_4096_takes_no_milliseconds():
    # 33 ms where every number of the row was compared with all children one by one; a chain of as many takes 0.06
    g = gen(96)
    B, T, V = 2, 4096, 32000
    p = torch.rand((B, 1, V), generator=g, device="cuda")
    p = (p / p.sum(-1, keepdim=True)).expand(B, T, V)
    ids = torch.randperm(V, generator=g, device="cuda")[:T].int().expand(B, T).contiguous()
    u = torch.full((B, T), 0.99999, device="cuda")
    acc, n, nxt = torch.zeros_like(ids), ints([0, 0]), ints([0, 0])
    times = []
    for _ in range(6):
        a, b = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
        a.record()
        ds.dep_verify_drafts(p, ids, u, acc, n, nxt, parents=star(T)[0].contiguous())
        b.record()
        torch.cuda.synchronize()
        times.append(a.elapsed_time(b))
    assert n.tolist() == [1, 1] and min(times) < 3.0, times
