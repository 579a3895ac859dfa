"""CPU tests of the host side of a round of drafts over a cache of 8 bits: argument checks through the C ABI (no call here gets as far as a device), layouts of the
packed descriptors, workspace sizes, frequencies, and the 64-bit forms' own numbers of 8 bits."""
import ctypes
import math
import random

import pytest
import torch

import draft_ref as ref
import paper_2305_13450_amd as ds

P = 0x10000          # an aligned address that nothing reads


def fill(d, kw):
    for k, v in kw.items():
        setattr(d.attn if isinstance(d, ds.TreeAttn8Desc) and k not in OWN8 else d, k, v)
    return d


OWN8 = ("block", "k_scale", "v_scale", "k_tail", "v_tail", "tail_batch", "tail_token", "tail_head")


def attn8(**kw):
    d = ds.TreeAttn8Desc()
    base = dict(batch=2, tokens=8, heads=8, kv_heads=2, head_dim=128, dtype=ds.BF16, capacity=128, q=P, k_new=P, v_new=P, k_cache=P, v_cache=P, cached=P, out=P,
                q_batch=8 * 1024, q_token=1024, q_head=128, new_batch=8 * 256, new_token=256, new_head=128, cache_batch=128 * 256, cache_token=256, cache_head=128,
                out_batch=8 * 1024, out_token=1024, out_head=128, block=64, k_scale=P, v_scale=P, k_tail=P, v_tail=P, tail_batch=64 * 256, tail_token=256, tail_head=128)
    return fill(d, {**base, **kw})


def append8(**kw):
    base = dict(batch=2, tokens=8, kv_heads=2, head_dim=128, dtype=ds.BF16, capacity=128, block=64, n_max=8, k_new=P, v_new=P, k_cache=P, v_cache=P, k_scale=P, v_scale=P,
                k_tail=P, v_tail=P, cached=P, cached_out=2 * P, new_batch=8 * 256, new_token=256, new_head=128, cache_batch=128 * 256, cache_token=256, cache_head=128,
                tail_batch=64 * 256, tail_token=256, tail_head=128)
    return fill(ds.CacheAppend8Desc(), {**base, **kw})


def norm(**kw):
    base = dict(batch=2, tokens=8, heads=8, kv_heads=2, head_dim=128, dtype=ds.BF16, rotary_dim=128, norm=1, eps=1e-6, q=P, k=P, q_out=2 * P, k_out=2 * P, freq=P)
    for t, h in (("q", 8), ("k", 2), ("q_out", 8), ("k_out", 2)):
        base.update({t + "_batch": 8 * h * 128, t + "_token": h * 128, t + "_head": 128})
    return fill(ds.QkNormRopeDesc(), {**base, **kw})


def verify(**kw):
    base = dict(batch=2, tokens=8, vocab=1000, p=P, p_batch=8000, p_token=1000, ids=P, u=P, accepted=P, n_accepted=P, next=2 * P)
    return fill(ds.VerifyDraftsDesc(), {**base, **kw})


def call(name, d):
    f = getattr(ds._lib(), name)
    r = None if d is None else ctypes.byref(d)
    return f(r, P, 1 << 40, None) if name in ("dep_tree_attn8", "dep_verify_drafts") else f(r, None)


SIZES = [dict(batch=0), dict(kv_heads=0), dict(head_dim=0), dict(dtype=2), dict(dtype=-1), dict(batch=-4), dict(tokens=0), dict(tokens=65537), dict(batch=(1 << 20) + 1)]
BLOCKS = [dict(block=0), dict(block=16), dict(block=48), dict(block=256), dict(block=-64), dict(capacity=0), dict(capacity=100), dict(capacity=-64), dict(block=128, capacity=64)]
BAD = {
    "dep_tree_attn8": (attn8, SIZES + BLOCKS + [
        dict(heads=7), dict(heads=1), dict(max_cached=-1), dict(q=0), dict(k_new=0), dict(v_new=P + 2), dict(k_cache=0), dict(v_cache=P + 8), dict(cached=0), dict(cached=P + 1),
        dict(out=0), dict(lse=P + 2), dict(drafted=P + 2), dict(tree=P + 4), dict(k_scale=0), dict(v_scale=0), dict(v_scale=P + 2), dict(k_tail=0), dict(v_tail=P + 8),
        dict(q_token=1025), dict(new_token=120), dict(cache_token=0), dict(cache_token=264), dict(cache_head=136), dict(cache_batch=8), dict(cache_token=112), dict(out_token=0),
        dict(tail_token=100), dict(tail_token=64), dict(tail_head=-8), dict(tail_token=(1 << 24) + 8), dict(scale=-1.0), dict(scale=float("nan")), dict(tree=P, tree_batch=7)]),
    "dep_cache_append8": (append8, SIZES + BLOCKS + [
        dict(n_max=0), dict(n_max=9), dict(n_max=65537, accepted=P), dict(k_new=0), dict(v_new=0), dict(k_cache=0), dict(v_cache=P + 8), dict(k_scale=0), dict(v_scale=P + 1),
        dict(k_tail=0), dict(v_tail=0), dict(cached=0), dict(cached_out=0), dict(cached_out=P), dict(accepted=P + 2), dict(n_accepted=P + 1), dict(n_out=P), dict(n_out=2 * P),
        dict(n_out=3 * P, n_accepted=3 * P), dict(new_head=12), dict(cache_token=64), dict(cache_head=64), dict(cache_token=264), dict(cache_batch=0), dict(tail_batch=0), dict(tail_head=0)]),
    "dep_qk_norm_rope": (norm, SIZES + [
        dict(heads=7), dict(heads=1), dict(rotary_dim=-16), dict(rotary_dim=8), dict(rotary_dim=144), dict(rotary_dim=100), dict(interleaved=2), dict(norm=-1), dict(eps=-1.0),
        dict(eps=float("inf")), dict(eps=float("nan")), dict(q=0), dict(k=0), dict(q_out=0), dict(k_out=P + 8), dict(freq=0), dict(freq=P + 8), dict(q_gain=P + 4), dict(k_gain=P + 8),
        dict(start=P + 2), dict(depth=P + 1), dict(drafted=P + 2), dict(q_token=1025), dict(k_head=-8), dict(q_out_token=0), dict(k_out_head=64), dict(q_out=P, q_out_token=2048),
        dict(k_out=P, k_out_head=256), dict(depth=P, depth_batch=7), dict(depth=P, depth_batch=-1)]),
    "dep_verify_drafts": (verify, [
        dict(batch=0), dict(tokens=0), dict(tokens=65537), dict(vocab=0), dict(vocab=(1 << 24) + 1), dict(batch=(1 << 20) + 1), dict(p=0), dict(p=P + 2), dict(q=P + 1), dict(ids=0),
        dict(parents=P + 2), dict(drafted=P + 2), dict(u=0), dict(accepted=0), dict(n_accepted=0), dict(next=0), dict(next=P), dict(p_token=-1), dict(p_batch=-8), dict(p_batch=1 << 41),
        dict(q=P, q_token=-4), dict(parents=P, parents_batch=7), dict(parents=P, parents_batch=-8)]),
}


@pytest.mark.parametrize("name", list(BAD))
def test_refusals(name):
    make, bad = BAD[name]
    for kw in bad:
        assert call(name, make(**kw)) == ds.EINVAL, kw
    if name != "dep_verify_drafts":
        for kw in (dict(head_dim=80), dict(head_dim=256)):
            assert call(name, make(**kw)) == ds.ENOTIMPL, kw
    assert call(name, None) == ds.EINVAL


def test_launches_too_large_are_refused():
    assert call("dep_cache_append8", append8(batch=1 << 20, kv_heads=64, n_max=8)) == ds.ENOTIMPL
    assert call("dep_qk_norm_rope", norm(batch=1 << 20, tokens=64)) == ds.ENOTIMPL
    assert call("dep_verify_drafts", verify(tokens=4097)) == ds.ENOTIMPL
    n = ctypes.c_size_t(0)
    f = ds._lib().depsync_tree_attn8_workspace
    assert f(ctypes.byref(attn8(batch=1 << 20, capacity=1 << 20, heads=64, kv_heads=64)), 256, ctypes.byref(n)) == ds.ENOTIMPL


def test_workspaces():
    n = ctypes.c_size_t(1)
    f = ds._lib().depsync_tree_attn8_workspace
    assert f(ctypes.byref(attn8(capacity=64)), 256, ctypes.byref(n)) == ds.OK
    assert f(ctypes.byref(attn8(capacity=64000)), 256, ctypes.byref(n)) == ds.OK and n.value > 0 and n.value % (2 * 8 * 4 * 130 * 4) == 0
    long = n.value
    assert f(ctypes.byref(attn8(capacity=64000, max_cached=300)), 256, ctypes.byref(n)) == ds.OK and n.value < long
    assert f(ctypes.byref(attn8(block=16)), 256, ctypes.byref(n)) == ds.EINVAL
    assert f(ctypes.byref(attn8()), 256, None) == ds.EINVAL and f(None, 256, ctypes.byref(n)) == ds.EINVAL
    g = ds._lib().depsync_verify_drafts_workspace
    assert g(ctypes.byref(verify()), ctypes.byref(n)) == ds.OK
    assert g(ctypes.byref(verify(vocab=0)), ctypes.byref(n)) == ds.EINVAL and g(ctypes.byref(verify()), None) == ds.EINVAL and g(None, ctypes.byref(n)) == ds.EINVAL


def flat(desc):
    """Names and kinds of a descriptor's fields in order, nested ones opened."""
    for name, kind in desc._fields_:
        if issubclass(kind, ctypes.Structure):
            yield from flat(kind)
        else:
            yield name, kind


@pytest.mark.parametrize("packs,desc", [((ds._P_APPEND8,), ds.CacheAppend8Desc), ((ds._P_NORM,), ds.QkNormRopeDesc), ((ds._P_VERIFY,), ds.VerifyDraftsDesc),
                                        ((ds._P_TREE, ds._P_TREE8), ds.TreeAttn8Desc)])
def test_packed_descriptors_have_the_headers_layout(packs, desc):
    fields = list(flat(desc))
    numbers = [i + 1 for i in range(len(fields))]
    raw, left = b"", list(numbers)
    for p in packs:
        n = len(p.unpack(bytes(p.size)))
        raw += p.pack(*left[:n])
        left = left[n:]
    assert not left and len(raw) == ctypes.sizeof(desc)
    d = desc.from_buffer_copy(raw)
    got = [getattr(d.attn if isinstance(d, ds.TreeAttn8Desc) and name not in OWN8 else d, name) for name, _ in fields]
    assert [int(x) for x in got] == numbers


def test_frequencies():
    assert ds.rope_frequencies([0.0]).tolist() == [0]
    quarter = ds.rope_frequencies([math.pi / 2]).item()
    assert abs(quarter - 2 ** 62) <= 2 ** 11                      # (pi / 2 itself is rounded)
    back = ds.rope_frequencies([-math.pi / 2]).item()
    assert back == -quarter
    r = random.Random(3)
    for _ in range(50):
        x, n = r.uniform(0, 7), r.randrange(1 << 31)
        f = ds.rope_frequencies([x]).item() % 2 ** 64
        turns = (n * f % 2 ** 64) / 2 ** 64
        assert abs(math.cos(2 * math.pi * turns) - math.cos(math.fmod(n * x, 2 * math.pi))) < 1e-5
    for bad in ([float("nan")], [[1.0]], [float("inf")]):
        with pytest.raises(ValueError):
            ds.rope_frequencies(bad)


def test_numbers_of_8_bits_of_the_reference():
    table = torch.tensor([ref.e4m3_value(i) for i in range(256)])
    assert torch.equal(torch.arange(256, dtype=torch.uint8).view(torch.float8_e4m3fn).double().nan_to_num(9e9), table.double().nan_to_num(9e9))
    for top, want in ((0.0, 0.0), (448.0, 1.0), (449.0, 2.0), (1.0, 2.0 ** -8), (1.75, 2.0 ** -8), (1.76, 2.0 ** -7), (3e38, 2.0 ** 120), (1e-44, 2.0 ** -126)):
        assert ref.scale_of(top) == want
    x = torch.randn((64, 32), dtype=torch.float64).bfloat16()
    y, s = ref.quantise(x)
    assert torch.equal((x.float() / s).to(torch.float8_e4m3fn).double(), y)


def test_verification_of_the_reference():
    # by hand: root, children of tokens 1 and 2; p = (1/8, 1/2, 3/8), the drafts drawn from q = (0, 3/4, 1/4)
    p = torch.tensor([[[0.125, 0.5, 0.375], [1.0, 0, 0], [0, 0, 1.0]]])
    q = torch.tensor([[[0.0, 0.75, 0.25], [1, 0, 0], [1, 0, 0]]])
    ids, parents = torch.tensor([[0, 1, 2]]), torch.tensor([-1, 0, 0])
    u = lambda *x: torch.tensor([list(x)])
    assert ref.verify(p, ids, u(0.5, 0.6, 0.9), q, parents) == [([0, 1], 0)]                  # 0.6 * 0.75 < 0.5
    # refused: max(p - q, 0) = (1/8, 0, 1/8), R = 1/4; token 2: 0.9 * 0.25 * 0.25 < 0.125 stays
    assert ref.verify(p, ids, u(0.5, 0.7, 0.9), q, parents) == [([0, 2], 2)]
    # without q: 0.7 >= 0.5 refused, then of R = 1/2 token 2 has 3/8: 0.7 * 0.5 < 0.375 stays, 0.8 * 0.5 does not; what is left is token 0
    assert ref.verify(p, ids, u(0.5, 0.7, 0.7), None, parents) == [([0, 2], 2)]
    assert ref.verify(p, ids, u(0.9, 0.7, 0.8), None, parents) == [([0], 0)]
