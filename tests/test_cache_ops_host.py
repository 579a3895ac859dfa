"""CPU tests of the cache operators' host side: argument checks through the C ABI (no call here gets as far as a device), workspace
sizes, and the words of a tree."""
import ctypes

import pytest
import torch

import paper_2305_13450_amd as ds

P = 0x10000          # an aligned address that nothing reads


def tree(**kw):
    d = ds.TreeAttnDesc()
    d.batch, d.tokens, d.heads, d.kv_heads, d.head_dim, d.dtype, d.capacity = 2, 8, 8, 2, 128, ds.BF16, 100
    d.q = d.k_new = d.v_new = d.k_cache = d.v_cache = d.cached = d.out = P
    d.q_batch, d.q_token, d.q_head = 8 * 1024, 1024, 128
    d.new_batch, d.new_token, d.new_head = 8 * 256, 256, 128
    d.cache_batch, d.cache_token, d.cache_head = 100 * 256, 256, 128
    d.out_batch, d.out_token, d.out_head = 8 * 1024, 1024, 128
    for k, v in kw.items():
        setattr(d, k, v)
    return d


def append(**kw):
    d = ds.CacheAppendDesc()
    d.batch, d.tokens, d.kv_heads, d.head_dim, d.dtype, d.capacity, d.n_max = 2, 8, 2, 128, ds.BF16, 100, 8
    d.k_new = d.v_new = d.k_cache = d.v_cache = d.cached = P
    d.cached_out = 2 * P
    d.new_batch, d.new_token, d.new_head = 8 * 256, 256, 128
    d.cache_batch, d.cache_token, d.cache_head = 100 * 256, 256, 128
    for k, v in kw.items():
        setattr(d, k, v)
    return d


def weights(**kw):
    d = ds.CacheWeightsDesc()
    d.batch, d.tokens, d.heads, d.kv_heads, d.head_dim, d.dtype, d.capacity, d.n_max = 2, 8, 8, 2, 128, ds.BF16, 100, 8
    d.q = d.lse = d.k_cache = d.cached = d.weights = P
    d.q_batch, d.q_token, d.q_head = 8 * 1024, 1024, 128
    d.cache_batch, d.cache_token, d.cache_head = 100 * 256, 256, 128
    for k, v in kw.items():
        setattr(d, k, v)
    return d


def evict(**kw):
    d = ds.CacheEvictDesc()
    d.batch, d.kv_heads, d.head_dim, d.dtype, d.capacity, d.budget, d.recent = 2, 2, 128, ds.BF16, 100, 50, 10
    d.k_cache = d.v_cache = d.weights = d.pos = d.cached = P
    d.cached_out = 2 * P
    d.cache_batch, d.cache_token, d.cache_head = 100 * 256, 256, 128
    for k, v in kw.items():
        setattr(d, k, v)
    return d


OTHER = dict(k_out=3 * P, v_out=3 * P, weights_out=3 * P, pos_out=3 * P, capacity_out=60, out_batch=60 * 256, out_token=256, out_head=128)


def call(name, d):
    f = getattr(ds._lib(), name)
    return f(ctypes.byref(d), P, 1 << 40, None) if name in ("dep_tree_attn", "dep_cache_evict") else f(ctypes.byref(d), None)


SIZES = [dict(batch=0), dict(kv_heads=0), dict(head_dim=0), dict(dtype=2), dict(capacity=-1), dict(batch=-4)]
BAD = {
    "dep_tree_attn": (tree, SIZES + [
        dict(tokens=0), dict(tokens=65537), dict(heads=7), dict(heads=1), dict(max_cached=-1), dict(q=0), dict(k_new=0), dict(v_new=P + 2), dict(k_cache=0),
        dict(v_cache=P + 8), dict(cached=0), dict(cached=P + 1), dict(out=0), dict(out=P + 4), dict(lse=P + 2), dict(drafted=P + 2), dict(tree=P + 4),
        dict(q_token=1025), dict(q_head=-8), dict(new_token=120), dict(new_token=(1 << 24) + 8), dict(cache_token=0), dict(cache_head=4), dict(out_token=0),
        dict(out_head=64), dict(out_batch=-8), dict(scale=-1.0), dict(scale=float("inf")), dict(scale=float("nan")), dict(tree=P, tree_batch=7), dict(tree=P, tree_batch=-1)]),
    "dep_cache_append": (append, SIZES + [
        dict(tokens=0), dict(capacity=0), dict(n_max=0), dict(n_max=9), dict(k_new=0), dict(v_new=0), dict(k_cache=0), dict(v_cache=P + 8), dict(cached=0),
        dict(cached_out=0), dict(cached_out=P), dict(accepted=P + 2), dict(n_accepted=P + 1), dict(weights=P + 2), dict(pos=P), dict(pos=P, start=P + 2),
        dict(new_head=12), dict(cache_token=64), dict(cache_head=64), dict(cache_batch=0)]),
    "dep_cache_weights": (weights, SIZES + [
        dict(tokens=0), dict(heads=9), dict(capacity=0), dict(max_cached=-2), dict(n_max=9), dict(n_max=0), dict(q=P + 8), dict(lse=0), dict(k_cache=0), dict(cached=0),
        dict(weights=0), dict(accepted=P + 2), dict(q_batch=4), dict(cache_token=100), dict(scale=float("nan"))]),
    "dep_cache_evict": (evict, SIZES + [
        dict(capacity=0), dict(budget=0), dict(recent=-1), dict(recent=51), dict(max_cached=-1), dict(k_cache=0), dict(v_cache=0), dict(weights=0), dict(pos=0),
        dict(pos=P + 2), dict(cached=0), dict(cached_out=0), dict(cached_out=P), dict(cache_token=64), dict(cache_head=0), dict(v_out=P), dict(weights_out=P),
        {**OTHER, "v_out": 0}, {**OTHER, "pos_out": 0}, {**OTHER, "k_out": P}, {**OTHER, "weights_out": P}, {**OTHER, "capacity_out": 49}, {**OTHER, "out_token": 8},
        {**OTHER, "out_head": 0}]),
}


@pytest.mark.parametrize("name", list(BAD))
def test_refusals(name):
    make, bad = BAD[name]
    for kw in bad:
        assert call(name, make(**kw)) == ds.EINVAL, kw
    for kw in (dict(head_dim=80), dict(head_dim=256)):
        assert call(name, make(**kw)) == ds.ENOTIMPL, kw
    f = getattr(ds._lib(), name)
    assert (f(None, P, 1 << 40, None) if name in ("dep_tree_attn", "dep_cache_evict") else f(None, None)) == ds.EINVAL


def test_launches_too_large_are_refused():
    assert call("dep_cache_append", append(batch=1 << 20, n_max=8, tokens=8, kv_heads=64)) == ds.ENOTIMPL
    assert call("dep_cache_weights", weights(batch=1 << 20, capacity=1 << 20)) == ds.ENOTIMPL
    assert call("dep_cache_evict", evict(batch=1 << 20, kv_heads=64)) == ds.ENOTIMPL
    n = ctypes.c_size_t(0)
    assert ds._lib().depsync_tree_attn_workspace(ctypes.byref(tree(batch=1 << 20, capacity=1 << 20, heads=64, kv_heads=64)), 256, ctypes.byref(n)) == ds.ENOTIMPL


def test_workspaces():
    n = ctypes.c_size_t(1)
    f = ds._lib().depsync_tree_attn_workspace
    assert f(ctypes.byref(tree(capacity=0)), 256, ctypes.byref(n)) == ds.OK and n.value == 0          # one block of keys: one part
    assert f(ctypes.byref(tree(capacity=50000)), 256, ctypes.byref(n)) == ds.OK and n.value % (2 * 8 * 4 * 130 * 4) == 0 and n.value > 0
    long = n.value
    assert f(ctypes.byref(tree(capacity=50000, max_cached=300)), 256, ctypes.byref(n)) == ds.OK and n.value < long
    assert f(ctypes.byref(tree()), 256, None) == ds.EINVAL and f(None, 256, ctypes.byref(n)) == ds.EINVAL
    g = ds._lib().depsync_cache_evict_workspace
    assert g(ctypes.byref(evict()), ctypes.byref(n)) == ds.OK and n.value >= 4 * (1 + 2 * 50) * 4
    assert g(ctypes.byref(evict(budget=0)), ctypes.byref(n)) == ds.EINVAL and g(ctypes.byref(evict()), None) == ds.EINVAL
    # a workspace that is missing, too small or unaligned
    d = evict()
    for ptr, size in ((None, 1 << 30), (P, n.value - 4), (P + 4, 1 << 30)):
        assert ds._lib().dep_cache_evict(ctypes.byref(d), ptr, size, None) == ds.EINVAL


def test_tree_words():
    m = ds.tree_mask([-1, 0, 1, 1, -7])
    assert m.tolist() == [[1], [3], [7], [11], [16]]
    chain = ds.tree_mask(torch.arange(130) - 1)
    assert chain.shape == (130, 3) and chain[63].tolist() == [-1, 0, 0] and chain[64].tolist() == [-1, 1, 0] and chain[129].tolist() == [-1, -1, 3]
    assert ds.tree_mask([[-1, 0], [-1, -1]]).tolist() == [[[1], [3]], [[1], [2]]]
    for bad in ([0], [-1, 1], [-1, 2, 0]):
        with pytest.raises(ValueError):
            ds.tree_mask(bad)
    with pytest.raises(ValueError):
        ds.tree_mask(torch.zeros((0,), dtype=torch.int64))


def test_token_strides_of_the_queries_of_weights():
    for kw in (dict(q_token=64), dict(q_token=0), dict(q_token=(1 << 24) + 8)):
        assert call("dep_cache_weights", weights(**kw)) == ds.EINVAL, kw
