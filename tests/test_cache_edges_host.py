"""CPU tests of the cache operators' newer arguments: refusals through the C ABI, and the packed descriptors against their ctypes forms."""
import ctypes

import paper_2305_13450_amd as ds
import test_cache_ops_host as host

P = host.P


def test_refusals_of_the_count_of_appended_rows():
    for kw in (dict(n_out=P + 2), dict(n_out=P), dict(n_out=2 * P), dict(n_accepted=5 * P, n_out=5 * P)):
        assert host.call("dep_cache_append", host.append(**kw)) == ds.EINVAL, kw


def test_packed_descriptors_have_the_size_of_their_classes():
    for packed, cls in ((ds._P_TREE, ds.TreeAttnDesc), (ds._P_APPEND, ds.CacheAppendDesc), (ds._P_WEIGHTS, ds.CacheWeightsDesc), (ds._P_EVICT, ds.CacheEvictDesc)):
        assert packed.size == ctypes.sizeof(cls)
