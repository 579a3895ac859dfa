"""CPU tests that arrays which a call writes while it reads others may not be those others: refused before anything reaches a device."""
import ctypes

import pytest

import paper_2305_13450_amd as ds
from test_cache_ops_host import append
from test_draft_ops_host import BAD, append8, verify

P = 0x10000          # aligned addresses that nothing reads are its multiples


def call(name, d):
    f = getattr(ds._lib(), name)
    return f(ctypes.byref(d), P, 1 << 40, None) if name == "dep_verify_drafts" else f(ctypes.byref(d), None)


def verify_apart(**kw):
    return verify(**{**dict(p=P, q=2 * P, ids=3 * P, parents=4 * P, drafted=5 * P, u=6 * P, accepted=7 * P, n_accepted=8 * P, next=9 * P, q_batch=8000, q_token=1000), **kw})


@pytest.mark.parametrize("written", ["accepted", "n_accepted", "next"])
def test_verification_writes_arrays_of_its_own(written):
    for other in ("p", "q", "ids", "parents", "drafted", "u", "accepted", "n_accepted", "next"):
        if other != written:
            assert call("dep_verify_drafts", verify_apart(**{written: getattr(verify_apart(), other)})) == ds.EINVAL, other


def test_refusals_of_verification_with_arrays_apart():
    for kw in BAD["dep_verify_drafts"][1]:
        assert call("dep_verify_drafts", verify_apart(**kw)) == ds.EINVAL, kw


@pytest.mark.parametrize("written", ["cached_out", "n_out"])
def test_the_append_to_8_bits_writes_lengths_of_its_own(written):
    apart = dict(cached=P, cached_out=2 * P, accepted=3 * P, n_accepted=4 * P, n_out=5 * P)
    for other in apart:
        if other != written:
            assert call("dep_cache_append8", append8(**{**apart, written: apart[other]})) == ds.EINVAL, other


@pytest.mark.parametrize("written", ["cached_out", "n_out", "weights", "pos"])
def test_the_append_writes_arrays_of_its_own(written):
    apart = dict(cached=P, cached_out=2 * P, accepted=3 * P, n_accepted=4 * P, n_out=5 * P, start=6 * P, weights=7 * P, pos=8 * P)
    for other in apart:
        if other != written:
            assert call("dep_cache_append", append(**{**apart, written: apart[other]})) == ds.EINVAL, other
