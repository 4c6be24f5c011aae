"""What the Python calls over paged caches refuse by themselves, before any GPU work: with a PossError, not with whatever an index or a narrower integer makes of it."""
import os

import pytest

import paper_2506_03566_amd as P
from paper_2506_03566_amd.binding import PossKvCache


def _cache():
    if not os.path.exists(P.LIB_PATH):
        pytest.skip("libposs.so not built (run __graft_entry__.build())")
    import torch
    P.Rope(32)                                             # (looks the library and the types up)
    cache = P.KvCache.__new__(P.KvCache)
    k, v, table = torch.zeros(4, 2, 32, 64), torch.zeros(4, 2, 64, 32), torch.zeros(2, 2, dtype=torch.int32)
    cache._set(PossKvCache(0, 2, 64, 32, 4, 2, 2, 2, 4096, 4096, k.data_ptr(), v.data_ptr(), table.data_ptr()), torch.float32, (k, v, table))
    return cache, torch


def refused(f, *args, **kw):
    with pytest.raises(P.PossError) as e:
        f(*args, **kw)
    assert e.value.code == P.E_INVALID_ARG


def test_tensors_of_other_dimensions():
    cache, torch = _cache()
    q, out, lengths, ints = torch.zeros(2, 4, 64), torch.zeros(2, 4, 64), torch.zeros(2, dtype=torch.int32), torch.zeros(3, dtype=torch.int32)
    for bad in (q[0, 0, 0], q[0, 0], q[0], q[None]):
        refused(P.kv_attend, cache, bad, lengths, out)
        refused(P.kv_attend, cache, q, lengths, bad)
    k = torch.zeros(3, 2, 64)
    for bad in (k[0, 0, 0], k[0, 0], k[0], k[None]):
        refused(P.kv_append, cache, bad, k, ints)
        refused(P.kv_append, cache, k, bad, ints)
        refused(P.kv_append, cache, k, k, ints, q=bad)
        refused(P.kv_append, cache, k, k, ints, q=k, q_out=bad)
    refused(P.kv_attend, cache, q, lengths, out)           # no GPU tensors
    refused(P.kv_append, cache, k, k, ints)


def test_numbers_beyond_32_bits():
    """ctypes keeps an integer's lowest 32 bits: 2^32 + 5 would be taken for 5."""
    cache, torch = _cache()
    q, out, lengths = torch.zeros(2, 4, 64), torch.zeros(2, 4, 64), torch.zeros(2, dtype=torch.int32)
    for wide in ((1 << 32) + 5, 1 << 31, -(1 << 32) + 5, -(1 << 32)):
        refused(P.kv_attend, cache, q, lengths, out, max_len=wide)
        refused(P.kv_attend, cache, q, lengths, out, max_len=wide, scratch=torch.zeros(1 << 16, dtype=torch.uint8))
        refused(P.kv_attend_scratch, cache, 4, max_len=wide)
        refused(P.kv_attend_scratch, cache, wide - 1)
        refused(P.logprobs_scratch, wide, 1000, 2, device="cpu")
        refused(P.logprobs_scratch, 3, wide, 2, device="cpu")
        refused(P.logprobs_scratch, 3, 1000, wide, device="cpu")
        refused(P.Rope, wide - 1)
    assert P.logprobs_scratch(3, 1000, 2, device="cpu").nbytes > 0 and P.kv_attend_scratch(cache, 4, max_len=5).nbytes > 0


def test_frequencies_and_magnitudes_that_are_not_finite():
    """Numbers that are finite as they come but give none: an infinite frequency turns every angle into NaN, a magnitude beyond float32 every value."""
    _cache()
    import math
    for kw in (dict(magnitude=1e39), dict(magnitude=-1e300), dict(theta=1e-320), dict(theta=1e-200, scaling="linear", factor=1e-200), dict(scaling="linear", factor=1e-320),
               dict(theta=1e-320, scaling="bands", factor=2.0), dict(scaling="base", factor=1e-320)):
        refused(P.Rope, 64, **kw)
    for kw in (dict(magnitude=3e38), dict(theta=1e-300), dict(scaling="linear", factor=1e-300), dict(scaling="base", factor=1e300)):
        assert all(math.isfinite(f) for f in P.Rope(64, **kw).frequencies)


def test_a_scale_that_float32_does_not_hold_in_the_log2_domain():
    """Scores are formed times scale * log2(e): where that is infinite, a score of 0 would be NaN."""
    cache, torch = _cache()
    lib = P.load_library()
    need = lib.poss_kv_attend_scratch_bytes(cache.ref, 4, 0, 0)
    a = 1 << 20                                            # (never followed: the scratch is too small)
    for scale in (2.4e38, -2.4e38, 3.4e38):
        assert lib.poss_kv_attend(cache.ref, 4, a, 256, 2 * a, 256, a, 0, scale, None, None, None, a, need - 1, None) == P.E_INVALID_ARG
        assert b"scale" in lib.poss_last_error(None)
    assert lib.poss_kv_attend(cache.ref, 4, a, 256, 2 * a, 256, a, 0, 2.3e38, None, None, None, a, need - 1, None) == P.E_CAPACITY
