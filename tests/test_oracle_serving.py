"""The float64 formulas of serving over paged caches against closed forms, and what the library refuses before any GPU work."""
import ctypes
import math
import os

import numpy as np
import pytest

import paper_2506_03566_amd as P
from paper_2506_03566_amd.binding import PossKvCache, PossRope
from oracle import serving as o


def _lib():
    if not os.path.exists(P.LIB_PATH):
        pytest.skip("libposs.so not built (run __graft_entry__.build())")
    return P.load_library()


@pytest.mark.parametrize("interleaved", [False, True])
def test_rotation_keeps_lengths_and_depends_on_differences(interleaved):
    rng = np.random.default_rng(1)
    w = o.rope_frequencies(32)
    q, k = rng.normal(size=(1, 1, 48)), rng.normal(size=(1, 1, 48))
    dots = [(o.rotate(q, [a], w, interleaved) * o.rotate(k, [b], w, interleaved)).sum() for a, b in ((5, 3), (1005, 1003), (2, 0))]
    assert np.allclose(dots, dots[0], atol=1e-9)
    y = o.rotate(q, [7], w, interleaved)
    assert np.allclose((y ** 2).sum(), (q ** 2).sum()) and np.array_equal(y[..., 32:], q[..., 32:])
    assert np.allclose(o.rotate(y, [7], w, interleaved, inverse=True), q)
    one = np.zeros((1, 1, 4))
    one[0, 0, 0] = 1.0                                     # the first pair turns by a radian a position
    assert np.allclose(o.rotate(one, [1], np.array([1.0, 0.5]), interleaved)[0, 0], [math.cos(1), math.sin(1), 0, 0] if interleaved else [math.cos(1), 0, math.sin(1), 0])


def test_scaled_frequencies():
    w = o.rope_frequencies(128, 500000.0)
    assert w[0] == 1 and np.isclose(w[-1], 500000.0 ** (-126 / 128))
    assert np.allclose(o.rope_frequencies(128, 500000.0, "linear", 4.0), w / 4)
    base = o.rope_frequencies(128, 500000.0, "base", 4.0)
    assert base[0] == 1 and np.isclose(base[-1], w[-1] / 4)      # the slowest pair turns as if positions were divided
    for scaling in ("bands", "ramp"):
        s = o.rope_frequencies(128, 500000.0, scaling, 8.0, 1.0, 4.0, 8192)
        turns = 8192 * w / (2 * np.pi)
        assert np.allclose(s[turns > 6], w[turns > 6]) and np.allclose(s[turns < 0.7], w[turns < 0.7] / 8)
        assert (np.diff(s) < 0).all() and (s <= w * (1 + 1e-15)).all() and (s >= w / 8 * (1 - 1e-15)).all()


@pytest.mark.parametrize("rot", [4, 32, 96, 128, 256])
@pytest.mark.parametrize("scaling", ["none", "linear", "base", "bands", "ramp"])
def test_the_library_fills_in_the_same_frequencies(rot, scaling):
    _lib()
    r = P.Rope(rot, 500000.0, interleaved=True, scaling=scaling, factor=8.0, low=1.0, high=32.0, original=4096, magnitude=1.25)
    assert np.allclose(r.frequencies, o.rope_frequencies(rot, 500000.0, scaling, 8.0, 1.0, 32.0, 4096), rtol=1e-13, atol=0)
    assert r.c.rot_dim == rot and r.c.interleaved == 1 and r.c.magnitude == 1.25
    own = P.Rope(rot, frequencies=[0.5] * (rot // 2))
    assert own.frequencies == [0.5] * (rot // 2)


def test_rope_refusals():
    _lib()
    for kw in (dict(rot_dim=0), dict(rot_dim=7), dict(rot_dim=258), dict(theta=0.0), dict(theta=float("nan")), dict(scaling="linear", factor=0.0), dict(scaling="other"),
               dict(scaling="bands", factor=2.0, low=4.0, high=4.0), dict(scaling="ramp", factor=2.0, original=0), dict(scaling="ramp", factor=2.0, theta=1.0), dict(scaling="base", rot_dim=2, factor=2.0),
               dict(magnitude=float("inf")), dict(frequencies=[1.0]), dict(frequencies=[float("nan")] * 32)):
        with pytest.raises(P.PossError) as e:
            P.Rope(**{"rot_dim": 64, **kw})
        assert e.value.code == P.E_INVALID_ARG, kw


def test_attention_and_eviction_by_hand():
    q, k, v = np.array([[2.0, 0.0], [0.0, 1.0]]), np.array([[[1.0, 0.0], [0.0, 1.0]]]), np.array([[[1.0, 2.0], [3.0, 4.0]]])
    out, lse, p, _ = o.attend(q, k, v, 0.5)
    e = math.e
    assert np.allclose(p, [[e / (e + 1), 1 / (e + 1)], [1 / (1 + e ** 0.5), e ** 0.5 / (1 + e ** 0.5)]])
    assert np.allclose(out, p @ v[0]) and np.allclose(lse, [math.log(e + 1), math.log(1 + e ** 0.5)])
    out, lse, p, _ = o.attend(q, k[:, :0], v[:, :0], 0.5)
    assert not out.any() and (lse == -np.inf).all() and p.shape == (2, 0)
    # six slots to three: slot 0 by its position, slot 5 the newest, then the heaviest, the lower of two equal ones; slots 1 and 2 are holes
    assert o.evict([.1, .2, .2, .9, .9, 0], [0, 7, 8, 9, 10, 11], 6, 3, 1, 1) == [0, 3, 5]
    assert o.evict([.1, .2, .2, .9, .9, 0], [0, 7, 8, 9, 10, 11], 6, 3, 0, 0) == [3, 1, 4]
    assert o.evict([math.nan, math.inf, -1.0, 0.0], [0, 1, 2, 3], 4, 2, 0, 0) == [3, 1]
    assert o.evict([1.0] * 4, [3, 2, 1, 0], 3, 3, 0, 0) == [0, 1, 2] and o.evict([1.0] * 4, [0] * 4, 0, 3, 0, 0) == []
    assert o.evict([1.0] * 6, [5, 4, 3, 2, 1, 0], 6, 3, 0, 2) == [0, 1, 2]        # age is a position's, not a slot's


def test_log_probabilities_by_hand():
    lp, h = o.logprobs(np.array([[0.0, math.log(3.0), -np.inf], [1.0, 1.0, 1.0]]))
    assert np.allclose(np.exp(lp), [[.25, .75, 0], [1 / 3] * 3]) and np.allclose(h, [-.25 * math.log(.25) - .75 * math.log(.75), math.log(3)])
    for bad in ([np.nan, 0, 0], [np.inf, 0, 0], [-np.inf] * 3):
        lp, h = o.logprobs(np.array([bad]))
        assert np.isnan(lp).all() and np.isnan(h).all()
    assert o.best([1.0, np.nan, 2.0, 2.0, -np.inf], 5) == [2, 3, 0, 4, 1]


# ---------------------------------------------------------------- refusals, without a GPU (the pointers are never followed)
A = 1 << 20


def cache(**kw):
    c = dict(dtype=1, n_kv_heads=2, head_dim=64, page_tokens=32, n_pages=4, n_seq=2, table_pages=2, table_stride=2, k_page_stride=4096, v_page_stride=4096, k=A, v=2 * A, page_table=3 * A)
    c.update(kw)
    return PossKvCache(**c)


BAD_CACHES = [dict(dtype=3), dict(dtype=-1), dict(n_kv_heads=0), dict(n_kv_heads=65536), dict(head_dim=0), dict(head_dim=48), dict(head_dim=288), dict(page_tokens=16), dict(page_tokens=48), dict(n_pages=0),
              dict(n_seq=-1), dict(n_seq=65536), dict(table_pages=0), dict(table_pages=1 << 26, table_stride=1 << 26), dict(table_stride=1), dict(k_page_stride=4088), dict(v_page_stride=4092),
              dict(k_page_stride=4100), dict(k=None), dict(v=None), dict(page_table=None), dict(k=A + 8), dict(v=A + 2), dict(page_table=A + 2)]


def test_bad_caches_are_refused_by_every_call():
    lib = _lib()
    rope = PossRope(64, 0, 1.0)
    for kw in [None, *BAD_CACHES]:
        c = ctypes.byref(cache(**kw)) if kw is not None else None
        assert lib.poss_kv_append(c, ctypes.byref(rope), 1, 0, None, 0, None, 0, A, 128, A, 128, None, A, A, None, None) == P.E_INVALID_ARG, kw
        assert lib.poss_last_error(None).startswith(b"poss_kv_append: ")
        assert lib.poss_kv_attend_scratch_bytes(c, 4, 0, 0) == 0
        assert lib.poss_kv_attend(c, 4, A, 256, 2 * A, 256, A, 0, 1.0, None, None, None, A, 1 << 30, None) == P.E_INVALID_ARG, kw
        assert lib.poss_last_error(None).startswith(b"poss_kv_attend: ")
        assert lib.poss_kv_evict(c, A, A, A, 4, 0, 0, A, 2 * A, 2 * A, 2 * A, None) == P.E_INVALID_ARG, kw
        assert lib.poss_last_error(None).startswith(b"poss_kv_evict: ")


def test_append_refusals():
    lib = _lib()
    c, rope = ctypes.byref(cache()), PossRope(64, 0, 1.0)
    good = dict(cache=c, rope=ctypes.byref(rope), rows=2, hq=4, q=A, q_row=256, q_out=A, q_out_row=256, k=A, k_row=128, v=A, v_row=128, seq=A, slots=A, positions=A, noted=A)

    def call(**kw):
        return lib.poss_kv_append(*{**good, **kw}.values(), None)
    for kw in (dict(rows=-1), dict(hq=-1), dict(hq=65536), dict(q=None), dict(q_out=None), dict(k=None), dict(v=None), dict(slots=None), dict(positions=None), dict(rope=None, positions=None), dict(k_row=127),
               dict(v_row=0), dict(q_row=255), dict(q_out_row=264), dict(k=A + 1), dict(v=A + 1), dict(q=A + 1), dict(slots=A + 2), dict(seq=A + 1), dict(noted=A + 2), dict(positions=A + 1)):
        assert call(**kw) == P.E_INVALID_ARG, kw
    for rot in (0, 3, 66, 258):
        assert call(rope=ctypes.byref(PossRope(rot, 0, 1.0))) == P.E_INVALID_ARG, rot
    assert call(rows=0, k=None) == P.POSS_OK and call(cache=ctypes.byref(cache(n_seq=0, k=None))) == P.POSS_OK


def test_rotary_refusals():
    lib = _lib()
    good = dict(t=1, x=A, x_row=128, x_head=64, y=2 * A, y_row=128, y_head=64, rows=2, heads=2, dim=64, positions=A, rope=ctypes.byref(PossRope(64, 0, 1.0)), inverse=0)

    def call(**kw):
        return lib.poss_rotary(*{**good, **kw}.values(), None)
    for kw in (dict(t=3), dict(rows=-1), dict(heads=0), dict(dim=1), dict(dim=62), dict(rope=None), dict(x=None), dict(y=None), dict(positions=None), dict(x=A + 1), dict(positions=A + 2), dict(x_head=63),
               dict(y_row=63), dict(y=A, y_row=256), dict(y=A, y_head=128), dict(rope=ctypes.byref(PossRope(63, 0, 1.0)))):
        assert call(**kw) == P.E_INVALID_ARG, kw
    assert call(rows=0, x=None) == P.POSS_OK


def test_attend_refusals():
    lib = _lib()
    c = ctypes.byref(cache())
    need = lib.poss_kv_attend_scratch_bytes(c, 4, 0, 1)
    assert 0 < lib.poss_kv_attend_scratch_bytes(c, 4, 5, 0) <= lib.poss_kv_attend_scratch_bytes(c, 4, 5, 1) <= need
    good = dict(cache=c, hq=4, q=A, q_row=256, out=2 * A, out_row=256, lengths=A, max_len=0, scale=0.125, lse=A, weights=A, weights_out=A, scratch=A, bytes=need)

    def call(**kw):
        return lib.poss_kv_attend(*{**good, **kw}.values(), None)
    for kw in (dict(hq=0), dict(hq=3), dict(hq=65536), dict(max_len=-1), dict(max_len=65), dict(scale=math.inf), dict(scale=math.nan), dict(weights_out=None), dict(q=None), dict(out=None), dict(lengths=None),
               dict(scratch=None), dict(q=A + 8), dict(out=A + 2), dict(q_row=260), dict(out_row=252), dict(q_row=248), dict(lengths=A + 1), dict(lse=A + 2), dict(weights=A + 1), dict(weights_out=A + 3),
               dict(scratch=A + 128)):
        assert call(**kw) == P.E_INVALID_ARG, kw
    assert call(bytes=need - 1) == P.E_CAPACITY
    assert call(cache=ctypes.byref(cache(n_seq=0)), q=None) == P.POSS_OK


def test_evict_refusals():
    lib = _lib()
    good = dict(cache=ctypes.byref(cache()), weights=A, positions=A, lengths=A, budget=8, first=2, recent=6, kept=A, weights_out=2 * A, positions_out=2 * A, lengths_out=2 * A)

    def call(**kw):
        return lib.poss_kv_evict(*{**good, **kw}.values(), None)
    for kw in (dict(budget=0), dict(budget=7), dict(first=-1), dict(recent=-1), dict(first=3), dict(weights=None), dict(positions=None), dict(lengths=None), dict(kept=None), dict(weights_out=None),
               dict(positions_out=None), dict(lengths_out=None), dict(weights_out=A), dict(positions_out=A), dict(lengths_out=A), dict(kept=A + 1), dict(weights=A + 2)):
        assert call(**kw) == P.E_INVALID_ARG, kw
    assert call(cache=ctypes.byref(cache(n_seq=0)), weights=None) == P.POSS_OK


def test_logprobs_refusals():
    lib = _lib()
    need = lib.poss_logprobs_scratch_bytes(3, 1000, 5)
    assert need > 0
    for bad in ((-1, 1000, 5), (3, 0, 0), (3, 1000, 33), (3, 4, 5), (3, 1000, -1), (3, (1 << 30) + 1, 1)):
        assert lib.poss_logprobs_scratch_bytes(*bad) == 0
    good = dict(t=1, x=A, ldx=1000, rows=3, vocab=1000, temperature=1.0, tokens=A, n_tokens=1, logp=A, entropy=A, n_top=5, ids=A, top=A, scratch=A, bytes=need)

    def call(**kw):
        return lib.poss_logprobs(*{**good, **kw}.values(), None)
    for kw in (dict(t=3), dict(rows=-1), dict(vocab=0), dict(ldx=999), dict(temperature=0.0), dict(temperature=-1.0), dict(temperature=math.inf), dict(temperature=math.nan), dict(temperature=1e-40), dict(n_tokens=-1), dict(n_top=33),
               dict(x=None), dict(tokens=None), dict(logp=None), dict(ids=None), dict(top=None), dict(scratch=None), dict(x=A + 1), dict(tokens=A + 2), dict(scratch=A + 64), dict(entropy=A + 2)):
        assert call(**kw) == P.E_INVALID_ARG, kw
    assert call(bytes=need - 1) == P.E_CAPACITY
    assert call(rows=0, x=None) == P.POSS_OK


def test_context_cache_refusals():
    assert _lib().poss_get_kv_cache(None, 0, -1, 0, None) == P.E_INVALID_ARG
