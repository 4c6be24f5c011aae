"""poss_kv_attend over values that are not finite, against the definition in float64: sum p v with p = softmax > 0 wherever a score is above -infinity.  An infinite value gives an
infinity of its sign however small its probability; two of opposite signs, a NaN, or an infinite value at a score of -infinity (0 times it) give NaN.  It concerns its own dim
of its own sequence and key head: the other dims, the log of the sum and the weights are what they are without it.

Tolerance of what is finite: as tests/test_gpu_kv_attend.py derives it; sums are taken relative to another maximum where such values are, which that covers."""
import numpy as np
import pytest

from gpu_util import have_gpu

pytestmark = pytest.mark.gpu

if have_gpu():
    import torch
    from oracle import serving as o
    from test_gpu_kv_attend import Case, TYPES, f64


def put(c, b, h, slot, d, x):
    c.cache.tensors[1][c.table[b, slot // c.page], h, d, slot % c.page] = x


def check(c, odd, scale=None):
    """odd: (sequence, key head, slot, dim, value) to put among c's values."""
    scale = c.dh ** -0.5 if scale is None else scale
    before = torch.rand(c.n, c.hkv, c.slots, device="cuda")
    for b, h, slot, d, _ in odd:
        put(c, b, h, slot, d, 0.0)
    plain_w = before.clone()
    _, plain_lse = c.attend(weights_out=plain_w, scale=scale)
    for at in odd:
        put(c, *at)
    wo = before.clone()
    out, lse = c.attend(weights_out=wo, scale=scale)
    alone, lse2 = c.attend(scale=scale)
    assert torch.equal(lse, plain_lse) and torch.equal(wo, plain_w) and torch.equal(lse2, lse)
    again, _ = c.attend(scale=scale)
    assert torch.equal(alone.nan_to_num(7.0), again.nan_to_num(7.0)) and torch.equal(alone.isnan(), again.isnan())
    k, v, q = f64(c.cache.tensors[0]), f64(c.cache.tensors[1]), f64(c.q)
    half, tiny = torch.finfo(TYPES[c.t]).eps / 2, float(torch.finfo(TYPES[c.t]).smallest_normal) * torch.finfo(TYPES[c.t]).eps
    seen = dict(inf=0, nan=0)
    for b in range(c.n):
        n = int(c.lengths[b])
        if n <= 0:
            continue
        kk, vv = o.gather(k, c.table[b], n, c.page), o.gather(v, c.table[b], n, c.page, values=True)
        for h in range(c.hq):
            kh = h // (c.hq // c.hkv)
            with np.errstate(invalid="ignore"):
                s = kk[kh] @ q[b, h] * scale
                p = np.exp(s - s.max())
                p /= p.sum()
                want = (p[:, None] * vv[kh]).sum(axis=0)
            assert (p[s > -np.inf] > 0).all()
            live = np.where(np.isfinite(vv[kh]), vv[kh], 0.0)
            dots = np.abs(np.where(np.isfinite(kk[kh]), kk[kh], 0.0)) @ np.abs(q[b, h]) * abs(scale)
            delta = (c.dh + 16) * 2.0 ** -23 * dots.max() + 2.0 ** -21 * (np.abs(s[s > -np.inf]).max() + 1)
            for got in (f64(out)[b, h], f64(alone)[b, h]):
                assert np.array_equal(np.isnan(got), np.isnan(want)), (b, h, np.flatnonzero(np.isnan(got) != np.isnan(want))[:5])
                assert np.array_equal(got[np.isinf(want)], want[np.isinf(want)]), (b, h)
                ok = np.isfinite(want)
                bound = (2 * delta + (n + 64) * 2.0 ** -22 + 2.0 ** -16) * (p @ np.abs(live)) * (1 + half) + half * np.abs(np.where(ok, want, 0.0)) + tiny
                assert (np.abs(got[ok] - want[ok]) <= bound[ok]).all(), (b, h)
            seen["inf"] += int(np.isinf(want).sum())
            seen["nan"] += int(np.isnan(want).sum())
    return seen


INF, NAN = float("inf"), float("nan")
SHAPES = [  # lengths, hq, hkv, dh, page
    ([1, 2, 0, 33], 4, 2, 64, 32), ([70, 300], 8, 2, 128, 64), ([9000], 8, 2, 64, 128), ([700, 3, 1500], 5, 5, 96, 64), ([600, 31], 34, 2, 32, 32), ([500, 400], 4, 1, 160, 32), ([450, 90], 6, 3, 192, 64),
    ([300, 600], 4, 2, 256, 128), ([900], 3, 1, 224, 32), ([400, 3] * 20, 8, 2, 64, 32)]


@pytest.mark.parametrize("t", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("lengths,hq,hkv,dh,page", SHAPES)
def test_infinite_values_by_the_definition(t, lengths, hq, hkv, dh, page):
    print(f"infinite values {t} lengths {lengths[:6]} heads {hq}/{hkv} of {dh} page {page}", flush=True)
    c = Case(t, lengths, hq, hkv, dh, page, seed=sum(lengths) + dh)
    rng = np.random.default_rng(dh + len(lengths))
    odd = []
    for b, n in enumerate(lengths):
        if n == 0:
            continue
        at = lambda: int(rng.integers(n))                    # noqa: E731
        h = int(rng.integers(hkv))
        odd += [(b, h, at(), 0, INF), (b, h, at(), 1, -INF), (b, h, n - 1, 2, INF), (b, h, 0, 3, -INF), (b, h, at(), 4, NAN)]
        if n > 2:
            odd += [(b, h, 0, 5, INF), (b, h, n - 1, 5, -INF), (b, h, 0, 6, INF), (b, h, n // 2, 6, INF), (b, h, n - 1, 6, INF), (b, h, n // 3, 7, INF), (b, h, n // 2, 7, NAN)]
    seen = check(c, odd)
    assert seen["inf"] and seen["nan"]


@pytest.mark.parametrize("t", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("n", [1, 2, 32, 48, 256, 1000, 4096])
def test_equal_probabilities(t, n):
    """1 / n of each: a number of the type, or not."""
    c = Case(t, [n], 4, 2, 64, 64, seed=n)
    c.q.zero_()
    assert check(c, [(0, 0, 0, 3, INF), (0, 1, n - 1, 5, -INF), (0, 1, n // 2, 9, INF)])["inf"] == 6


@pytest.mark.parametrize("t", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("n", [60, 200, 3000])
def test_probabilities_that_float32_does_not_hold(t, n):
    """Slots 200 below the largest score, in its block and others, before and behind it: above zero all the same.  At a score of -infinity the probability is 0."""
    c = Case(t, [n, n], 2, 1, 64, 32, seed=n)
    k, v, table = c.cache.tensors
    c.q.zero_()
    c.q[:, :, 0] = 8.0
    k[:, :, :, 0] = torch.where(k[:, :, :, 0].isnan(), k[:, :, :, 0], torch.full_like(k[:, :, :, 0], -200.0))
    top = n // 2
    for b in range(2):
        k[c.table[b, top // 32], 0, top % 32, 0] = 0.0
    seen = check(c, [(0, 0, s, d, INF) for d, s in enumerate([0, 1, top - 1, top, top + 1, n - 1])] + [(1, 0, 0, 0, -INF), (1, 0, 1, 8, INF), (1, 0, n - 1, 8, -INF)])
    assert seen["inf"] == 14 and seen["nan"] == 2
    k[c.table[1, 0], 0, 5, 0] = -np.inf
    seen = check(c, [(1, 0, 5, 11, INF), (1, 0, 6, 12, INF)])
    assert seen["nan"] >= 2 and seen["inf"] >= 2


@pytest.mark.parametrize("t", ["bf16", "f16", "f32"])
def test_infinities_behind_the_length_and_in_other_heads(t):
    c = Case(t, [45, 20], 4, 2, 64, 32, seed=11)
    for b, h, slot in ((0, 0, 45), (0, 1, 63), (1, 0, 20), (1, 1, 31)):
        put(c, b, h, slot, 5, INF)
    assert check(c, []) == dict(inf=0, nan=0)
    assert check(c, [(0, 1, 44, 5, INF)]) == dict(inf=2, nan=0)


@pytest.mark.parametrize("t", ["bf16", "f32"])
def test_sums_beyond_float32_are_not_numbers(t):
    """Finite values whose sum float32 does not hold: infinity, or NaN of two, never a number; dims beside them as ever."""
    c = Case(t, [200], 2, 1, 64, 32, seed=12)
    c.q.zero_()
    for s in range(200):
        put(c, 0, 0, s, 3, 3e38)
        put(c, 0, 0, s, 4, 3e38 if s < 100 else -3e38)
    out, _ = c.attend()
    assert bool((out[0, :, 3] == INF).all()) and not bool(out[0, :, 4].isfinite().any()) and bool(out[0, :, 5:].isfinite().all())
