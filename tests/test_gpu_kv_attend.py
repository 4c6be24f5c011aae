"""poss_kv_attend against float64 attention over the same pages.

Tolerance, for a row of n slots.  A score sums dim exact products (float32 caches: rounded ones): off by at most (dim + 16) half steps and as many truncations,
(dim + 16) * 2^-23 * scale * sum |q k|; its scaling, difference to the maximum and exponential by 2^-21 * (max |s| + 1).  Call that delta, the largest over the slots.  A probability
is off by 2 delta (numerator and sum) and the sums by (n + 64) * 2^-23 in any order; a bf16 probability enters the product with 16 bits.  So the output is off by
(2 delta + (n + 64) * 2^-22 + 2^-16) * sum p |v|, and half a step of its type."""
import numpy as np
import pytest

from gpu_util import have_gpu

pytestmark = pytest.mark.gpu

if have_gpu():
    import torch
    import paper_2506_03566_amd as P
    from oracle import serving as o
    TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}


def f64(t):
    return t.double().cpu().numpy()


class Case:
    def __init__(self, t, lengths, hq, hkv, dh, page, seed=0, loud=1.0, spare=3, slots=None, apart=0):
        rng = np.random.default_rng(seed)
        self.t, self.lengths, self.hq, self.hkv, self.dh, self.page = t, np.array(lengths, np.int32), hq, hkv, dh, page
        n = len(lengths)
        per = -(-max(slots or 0, 1, *lengths) // page)
        used = [-(-max(l, 0) // page) for l in lengths]
        pages = sum(used) + spare
        order = rng.permutation(pages).astype(np.int32)
        table = np.full((n, per), -1, np.int32)              # entries behind a sequence's last page are no pages
        i = 0
        for b in range(n):
            table[b, :used[b]] = order[i:i + used[b]]
            i += used[b]
        self.table = table

        def pool(a, b):
            size = hkv * a * b + apart
            p = torch.full((pages * size,), float("nan"), dtype=TYPES[t], device="cuda").as_strided((pages, hkv, a, b), (size, a * b, b, 1))
            return p
        k, v = pool(page, dh), pool(dh, page)
        kn, vn = rng.normal(size=(pages, hkv, page, dh)) * loud, rng.normal(size=(pages, hkv, dh, page))
        for b in range(n):                                   # what lies behind a length stays NaN
            for j in range(used[b]):
                live = min(page, self.lengths[b] - j * page)
                k[table[b, j], :, :live] = torch.from_numpy(kn[j + b, :, :live]).to(TYPES[t]).cuda()
                v[table[b, j], :, :, :live] = torch.from_numpy(vn[j + b, :, :, :live]).to(TYPES[t]).cuda()
        self.cache = P.KvCache(k, v, torch.from_numpy(table).cuda())
        self.q = torch.from_numpy(rng.normal(size=(n, hq, dh)) * loud).to(TYPES[t]).cuda()
        self.len_dev = torch.from_numpy(self.lengths).cuda()
        self.rng, self.n, self.slots = rng, n, per * page

    def attend(self, weights=None, **kw):
        out = torch.full((self.n, self.hq, self.dh), 9.0, dtype=TYPES[self.t], device="cuda")
        lse = torch.full((self.n, self.hq), 9.0, device="cuda")
        wo = kw.pop("weights_out", None)
        P.kv_attend(self.cache, self.q, kw.pop("lengths", self.len_dev), out, lse=lse, weights=weights, weights_out=wo, **kw)
        return out, lse

    def check(self, out, lse, scale, weights=None, weights_out=None, before=None, rows=None):
        k, v, _ = (f64(x) if x.is_floating_point() else None for x in self.cache.tensors)
        q, out, lse = f64(self.q), f64(out), f64(lse)
        half = torch.finfo(TYPES[self.t]).eps / 2
        tiny = float(torch.finfo(TYPES[self.t]).smallest_normal) * half * 2
        for b in range(self.n) if rows is None else rows:
            n = max(int(self.lengths[b]), 0)
            kk, vv = o.gather(k, self.table[b], n, self.page), o.gather(v, self.table[b], n, self.page, values=True)
            want, wl, p, s = o.attend(q[b], kk, vv, scale)
            if n == 0:
                assert not out[b].any() and (lse[b] == -np.inf).all()
            else:
                g = self.hq // self.hkv
                dots = np.stack([np.abs(kk[h // g]) @ np.abs(q[b, h]) for h in range(self.hq)]) * abs(scale)
                delta = ((self.dh + 16) * 2.0 ** -23 * dots.max(axis=1) + 2.0 ** -21 * (np.abs(s).max(axis=1) + 1))
                rel = 2 * delta + (n + 64) * 2.0 ** -22 + 2.0 ** -16
                mag = np.stack([p[h] @ np.abs(vv[h // g]) for h in range(self.hq)])
                bound = rel[:, None] * mag * (1 + half) + half * np.abs(want) + tiny
                err = np.abs(out[b] - want)
                assert (err <= bound).all(), (b, n, float((err / bound).max()), np.argwhere(~(err <= bound))[:3])
                assert (np.abs(lse[b] - wl) <= delta + (n + 64) * 2.0 ** -23 + 2.0 ** -22 * (1 + np.abs(wl))).all()
            if weights_out is not None:
                got = f64(weights_out[b])
                base = f64(weights[b])[:, :n] if weights is not None else 0.0
                if n:
                    share = p.reshape(self.hkv, -1, n)
                    wb = (rel.reshape(self.hkv, -1, 1) * share).sum(axis=1)
                    want_w = base + share.sum(axis=1)
                    assert (np.abs(got[:, :n] - want_w) <= wb + 2.0 ** -23 * np.abs(want_w) + 2.0 ** -120).all()
                assert np.array_equal(got[:, n:], f64(before[b])[:, n:])       # slots beyond the length: as they were


SHAPES = [  # lengths, hq, hkv, dh, page
    ([1], 1, 1, 64, 32), ([0], 4, 2, 64, 32), ([2], 8, 1, 128, 64), ([31, 32, 33], 4, 4, 64, 32), ([17], 32, 8, 128, 64), ([64, 0, 1, 63, 65, 128, 129], 8, 2, 128, 64), ([500, 1, 0, 700], 5, 5, 64, 128),
    ([255, 256, 257], 6, 2, 96, 32), ([1000], 16, 1, 128, 64), ([333, 90], 34, 2, 64, 32), ([4000, 3, 0, 1500, 2049], 8, 2, 128, 128), ([3000], 40, 40, 128, 64), ([700, 701], 8, 1, 256, 32),
    ([1, 2, 3, 4, 5] * 30, 4, 2, 32, 32), ([100, 1200], 48, 1, 160, 64), ([900], 9, 3, 192, 32), ([411, 60], 4, 2, 224, 128), ([9001], 8, 8, 64, 64),
    ([300, 5, 0, 129] * 20 + [4000], 16, 2, 64, 32), ([90, 40] * 100, 6, 3, 96, 64), ([200, 31], 40, 1, 64, 32), ([400, 3] * 20, 8, 2, 64, 32),
    ([255, 0, 256], 17, 1, 32, 128), ([512] * 40, 34, 2, 128, 64)]


@pytest.mark.parametrize("t", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("lengths,hq,hkv,dh,page", SHAPES)
def test_attention_and_weights(t, lengths, hq, hkv, dh, page):
    print(f"attend {t} lengths {lengths[:8]} heads {hq}/{hkv} of {dh} page {page}", flush=True)
    c = Case(t, lengths, hq, hkv, dh, page, seed=sum(lengths) + dh, apart=64 if page == 32 else 0)
    scale = dh ** -0.5
    out, lse = c.attend()
    c.check(out, lse, scale)
    before = torch.rand(c.n, hkv, c.slots, device="cuda")
    w = torch.rand(c.n, hkv, c.slots, device="cuda")
    wo = before.clone()
    out2, lse2 = c.attend(weights=w, weights_out=wo)
    c.check(out2, lse2, scale, w, wo, before)
    fresh = before.clone()
    c.attend(weights_out=fresh)                              # weights from nothing
    c.check(out2, lse2, scale, None, fresh, before)
    c.attend(weights=w, weights_out=w)                       # in place, the same sums
    live = torch.arange(c.slots, device="cuda") < c.len_dev[:, None, None]
    assert torch.equal(torch.where(live, w, 0), torch.where(live, wo, 0))


@pytest.mark.parametrize("t", ["bf16", "f16", "f32"])
def test_a_bound_on_the_lengths_changes_nothing_but_the_split(t):
    c = Case(t, [300, 7, 0, 299], 8, 2, 128, 64, seed=3, slots=4096)
    for most in (300, 301, 2000, 4096, 0):
        wo = torch.zeros(c.n, 2, c.slots, device="cuda")
        out, lse = c.attend(weights_out=wo, max_len=most)
        c.check(out, lse, 128 ** -0.5, None, wo, torch.zeros_like(wo))


@pytest.mark.parametrize("t", ["bf16", "f16", "f32"])
def test_loud_scores_scales_and_strides(t):
    c = Case(t, [600, 33], 8, 2, 64, 32, seed=4, loud=6.0)
    for scale in (0.125, 1.0, -0.3, 0.0):
        out, lse = c.attend(scale=scale)
        c.check(out, lse, scale)
    wide = torch.full((2, 3 * 8 * 64), float("nan"), dtype=TYPES[t], device="cuda")
    q = wide[:, 8 * 64:16 * 64].view(2, 8, 64)
    q.copy_(c.q)
    c.q = q                                                  # a part of a wider matrix, and one for the results
    room = torch.full((2, 5, 8, 64), 3.0, dtype=TYPES[t], device="cuda")
    lse = torch.empty(2, 8, device="cuda")
    P.kv_attend(c.cache, q, c.len_dev, room[:, 2], lse=lse)
    c.check(room[:, 2], lse, 0.125)
    assert bool((room[:, [0, 1, 3, 4]] == 3).all())


@pytest.mark.parametrize("t", ["bf16", "f16", "f32"])
def test_many_small_probabilities_beside_a_large_one(t):
    """Each 2^-15 to 2^-17 of the largest, together as much as it: what a 16-bit number cannot hold of one must not be lost of all."""
    n = 40000
    c = Case(t, [n], 2, 1, 64, 128, seed=8)
    k, v, _ = c.cache.tensors
    k[:] = torch.where(k.isnan(), k, 0)
    c.q[:] = 0
    c.q[:, :, 0] = 8.0
    k[:, :, :, 0] = torch.where(k[:, :, :, 0].isnan(), k[:, :, :, 0], -11.0 + torch.rand_like(k[:, :, :, 0].float()).mul_(0.5).to(TYPES[t]) - 0.25)
    k[c.table[0, 0], 0, 77, 0] = 0.0
    v[:] = torch.where(v.isnan(), v, v.abs() + 0.5)
    v[c.table[0, 0], 0, :, 77] = 0.0                         # the large one's value: the others' are the result
    wo = torch.zeros(1, 1, c.slots, device="cuda")
    out, lse = c.attend(weights_out=wo)
    c.check(out, lse, 0.125, None, wo, torch.zeros_like(wo))


@pytest.mark.parametrize("t", ["bf16", "f16", "f32"])
def test_pages_that_are_not_there_and_lengths_beyond_the_bound(t):
    """A row with such a slot is NaN, the others are as ever; nothing outside the pages is read."""
    c = Case(t, [200, 130, 64, 1], 4, 2, 64, 32, seed=5, slots=512)
    table = c.table.copy()
    table[0, 3] = -1
    table[2, 1] = 10 ** 6
    good = c.cache.tensors
    c.cache = P.KvCache(good[0], good[1], torch.from_numpy(table).cuda())
    wo = torch.zeros(4, 2, c.slots, device="cuda")
    out, lse = c.attend(weights_out=wo)
    assert bool(wo[0, :, :200].isnan().all()) and bool(wo[2, :, :64].isnan().all()) and not bool(wo[0, :, 200:].any()) and not bool(wo[[1, 3]].isnan().any())
    assert bool(out[[0, 2]].isnan().all()) and bool(lse[[0, 2]].isnan().all())
    c.check(out, lse, 0.125, rows=[1, 3])
    c.cache = P.KvCache(*good)
    lengths = torch.tensor([200, 513, -5, 2 ** 31 - 1], dtype=torch.int32, device="cuda")
    wo = torch.zeros(4, 2, c.slots, device="cuda")
    out, lse = c.attend(lengths=lengths, weights_out=wo)
    assert bool(out[[1, 3]].isnan().all()) and bool(lse[[1, 3]].isnan().all()) and not bool(out[2].any()) and bool((lse[2] == -np.inf).all())
    c.check(out, lse, 0.125, rows=[0])
    assert not bool(wo[1:].any()) and not bool(wo[0].isnan().any())
    out, lse = c.attend(lengths=torch.tensor([200, 129, 64, 1], dtype=torch.int32, device="cuda"), max_len=199)
    assert bool(out[0].isnan().all()) and not bool(out[1:].isnan().any())


@pytest.mark.parametrize("t", ["bf16", "f16", "f32"])
def test_special_keys_and_values(t):
    """Keys that give a score of -infinity take no weight; a NaN is a row's own affair."""
    c = Case(t, [70, 70, 70], 2, 1, 64, 32, seed=6)
    k, v, _ = c.cache.tensors
    q = c.q
    q[:, :, 0] = 1.0
    k[c.table[0, 1], 0, 5, 0] = -np.inf                      # slot 37 of row 0
    k[c.table[1, 0], 0, 9, 3] = np.nan
    v[c.table[2, 2], 0, 7, 2] = np.nan                       # slot 66 of row 2, one value
    wo = torch.zeros(3, 1, c.slots, device="cuda")
    out, lse = c.attend(weights_out=wo)
    assert bool(out[1].isnan().all()) and bool(lse[1].isnan().all())
    assert not bool(out[0].isnan().any()) and float(wo[0, 0, 37]) == 0.0
    assert bool(out[2, :, 7].isnan().all()) and not bool(out[2, :, 8:].isnan().any()) and not bool(out[2, :, :7].isnan().any()) and not bool(lse[2].isnan().any())
    k[c.table[0, 1], 0, 5, 0] = 0.0
    k[:, :, :, 0] = torch.where(k[:, :, :, 0].isnan(), k[:, :, :, 0], torch.full_like(k[:, :, :, 0], -np.inf))
    out, lse = c.attend()                                    # every score -infinity: no distribution
    assert bool(out[0].isnan().all()) and not bool((lse[0] > -np.inf).any())


def test_the_same_call_gives_the_same_bits_and_shared_pages_are_read():
    c = Case("bf16", [5000, 17, 0, 2500], 8, 2, 128, 64, seed=7)
    first = c.attend()
    for _ in range(3):
        again = c.attend()
        assert torch.equal(first[0], again[0]) and torch.equal(first[1], again[1])
    k, v, table = c.cache.tensors
    shared = P.KvCache(k, v, table[:1].expand(4, -1).contiguous())
    out, lse = torch.empty(4, 8, 128, dtype=torch.bfloat16, device="cuda"), torch.empty(4, 8, device="cuda")
    q = c.q[:1].expand(4, -1, -1).contiguous()
    P.kv_attend(shared, q, torch.full((4,), 5000, dtype=torch.int32, device="cuda"), out, lse=lse)
    c.q, c.lengths, c.table, c.n = q, np.full(4, 5000, np.int32), np.repeat(c.table[:1], 4, axis=0), 4
    c.check(out, lse, 128 ** -0.5)


def test_refused_arguments():
    c = Case("bf16", [40, 3], 4, 2, 64, 32)
    out = torch.empty_like(c.q)
    for kw in (dict(q=c.q[:, :3]), dict(q=c.q.half()), dict(out=out[:1]), dict(lengths=c.len_dev.long()), dict(lse=torch.zeros(2, 3, device="cuda")), dict(weights=torch.zeros(2, 2, 64, device="cuda")),
               dict(weights_out=torch.zeros(2, 2, 63, device="cuda")), dict(max_len=65), dict(scale=float("nan")), dict(scratch=torch.zeros(16, dtype=torch.uint8, device="cuda")), dict(lengths=c.len_dev.cpu())):
        with pytest.raises(P.PossError):
            P.kv_attend(**{"cache": c.cache, "q": c.q, "lengths": c.len_dev, "out": out, **kw})
    with pytest.raises(P.PossError):
        P.kv_attend_scratch(c.cache, 3)
