"""poss_kv_evict: what stays, where it lies and what is left alone, equal to the plain rule."""
import numpy as np
import pytest

from gpu_util import have_gpu

pytestmark = pytest.mark.gpu

if have_gpu():
    import torch
    import paper_2506_03566_amd as P
    from oracle import serving as o
    TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}


def make(t, n_seq, slots, hkv, dh, page, seed, holes=(), apart=0):
    rng = np.random.default_rng(seed)
    per = -(-slots // page)
    pages = n_seq * per + 2
    table = rng.permutation(pages)[:n_seq * per].reshape(n_seq, per).astype(np.int32)
    for b, j in holes:
        table[b, j] = -1

    def pool(a, b):
        size = hkv * a * b + apart
        p = torch.full((pages * size,), 5.0, dtype=TYPES[t], device="cuda").as_strided((pages, hkv, a, b), (size, a * b, b, 1))
        p.copy_(torch.randn(pages, hkv, a, b, generator=torch.Generator("cuda").manual_seed(seed), device="cuda"))
        return p
    return P.KvCache(pool(page, dh), pool(dh, page), torch.from_numpy(table).cuda()), table, rng


def run(cache, weights, positions, lengths, budget, first, recent):
    n, h, s = cache.n_seq, cache.heads, cache.slots
    kept = torch.full((n, h, budget), -9, dtype=torch.int32, device="cuda")
    wo, po = torch.full((n, h, s), 9.0, device="cuda"), torch.full((n, h, s), -9, dtype=torch.int32, device="cuda")
    lo = torch.full((n,), -9, dtype=torch.int32, device="cuda")
    dev = lambda a: torch.from_numpy(a).cuda()              # noqa: E731
    P.kv_evict(cache, dev(weights), dev(positions), dev(lengths), budget, kept, wo, po, lo, first=first, recent=recent)
    return kept, wo, po, lo


def check(cache, table, weights, positions, lengths, budget, first, recent):
    k0, v0 = cache.tensors[0].cpu().clone(), cache.tensors[1].cpu().clone()
    kept, wo, po, lo = (x.cpu().numpy() for x in run(cache, weights, positions, lengths, budget, first, recent))
    page, (n, hkv, slots) = k0.shape[2], weights.shape
    k1, v1 = k0.clone(), v0.clone()
    for b in range(n):
        left = min(max(int(lengths[b]), 0), slots, budget)
        assert lo[b] == left
        for h in range(hkv):
            want = o.evict(weights[b, h], positions[b, h], lengths[b], budget, first, recent)
            assert len(want) == left and kept[b, h, :left].tolist() == want and (kept[b, h, left:] == -1).all(), (b, h)
            at = np.array(want, np.int64)
            assert np.array_equal(wo[b, h, :left], weights[b, h][at], equal_nan=True) and not wo[b, h, left:].any()
            assert np.array_equal(po[b, h, :left], positions[b, h][at]) and (po[b, h, left:] == -1).all()
            to = np.flatnonzero(at != np.arange(left))
            fp, tp = table[b, at[to] // page], table[b, to // page]
            ok = (fp >= 0) & (tp >= 0)
            fp, tp, fs, ts = fp[ok], tp[ok], at[to][ok] % page, to[ok] % page
            k1[tp, h, ts] = k0[fp, h, fs]
            v1[tp, h, :, ts] = v0[fp, h, :, fs]
    assert torch.equal(cache.tensors[0].cpu(), k1) and torch.equal(cache.tensors[1].cpu(), v1)
    again = run(cache, weights, positions, lengths, budget, first, recent)      # nothing it reads has been written: the same once more
    assert np.array_equal(again[0].cpu().numpy(), kept)
    assert torch.equal(cache.tensors[0].cpu(), k1) and torch.equal(cache.tensors[1].cpu(), v1)


SHAPES = [  # n_seq, slots, lengths, hkv, dh, page, budget, first, recent
    (1, 32, [32], 1, 64, 32, 31, 0, 0), (1, 64, [33], 2, 64, 32, 32, 4, 16), (3, 100, [100, 0, 1], 2, 128, 64, 50, 0, 10), (2, 96, [96, 95], 3, 32, 32, 1, 0, 0), (2, 96, [96, 40], 1, 96, 32, 1, 0, 1),
    (1, 1025, [1025], 8, 128, 64, 1024, 4, 256), (4, 2000, [2000, 1999, 700, 1300], 2, 64, 128, 700, 4, 100), (1, 5000, [5000], 2, 128, 64, 4000, 0, 0), (2, 300, [300, 299], 2, 256, 32, 300, 0, 0),
    (2, 200, [500, -3], 2, 64, 32, 64, 60, 4), (1, 9000, [8888], 1, 64, 128, 100, 3, 90), (2, 200, [200, 150], 1, 160, 64, 1000, 5, 10), (1, 40000, [40000], 2, 32, 128, 20001, 4, 1000),
    (2, 3000, [3000, 2500], 2, 64, 64, 1500, 2, 100), (1, 1300, [1290], 2, 64, 32, 1289, 0, 1), (2, 8000, [8000, 10], 1, 32, 64, 7000, 9, 0), (1, 20000, [20000], 1, 32, 128, 19999, 0, 0),
    (1, 9000, [9000], 1, 32, 128, 8000, 0, 0), (2, 30000, [30000, 20000], 1, 32, 64, 15000, 10, 3000), (1, 70000, [66000], 1, 32, 128, 30000, 0, 500), (1, 12000, [12000], 2, 64, 64, 3, 1, 1)]


@pytest.mark.parametrize("t", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("n_seq,slots,lengths,hkv,dh,page,budget,first,recent", SHAPES)
def test_evict_is_the_plain_rule(t, n_seq, slots, lengths, hkv, dh, page, budget, first, recent):
    print(f"evict {t} {n_seq} seqs of {slots} lengths {lengths} heads {hkv} of {dh} page {page} budget {budget} first {first} recent {recent}", flush=True)
    cache, table, rng = make(t, n_seq, slots, hkv, dh, page, seed=slots + budget, apart=64 if page == 32 else 0)
    s = cache.slots
    weights = np.exp(rng.normal(size=(n_seq, hkv, s)) * 2).astype(np.float32)
    weights[rng.random(size=weights.shape) < 0.3] = 0.0       # equal ones
    weights = np.where(rng.random(size=weights.shape) < 0.3, np.round(weights), weights).astype(np.float32)
    positions = np.argsort(rng.random(size=weights.shape), axis=2).astype(np.int32) + 1000      # slots in no order of age
    positions[:, :, 3] = 1
    check(cache, table, weights, positions, np.array(lengths, np.int32), budget, first, recent)


@pytest.mark.parametrize("how", ["equal", "zero", "special", "rising", "falling", "near", "negative"])
@pytest.mark.parametrize("slots", [64, 1500, 5000, 20000])
def test_weights_of_every_kind(how, slots):
    print(f"evict weights {how} slots {slots}", flush=True)
    cache, table, rng = make("bf16", 1, slots, 2, 64, 32, seed=slots)
    s = cache.slots
    w = {"equal": np.full(s, 0.25), "zero": np.where(np.arange(s) % 2, 0.0, -0.0), "rising": np.arange(s) * 1e-3, "falling": -np.arange(s) * 1e-3,
         "near": 1 + np.arange(s)[::-1] % 7 * 2.0 ** -23, "negative": -rng.random(s),
         "special": rng.choice(np.array([np.nan, np.inf, -np.inf, 0.0, 1e-40, -1e-40, 3.4e38, 1.0]), size=s)}[how]
    weights = np.broadcast_to(w, (1, 2, s)).astype(np.float32).copy()
    weights[0, 1] = rng.permutation(weights[0, 1])
    positions = np.broadcast_to(np.arange(s), (1, 2, s)).astype(np.int32).copy()
    for budget, first, recent in ((slots // 2, 0, 0), (slots - 1, 5, 20), (slots // 3, 0, slots // 3)):
        check(cache, table, weights, positions, np.array([slots], np.int32), budget, first, recent)


def test_positions_at_the_ends_and_repeated():
    """Positions of any value; where more slots than the budget would always stay, the lowest of them do."""
    cache, table, rng = make("f32", 1, 96, 1, 32, 32, seed=1)
    weights = rng.random(size=(1, 1, 96)).astype(np.float32)
    for p in (np.full(96, 7), np.full(96, -2 ** 31), np.full(96, 2 ** 31 - 1), np.r_[np.full(48, -2 ** 31), np.full(48, 2 ** 31 - 1)], -np.arange(96)):
        check(cache, table, weights, p.astype(np.int32).reshape(1, 1, 96), np.array([90], np.int32), 40, 3, 30)


def test_slots_without_a_page_are_left_out():
    cache, table, rng = make("bf16", 2, 160, 2, 64, 32, seed=2, holes=[(0, 0), (1, 4), (1, 2)])
    weights = rng.random(size=(2, 2, 160)).astype(np.float32)
    positions = np.broadcast_to(np.arange(160), (2, 2, 160)).astype(np.int32).copy()
    check(cache, table, weights, positions, np.array([160, 150], np.int32), 70, 2, 8)


def test_refused_arguments():
    cache, _, _ = make("bf16", 2, 64, 2, 64, 32, seed=3)
    f, i, l = torch.zeros(2, 2, 64, device="cuda"), torch.zeros(2, 2, 64, dtype=torch.int32, device="cuda"), torch.zeros(2, dtype=torch.int32, device="cuda")
    good = dict(cache=cache, weights=f, positions=i, lengths=l, budget=32, kept=torch.zeros(2, 2, 32, dtype=torch.int32, device="cuda"), weights_out=f.clone(), positions_out=i.clone(), lengths_out=l.clone())
    P.kv_evict(**good)
    for kw in (dict(budget=33), dict(budget=0), dict(first=20, recent=13), dict(first=-1), dict(weights=f[:1]), dict(weights=f.double()), dict(positions=i.long()), dict(weights_out=f), dict(positions_out=i),
               dict(lengths_out=l), dict(kept=good["kept"][:, :1]), dict(lengths=l.cpu())):
        with pytest.raises(P.PossError):
            P.kv_evict(**{**good, **kw})
