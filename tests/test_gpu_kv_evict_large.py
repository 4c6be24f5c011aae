"""poss_kv_evict where a launch moves fewer slots side by side than there are, up to the most that a sequence can have."""
import numpy as np
import pytest

from gpu_util import have_gpu

pytestmark = pytest.mark.gpu

if have_gpu():
    import torch
    import paper_2506_03566_amd as P
    from test_gpu_kv_evict import check, make, run


@pytest.mark.parametrize("t,hkv,dh,slots,budget", [("bf16", 1, 32, 300000, 280000), ("f32", 1, 96, 270000, 262145), ("f16", 2, 256, 263000, 262400), ("bf16", 1, 64, 600000, 540000)])
def test_more_slots_than_a_launch_moves_at_once(t, hkv, dh, slots, budget):
    print(f"evict {t} {slots} slots of {hkv} heads of {dh} to {budget}", flush=True)
    cache, table, rng = make(t, 1, slots, hkv, dh, 128, seed=slots)
    weights = rng.random(size=(1, hkv, cache.slots)).astype(np.float32)
    weights[:, :, budget - 300:budget] = 0.0                  # holes at the end, where a workgroup comes for the second time
    positions = np.broadcast_to(np.arange(cache.slots), weights.shape).astype(np.int32).copy()
    check(cache, table, weights, positions, np.array([slots], np.int32), budget, 4, 1000)


def test_a_small_cut_of_many_slots_moves_each_once():
    """Slots of three rounds of a workgroup, every one of them moved or none but one."""
    slots, budget = 800000, 600000
    cache, table, rng = make("bf16", 1, slots, 1, 32, 128, seed=3)
    weights = torch.ones(1, 1, cache.slots, device="cuda")
    weights[:, :, 100] = 0.0
    weights[:, :, budget:] = 0.5
    weights[:, :, 700001] = 2.0
    positions = torch.arange(cache.slots, device="cuda").int().expand(1, 1, -1).contiguous()
    k0, v0 = (x.clone() for x in cache.tensors[:2])
    kept, wo, po, lo = run(cache, weights.cpu().numpy(), positions.cpu().numpy(), np.array([slots], np.int32), budget, 0, 0)
    want = torch.arange(budget, device="cuda").int()
    want[100] = 700001
    assert torch.equal(kept[0, 0], want) and int(lo) == budget and float(wo[0, 0, 100]) == 2.0 and int(po[0, 0, 100]) == 700001
    pg = lambda s: (table[0, s // 128], s % 128)              # noqa: E731
    (fp, fs), (tp, ts) = pg(700001), pg(100)
    k0[tp, 0, ts], v0[tp, 0, :, ts] = k0[fp, 0, fs].clone(), v0[fp, 0, :, fs].clone()
    assert torch.equal(cache.tensors[0], k0) and torch.equal(cache.tensors[1], v0)


def test_the_most_slots_of_a_sequence():
    """2^30 slots of heads of 256, most of them without a page: one goes, and the last takes its place."""
    slots, page = 1 << 30, 128
    k, v = torch.randn(3, 1, page, 256, device="cuda").bfloat16(), torch.randn(3, 1, 256, page, device="cuda").bfloat16()
    table = torch.full((1, slots // page), -1, dtype=torch.int32, device="cuda")
    table[0, 0], table[0, -1], table[0, 1 << 22] = 2, 0, 1
    cache = P.KvCache(k, v, table)
    weights = torch.ones(1, 1, slots, device="cuda")
    weights[0, 0, 5] = 0.5
    positions = torch.arange(slots, dtype=torch.int32, device="cuda").view(1, 1, -1)
    kept, wo, po = torch.empty(1, 1, slots - 1, dtype=torch.int32, device="cuda"), torch.empty_like(weights), torch.empty_like(positions)
    lengths = torch.tensor([slots], dtype=torch.int32, device="cuda")
    lo = torch.empty_like(lengths)
    key, value = k[0, 0, page - 1].clone(), v[0, 0, :, page - 1].clone()
    k1, v1 = k.clone(), v.clone()
    print("2^30 slots to one less", flush=True)
    P.kv_evict(cache, weights, positions, lengths, slots - 1, kept, wo, po, lo)
    assert int(lo) == slots - 1 and int(kept[0, 0, 5]) == slots - 1 == int(po[0, 0, 5]) and float(wo[0, 0, 5]) == 1.0
    assert float(wo[0, 0, -1]) == 0.0 and int(po[0, 0, -1]) == -1
    kept[0, 0, 5] = po[0, 0, 5] = 5
    assert torch.equal(kept[0, 0], positions[0, 0, :-1]) and torch.equal(po[0, 0, :-1], positions[0, 0, :-1]) and bool((wo[0, 0, :-1] == 1).all())
    k1[2, 0, 5], v1[2, 0, :, 5] = key, value
    assert torch.equal(k, k1) and torch.equal(v, v1)
