"""poss_kv_attend where key heads, in tiles of sixteen query heads, are more than a launch's workgroups: one of them takes the whole batch of its tile, row after row."""
import pytest

from gpu_util import have_gpu

pytestmark = pytest.mark.gpu

if have_gpu():
    import torch
    from test_gpu_kv_attend import Case


@pytest.mark.parametrize("t,lengths,hq,hkv,dh,page", [("bf16", [520, 3, 0, 513], 513, 513, 32, 32), ("f32", [0, 520, 33], 513, 513, 32, 128), ("f16", [600, 1], 257 * 17, 257, 32, 64),
                                                      ("bf16", [530, 40], 130 * 17, 130, 192, 64), ("f32", [513, 0, 1], 257, 257, 128, 32)])
def test_more_tiles_than_workgroups(t, lengths, hq, hkv, dh, page):
    print(f"attend {t} lengths {lengths} heads {hq}/{hkv} of {dh}", flush=True)
    c = Case(t, lengths, hq, hkv, dh, page, seed=hkv)
    out, lse = c.attend()
    c.check(out, lse, dh ** -0.5)
    before = torch.rand(c.n, hkv, c.slots, device="cuda")
    wo = before.clone()
    out, lse = c.attend(weights_out=wo)
    c.check(out, lse, dh ** -0.5, None, wo, before)
