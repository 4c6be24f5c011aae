"""Rotation of many rows, alone and into a cache, against float64 where a wave takes whole pieces: heads of a single unit and of a few, rows on both sides of a wave each and past the last whole
workgroup, heads that lie apart or in another order, parts of wider heads, in place.

Tolerance.  The angle is the float64 product that the oracle forms too; cosine and sine, times the magnitude, are rounded once to float32 (half a step, 2^-24, each), the product b sin
once (2^-24 of it) and the fused multiply-add once (2^-24 of the result): 3 * 2^-24 * magnitude * (|a| + |b|), a thousandth more for products of these errors and for the sines' own in 64 bits.
Then half a step of the type, of a value that may be off by as much, and half of its smallest step (float32: the multiply-add was the rounding)."""
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


def assert_rotated(got, x, positions, rope, inverse, t):
    w, interleaved, magnitude = np.array(rope.frequencies), bool(rope.c.interleaved), float(rope.c.magnitude)
    want = o.rotate(x, positions, w, interleaved, magnitude, inverse)
    r = 2 * len(w)
    a, b = (slice(0, r, 2), slice(1, r, 2)) if interleaved else (slice(0, r // 2), slice(r // 2, r))
    pair = np.zeros_like(x)
    pair[..., a] = pair[..., b] = np.abs(x[..., a]) + np.abs(x[..., b])
    bound = 3.003 * 2.0 ** -24 * magnitude * pair
    if t != "f32":
        fi = torch.finfo(TYPES[t])
        bound = bound * (1 + fi.eps) + fi.eps / 2 * np.abs(want) + fi.smallest_normal * fi.eps / 2
    bound[..., r:] = 0
    err = np.abs(f64(got) - want)
    assert (err <= bound).all(), (float((err - bound).max()), np.argwhere(~(err <= bound))[:3])


def rows_of(rng, n, h, d, t, how):
    """[n, h, d] in a buffer of NaN: "plain", with heads and rows "apart", heads outermost ("turned"), or the first d of heads of 64 ("part")."""
    apart = {"plain": (h * d, d), "apart": (h * (d + 16) + 32, d + 16), "turned": (d, n * d + 48), "part": (h * 64, 64)}[how]
    buf = torch.full(((n - 1) * apart[0] + (h - 1) * apart[1] + max(d, 64),), float("nan"), dtype=TYPES[t], device="cuda")
    v = buf.as_strided((n, h, d), (*apart, 1))
    v.copy_(torch.from_numpy(rng.normal(size=(n, h, d)) * 3))
    return v, buf


SIZES = [(16, 16), (8, 8), (4, 4), (8, 4), (16, 8), (32, 16), (64, 64), (128, 96), (48, 48)]


@pytest.mark.parametrize("t", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("dh,rot", SIZES)
def test_rows_of_small_heads(t, interleaved, dh, rot):
    rope = P.Rope(rot, 10000.0, interleaved=interleaved, magnitude=1.25)
    for n, h in ((200, 2), (199, 3), (203, 9), (2047, 2), (2048, 3), (2100, 2), (2049, 1), (2050, 5), (200, 130)):
        for how in ("plain", "apart", "turned", "part"):
            if how == "part" and dh >= 64:
                continue
            print(f"rotary {t} interleaved {interleaved} {n}x{h}x{dh} rot {rot} {how}", flush=True)
            rng = np.random.default_rng(n * 10 + h)
            x, buf = rows_of(rng, n, h, dh, t, how)
            positions = rng.integers(-2000, 200000, size=n).astype(np.int32)
            pos, before = torch.from_numpy(positions).cuda(), f64(x)
            inverse = h % 2 == 0
            out, obuf = rows_of(rng, n, h, dh, t, how)
            P.rotary(x, pos, rope, out, inverse=inverse)
            assert_rotated(out, before, positions, rope, inverse, t)
            assert int(obuf.isnan().sum()) == obuf.numel() - n * h * dh and torch.equal(x.double().cpu(), torch.from_numpy(before))
            P.rotary(x, pos, rope, x, inverse=inverse)       # in place: the same bits
            assert torch.equal(x, out) and int(buf.isnan().sum()) == buf.numel() - n * h * dh


@pytest.mark.parametrize("t", ["f32", "bf16", "f16"])
def test_a_row_does_not_depend_on_how_many_there_are(t):
    """The same row alone, among 199, 200, 2047 and 2048."""
    for dh, rot, interleaved in ((16, 16, False), (8, 8, True), (128, 64, False), (96, 96, True)):
        rope = P.Rope(rot, interleaved=interleaved)
        x = torch.randn(2500, 4, dh, generator=torch.Generator("cuda").manual_seed(dh), device="cuda").to(TYPES[t])
        pos = (torch.arange(2500, device="cuda") * 37 % 5000).int()
        whole = P.rotary(x, pos, rope)
        for n in (1, 199, 200, 2047, 2048):
            assert torch.equal(P.rotary(x[:n], pos[:n], rope), whole[:n]), (dh, n)


@pytest.mark.parametrize("t", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("rows,n_seq,first", [(2047, 1, 0), (2048, 1, 5), (2049, 3, 0), (2051, 2, 3), (2600, 2600, 0)])
def test_append_of_many_rows(t, rows, n_seq, first):
    """On both sides of a wave a row, with rows past the last whole workgroup: what is where, and nothing elsewhere."""
    print(f"append {t} {rows} rows of {n_seq} sequences from slot {first}", flush=True)
    rng = np.random.default_rng(rows)
    hq, hkv, dh, page = 3, 2, 32, 32
    each = -(-rows // n_seq)
    per = -(-(each + first) // page)
    pages = n_seq * per
    k, v = (torch.full((pages, hkv, *s), float("nan"), dtype=TYPES[t], device="cuda") for s in ((page, dh), (dh, page)))
    table = rng.permutation(pages).reshape(n_seq, per).astype(np.int32)
    cache = P.KvCache(k, v, torch.from_numpy(table).cuda())
    seq, slots = (np.arange(rows) // each).astype(np.int32), (np.arange(rows) % each + first).astype(np.int32)
    slots[11] = -1
    positions = rng.integers(0, 100000, size=rows).astype(np.int32)
    rope = P.Rope(dh, magnitude=0.75)
    q, kn, vn = torch.from_numpy(rng.normal(size=(rows, hq + 2 * hkv, dh))).to(TYPES[t]).cuda().split([hq, hkv, hkv], dim=1)
    q_out = torch.empty(rows, hq, dh, dtype=TYPES[t], device="cuda")
    P.kv_append(cache, kn, vn, torch.from_numpy(slots).cuda(), torch.from_numpy(positions).cuda(), rope, seq=torch.from_numpy(seq).cuda(), q=q, q_out=q_out)
    assert_rotated(q_out, f64(q), positions, rope, False, t)
    there = np.flatnonzero(slots >= 0)
    pg, at = torch.from_numpy(table[seq[there], slots[there] // page].astype(np.int64)).cuda(), torch.from_numpy(slots[there].astype(np.int64) % page).cuda()
    assert_rotated(k[pg, :, at], f64(kn)[there], positions[there], rope, False, t)
    assert torch.equal(v[pg, :, :, at], vn[torch.from_numpy(there).cuda()])
    assert int((~k.isnan()).sum()) == int((~v.isnan()).sum()) == len(there) * hkv * dh
