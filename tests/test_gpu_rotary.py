"""poss_rotary and poss_kv_append against the float64 rotation.

Tolerance.  The angle is formed in 64 bits and may be reduced to a quarter turn's half, rounded to float32 there (2^-25); sine and cosine within two half steps of their
own (2^-23), times the magnitude (2^-24), a product and a fused multiply-add (2^-24 of each term): 11 * 2^-25 of magnitude * (|a| + |b|), 12 allowed; then half a step
of the type (and half of its smallest step)."""
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


def assert_rotated(got, x, positions, w, interleaved, magnitude, inverse, t):
    want = o.rotate(x, positions, w, interleaved, magnitude, inverse)
    r = 2 * len(w)
    mag = np.abs(x).copy()
    a, b = (slice(0, r, 2), slice(1, r, 2)) if interleaved else (slice(0, r // 2), slice(r // 2, r))
    mag[..., a] = mag[..., b] = mag[..., a] + mag[..., b]
    fi = torch.finfo(TYPES[t])
    bound = 12 * 2.0 ** -25 * abs(magnitude) * mag * (1 + fi.eps) + fi.eps / 2 * np.abs(want) + fi.smallest_normal * fi.eps
    bound[..., r:] = 0
    err = np.abs(f64(got) - want)
    assert (err <= bound).all(), (float((err - bound).max()), np.argwhere(err > bound)[:3])


def rows(rng, n, h, d, t, pad=0, shift=0, head_pad=0):
    """[n, h, d] with rows and heads apart, off alignment by `shift` values, NaN between."""
    buf = torch.full((n * (h * (d + head_pad) + pad) + shift + 64,), float("nan"), dtype=TYPES[t], device="cuda")
    v = buf[shift:].as_strided((n, h, d), (h * (d + head_pad) + pad, d + head_pad, 1), shift)
    v.copy_(torch.from_numpy(rng.normal(size=(n, h, d)) * 3))
    return v, buf


@pytest.mark.parametrize("t", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("n,h,d,rot,pad,shift,head_pad", [(1, 1, 2, 2, 0, 0, 0), (1, 8, 128, 128, 0, 0, 0), (3, 5, 128, 96, 0, 0, 0), (2, 3, 64, 64, 8, 0, 0), (7, 2, 80, 20, 3, 1, 0), (130, 4, 96, 32, 0, 0, 32),
                                                          (5, 1, 256, 256, 0, 0, 0), (17, 3, 33, 16, 0, 0, 0), (1, 40, 128, 64, 0, 8, 0), (300, 1, 64, 2, 0, 0, 0), (2, 2, 300, 256, 1, 3, 5),
                                                          (200, 5, 64, 64, 8, 0, 0), (261, 3, 128, 96, 0, 0, 0), (300, 2, 256, 256, 0, 0, 0), (250, 4, 96, 32, 0, 0, 32), (220, 40, 128, 128, 0, 8, 0),
                                                          (220, 2, 64, 64, 1, 1, 0), (1001, 1, 32, 16, 0, 0, 0)])
def test_rotary_against_float64(t, interleaved, n, h, d, rot, pad, shift, head_pad):
    print(f"rotary {t} interleaved {interleaved} {n}x{h}x{d} rot {rot} pad {pad} shift {shift} head_pad {head_pad}", flush=True)
    rng = np.random.default_rng(n * 100 + d)
    x, buf = rows(rng, n, h, d, t, pad, shift, head_pad)
    positions = rng.integers(-2000, 200000, size=n).astype(np.int32)
    positions[0] = 0
    rope = P.Rope(rot, 500000.0, interleaved=interleaved, scaling="ramp" if rot > 4 else "none", factor=4.0, magnitude=1.2)
    pos = torch.from_numpy(positions).cuda()
    before = f64(x)
    for inverse in (False, True):
        out = P.rotary(x, pos, rope, inverse=inverse)
        assert_rotated(out, before, positions, np.array(rope.frequencies), interleaved, float(np.float32(1.2)), inverse, t)
        wide, wbuf = rows(rng, n, h, d, t, pad + 8, shift, head_pad)
        assert P.rotary(x, pos, rope, wide, inverse=inverse).data_ptr() == wide.data_ptr() and torch.equal(wide, out)
        assert int(wbuf.isnan().sum()) == wbuf.numel() - n * h * d          # nothing between the rows is written
    out = P.rotary(x, pos, rope)
    P.rotary(x, pos, rope, x)                                               # in place: the same bits
    assert torch.equal(x, out) and int(buf.isnan().sum()) == buf.numel() - n * h * d


def test_rotary_far_positions_and_empty_calls():
    rope = P.Rope(64)
    x = torch.randn(4, 2, 64, device="cuda")
    pos = np.array([2 ** 31 - 1, -2 ** 31, 10 ** 9, 10 ** 6], np.int32)
    got = P.rotary(x, torch.from_numpy(pos).cuda(), rope)
    want = o.rotate(f64(x), pos, np.array(rope.frequencies))
    assert np.abs(f64(got) - want).max() < 1e-5            # 2^31 half steps of 2^-53 add 2^-22 to the angle on either side
    assert P.rotary(x[:0], torch.zeros(0, dtype=torch.int32, device="cuda"), rope).shape == (0, 2, 64)
    for bad in (dict(x=x[..., ::2]), dict(positions=torch.zeros(4, device="cuda")), dict(positions=torch.zeros(3, dtype=torch.int32, device="cuda")), dict(out=x.half()), dict(out=x[:, :1]),
                dict(rope=P.Rope(128)), dict(positions=torch.zeros(4, dtype=torch.int32)), dict(x=x[0])):
        with pytest.raises(P.PossError):
            P.rotary(**{"x": x, "positions": torch.zeros(4, dtype=torch.int32, device="cuda"), "rope": rope, **bad})


def test_a_gradient_is_the_rotation_back():
    """The gradient of sum(g . rotary(x)) is rotary(g, inverse), against differences of the float64 rotation."""
    rng = np.random.default_rng(5)
    w = np.array(P.Rope(32, interleaved=True, magnitude=1.5).frequencies)
    x, g, pos = rng.normal(size=(3, 2, 40)), rng.normal(size=(3, 2, 40)), np.array([3, 500, 70000], np.int32)
    grad = P.rotary(torch.from_numpy(g).float().cuda(), torch.from_numpy(pos).cuda(), P.Rope(32, interleaved=True, magnitude=1.5), inverse=True)
    for i in [(0, 0, 0), (1, 1, 7), (2, 0, 31), (2, 1, 32), (0, 1, 39)]:
        step = np.zeros_like(x)
        step[i] = 0.5
        d = (g * (o.rotate(x + step, pos, w, True, 1.5) - o.rotate(x - step, pos, w, True, 1.5))).sum()
        assert abs(float(grad[i]) - d) < 1e-5


# ---------------------------------------------------------------- into the cache
def make_cache(rng, t, n_seq, per, hkv, dh, page, spare=2, apart=0):
    """Pages full of NaN, a shuffled table; with `apart`, pages lie further apart than they are large."""
    pages = n_seq * per + spare

    def pool(a, b):
        size = hkv * a * b + apart
        return torch.full((pages * size,), float("nan"), dtype=TYPES[t], device="cuda").as_strided((pages, hkv, a, b), (size, a * b, b, 1))
    k, v = pool(page, dh), pool(dh, page)
    table = torch.from_numpy(rng.permutation(pages)[:n_seq * per].reshape(n_seq, per).astype(np.int32)).cuda()
    return P.KvCache(k, v, table)


APPENDS = [  # n_seq, rows, hq, hkv, dh, page, kind of rows
    (1, 1, 4, 2, 64, 32, "decode"), (5, 5, 8, 8, 128, 64, "decode"), (2, 70, 2, 1, 96, 32, "prompt"), (1, 300, 8, 2, 128, 64, "prompt"), (3, 200, 5, 5, 64, 128, "prompt"), (2, 33, 7, 1, 256, 32, "any"),
    (4, 90, 3, 3, 32, 64, "any"), (1, 129, 0, 4, 160, 128, "prompt"), (3, 65, 16, 2, 224, 32, "offset"),
    (2, 260, 4, 3, 64, 32, "any"), (3, 400, 2, 2, 128, 64, "offset"), (210, 210, 4, 2, 96, 32, "decode"), (1, 700, 0, 1, 32, 128, "offset"), (5, 333, 6, 6, 160, 64, "prompt")]


@pytest.mark.parametrize("t", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("n_seq,rows_,hq,hkv,dh,page,how", APPENDS)
def test_append(t, interleaved, n_seq, rows_, hq, hkv, dh, page, how):
    print(f"append {t} interleaved {interleaved} {n_seq} seqs {rows_} rows {hq}/{hkv} heads of {dh} page {page} {how}", flush=True)
    rng = np.random.default_rng(rows_ * 7 + dh)
    per = -(-(rows_ + 20) // page) + 1
    cache = make_cache(rng, t, n_seq, per, hkv, dh, page, apart=64 if how == "any" else 0)
    slots_all = per * page
    if how == "decode":
        seq, slots = np.arange(rows_), rng.integers(0, slots_all, size=rows_)
    elif how == "any":                                     # rows in any order, each at a place of its own
        at = rng.permutation(n_seq * slots_all)[:rows_]
        seq, slots = at // slots_all, at % slots_all
    else:
        each = -(-rows_ // n_seq)
        seq, slots = np.arange(rows_) // each, np.arange(rows_) % each + (0 if how == "prompt" else 3)
    seq, slots = seq.astype(np.int32), slots.astype(np.int32)
    if rows_ > 4:
        slots[2], slots[4] = -1, slots_all                 # padding, and one past the end
    if rows_ > 40:
        slots[30] = -2 ** 31
        if how != "decode":
            seq[17], seq[18] = -1, n_seq
    table = cache.tensors[2]
    if how == "any":
        table[0, 1] = -1                                   # pages that are not there
        table[n_seq - 1, 0] = 1 << 20
    positions = rng.integers(0, 100000, size=rows_).astype(np.int32)
    rot = dh if dh % 64 else dh // 2
    rope = P.Rope(rot, interleaved=interleaved, magnitude=0.75)
    wide = torch.from_numpy(rng.normal(size=(rows_, (hq + 2 * hkv) * dh + (8 if how == "any" else 0))).astype(np.float32)).to(TYPES[t]).cuda()
    q, k, v = (p.reshape(rows_, -1, dh) if p.shape[1] == 0 else p.view(rows_, -1, dh) for p in wide[:, :(hq + 2 * hkv) * dh].split([hq * dh, hkv * dh, hkv * dh], dim=1))
    noted = torch.full((n_seq, hkv, slots_all), -7, dtype=torch.int32, device="cuda")
    q_out = torch.empty(rows_, hq, dh, dtype=TYPES[t], device="cuda") if hq else None
    dev = lambda a: torch.from_numpy(a).cuda()              # noqa: E731
    seq_arg = None if how == "decode" else dev(seq)
    P.kv_append(cache, k, v, dev(slots), dev(positions), rope, seq=seq_arg, q=q if hq else None, q_out=q_out, slot_positions=noted)
    w = np.array(rope.frequencies)
    if hq:
        assert_rotated(q_out, f64(q), positions, w, interleaved, 0.75, False, t)
    ck, cv, tab, got_noted = cache.tensors[0].cpu(), cache.tensors[1].cpu(), table.cpu().numpy(), noted.cpu().numpy()
    want_noted, written = np.full_like(got_noted, -7), 0
    for r in range(rows_):
        b, s = seq[r], slots[r]
        if not (0 <= b < n_seq and 0 <= s < slots_all) or not 0 <= tab[b, s // page] < ck.shape[0]:
            continue
        pg = tab[b, s // page]
        assert_rotated(ck[pg, :, s % page][None], f64(k[r:r + 1]), positions[r:r + 1], w, interleaved, 0.75, False, t)
        assert torch.equal(cv[pg, :, :, s % page], v[r].cpu())
        want_noted[b, :, s] = positions[r]
        written += 1
    assert np.array_equal(got_noted, want_noted)
    assert int((~ck.isnan()).sum()) == int((~cv.isnan()).sum()) == written * hkv * dh
    # without a rope: as they are; queries in place
    plain = make_cache(np.random.default_rng(1), t, n_seq, per, hkv, dh, page)
    q2 = q.clone() if hq else None
    P.kv_append(plain, k, v, dev(slots), seq=seq_arg, q=q2)
    if hq:
        assert torch.equal(q2, q)
        P.kv_append(plain, k, v, dev(slots), dev(positions), rope, seq=seq_arg, q=q2)
        assert torch.equal(q2, q_out)
        P.kv_append(plain, k, v, dev(slots), seq=seq_arg)
    pk, ptab = plain.tensors[0].cpu(), plain.tensors[2].cpu().numpy()
    for r in range(rows_):
        if 0 <= seq[r] < n_seq and 0 <= slots[r] < slots_all:
            assert torch.equal(pk[ptab[seq[r], slots[r] // page], :, slots[r] % page], k[r].cpu())


def test_append_of_nothing_and_refused_arguments():
    rng = np.random.default_rng(0)
    c = make_cache(rng, "bf16", 2, 2, 2, 64, 32)
    k = torch.zeros(3, 2, 64, dtype=torch.bfloat16, device="cuda")
    s = torch.zeros(3, dtype=torch.int32, device="cuda")
    P.kv_append(c, k[:0], k[:0], s[:0])
    for kw in (dict(k=k.half()), dict(v=k[:2]), dict(slots=s.long()), dict(slots=s[:2]), dict(rope=P.Rope(64)), dict(rope=P.Rope(128), positions=s), dict(seq=s[:1]), dict(q=k[:, :, :32]),
               dict(slot_positions=torch.zeros(2, 2, 60, dtype=torch.int32, device="cuda"), positions=s), dict(k=k.transpose(1, 2)), dict(slots=s.cpu())):
        with pytest.raises(P.PossError):
            P.kv_append(**{"cache": c, "k": k, "v": k, "slots": s, **kw})
    pool = torch.zeros(4, 2, 32, 64, device="cuda")
    vals = torch.zeros(4, 2, 64, 32, device="cuda")
    table = torch.zeros(1, 2, dtype=torch.int32, device="cuda")
    P.KvCache(pool, vals, table)
    for bad in ((pool.half(), vals, table), (pool, vals.transpose(2, 3), table), (pool, pool, table), (pool, vals, table.long()), (pool, vals, table[0]), (pool, vals.cpu(), table)):
        with pytest.raises(P.PossError):
            P.KvCache(*bad)
