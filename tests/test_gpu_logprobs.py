"""poss_logprobs against float64.

Tolerance.  z = x / T may be formed with the rounded reciprocal: 2^-23 |z|; d = z - m: 2^-24 |d| more; an exponential 2^-22; a sum of V terms in chains of V / 256 and a tree:
(V / 256 + 64) * 2^-24.  So the sum of exponentials is off by r = sum p (|z| + |d|) * 2^-23 + 2^-22 + (V / 256 + 64) * 2^-24 of itself, a log-probability by
r + 2^-22 (|z| + |lse| + 1), the entropy by r + 2^-22 (log S + 1) + sum p |d| (2 r + 2^-21) + sum p (|z| + |d|) 2^-23."""
import numpy as np
import pytest

from gpu_util import have_gpu

pytestmark = pytest.mark.gpu

if have_gpu():
    import torch
    import paper_2506_03566_amd as P
    from oracle import serving as o
    TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}


def check(x, tokens, n_top, temperature, got):
    xs = x.double().cpu().numpy()
    rows, V = xs.shape
    logp, entropy, ids, top = (g.cpu().numpy().astype(np.float64) if g is not None else None for g in got)
    lp, h = o.logprobs(xs, temperature)
    lp[lp < -float(torch.finfo(torch.float32).max)] = -np.inf          # what float32 cannot hold is rounded to that
    with np.errstate(all="ignore"):
        z = xs / temperature
        m = z.max(axis=1, keepdims=True)
        d, p = z - m, np.exp(lp)
        lse = (z - lp)[np.arange(rows), np.argmax(z, axis=1)]
        spread = np.where(p > 0, p * (np.abs(z) + np.abs(d)), 0).sum(axis=1)
        r = spread * 2.0 ** -23 + 2.0 ** -22 + (V / 256 + 64) * 2.0 ** -24
        tol = (r + 2.0 ** -22 * (np.abs(lse) + 1))[:, None] + 2.0 ** -22 * np.where(np.isfinite(z), np.abs(z), 0)
        pd = np.where(p > 0, p * np.abs(d), 0).sum(axis=1)
        tol_h = r + 2.0 ** -22 * (np.abs(lse - m[:, 0]) + 1) + pd * (2 * r + 2.0 ** -21) + spread * 2.0 ** -23

    def near(a, b, tol):
        assert np.array_equal(np.isnan(a), np.isnan(b)), (a[np.isnan(a) != np.isnan(b)][:3], b[np.isnan(a) != np.isnan(b)][:3])
        inf = np.isinf(b)
        assert np.array_equal(a[inf], b[inf])
        ok = np.isfinite(b)
        err = np.abs(a - np.where(ok, b, 0))
        assert (err[ok] <= np.broadcast_to(tol, b.shape)[ok]).all(), float((err[ok] / np.broadcast_to(tol, b.shape)[ok]).max())
    near(entropy, h, tol_h)
    if tokens is not None:
        tk = tokens.cpu().numpy().reshape(rows, -1)
        there = (tk >= 0) & (tk < V)
        at = np.where(there, tk, 0)
        near(logp.reshape(rows, -1), np.where(there, np.take_along_axis(lp, at, 1), np.nan), np.take_along_axis(np.broadcast_to(tol, lp.shape), at, 1))
    if n_top:
        want = np.array([o.best(row, n_top) for row in xs])
        assert np.array_equal(ids, want), (np.argwhere(ids != want)[:3], ids[ids != want][:3], want[ids != want][:3])
        near(top, np.take_along_axis(lp, want, 1), np.take_along_axis(np.broadcast_to(tol, lp.shape), want, 1))
    else:
        assert ids.shape == (rows, 0)


def logits(rng, rows, V, t, pad=0, shift=0):
    """Rows of noise over [rows, V] with loud ids, forbidden ones and equal ones; `pad` values between rows that hold NaN."""
    x = rng.normal(size=(rows, V)) * 2
    x[:, rng.integers(0, V, size=max(1, V // 60))] = -np.inf
    x[:, rng.integers(0, V, size=max(1, V // 200))] += 9
    x[0] = np.round(x[0])                                    # equal ones
    buf = torch.full((rows * (V + pad) + shift + 8,), float("nan"), dtype=TYPES[t], device="cuda")
    v = buf[shift:shift + rows * (V + pad)].view(rows, V + pad)[:, :V]
    v.copy_(torch.from_numpy(x))
    return v


SHAPES = [(1, 1, 0, 0), (1, 2, 0, 0), (2, 3, 1, 1), (1, 63, 0, 0), (5, 64, 0, 0), (3, 65, 0, 3), (7, 1000, 24, 0), (61, 4096, 0, 0), (4, 4097, 0, 0), (3, 32000, 0, 0), (2, 32003, 0, 1), (1, 128256, 0, 0), (9, 50001, 7, 0),
          (300, 513, 0, 0), (2, 128256, 8, 8), (1, 200000, 0, 0)]


@pytest.mark.parametrize("t", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("rows,V,pad,shift", SHAPES)
def test_logprobs_against_float64(t, rows, V, pad, shift):
    rng = np.random.default_rng(rows * 31 + V)
    x = logits(rng, rows, V, t, pad, shift)
    for n_top, n_tokens, temperature in ((min(5, V), 1, 1.0), (min(32, V), 10, 0.7), (0, 3, 1.9), (min(1, V), 0, 1.0)):
        print(f"logprobs {t} {rows}x{V} pad {pad} shift {shift} top {n_top} tokens {n_tokens} temperature {temperature}", flush=True)
        tokens = torch.from_numpy(rng.integers(0, V, size=(rows, n_tokens) if n_tokens != 1 else rows).astype(np.int32)).cuda() if n_tokens else None
        if n_tokens == 10:
            tokens[0, 3], tokens[-1, 4], tokens[0, 5] = -1, V, -2 ** 31
        got = P.logprobs(x, tokens, n_top=n_top, temperature=temperature)
        assert (got[0] is None) == (tokens is None)
        check(x, tokens, n_top, temperature, got)


@pytest.mark.parametrize("t", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("V", [40, 2049, 33000])
def test_rows_of_every_kind(t, V):
    """Equal logits, rising and falling ones (every value a new best), the types' largest, and rows without a distribution."""
    print(f"logprobs kinds {t} {V}", flush=True)
    big = float(torch.finfo(TYPES[t]).max)
    rng = np.random.default_rng(V)
    ramp = np.arange(V) * 2.0 ** -6
    forbidden = np.full(V, -np.inf)
    one = forbidden.copy(); one[V // 2] = -3.0                     # noqa: E702
    few = forbidden.copy(); few[[1, V - 1]] = 2.0                  # noqa: E702
    nan, inf, nans = rng.normal(size=V), rng.normal(size=V), np.full(V, np.nan)
    nan[V // 3], inf[V // 4], nans[[3, V - 2]] = np.nan, np.inf, 1.0
    lowest = np.where(rng.random(V) < 0.5, -big, rng.normal(size=V))       # forbidden by the type's lowest value
    x = np.stack([np.zeros(V), ramp, -ramp, ramp[::-1] % 3, np.full(V, big), np.full(V, -big), lowest, one, few, forbidden, nan, inf, nans, np.full(V, np.nan), rng.normal(size=V) * 1e-6, rng.normal(size=V) * 60])
    x = torch.from_numpy(x).to(TYPES[t]).cuda()
    tokens = torch.from_numpy(rng.integers(0, V, size=(len(x), 4)).astype(np.int32)).cuda()
    for n_top in (32, 1):
        check(x, tokens, n_top, 1.0, P.logprobs(x, tokens, n_top=n_top))
    for temperature in (0.5, 2.0):
        check(x, None, 20, temperature, P.logprobs(x, n_top=20, temperature=temperature))


@pytest.mark.parametrize("t", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("rows,V", [(1100, 9000), (1300, 4103), (500, 13001)])
def test_many_rows_of_several_tiles(t, rows, V):
    """One workgroup, or two, walk a row tile by tile; the best against a stable sort."""
    print(f"logprobs tiles {t} {rows}x{V}", flush=True)
    x = logits(np.random.default_rng(rows), rows, V, t)
    logp, entropy, ids, top = (g.cpu().numpy() for g in P.logprobs(x, torch.zeros(rows, dtype=torch.int32, device="cuda"), n_top=7))
    xs = x.double().cpu().numpy()
    want = np.argsort(-xs, axis=1, kind="stable")[:, :7]
    assert np.array_equal(ids, want)
    lp, h = o.logprobs(xs)
    r = 2.0 ** -22 * 40 + (V / 256 + 64) * 2.0 ** -24          # magnitudes of z, d and lse here are below 20
    assert np.abs(top - np.take_along_axis(lp, want, 1)).max() <= r and np.abs(entropy - h).max() <= 8 * r
    fine = np.isfinite(lp[:, 0])
    assert np.array_equal(logp[~fine], lp[~fine, 0]) and np.abs(logp[fine] - lp[fine, 0]).max() <= r


def test_many_rows_and_given_outputs():
    rng = np.random.default_rng(3)
    x = logits(rng, 700, 3001, "bf16")
    tokens = torch.from_numpy(rng.integers(0, 3001, size=700).astype(np.int32)).cuda()
    outs = dict(logp=torch.empty(700, device="cuda"), entropy=torch.empty(700, device="cuda"), top_ids=torch.empty(700, 2, dtype=torch.int32, device="cuda"), top_logp=torch.empty(700, 2, device="cuda"))
    scratch = P.logprobs_scratch(700, 3001, 2)
    got = P.logprobs(x, tokens, n_top=2, scratch=scratch, **outs)
    assert all(g is outs[n] for g, n in zip(got, outs))
    check(x, tokens, 2, 1.0, got)
    first = [g.clone() for g in got]
    P.logprobs(x, tokens, n_top=2, scratch=scratch, **outs)
    assert all(torch.equal(a, b) for a, b in zip(first, got))
    assert P.logprobs(x[:0], n_top=2)[2].shape == (0, 2)


def test_refused_arguments():
    x = torch.zeros(3, 100, device="cuda")
    tk = torch.zeros(3, dtype=torch.int32, device="cuda")
    P.logprobs(x, tk)
    for kw in (dict(logits=x[0]), dict(logits=x.double()), dict(logits=x.t()), dict(tokens=tk.long()), dict(tokens=tk[:2]), dict(n_top=33), dict(n_top=-1), dict(temperature=0.0), dict(temperature=float("inf")),
               dict(entropy=torch.zeros(2, device="cuda")), dict(top_ids=torch.zeros(3, 1, device="cuda"), n_top=1), dict(scratch=torch.zeros(8, dtype=torch.uint8, device="cuda")), dict(tokens=tk.cpu())):
        with pytest.raises(P.PossError):
            P.logprobs(**{"logits": x, "tokens": tk, **kw})
