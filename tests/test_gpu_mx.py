"""Microscaled 4-bit quantisation and products against the float64 oracle, through the C ABI.

Tolerances.  Codes, scales and float32 / bfloat16 values: equal.  A product: every term is exact, so what differs is the order and the
rounding of K float32 additions (matrix instruction, K splits); a sum of n terms is off by at most n half steps of the sum of
magnitudes, and an adder that truncates by whole steps: (K + 16) * 2^-23 * sum |x w|, and half a step of the type for the result."""
import numpy as np
import pytest

from gpu_util import have_gpu

pytestmark = pytest.mark.gpu

if have_gpu():
    import torch
    import paper_2506_03566_amd as P
    from oracle import mx
    TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}


def rows_of(rng, M, K, t, pad=0, shift=0):
    """[M, K] of type t: noise over many powers of two with loud channels, rows `pad` values apart, `shift` values off alignment."""
    x = rng.normal(size=(M, K)) * np.exp2(rng.integers(-6, 5, size=(M, 1)))
    x[:, rng.integers(0, K, size=max(1, K // 50))] *= 32
    buf = torch.full((M * (K + pad) + shift + 8,), float("nan"), dtype=TYPES[t], device="cuda")
    v = buf[shift:shift + M * (K + pad)].view(M, K + pad)[:, :K]
    v.copy_(torch.from_numpy(x))
    return v


def f64(t):
    return t.double().cpu().numpy()


def weights(rng, N, K, spread=0):
    w = rng.normal(size=(N, K)) * 0.02
    if spread:
        w *= np.exp2(rng.integers(-spread, 1, size=(N, -(-K // 32))).astype(float)).repeat(32, axis=1)[:, :K]
    codes, scales = mx.quantize(w)
    return mx.dequantize(codes, scales, K), P.mx_pack(torch.from_numpy(codes).cuda(), torch.from_numpy(scales).cuda(), K)


def half_step(t):
    return torch.finfo(TYPES[t]).eps / 2


def assert_product(y, x, w, t):
    """y against x w^T within the derived bound; a NaN has to be one on both sides."""
    with np.errstate(invalid="ignore"):
        ref, mag = x @ w.T, np.abs(x) @ np.abs(w).T
    got = f64(y)
    assert np.array_equal(np.isnan(got), np.isnan(ref))
    fine = np.isfinite(ref)
    assert np.array_equal(got[~fine & ~np.isnan(ref)], ref[~fine & ~np.isnan(ref)])
    bound = (x.shape[1] + 16) * 2.0 ** -23 * mag[fine] * (1 + half_step(t)) + half_step(t) * np.abs(ref[fine]) + float(torch.finfo(TYPES[t]).smallest_normal) * torch.finfo(TYPES[t]).eps
    err = np.abs(got[fine] - ref[fine])
    assert (err <= bound).all(), (float((err / np.maximum(bound, 1e-300)).max()), float(err.max()))


# ---------------------------------------------------------------- quantisation
@pytest.mark.parametrize("t", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("M,K,pad,shift", [(1, 1, 0, 0), (1, 32, 0, 0), (3, 33, 0, 0), (2, 31, 2, 1), (5, 64, 0, 0), (7, 100, 4, 0), (61, 1408, 0, 0), (4, 4096, 8, 0),
                                           (131, 1001, 0, 0), (16, 520, 0, 4), (300, 8, 0, 0)])
def test_quantize_is_the_oracle(t, M, K, pad, shift):
    print(f"quantize {t} {M}x{K} pad {pad} shift {shift}", flush=True)
    x = rows_of(np.random.default_rng(M * 1000 + K), M, K, t, pad, shift)
    codes, scales = P.mx_quantize(x)
    want_c, want_s = mx.quantize(f64(x))
    assert np.array_equal(scales.cpu().numpy(), want_s) and np.array_equal(codes.cpu().numpy(), want_c)
    for ty in TYPES:
        out = torch.full((M, K + 3), 7.0, dtype=TYPES[ty], device="cuda")
        assert P.mx_dequantize(codes, scales, out[:, 1:K + 1]).data_ptr() == out[:, 1:].data_ptr()
        want = torch.from_numpy(mx.dequantize(want_c, want_s, K)).to(TYPES[ty])
        assert torch.equal(out[:, 1:K + 1].cpu(), want) and bool((out[:, 0] == 7).all()) and bool((out[:, K + 1:] == 7).all())


@pytest.mark.parametrize("t", ["f32", "bf16", "f16"])
def test_quantize_ties_borders_and_special_values(t):
    big = float(torch.finfo(TYPES[t]).max)
    tiny = float(torch.finfo(TYPES[t]).smallest_normal)
    eighths = np.arange(0, 64) / 8.0                       # every tie between neighbours, both signs, several scales
    rows = [np.concatenate([[6.0], eighths[1:32]]), np.concatenate([[7.875], eighths[32:63]]), np.concatenate([[-6.0], -eighths[1:32]])]
    for e in (-4, 3, 10):
        rows += [r * 2.0 ** e for r in rows[:3]]
    rows += [np.zeros(32), np.full(32, -0.0), np.full(32, big), np.full(32, -big), np.r_[big, np.full(31, tiny)], np.full(32, tiny), np.full(32, tiny / 4), np.r_[tiny, np.full(31, tiny / 8)],
             np.r_[tiny * 3, tiny * np.arange(31) / 8]]
    for bad in (np.inf, -np.inf, np.nan):
        r = np.ones(32)
        r[17] = bad
        rows.append(r)
    x = torch.from_numpy(np.stack(rows)).to(TYPES[t]).cuda()
    codes, scales = P.mx_quantize(x)
    want_c, want_s = mx.quantize(f64(x))
    assert np.array_equal(scales.cpu().numpy(), want_s) and np.array_equal(codes.cpu().numpy(), want_c)
    back = P.mx_dequantize(codes, scales, torch.empty_like(x))
    want = torch.from_numpy(mx.dequantize(want_c, want_s, 32)).to(TYPES[t])
    assert torch.equal(back.cpu().nan_to_num(nan=1e4), want.nan_to_num(nan=1e4)) and torch.equal(back.cpu().isnan(), want.isnan())


def test_every_code_and_scale_comes_back():
    codes = np.tile(np.arange(256, dtype=np.uint8).reshape(16, 16), (16, 1))
    scales = np.arange(256, dtype=np.uint8).reshape(256, 1)
    for t in TYPES:
        y = P.mx_dequantize(torch.from_numpy(codes).cuda(), torch.from_numpy(scales).cuda(), torch.empty(256, 32, dtype=TYPES[t], device="cuda")).cpu()
        want = torch.from_numpy(mx.dequantize(codes, scales, 32)).to(TYPES[t])
        assert torch.equal(y.isnan(), want.isnan()) and torch.equal(y.nan_to_num(nan=3.0), want.nan_to_num(nan=3.0))


# ---------------------------------------------------------------- products
SHAPES = [(1, 1, 1), (1, 16, 32), (2, 17, 33), (1, 512, 512), (3, 130, 100), (16, 128, 1000), (17, 64, 128), (10, 5120, 640), (33, 1000, 1001), (61, 1720, 2048), (64, 96, 4096),
          (100, 300, 136), (128, 512, 1408), (129, 257, 520), (244, 640, 1728), (300, 1000, 264), (1001, 520, 512), (600, 2048, 256)]


@pytest.mark.parametrize("t", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("M,N,K", SHAPES)
def test_gemm_against_float64(t, M, N, K):
    print(f"mx_gemm {t} M={M} N={N} K={K}", flush=True)
    rng = np.random.default_rng(M + N + K)
    x = rows_of(rng, M, K, t)
    w, packed = weights(rng, N, K)
    for ty in TYPES:
        if ty == "f16":                                    # (within its range)
            x.clamp_(-200, 200)
        y = torch.full((M, N + 5), 7.0, dtype=TYPES[ty], device="cuda")
        assert P.mx_gemm(x, packed, y[:, 2:N + 2]) is not None
        assert bool((y[:, :2] == 7).all()) and bool((y[:, N + 2:] == 7).all())
        assert_product(y[:, 2:N + 2], f64(x), w, ty)


@pytest.mark.parametrize("t,M,pad,shift", [("bf16", 1, 0, 1), ("bf16", 40, 3, 0), ("f16", 300, 8, 4), ("f16", 16, 8, 0), ("f32", 70, 4, 0), ("f32", 20, 1, 3), ("bf16", 300, 0, 1), ("bf16", 520, 1, 0)])
def test_gemm_of_strided_and_unaligned_rows(t, M, pad, shift):
    rng = np.random.default_rng(M + pad)
    N, K = 176, 392
    x = rows_of(rng, M, K, t, pad, shift)
    w, packed = weights(rng, N, K)
    buf = torch.full((M * (N + 3) + 1,), 7.0, device="cuda")
    y = buf[1:].view(M, N + 3)[:, :N]
    P.mx_gemm(x, packed, y)
    assert_product(y, f64(x), w, "f32")
    assert bool((buf[1:].view(M, N + 3)[:, N:] == 7).all())


@pytest.mark.parametrize("M,N,K", SHAPES)
def test_both_microscaled_against_float64(M, N, K):
    print(f"mx_gemm_mx M={M} N={N} K={K}", flush=True)
    rng = np.random.default_rng(M * 3 + N + K)
    codes, scales = mx.quantize(rng.normal(size=(M, K)) * np.exp2(rng.integers(-12, 12, size=(M, K // 32 + 1)).repeat(32, axis=1)[:, :K].astype(float)))
    x = mx.dequantize(codes, scales, K)
    w, packed = weights(rng, N, K)
    c, s = torch.from_numpy(codes).cuda(), torch.from_numpy(scales).cuda()
    for ty in ("f32", "bf16"):
        y = torch.full((M, N + 5), 7.0, dtype=TYPES[ty], device="cuda")
        P.mx_gemm_mx(c, s, packed, y[:, 2:N + 2])
        assert bool((y[:, :2] == 7).all()) and bool((y[:, N + 2:] == 7).all())
        assert_product(y[:, 2:N + 2], x, w, ty)


# sizes of the largest tiles: several rounds of them with edges in rows and columns, a K of one group of k-steps and of several, K splits
def large(M, N, K, t):
    g = torch.Generator(device="cuda").manual_seed(M + N + K)
    x = (torch.randn(M, K, generator=g, device="cuda") * torch.exp2(torch.randint(-3, 4, (M, 1), generator=g, device="cuda").float())).to(t)
    codes, scales = P.mx_quantize(torch.randn(N, K, generator=g, device="cuda") * 0.02)
    w = P.mx_dequantize(codes, scales, torch.empty(N, K, device="cuda")).double()
    return x, w, P.mx_pack(codes, scales, K)


def check_large(product, x, w, M, N, K):
    ref, mag = x @ w.T.contiguous(), x.abs() @ w.abs().T.contiguous()
    for ty, left, right in (("bf16", 0, 0), ("f32", 0, 8), ("f16", 0, 1), ("f32", 3, 2)):       # 16-byte pieces of a row, and single values
        y = torch.full((M + 1, left + N + right), 7.0, dtype=TYPES[ty], device="cuda")
        product(y[:M, left:left + N])
        assert bool((y[M] == 7).all()) and bool((y[:, :left] == 7).all()) and bool((y[:, left + N:] == 7).all())
        got = y[:M, left:left + N].double()
        bound = (K + 16) * 2.0 ** -23 * mag * (1 + half_step(ty)) + half_step(ty) * ref.abs() + float(torch.finfo(TYPES[ty]).smallest_normal) * torch.finfo(TYPES[ty]).eps
        worst = float(((got - ref).abs() / bound).max())
        assert worst <= 1, (ty, left, worst)               # (a NaN fails too)


@pytest.mark.parametrize("t,M,N,K", [("bf16", 5000, 2992, 2100), ("f16", 3000, 5001, 2104), ("bf16", 500, 4100, 13000), ("f16", 5000, 777, 9000), ("f32", 1500, 2500, 2100)])
def test_gemm_of_large_tiles(t, M, N, K):
    x, w, packed = large(M, N, K, TYPES[t])
    check_large(lambda y: P.mx_gemm(x, packed, y), x.double(), w, M, N, K)


@pytest.mark.parametrize("M,N,K", [(4100, 2992, 520), (5000, 5001, 700), (8200, 8200, 500), (2100, 9001, 1100), (3000, 4104, 2100), (5000, 777, 9000), (1030, 4001, 9000)])
def test_both_microscaled_of_large_tiles(M, N, K):
    x, w, packed = large(M, N, K, torch.bfloat16)
    codes, scales = P.mx_quantize(x)
    x = P.mx_dequantize(codes, scales, torch.empty(M, K, device="cuda")).double()
    check_large(lambda y: P.mx_gemm_mx(codes, scales, packed, y), x, w, M, N, K)


@pytest.mark.parametrize("M", [1, 40, 300])
def test_scales_far_apart_in_a_row(M):
    """bf16 and float32 activations: 100 powers of two in a row of weights; fp16: the 36 that its operands reach."""
    rng = np.random.default_rng(M)
    N, K = 48, 512
    for t, spread in (("bf16", 100), ("f32", 100), ("f16", 36)):
        w, packed = weights(rng, N, K, spread)
        x = torch.from_numpy(rng.normal(size=(M, K))).to(TYPES[t]).cuda()
        y = torch.empty(M, N, device="cuda")
        P.mx_gemm(x, packed, y)
        assert_product(y, f64(x), w, "f32")
        one = torch.zeros(M, K, dtype=TYPES[t], device="cuda")     # each block alone: nothing of a small one is lost
        for b in range(0, K, 32 * 5):
            one.zero_()
            one[:, b + 3] = 1.0
            P.mx_gemm(one, packed, y)
            assert np.array_equal(f64(y), np.broadcast_to(w[:, b + 3].astype(np.float32).astype(float), (M, N)))


@pytest.mark.parametrize("scale", [0, 30, 140, 220, 254])
def test_scales_at_the_ends_of_the_range(scale):
    """Foreign codes and scales: results that leave float32's range do so once, at the end."""
    rng = np.random.default_rng(scale)
    codes = rng.integers(0, 256, size=(32, 64), dtype=np.uint8)
    scales = np.full((32, 4), scale, np.uint8)
    scales[5] = 100
    codes[6], scales[6] = 0, [254, 0, 90, 1]               # zeros, whatever their scales
    codes[7, 16:], scales[7] = 0, [100, 254, 254, 254]     # blocks of zeros do not count for the row's largest scale
    w = mx.dequantize(codes, scales, 128)
    packed = P.mx_pack(torch.from_numpy(codes).cuda(), torch.from_numpy(scales).cuda(), 128)
    for t, M in (("bf16", 3), ("f16", 70), ("f32", 300)):
        x = torch.from_numpy(rng.normal(size=(M, 128))).to(TYPES[t]).cuda()
        y = P.mx_gemm(x, packed, torch.empty(M, 32, device="cuda"))
        with np.errstate(over="ignore"):
            ref = f64(x) @ w.T
        got, mag = f64(y), np.abs(f64(x)) @ np.abs(w).T
        far = np.abs(ref) - 150 * 2.0 ** -23 * mag > np.finfo(np.float32).max
        near = np.abs(ref) + 150 * 2.0 ** -23 * mag < np.finfo(np.float32).max
        assert np.array_equal(got[far], np.sign(ref[far]) * np.inf)
        assert (np.abs(got - ref)[near] <= (150 * 2.0 ** -23 * mag + 2.0 ** -149)[near]).all()


@pytest.mark.parametrize("M", [1, 5, 40, 200, 300])
def test_infinities_nan_and_rows_of_zeros(M):
    rng = np.random.default_rng(M)
    N, K = 80, 200
    w, packed = weights(rng, N, K)
    codes, scales = mx.quantize(w)
    codes, scales = codes.copy(), scales.copy()
    codes[3] = 0                                           # a column of zeros
    scales[9, 2] = 255                                     # a column of NaN
    codes[12] |= 0x11                                      # no zero among its weights but in the padding
    w = mx.dequantize(codes, scales, K)
    packed = P.mx_pack(torch.from_numpy(codes).cuda(), torch.from_numpy(scales).cuda(), K)
    for t in TYPES:
        x = torch.from_numpy(rng.normal(size=(M, K))).to(TYPES[t]).cuda()
        x[0, K - 1] = float("inf")                         # next to the columns that do not exist
        if M > 4:
            x[2, 7], x[3], x[4, 40] = float("nan"), 0.0, float("-inf")
        y = P.mx_gemm(x, packed, torch.empty(M, N, device="cuda"))
        assert_product(y, f64(x), w, "f32")
    c, s = P.mx_quantize(x)
    y = P.mx_gemm_mx(c, s, packed, torch.empty(M, N, device="cuda"))
    assert_product(y, mx.dequantize(c.cpu().numpy(), s.cpu().numpy(), K), w, "f32")


def test_a_row_of_no_rows():
    w, packed = weights(np.random.default_rng(0), 40, 64)
    for t in TYPES.values():
        x, y = torch.empty(0, 64, dtype=t, device="cuda"), torch.empty(0, 40, dtype=t, device="cuda")
        c, s = P.mx_quantize(x)
        assert c.shape == (0, 32) and s.shape == (0, 2)
        assert P.mx_dequantize(c, s, x).shape == (0, 64) and P.mx_gemm(x, packed, y).shape == (0, 40) and P.mx_gemm_mx(c, s, packed, y).shape == (0, 40)


# ---------------------------------------------------------------- as a program uses them
def test_a_decoder_mlp_in_four_bits():
    """gate, up and down of a feed-forward layer on a tree's rows: quantised on the GPU, activations as they are and in 4 bits; the
    same calls on a side stream and replayed from a graph give the same bits."""
    rng = np.random.default_rng(5)
    d, F, M = 512, 1408, 61
    make = lambda n, k: torch.from_numpy(rng.normal(size=(n, k)) * 0.05).to(torch.bfloat16).cuda()  # noqa: E731
    ws, dense = [], []
    for n, k in ((F, d), (F, d), (d, F)):
        c, s = P.mx_quantize(make(n, k))
        ws.append(P.mx_pack(c, s, k))
        dense.append(mx.dequantize(c.cpu().numpy(), s.cpu().numpy(), k))
    x = make(M, d) * 20
    scratch = [P.mx_gemm_scratch(t, M, F, F) for t in (torch.bfloat16, None)]

    def layer(x, four, stream=None):
        def product(a, w, y):
            if not four:
                return P.mx_gemm(a, w, y, scratch[0], stream)
            return P.mx_gemm_mx(*P.mx_quantize(a, stream=stream), w, y, scratch[1], stream)
        g = product(x, ws[0], torch.empty(M, F, device="cuda"))
        u = product(x, ws[1], torch.empty(M, F, device="cuda"))
        a = (torch.nn.functional.silu(g) * u).to(torch.bfloat16)
        return g, u, a, product(a, ws[2], torch.empty(M, d, device="cuda"))

    def held(a, four):
        if not four:
            return f64(a)
        return mx.dequantize(*mx.quantize(f64(a)), a.shape[1])
    for four in (False, True):
        g, u, a, y = layer(x, four)
        assert_product(g, held(x, four), dense[0], "f32")
        assert_product(u, held(x, four), dense[1], "f32")
        assert_product(y, held(a, four), dense[2], "f32")
        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):
            again = layer(x, four)
            named = layer(x, four, stream=side)
        side.synchronize()
        assert all(torch.equal(p, q) for p, q in zip((g, u, a, y), again)) and all(torch.equal(p, q) for p, q in zip((g, u, a, y), named))
        xin = x.clone()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            captured = layer(xin, four)
        for k in range(4):
            new = make(M, d) * (k + 1)
            xin.copy_(new)
            graph.replay()
            torch.cuda.synchronize()
            eager = layer(new, four)
            assert all(torch.equal(p, q) for p, q in zip(captured, eager)), k


def test_the_same_call_gives_the_same_bits():
    rng = np.random.default_rng(11)
    for M, N, K in ((1, 1000, 4096), (40, 1000, 4096), (200, 512, 4096), (700, 300, 1024)):
        _, packed = weights(rng, N, K)
        x = rows_of(rng, M, K, "bf16")
        c, s = P.mx_quantize(x)
        y, z = (torch.empty(M, N, device="cuda") for _ in range(2))
        first, both = P.mx_gemm(x, packed, y).clone(), P.mx_gemm_mx(c, s, packed, z).clone()
        for _ in range(5):
            assert torch.equal(P.mx_gemm(x, packed, y), first) and torch.equal(P.mx_gemm_mx(c, s, packed, z), both)


@pytest.mark.parametrize("M,N,K", [(5000, 5000, 2100), (5000, 777, 9000)])
def test_large_tiles_give_the_same_bits_eager_and_replayed(M, N, K):
    x, _, packed = large(M, N, K, torch.bfloat16)
    codes, scales = P.mx_quantize(x)
    ys = [torch.empty(M, N, dtype=torch.bfloat16, device="cuda") for _ in range(2)]
    scratch = [P.mx_gemm_scratch(t, M, N, K) for t in (torch.bfloat16, None)]

    def run():
        P.mx_gemm(x, packed, ys[0], scratch[0])
        P.mx_gemm_mx(codes, scales, packed, ys[1], scratch[1])
    run()
    first = [y.clone() for y in ys]
    for _ in range(5):
        run()
        assert all(torch.equal(a, b) for a, b in zip(ys, first))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        run()
    for _ in range(4):
        for y, s in zip(ys, scratch):
            y.fill_(3.0)
            s.fill_(255)
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(ys, first))


def test_two_streams_at_once_with_scratch_of_their_own():
    rng = np.random.default_rng(12)
    M, N, K = 40, 512, 8192                                # (planes of several splits in scratch)
    _, packed = weights(rng, N, K)
    xs = [rows_of(rng, M, K, "bf16") for _ in range(2)]
    want = [P.mx_gemm(x, packed, torch.empty(M, N, device="cuda")) for x in xs]
    want_q = [P.mx_gemm_mx(*P.mx_quantize(x), packed, torch.empty(M, N, device="cuda")) for x in xs]
    streams = [torch.cuda.Stream() for _ in xs]
    scratch = [P.mx_gemm_scratch(t, M, N, K) for t in (torch.bfloat16, torch.bfloat16, None, None)]
    got = [torch.empty(M, N, device="cuda") for _ in range(4)]
    torch.cuda.synchronize()
    for _ in range(20):
        for i, st in enumerate(streams):
            P.mx_gemm(xs[i], packed, got[i], scratch[i], st)
            c, s = P.mx_quantize(xs[i], stream=st)
            P.mx_gemm_mx(c, s, packed, got[2 + i], scratch[2 + i], st)
    torch.cuda.synchronize()
    assert all(torch.equal(got[i], want[i]) and torch.equal(got[2 + i], want_q[i]) for i in range(2))


def test_rows_behind_four_gib():
    """Offsets that pass 32 bits: the last rows of matrices of 4.5 GB."""
    K, rows = 4096, 550_000
    x = torch.zeros(rows, K, dtype=torch.bfloat16, device="cuda")
    x[-3:] = torch.randn(3, K, device="cuda").to(torch.bfloat16)
    codes, scales = P.mx_quantize(x)
    want_c, want_s = mx.quantize(f64(x[-3:]))
    assert np.array_equal(codes[-3:].cpu().numpy(), want_c) and np.array_equal(scales[-3:].cpu().numpy(), want_s) and not bool(codes[:-3].any())
    w, packed = weights(np.random.default_rng(2), 16, K)
    y = P.mx_gemm(x, packed, torch.full((rows, 16), 5.0, device="cuda"))
    assert_product(y[-3:], f64(x[-3:]), w, "f32")
    assert not bool(y[:-3].any())
    y = P.mx_gemm_mx(codes, scales, packed, y.fill_(5.0))
    assert_product(y[-3:], mx.dequantize(want_c, want_s, K), w, "f32")
    assert not bool(y[:-3].any())
    P.mx_dequantize(codes, scales, x.fill_(9.0))
    assert np.array_equal(f64(x[-3:]), mx.dequantize(want_c, want_s, K)) and not bool(x[:-3].any())
