"""Microscaled products at the ends of the numbers' range, against float64, through the C ABI."""
import numpy as np
import pytest

from gpu_util import have_gpu, prefill_in_step, tol_for

pytestmark = pytest.mark.gpu

if have_gpu():
    import torch
    import paper_2506_03566_amd as P
    from oracle import mx
    TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
    # powers of two that a block may lie below its row's largest and lose nothing
    REACH = {"f32": 126, "bf16": 126, "f16": 36, "mx": 126}


def f64(t):
    return t.double().cpu().numpy()


def one_hot_product(kind, M, K, col, packed, N):
    """Rows of X that are one in one column and zero elsewhere: a column of the weights, M times."""
    y = torch.full((M, N), 7.0, device="cuda")
    if kind == "mx":
        x = np.zeros((M, K))
        x[:, col] = 1.0
        codes, scales = mx.quantize(x)
        return f64(P.mx_gemm_mx(torch.from_numpy(codes).cuda(), torch.from_numpy(scales).cuda(), packed, y))
    x = torch.zeros(M, K, dtype=TYPES[kind], device="cuda")
    x[:, col] = 1.0
    return f64(P.mx_gemm(x, packed, y))


@pytest.mark.parametrize("M", [1, 40, 300])
@pytest.mark.parametrize("top", [254, 252, 200, 140])
def test_blocks_far_below_the_largest_of_their_row(top, M):
    """Blocks of ordinary codes from 0 to `top` powers of two below the largest block of their row, each taken alone: its weights come out as they
    are within reach, and beyond it off by no more than their own size (rounded to the operand's type, or zero), never enlarged."""
    rng = np.random.default_rng(top + M)
    N, below = 32, [0, 20, 36, 37, 60, 100, 126, 127, 128, 130, 160, 200, 250, 252, 253, 254]
    K = 32 * len(below)
    codes = rng.integers(0, 256, size=(N, K // 2), dtype=np.uint8)
    codes[:, 0] |= 0x11                                    # (the largest block of a row is not all zero)
    scales = np.repeat(np.maximum(top - np.array(below), 0)[None], N, axis=0).astype(np.uint8)
    w = mx.dequantize(codes, scales, K)
    packed = P.mx_pack(torch.from_numpy(codes).cuda(), torch.from_numpy(scales).cuda(), K)
    for kind in REACH:
        print(f"far blocks {kind} top {top} M {M}", flush=True)
        for b in range(len(below)):
            col = b * 32 + 5 + b % 3
            got, want = one_hot_product(kind, M, K, col, packed, N), np.broadcast_to(w[:, col], (M, N))
            with np.errstate(over="ignore"):
                want = want.astype(np.float32).astype(float)
            if top - int(scales[0, b]) <= REACH[kind]:
                assert np.array_equal(got, want), (kind, b)
            else:
                assert (np.abs(got - want) <= np.abs(want)).all(), (kind, b, float(np.abs(got).max()), float(np.abs(want).max()))


def test_far_blocks_of_a_layers_matrix():
    """A context whose down projections hold one block of 2^130 times ordinary weights in every row, over activations that are exactly zero, and
    2^-10 times ordinary weights beside it: those count for what they are, or for nothing (far below the tolerance either way)."""
    from synth import get_config, make_prompt, make_weights
    from synth.gen import to_float64, to_storage
    from synth.gpu import weights_to_device
    from oracle.model import Weights
    from oracle.poss import PossOracle
    from oracle.tree import Tree
    from test_gpu_mx_context import rounded
    cfg, storage = get_config("t_mid_bf16"), make_weights(get_config("t_mid_bf16"))
    for name in list(storage):
        if name.split(".")[-1] not in ("w_up", "w_down"):
            continue
        w = to_float64(storage[name], cfg.dtype).copy()
        if name.endswith("w_up"):
            w[:32] = 0
        else:
            w[:, :32] *= 2.0 ** 130
            w[:, 32:] *= 2.0 ** -10
            assert np.abs(w).max() < 2.0 ** 127
        storage[name] = to_storage(w, cfg.dtype)
    ctx, o = P.Poss(cfg, weights_to_device(cfg, storage), mx=True), PossOracle(Weights(cfg, rounded(cfg, storage)), cfg, act=cfg.dtype)
    prompt = make_prompt(cfg)
    prefill_in_step(ctx, o, prompt, tol_for(cfg))
    tree = Tree([o.tokens[-1], 5, 9, 11], [-1, 0, 0, 1])
    logits = torch.zeros(4, cfg.vocab, device="cuda")
    ctx.verify_tree(P.TreeArrays.from_lists(tree.token, tree.parent), logits_out=logits)
    _, ologits, _ = o.verify_tree(tree)
    assert np.abs(logits.cpu().numpy() - ologits).max() <= tol_for(cfg)
    ctx.close()


@pytest.mark.parametrize("M", [1, 40, 300])
@pytest.mark.parametrize("top", [254, 253, 252, 200, 140, 128, 127, 126, 103, 102, 20, 0])
def test_weights_of_all_scales_come_out_as_they_are(top, M):
    """With activations that reach as far as float32, a weight that is taken alone is exact, subnormal results among them: in rows whose largest scale is at
    most 127 at any distance from it, in others up to 127 powers of two below it, and off by no more than its own size beyond."""
    rng = np.random.default_rng(top * 3 + M)
    N, below = 32, [0, 1, 24, 36, 100, 126, 127, 128, 130, 199, 200, 250, 251, 252]
    K = 32 * len(below)
    codes = rng.integers(0, 256, size=(N, K // 2), dtype=np.uint8)
    codes[:, 0] |= 0x11
    scales = np.repeat(np.maximum(top - np.array(below), 0)[None], N, axis=0).astype(np.uint8)
    w = mx.dequantize(codes, scales, K)
    packed = P.mx_pack(torch.from_numpy(codes).cuda(), torch.from_numpy(scales).cuda(), K)
    for kind in ("bf16", "f32", "mx"):
        print(f"all scales {kind} top {top} M {M}", flush=True)
        for b in range(len(below)):
            col = b * 32 + 5 + b % 3
            with np.errstate(over="ignore"):
                want = np.broadcast_to(w[:, col].astype(np.float32).astype(float), (M, N))
            got = one_hot_product(kind, M, K, col, packed, N)
            if top <= 127 or top - int(scales[0, b]) <= 127:
                assert np.array_equal(got, want), (kind, b, got[0, :4].tolist(), want[0, :4].tolist())
            else:
                assert (np.abs(got - want) <= np.abs(want)).all(), (kind, b)


def close(got, ref, mag, K, t):
    """Within (K + 16) 2^-23 of the sum of magnitudes and half a step of the type, as float32 sums of exact products are; nothing infinite."""
    half = torch.finfo(TYPES[t]).eps / 2
    bound = (K + 16) * 2.0 ** -23 * mag * (1 + half) + half * np.abs(ref) + float(torch.finfo(TYPES[t]).smallest_normal) * torch.finfo(TYPES[t]).eps
    assert np.isfinite(got).all()
    assert (np.abs(got - ref) <= bound).all(), float((np.abs(got - ref) / bound).max())


@pytest.mark.parametrize("kind", ["bf16", "f32", "f16", "mx"])
@pytest.mark.parametrize("M,N,K", [(1, 48, 96), (3, 48, 2000), (40, 300, 1000), (300, 640, 520), (2100, 2500, 1100)])
def test_activations_of_the_types_largest_values(kind, M, N, K):
    """Rows with one, two or eight values next to the type's largest and lowest: results that float32 holds are not infinite.  Weights lie within 0.1,
    so that the sum of magnitudes stays below 0.9 of the range; some rows of W are 2^-70 of that, with whole rows of such values allowed."""
    print(f"large {kind} {M} {N} {K}", flush=True)
    rng = np.random.default_rng(M + N + K)
    big = float(torch.finfo(torch.float16 if kind == "f16" else torch.bfloat16).max) * (0.9 if kind == "mx" else 1.0)
    x = rng.normal(size=(M, K))
    for m in range(M):
        at = rng.choice(K, size=(1, 2, 8)[m % 3], replace=False)
        x[m, at] = big * np.where(rng.random(len(at)) < 0.7, -1.0, 1.0)
    wv = np.clip(rng.normal(size=(N, K)) * 0.02, -0.08, 0.08)
    wv[::5] *= 2.0 ** -70
    codes, scales = mx.quantize(wv)
    w = mx.dequantize(codes, scales, K)
    assert np.abs(w).max() <= 0.1
    packed = P.mx_pack(torch.from_numpy(codes).cuda(), torch.from_numpy(scales).cuda(), K)
    if kind == "mx":
        xc, xs = mx.quantize(x)
        assert xs.max() == 252
        x64 = mx.dequantize(xc, xs, K)
        product = lambda y: P.mx_gemm_mx(torch.from_numpy(xc).cuda(), torch.from_numpy(xs).cuda(), packed, y)  # noqa: E731
    else:
        xt = torch.from_numpy(x).to(TYPES[kind]).cuda()
        x64 = f64(xt)
        product = lambda y: P.mx_gemm(xt, packed, y)  # noqa: E731
    ref, mag = x64 @ w.T, np.abs(x64) @ np.abs(w).T
    assert mag.max() < 0.9 * float(torch.finfo(torch.float32).max)
    for t in ("f32", "bf16"):
        close(f64(product(torch.empty(M, N, dtype=TYPES[t], device="cuda"))), ref, mag, K, t)
    if kind in ("bf16", "f32"):                            # every activation the lowest value: rows of small weights
        xt.fill_(-big)
        y = f64(P.mx_gemm(xt, packed, torch.empty(M, N, device="cuda")))[:, ::5]
        x64 = f64(xt)
        close(y, x64 @ w[::5].T, np.abs(x64) @ np.abs(w[::5]).T, K, "f32")


@pytest.mark.parametrize("M", [1, 40, 300])
def test_infinities_over_far_blocks(M):
    """An infinite activation over a weight that is small but not zero gives an infinity, over a weight of zero a NaN."""
    rng = np.random.default_rng(M)
    N, K = 32, 96
    codes = rng.integers(0, 256, size=(N, K // 2), dtype=np.uint8)
    codes[:, 16:] = np.where(codes[:, 16:] & 0x70, codes[:, 16:], codes[:, 16:] | 0x10)      # (odd columns behind the first block: not zero)
    codes[3, 24] = 0x05                                    # a zero at column 49 of row 3
    scales = np.repeat(np.array([[120, 10, 1]], np.uint8), N, axis=0)
    w = mx.dequantize(codes, scales, K)
    packed = P.mx_pack(torch.from_numpy(codes).cuda(), torch.from_numpy(scales).cuda(), K)
    for kind in ("bf16", "f32"):
        x = torch.ones(M, K, dtype=TYPES[kind], device="cuda")
        x[:, 49], x[0, 49], x[0, 95] = float("inf"), 1.0, float("-inf")
        with np.errstate(invalid="ignore"):
            ref = f64(x) @ w.T
        got = f64(P.mx_gemm(x, packed, torch.empty(M, N, device="cuda")))
        assert np.array_equal(np.isnan(got), np.isnan(ref)) and np.isnan(ref).any() == (M > 1)
        assert np.array_equal(got[np.isinf(ref)], ref[np.isinf(ref)]) and np.isfinite(got[np.isfinite(ref)]).all()
