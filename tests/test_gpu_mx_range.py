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
