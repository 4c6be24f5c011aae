"""Products with weights of 4 bits, and the quantisation before them, as cases that can be timed and compared.

The number format is microscaled: 32 values of a row share a power of two (a byte, e8m0), each value is a sign, two bits of exponent
and one of mantissa (e2m1: 0, 0.5, 1, 1.5, 2, 3, 4, 6).  Three kinds of case:

"codes": rows to codes and scales, and those back to values, as a program does that checks what its weights lose.
"gemm":  Y = X W^T with a microscaled W and activations as they are (float32, bfloat16, float16).
"both":  activations quantised on the way, then the product of two microscaled operands.

The plain form computes in float32 with elementary operations and rounds once at the end.
"""
import math

import torch

own = False

TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
SIZE = {"f32": 4, "bf16": 2, "f16": 2}
BLOCK = 32


def listed():
    return [
        # one token's activations: two launches, latency is all there is
        dict(name="codes_row", kind="codes", t="bf16", M=1, K=4096),
        # float32 rows that end inside a block
        dict(name="codes_ragged", kind="codes", t="f32", M=131, K=1001),
        # a tree's rows before the down projection
        dict(name="codes_tree", kind="codes", t="f16", M=61, K=13824),
        # a weight matrix when a model is loaded
        dict(name="codes_weight", kind="codes", t="bf16", M=28672, K=4096),
        # plain decoding: one row through the projections of queries, keys and values
        dict(name="gemm_row", kind="gemm", t="bf16", y="bf16", M=1, N=6144, K=4096),
        # a drafting pass: ten rows through the down projection
        dict(name="gemm_draft", kind="gemm", t="f16", y="f32", M=10, N=5120, K=13824),
        # verification of a tree: gate and up
        dict(name="gemm_tree", kind="gemm", t="bf16", y="bf16", M=61, N=28672, K=4096),
        # float32 activations, odd sizes, K that ends inside a block
        dict(name="gemm_ragged", kind="gemm", t="f32", y="f32", M=131, N=1720, K=5000),
        # a chunk of a prompt
        dict(name="gemm_prompt", kind="gemm", t="bf16", y="bf16", M=4096, N=14336, K=4096),
        # sixteen rows, both operands in 4 bits
        dict(name="both_rows", kind="both", t="bf16", y="f32", M=16, N=4096, K=14336),
        # four sequences' trees in one launch
        dict(name="both_batch", kind="both", t="f16", y="f16", M=244, N=5120, K=5120),
        # a long prompt: the matrix cores are the bound
        dict(name="both_prompt", kind="both", t="bf16", y="bf16", M=8192, N=28672, K=4096),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["codes", "gemm", "gemm", "both", "both"])
    t = rng.choice(["bf16", "bf16", "f16", "f32"])
    rows = rng.choice(["one", "few", "tree", "batch", "prompt"])
    M = {"one": 1, "few": rng.randint(2, 16), "tree": rng.randint(17, 128), "batch": rng.randint(129, 512), "prompt": _log_int(rng, 513, 6000)}[rows]
    K = _log_int(rng, 64, 14336)
    if rng.random() < 0.6:                                 # widths of models: multiples of 64
        K = max(64, K // 64 * 64)
    if kind == "codes":
        return dict(kind=kind, t=t, M=_log_int(rng, 1, 16384), K=_log_int(rng, 16, 4096))
    N = _log_int(rng, 64, 28672)
    if rng.random() < 0.6:
        N = max(64, N // 64 * 64)
    most = (8192 * 28672 if kind == "both" else 4096 * 14336 if t != "f32" else 4096 * 4096) * 4096
    N = max(1, min(N, most // (M * K)))                    # no more work than the largest listed case of its kind
    return dict(kind=kind, t=t, y=rng.choice(["bf16", "f16", "f32"]), M=M, N=N, K=K)


# ---------------------------------------------------------------- what the program has in hand
def _blocks(K):
    return (K + BLOCK - 1) // BLOCK


def _made(case, seed):
    """The 16- or 32-bit matrices of a case: activations with a few loud channels and, of several rows, one of zeros; weights."""
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    M, K = case["M"], case["K"]
    x = torch.randn(M, K, generator=g, device="cuda")
    if case["kind"] == "codes" and M > 4096:
        x *= 0.02                                          # a weight matrix
    else:
        loud = torch.randint(0, K, (max(1, K // 200),), generator=g, device="cuda")
        x[:, loud] *= 16.0
        if M > 4:
            x[M // 2] = 0.0
    w = None
    if case["kind"] != "codes":
        w = torch.randn(case["N"], K, generator=g, device="cuda") * 0.02
    return x.to(TYPES[case["t"]]), w


def _quantized(x):
    """Codes [rows, blocks * 16] (the even column in the low half) and scales [rows, blocks], by elementary operations."""
    rows, K = x.shape
    nb = _blocks(K)
    v = torch.zeros(rows, nb * BLOCK, device=x.device)
    v[:, :K] = x.float()
    v = v.view(rows, nb, BLOCK)
    field = (v.abs().amax(dim=2).view(torch.int32) >> 23) & 255
    scale = torch.where(field == 255, field, (field - 2).clamp(min=0))
    v = v * _power(-(scale - 127))[:, :, None]             # a power of two: exact
    a = v.abs()
    index = torch.where(a < 2, (a * 2).round(), torch.where(a < 4, a.round() + 2, (a / 2).round().clamp(max=3) + 4)).to(torch.uint8)
    index |= torch.signbit(v).to(torch.uint8) << 3
    index = index.view(rows, nb * BLOCK)
    return index[:, 0::2] | (index[:, 1::2] << 4), scale.to(torch.uint8)


def _power(e):
    """2^e in float32 for -127 <= e <= 127."""
    return torch.where(e > -127, ((e + 127).clamp(min=1) << 23).view(torch.float32), torch.full_like(e, 2.0 ** -127, dtype=torch.float32))


def _values(codes, scales, K):
    """What codes and scales stand for, in float32."""
    rows, nb = scales.shape
    grid = torch.tensor([0, .5, 1, 1.5, 2, 3, 4, 6, -0., -.5, -1, -1.5, -2, -3, -4, -6], device=codes.device)
    v = torch.stack([grid[(codes & 15).int()], grid[(codes >> 4).int()]], dim=2).view(rows, nb, BLOCK)
    s = torch.where(scales == 255, torch.full_like(scales, float("nan"), dtype=torch.float32), _power(scales.int() - 127))
    return (v * s[:, :, None]).view(rows, nb * BLOCK)[:, :K]


def prepare(case, seed):
    x, w = _made(case, seed)
    M, K = x.shape
    nb = _blocks(K)
    s = dict(case=case, x=x, codes=torch.empty(M, nb * 16, dtype=torch.uint8, device="cuda"),
             scales=torch.empty(M, nb, dtype=torch.uint8, device="cuda"))
    s["out"] = torch.empty(M, case.get("N", K), dtype=TYPES[case.get("y", case["t"])], device="cuda")
    if w is not None:
        s["w_codes"], s["w_scales"] = _quantized(w)
        if own:                                            # the weights laid out once, the workspace a program keeps
            import paper_2506_03566_amd as P
            s["w"] = P.mx_pack(s["w_codes"], s["w_scales"], K)
            s["scratch"] = P.mx_gemm_scratch(TYPES[case["t"]] if case["kind"] == "gemm" else None, M, case["N"], K)
    return s


# ---------------------------------------------------------------- one pass
def run(s):
    kind, x = s["case"]["kind"], s["x"]
    K = x.shape[1]
    if own:
        import paper_2506_03566_amd as P
        if kind == "gemm":
            return P.mx_gemm(x, s["w"], s["out"], scratch=s["scratch"])
        P.mx_quantize(x, s["codes"], s["scales"])
        if kind == "codes":
            return P.mx_dequantize(s["codes"], s["scales"], s["out"])
        return P.mx_gemm_mx(s["codes"], s["scales"], s["w"], s["out"], scratch=s["scratch"])
    if kind == "codes":
        return _values(*_quantized(x), K).to(s["out"].dtype)
    a = x.float() if kind == "gemm" else _values(*_quantized(x), K)
    return (a @ _values(s["w_codes"], s["w_scales"], K).t()).to(s["out"].dtype)


def work(case):
    M, K, nb = case["M"], case["K"], _blocks(case["K"])
    if case["kind"] == "codes":                            # values in, codes and scales out, values out
        return {"bytes": 2 * M * K * SIZE[case["t"]] + M * nb * 17, "flops": 4 * M * K}
    N = case["N"]
    return {"bytes": M * K * SIZE[case["t"]] + N * nb * 17 + M * N * SIZE[case["y"]], "flops": 2 * M * N * K}


# ---------------------------------------------------------------- the definition, in 64 bits
def _nearest(x):
    """What the microscaled form of x stands for, from the definition: the nearest of the eight magnitudes times the block's
    power of two, the even code of two that are equally near."""
    rows, K = x.shape
    out = torch.empty(rows, K, dtype=torch.float64, device=x.device)
    middle = [.25, .75, 1.25, 1.75, 2.5, 3.5, 5.]
    grid = torch.tensor([0, .5, 1, 1.5, 2, 3, 4, 6], dtype=torch.float64, device=x.device)
    step = max(1, (1 << 25) // K)
    for r in range(0, rows, step):
        v = torch.nn.functional.pad(x[r:r + step].double(), (0, -K % BLOCK))
        v = v.view(v.shape[0], -1, BLOCK)
        top = v.abs().amax(dim=2, keepdim=True)
        e = torch.floor(torch.log2(top.clamp(min=2.0 ** -200)))
        e = e - (torch.exp2(e) > top).double() + (torch.exp2(e + 1) <= top).double()      # where the logarithm was rounded over a border
        s = torch.exp2((e - 2).clamp(min=-127))
        a = v.abs() / s
        code = torch.zeros_like(a, dtype=torch.long)
        for i, m in enumerate(middle):
            code += (a > m) if i % 2 == 0 else (a >= m)
        out[r:r + step] = (torch.sign(v) * grid[code] * s).reshape(v.shape[0], -1)[:, :K]
    return out


def exact(case, seed):
    x, w = _made(case, seed)
    if case["kind"] == "codes":
        return _nearest(x)
    a = x.double() if case["kind"] == "gemm" else _nearest(x)
    # prepare() quantises the weights: what the product takes is what its codes stand for
    b = _nearest(w)
    return a @ b.t()
