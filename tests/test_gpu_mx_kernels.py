"""Every kernel of the microscaled products against float64: contiguous results, whose rows are written in pieces of 16 bytes, and results in the
middle of longer rows; scratch full of NaN before each call.  Tolerances as in test_gpu_mx.py."""
import pytest

from gpu_util import have_gpu
from mx_sizes import SIZES

pytestmark = pytest.mark.gpu

if have_gpu():
    import torch
    import paper_2506_03566_amd as P
    from test_gpu_mx import TYPES, check_large, large

CASES = [(t, *s[1:]) for s in SIZES for t in (("bf16", "f16") if s[0] == "16" else (s[0],))]


@pytest.mark.parametrize("kind,M,N,K,tile,splits", CASES)
def test_product_against_float64(kind, M, N, K, tile, splits):
    print(f"kernel {tile} x {splits}: {kind} M={M} N={N} K={K}", flush=True)
    x, w, packed = large(M, N, K, torch.bfloat16 if kind == "mx" else TYPES[kind])
    scratch = P.mx_gemm_scratch(None if kind == "mx" else x.dtype, M, N, K)
    if kind == "mx":
        codes, scales = P.mx_quantize(x)
        x64 = P.mx_dequantize(codes, scales, torch.empty(M, K, device="cuda")).double()
        check_large(lambda y: P.mx_gemm_mx(codes, scales, packed, y, scratch.fill_(255)), x64, w, M, N, K)
    else:
        check_large(lambda y: P.mx_gemm(x, packed, y, scratch.fill_(255)), x.double(), w, M, N, K)
