"""The microscaled format's oracle against values written out by hand, and what the C entry points refuse before any GPU work."""
import os

import numpy as np
import pytest

import paper_2506_03566_amd as P
from oracle import mx


def test_values_of_every_code_and_scale():
    codes = np.arange(16, dtype=np.uint8)
    codes = (codes[0::2] | codes[1::2] << 4).reshape(1, 8)
    codes = np.concatenate([codes, np.zeros((1, 8), np.uint8)], axis=1)
    for s in (0, 1, 100, 127, 254):
        v = mx.dequantize(codes, np.array([[s]], np.uint8), 32)[0]
        assert v[:8].tolist() == [m * 2.0 ** (s - 127) for m in (0, .5, 1, 1.5, 2, 3, 4, 6)]
        assert v[8:16].tolist() == [-m * 2.0 ** (s - 127) for m in (0, .5, 1, 1.5, 2, 3, 4, 6)]
    assert np.isnan(mx.dequantize(codes, np.array([[255]], np.uint8), 32)).all()


def test_rounding_ties_and_saturation_by_hand():
    x = np.zeros((1, 32))
    x[0, :16] = [6, .25, .26, .75, 1.25, 1.75, 2.5, 3.5, 5, 5.01, -.25, -.75, -5, 7.9, .24, -7.99]   # the largest lies in [4, 8): scale 1
    codes, scales = mx.quantize(x)
    assert scales.tolist() == [[127]]
    assert mx.dequantize(codes, scales, 16)[0].tolist() == [6, 0, .5, 1, 1, 2, 2, 4, 4, 6, 0, -1, -4, 6, 0, -6]


@pytest.mark.parametrize("top,byte", [(8.0, 128), (7.99, 127), (4.0, 127), (3.99, 126), (1.0, 125), (2.0 ** -125, 0), (2.0 ** -149, 0), (0.0, 0),
                                      (2.0 ** 127, 252), (np.inf, 255), (np.nan, 255)])
def test_scale_of_a_block(top, byte):
    x = np.zeros((1, 40))
    x[0, 7] = -top
    assert mx.quantize(x)[1].tolist() == [[byte, 0]]


def test_a_value_moves_by_at_most_half_its_step():
    rng = np.random.default_rng(1)
    x = rng.normal(size=(50, 77)) * np.exp2(rng.integers(-20, 20, (50, 1)))
    codes, scales = mx.quantize(x)
    assert codes.shape == (50, 48) and scales.shape == (50, 3)
    y, s = mx.dequantize(codes, scales, 77), np.repeat(np.exp2(scales.astype(float) - 127), 32, axis=1)[:, :77]
    a = np.abs(x) / s
    step = np.where(a < 2, .5, np.where(a < 4, 1., 2.))
    assert (np.abs(y - x) <= np.where(a > 6, a - 6, step / 2) * s * (1 + 1e-12)).all() and a.max() < 8 and a.max() >= 4


def _lib():
    if not os.path.exists(P.LIB_PATH):
        pytest.skip("libposs.so not built (run __graft_entry__.build())")
    return P.load_library()


def test_refusals_need_no_gpu():
    lib = _lib()
    bad, cap = P.E_INVALID_ARG, P.E_CAPACITY
    a, o = 1 << 20, 1 << 30                                # addresses that are never followed
    assert lib.poss_mx_quantize(3, a, 32, 1, 32, o, o, None) == bad
    assert lib.poss_mx_quantize(1, a, 31, 1, 32, o, o, None) == bad          # rows that overlap
    assert lib.poss_mx_quantize(1, a, 32, -1, 32, o, o, None) == bad
    assert lib.poss_mx_quantize(1, a, 32, 1, 0, o, o, None) == bad
    assert lib.poss_mx_quantize(1, None, 32, 1, 32, o, o, None) == bad and b"null" in lib.poss_last_error(None)
    assert lib.poss_mx_quantize(1, a + 1, 32, 1, 32, o, o, None) == bad      # x not aligned to its type
    assert lib.poss_mx_quantize(1, a, 32, 1, 32, o + 8, o, None) == bad
    assert lib.poss_mx_quantize(1, None, 32, 0, 32, None, None, None) == P.POSS_OK       # no rows, no work
    assert lib.poss_mx_dequantize(-1, o, o, 1, 32, a, 32, None) == bad
    assert lib.poss_mx_dequantize(0, o, o, 1, 32, a + 2, 32, None) == bad
    assert lib.poss_mx_dequantize(0, o, o, 1, 32, a, 16, None) == bad
    assert lib.poss_mx_dequantize(0, None, o, 1, 32, a, 32, None) == bad
    assert lib.poss_mx_dequantize(0, None, None, 0, 32, None, 32, None) == P.POSS_OK
    assert lib.poss_mx_packed_bytes(0, 32) == 0 and lib.poss_mx_packed_bytes(16, 0) == 0
    assert lib.poss_mx_packed_bytes(4096, 4096) >= 4096 * 4096 // 2 + 4096 * 128
    assert lib.poss_mx_pack(a, a, 0, 32, o, None) == bad and lib.poss_mx_pack(a, a, 16, 32, None, None) == bad
    assert lib.poss_mx_pack(a, a, 16, 32, o + 16, None) == bad
    for dt in (0, 1, 2, 4):
        assert lib.poss_mx_gemm_scratch_bytes(dt, 0, 1, 1) >= 256
        assert lib.poss_mx_gemm_scratch_bytes(dt, -1, 1, 1) == lib.poss_mx_gemm_scratch_bytes(dt, 1, 0, 1) == lib.poss_mx_gemm_scratch_bytes(dt, 1, 1, 0) == 0
    assert lib.poss_mx_gemm_scratch_bytes(3, 1, 1, 1) == 0
    assert lib.poss_mx_packed_bytes(16, (1 << 21) + 1) == lib.poss_mx_packed_bytes((1 << 27) + 1, 32) == 0
    for big in ((1, 16, (1 << 21) + 1), (1, (1 << 27) + 1, 32), ((1 << 24) + 1, 16, 32), (1 << 24, (1 << 14) + 1, 32)):
        assert [lib.poss_mx_gemm_scratch_bytes(dt, *big) for dt in (0, 1, 2, 4)] == [0] * 4
    need = lib.poss_mx_gemm_scratch_bytes(1, 2, 16, 32)

    def gemm(xt=1, x=a, ldx=32, w=o, yt=1, y=a, ldy=16, M=2, N=16, K=32, scratch=o, n=need):
        return lib.poss_mx_gemm(xt, x, ldx, w, yt, y, ldy, M, N, K, scratch, n, None)
    for over in (dict(xt=3), dict(xt=4), dict(yt=-1), dict(x=None), dict(w=None), dict(y=None), dict(scratch=None), dict(ldx=31), dict(ldy=15), dict(M=-1), dict(N=0), dict(K=0),
                 dict(w=o + 64), dict(scratch=o + 64), dict(x=a + 1), dict(y=a + 1)):
        assert gemm(**over) == bad, over
    assert gemm(n=need - 1) == cap
    assert gemm(M=0, x=None, y=None) == P.POSS_OK

    def both(x=o, s=o, w=o, yt=1, y=a, ldy=16, M=2, N=16, K=32, scratch=o, n=1 << 24):
        return lib.poss_mx_gemm_mx(x, s, w, yt, y, ldy, M, N, K, scratch, n, None)
    for over in (dict(x=None), dict(s=None), dict(w=None), dict(y=None), dict(scratch=None), dict(yt=4), dict(x=o + 8), dict(ldy=1), dict(M=-1), dict(N=0), dict(K=0), dict(w=o + 64)):
        assert both(**over) == bad, over
    assert both(n=16) == cap and both(M=0) == P.POSS_OK


def test_the_binding_refuses_what_the_kernels_would_misread():
    """Shapes, types and layouts are looked at before anything is launched (host tensors: no GPU is needed to be refused)."""
    import torch
    u8 = torch.uint8

    def refused(f, *a, **k):
        with pytest.raises(P.PossError) as e:
            f(*a, **k)
        return e.value.code == P.E_INVALID_ARG
    _lib()
    x, y = torch.zeros(4, 64, dtype=torch.bfloat16), torch.zeros(4, 16)
    codes, scales = torch.zeros(4, 32, dtype=u8), torch.zeros(4, 2, dtype=u8)
    w = P.MxWeight(torch.zeros(P.load_library().poss_mx_packed_bytes(16, 64), dtype=u8), 16, 64)
    assert refused(P.MxWeight, torch.zeros(4096, dtype=u8), 16, 64)        # too few bytes
    assert refused(P.mx_quantize, x, codes, scales)                        # host memory
    assert refused(P.mx_quantize, x.t())                                   # rows that are not contiguous
    assert refused(P.mx_quantize, x[0])                                    # not a matrix
    assert refused(P.mx_quantize, x[:1].expand(4, 64), codes, scales)      # rows that overlap
    assert refused(P.mx_quantize, x, codes[:, :16], scales)
    assert refused(P.mx_quantize, x, codes.to(torch.int8), scales)
    assert refused(P.mx_dequantize, codes, scales, torch.zeros(4, 65))
    assert refused(P.mx_dequantize, codes, scales[:3], torch.zeros(4, 64))
    assert refused(P.mx_gemm, x[:, :32], w, y)
    assert refused(P.mx_gemm, x, w, y[:3])
    assert refused(P.mx_gemm, x.double(), w, y)
    assert refused(P.mx_gemm_mx, codes[:2], scales, w, y)
    assert refused(P.mx_gemm_mx, codes, scales, w, y[:, :8])
    assert refused(P.mx_pack, codes, scales, 128)
    assert refused(P.mx_gemm_scratch, torch.int8, 4, 16, 64)
    assert refused(P.mx_gemm_scratch, None, -1, 16, 64)
    assert refused(P.mx_gemm_scratch, None, 4, (1 << 32) + 16, 64)         # (would pass as 16 in 32 bits)
    assert refused(P.mx_gemm, x, w, y, torch.zeros(4, 600, dtype=u8)[:, :512])   # scratch with gaps


def test_workspace_of_microscaled_layers():
    import ctypes
    from synth import CONFIGS
    lib = _lib()
    for name, cfg in CONFIGS.items():
        c = P.make_config(cfg)
        small, full = lib.poss_workspace_bytes_mx(ctypes.byref(c)), lib.poss_workspace_bytes(ctypes.byref(c))
        assert small == 0 if cfg.dtype == 0 else 0 < small < full, name
    assert lib.poss_workspace_bytes_mx(None) == 0
    out = ctypes.c_void_p()
    c = P.make_config(CONFIGS["t_mid_bf16"])
    assert lib.poss_load_mx(ctypes.byref(c), None, None, 0, None, ctypes.byref(out)) == P.E_INVALID_ARG


def test_microscaled_layers_of_any_width_up_to_the_products_limit():
    import ctypes
    from synth import CONFIGS
    lib = _lib()
    base = CONFIGS["t_mid_bf16"]

    def size(**over):
        c = P.make_config(base)
        for k, v in over.items():
            setattr(c, k, v)
        return lib.poss_workspace_bytes_mx(ctypes.byref(c)), lib.poss_workspace_bytes(ctypes.byref(c))

    small, full = size(d_ffn=1 << 21, n_layers=1)
    assert 0 < small < full
    small, full = size(d_ffn=(1 << 21) + 8, n_layers=1)
    assert small == 0 < full
