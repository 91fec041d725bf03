"""The grouped products' refusals (the C calls check on the host, nothing is launched) and the tests' own 64-bit formulas against
differences."""
import ctypes as C

import numpy as np
import pytest
import torch

import grouped_ref as ref
import paper_2508_17624_amd as ew

ONE = C.c_void_p(256)   # never dereferenced
INVALID, WORKSPACE, UNSUPPORTED = -1, -5, -6


def gemm(x=ONE, dtype=ew.EW_BF16, tokens=4, rows=4, k=2, K=8, N=8, P=3, counts=ONE, offsets=ONE, w=ONE, y=ONE):
    return ew.lib().moe_grouped_gemm(x, dtype, tokens, rows, k, K, N, P, 0, counts, offsets, None, w, y, None)


def wgrad(dy=ONE, x=ONE, dtype=ew.EW_BF16, rows=4, k=2, K=8, N=8, P=3, counts=ONE, first=0, n=3, dw_dtype=ew.EW_F32, accumulate=0, dw=ONE):
    return ew.lib().moe_grouped_gemm_wgrad(dy, x, dtype, 4, rows, k, K, N, P, counts, ONE, None, first, n, dw_dtype, accumulate, dw, None)


def backward(dtype=ew.EW_BF16, rows=4, H=8, I=8, P=3, dx=ONE, first=0, n=3, dw_dtype=ew.EW_F32, accumulate=0, d13=ONE, ws=ONE, ws_bytes=1 << 30, x=ONE):
    return ew.lib().moe_grouped_ffn_backward(x, ONE, dtype, 4, rows, 2, H, I, P, ONE, ONE, None, ONE, ONE, dx, first, n, dw_dtype, accumulate, d13, ONE, ws,
                                             ws_bytes, None)


def test_grouped_products_refuse_on_the_host():
    for bad in (dict(x=None), dict(w=None), dict(y=None), dict(counts=None), dict(offsets=None), dict(dtype=2), dict(K=0), dict(N=0), dict(P=0), dict(k=0),
                dict(rows=-1), dict(tokens=-1)):
        assert gemm(**bad) == INVALID and b"moe_grouped_gemm" in ew.lib().ew_last_error(), bad
    assert gemm(rows=0) == 0 and gemm(rows=0, x=None, y=None, w=None) == 0     # no rows: nothing to do
    for bad in (dict(dy=None), dict(dw=None), dict(counts=None), dict(dtype=9), dict(dw_dtype=5), dict(dtype=ew.EW_F32, dw_dtype=ew.EW_BF16), dict(first=-1),
                dict(first=1, n=3), dict(n=-1), dict(first=3, n=2 ** 31 - 1), dict(K=0), dict(k=0)):
        assert wgrad(**bad) == INVALID, bad
    assert wgrad(accumulate=1, dw_dtype=ew.EW_BF16) == UNSUPPORTED
    assert wgrad(n=0) == 0 and wgrad(n=0, dw=None) == 0
    for bad in (dict(dtype=3), dict(H=0), dict(I=0), dict(P=0), dict(first=2, n=2), dict(x=None), dict(dtype=ew.EW_F32, dw_dtype=ew.EW_BF16)):
        assert backward(**bad) == INVALID, bad
    need = ew.lib().moe_grouped_ffn_backward_workspace_bytes(4, 8, ew.EW_BF16)
    for bad in (dict(ws=None), dict(ws=C.c_void_p(264)), dict(ws_bytes=need - 1)):
        assert backward(**bad) == WORKSPACE, bad
    assert backward(accumulate=1, dw_dtype=ew.EW_BF16) == UNSUPPORTED
    assert backward(dx=None, n=0) == 0                                          # no gradient asked for
    un = ew.lib().moe_unpermute_backward
    assert un(None, None, ONE, ONE, 4, 2, 8, 1, ONE, None, None) == INVALID
    assert un(ONE, ONE, ONE, ONE, 4, 2, 8, 1, ONE, None, None) == INVALID       # y_sorted without dw
    assert un(ONE, None, ONE, ONE, 4, 2, 8, 1, ONE, ONE, None) == INVALID       # dw without y_sorted
    assert un(ONE, None, ONE, ONE, 4, 2, 8, 7, ONE, None, None) == INVALID
    assert un(ONE, None, ONE, ONE, 1 << 30, 2, 8, 1, ONE, None, None) == UNSUPPORTED
    assert un(None, None, None, None, 0, 2, 8, 1, None, None, None) == 0


def test_four_bit_calls_refuse_on_the_host():
    lib = ew.lib()
    assert lib.moe_w4_expert_bytes(2816, 2048) == 2816 * 2048 * 17 // 32
    for N, K in ((16, 33), (1, 32), (0, 32), (16, 0), (-1, 64)):
        assert lib.moe_w4_expert_bytes(N, K) == 0
        with pytest.raises(ew.EWError):
            ew.moe_w4_expert_bytes(N, K)
    for call in (lib.moe_quantize_w4, lib.moe_dequantize_w4):
        assert call(ONE, 1, 2, 16, 48, ONE, None) == UNSUPPORTED
        assert call(None, 1, 2, 16, 64, ONE, None) == INVALID and call(ONE, 1, 2, 16, 64, None, None) == INVALID
        assert call(ONE, 4, 2, 16, 64, ONE, None) == INVALID and call(ONE, 1, -1, 16, 64, ONE, None) == INVALID
        assert call(C.c_void_p(264), 1, 2, 16, 64, ONE, None) == INVALID        # not aligned to 16 bytes
        assert call(None, 1, 0, 16, 64, None, None) == 0
    assert lib.moe_grouped_gemm_w4(ONE, 4, 4, 2, 40, 16, 3, ONE, ONE, None, ONE, ONE, None) == UNSUPPORTED
    assert lib.moe_grouped_gemm_w4(ONE, 4, 4, 2, 64, 16, 3, ONE, ONE, None, None, ONE, None) == INVALID
    assert lib.moe_grouped_gemm_w4(ONE, 0, 0, 2, 64, 16, 3, None, None, None, None, None, None) == 0
    ffn = lib.moe_grouped_ffn_w4
    need = lib.moe_grouped_ffn_w4_workspace_bytes(4, 128)
    assert need >= 4 * 128 * 2 and lib.moe_grouped_ffn_w4_workspace_bytes(0, 128) == 0
    assert ffn(ONE, 4, 4, 2, 128, 40, 3, ONE, ONE, None, ONE, ONE, ONE, ONE, need, None) == UNSUPPORTED
    assert ffn(ONE, 4, 4, 2, 128, 128, 3, ONE, ONE, None, ONE, ONE, ONE, ONE, need - 1, None) == WORKSPACE
    assert ffn(ONE, 4, 4, 2, 128, 128, 3, ONE, ONE, None, ONE, ONE, ONE, None, need, None) == WORKSPACE
    assert ffn(ONE, 4, 4, 2, 128, 128, 3, ONE, ONE, None, None, ONE, ONE, ONE, need, None) == INVALID


def test_launches_too_large_are_refused():
    """2^24 tiles of 256 threads are more than a launch can have; 2 I has to fit an int."""
    many = 2 ** 31 - 1
    assert gemm(dtype=ew.EW_F32, rows=many, K=7, N=7, k=1) == UNSUPPORTED and b"too many" in ew.lib().ew_last_error()
    assert gemm(rows=many, K=8, N=8 * 256 * 4, k=1) == UNSUPPORTED
    assert wgrad(dtype=ew.EW_F32, K=2 ** 18, N=2 ** 18) == UNSUPPORTED
    assert ew.lib().moe_grouped_gemm_w4(ONE, 4, many, 1, 128, 16 * 64 * 4, 2 ** 30, ONE, ONE, None, ONE, ONE, None) == UNSUPPORTED
    assert backward(I=2 ** 30) == INVALID
    assert ew.lib().moe_grouped_ffn_w4(ONE, 4, 4, 2, 128, 2 ** 30, 3, ONE, ONE, None, ONE, ONE, ONE, ONE, 2 ** 40, None) == INVALID


def test_bindings_refuse_what_does_not_fit():
    """Tensors on the host, of another type, too small or not contiguous never reach the library."""
    x, c, off = torch.zeros(4, 64, dtype=torch.bfloat16), torch.zeros(3, dtype=torch.int32), torch.zeros(4, dtype=torch.int32)
    w = torch.zeros(3, 16, 64, dtype=torch.bfloat16)
    with pytest.raises(ValueError, match="current HIP device"):
        ew.moe_grouped_gemm(x, 1, 16, 3, c, off, None, w)
    need = ew.binding._need
    with pytest.raises(TypeError):
        need("w", w.float(), torch.bfloat16, 1, x)
    with pytest.raises(ValueError, match="contiguous"):
        need("w", w.transpose(1, 2), torch.bfloat16, 1, x)
    with pytest.raises(ValueError, match="needed"):
        need("w", w, torch.bfloat16, w.numel() + 1, x)
    with pytest.raises(ValueError, match="2-D"):
        ew.moe_grouped_gemm(x.t(), 1, 16, 3, c, off, None, w)
    with pytest.raises(TypeError):
        ew.moe_grouped_gemm_w4(x.float(), 1, 16, 3, c, off, None, 0)
    with pytest.raises(TypeError):
        ew.moe_grouped_ffn_w4(x.float(), 1, 16, 3, c, off, None, 0, 0)
    with pytest.raises(ValueError, match="dy"):
        ew.moe_grouped_gemm_wgrad(x.float(), x, 1, 3, c, off, None)


def test_reference_gradients_agree_with_differences():
    g = torch.Generator().manual_seed(0)
    H, I, offsets = 6, 5, torch.tensor([0, 3, 3, 7])
    x, dy = torch.randn((7, H), generator=g, dtype=torch.float64), torch.randn((7, H), generator=g, dtype=torch.float64)
    w13, w2 = torch.randn((3, 2 * I, H), generator=g, dtype=torch.float64), torch.randn((3, H, I), generator=g, dtype=torch.float64)

    def loss():
        return float((ref.ffn(x, w13, w2, offsets, False)[0] * dy).sum())

    (dx, _), (d13, _), (d2, _) = ref.ffn_backward(x, dy, w13, w2, offsets, False, False)
    rng = np.random.default_rng(1)
    for t, d in ((x, dx), (w13, d13), (w2, d2)):
        for _ in range(12):
            i = tuple(int(rng.integers(n)) for n in t.shape)
            old, eps = float(t[i]), 1e-6
            t[i] = old + eps
            up = loss()
            t[i] = old - eps
            down = loss()
            t[i] = old
            assert abs((up - down) / (2 * eps) - float(d[i])) <= 1e-7 * (1 + abs(float(d[i])))


def test_reference_quantiser_is_the_nearest_value():
    rng = np.random.default_rng(2)
    w = rng.standard_normal((1, 8, 64)) * 0.1
    codes, scales = ref.quantize_w4(w)
    v = ref.values_w4(codes, scales)
    step = 2.0 ** (scales[..., None].astype(float) - 127)
    inside = np.abs(w.reshape(1, 8, 2, 32)) <= 6 * step
    off = np.abs(v - w).reshape(1, 8, 2, 32)
    assert (off[inside] <= np.broadcast_to(step, off.shape)[inside]).all() and (off <= 2 * step).all()
    assert np.array_equal(ref.pack_w4(codes, scales)[0, :4], codes.reshape(-1, 2)[:4, 0] | codes.reshape(-1, 2)[:4, 1] << 4)
