"""Calls of the grouped products and the 4-bit experts that are refused before anything is launched, and which kernel takes which form.
Nothing here reaches a GPU: addresses are never dereferenced, tensors lie on the host."""
import ctypes as C

import pytest
import torch

import paper_2508_17624_amd as ew

ONE = C.c_void_p(256)   # never dereferenced
INVALID, UNSUPPORTED = -1, -6


def rows_on_host():
    """(x, dy, counts, offsets) of two tokens, one row each, on the host: any call that gets past the checks of types and sizes ends at the
    check of devices."""
    x = torch.zeros(2, 64, dtype=torch.bfloat16)
    return x, x.clone(), torch.zeros(3, dtype=torch.int32), torch.zeros(4, dtype=torch.int32)


@pytest.mark.parametrize("dtype", [torch.float16, torch.int16, torch.uint8, torch.float64, torch.int32])
def test_weight_gradients_of_other_types_are_refused(dtype):
    """The kernels write float32 or bfloat16: into 2-byte tensors of another type they would put wrong numbers, and past the end of 1-byte ones."""
    x, dy, c, off = rows_on_host()
    with pytest.raises(TypeError, match="unsupported dtype"):
        ew.moe_grouped_ffn_backward(x, dy, 1, 32, 3, c, off, None, 0, 0, dw_dtype=dtype)
    out = torch.zeros(3, 64, 64, dtype=dtype)
    with pytest.raises(TypeError, match="unsupported dtype"):
        ew.moe_grouped_gemm_wgrad(dy, x, 1, 3, c, off, None, dtype=dtype, out=out)


def test_a_layer_refuses_a_pool_of_other_experts():
    """A pass over a pool of 4-bit experts would read bf16 weights 3.8 times too far apart, past the end of the pool's range."""
    from paper_2508_17624_amd.layer import MoELayer, MoEStack
    M, H, I, k = 4, 64, 32, 2
    Wg = torch.zeros(M, H)
    sizes = {"4 bits": (ew.moe_w4_expert_bytes(2 * I, H), ew.moe_w4_expert_bytes(H, I)), "bf16": (2 * I * H * 2, H * I * 2),
             "f32": (2 * I * H * 4, H * I * 4), "other H": (2 * I * H * 4, H * I * 2)}
    for name, (b13, b2) in sizes.items():
        pool = ew.ExpertPool(1, M, 1, 2, b13, b2, flags=ew.EW_POOL_FAKE)
        for dtype, fits in ((torch.bfloat16, "bf16"), (torch.float32, "f32")):
            if name == fits:
                assert MoELayer(pool, 0, Wg, None, None, k, I, 8, dtype).H == H
                continue
            with pytest.raises(ValueError, match="bytes"):
                MoELayer(pool, 0, Wg, None, None, k, I, 8, dtype)
            with pytest.raises(ValueError, match="bytes"):
                MoEStack(pool, [Wg], [(None, None)], k, I, 8, dtype)
        pool.close()


def test_a_layer_takes_a_pool_that_states_no_sizes():
    """Weights that lie elsewhere than in an ExpertPool: an object with M, N, P and view() is enough."""
    from types import SimpleNamespace
    from paper_2508_17624_amd.layer import MoELayer
    pool = SimpleNamespace(M=4, N=1, P=6, view=lambda layer: (256, 512, 1024, 6))
    assert MoELayer(pool, 0, torch.zeros(4, 64), None, None, 2, 32, 8, torch.bfloat16).w2_base == 512


def test_a_pool_refuses_weights_shorter_than_its_experts():
    """4-bit experts handed to a bf16 pool, or too few of them, would be copied from past the end of the tensor."""
    M, H, I = 3, 64, 32
    pool = ew.ExpertPool(1, M, 1, 2, 2 * I * H * 2, H * I * 2, flags=ew.EW_POOL_FAKE)
    w13, w2 = torch.zeros(M, 2 * I, H, dtype=torch.bfloat16), torch.zeros(M, H, I, dtype=torch.bfloat16)
    packed = torch.zeros(M, ew.moe_w4_expert_bytes(2 * I, H), dtype=torch.uint8)
    for a, b in ((packed, w2), (w13[:2], w2), (w13, w2[:2])):
        with pytest.raises(ValueError, match="bytes"):
            pool.map(0, 0, list(range(M)), a, b)
    pool.map(0, 0, list(range(M)), w13, w2)
    pool.close()


def test_sizes_whose_loops_would_wrap_are_refused():
    """A contraction, a width or a slot's rows within a step of 2^31: the index of the step behind the last one has no 32-bit value."""
    lib, most = ew.lib(), 2 ** 31 - 1024
    for big in (2 ** 31 - 1, most + 1):
        for dtype in (ew.EW_F32, ew.EW_BF16):
            for K, N in ((big, 1), (1, big)):
                assert lib.moe_grouped_gemm(ONE, dtype, 1, 1, 1, K, N, 1, 0, ONE, ONE, ONE, ONE, ONE, None) == UNSUPPORTED
                assert lib.moe_grouped_gemm_wgrad(ONE, ONE, dtype, 1, 1, 1, K, N, 1, ONE, ONE, ONE, 0, 1, ew.EW_F32, 0, ONE, None) == UNSUPPORTED
            assert lib.moe_grouped_gemm(ONE, dtype, big, big, 1, 1, 1, 1, 0, ONE, ONE, ONE, ONE, ONE, None) == UNSUPPORTED
            assert lib.moe_grouped_gemm_wgrad(ONE, ONE, dtype, big, big, 1, 1, 1, 1, ONE, ONE, ONE, 0, 1, ew.EW_F32, 0, ONE, None) == UNSUPPORTED
            for H, I, rows in ((big, 1, 1), (1, 2 ** 30 - 1, 1), (1, 1, big)):
                assert lib.moe_grouped_ffn_backward(ONE, ONE, dtype, rows, rows, 1, H, I, 1, ONE, ONE, ONE, ONE, ONE, ONE, 0, 1, ew.EW_F32, 0, ONE, ONE, ONE,
                                                    2 ** 62, None) == UNSUPPORTED
            assert lib.moe_unpermute_backward(ONE, None, ONE, ONE, 1, 1, big, dtype, ONE, None, None) == UNSUPPORTED
    big = 2 ** 31 - 512
    assert lib.moe_grouped_gemm_w4(ONE, 1, 1, 1, big, 1, 1, ONE, ONE, ONE, ONE, ONE, None) == UNSUPPORTED
    assert lib.moe_grouped_ffn_w4(ONE, 1, 1, 1, big, 32, 1, ONE, ONE, ONE, ONE, ONE, ONE, ONE, 2 ** 40, None) == UNSUPPORTED
    assert b"at most" in lib.ew_last_error()


@pytest.mark.parametrize("tokens,rows", [(2 ** 29, 2 ** 27), (2 ** 22 - 1, 2 ** 22 - 1)])
def test_launches_of_too_many_tiles_are_refused(tokens, rows):
    """2^24 tiles of 256 threads are more than a launch can have, whatever the sizes themselves are."""
    lib, wide = ew.lib(), 2 ** 15
    assert lib.moe_grouped_gemm(ONE, ew.EW_F32, tokens, rows, 1, 7, wide + 1, 4, 0, ONE, ONE, ONE, ONE, ONE, None) == UNSUPPORTED
    assert b"too many for one launch" in lib.ew_last_error()
    assert lib.moe_grouped_gemm(ONE, ew.EW_BF16, tokens, rows, 1, 8, 64 * wide, 4, 0, ONE, ONE, ONE, ONE, ONE, None) == UNSUPPORTED
    assert b"too many for one launch" in lib.ew_last_error()


def test_bindings_refuse_numbers_that_do_not_fit_32_bits():
    """ctypes hands the low 32 bits on: 2^32 + 4 rows would run as 4, 2^32 features as none."""
    x, dy, c, off = rows_on_host()
    w, big = torch.zeros(3, 16, 64, dtype=torch.bfloat16), 2 ** 32 + 4
    por = torch.zeros(1, dtype=torch.int32).expand(big)          # no memory behind it
    wide, many = torch.empty(big, 0), torch.zeros(1, 1).expand(big, 1)
    for call in (lambda: ew.moe_grouped_gemm(x, 1, 16, 3, c, off, por, w, num_rows=big), lambda: ew.moe_grouped_gemm(x, 1, big, 3, c, off, None, 0),
                 lambda: ew.moe_grouped_gemm(x, big, 16, 3, c, off, por, w, num_rows=2), lambda: ew.moe_grouped_gemm(x, 1, 16, big, c, off, None, 0),
                 lambda: ew.moe_grouped_gemm(x, 2 ** 31, 16, 3, c, off, None, w), lambda: ew.moe_grouped_gemm_wgrad(dy, x, 1, big, c, off, None, num_slots=1),
                 lambda: ew.moe_grouped_ffn_backward(x, dy, 1, big, 3, c, off, None, 0, 0), lambda: ew.moe_grouped_gemm_w4(x, 1, big, 3, c, off, None, 0),
                 lambda: ew.moe_grouped_ffn_w4(x, 1, 2 ** 30, 3, c, off, None, 0, 0), lambda: ew.moe_unpermute_backward(wide, None, many),
                 lambda: ew.moe_grouped_gemm_wgrad(dy, x, 1, 3, c, off, None, first_slot=2 ** 32 + 1, num_slots=1),
                 lambda: ew.moe_grouped_ffn_backward(x, dy, 1, 32, 3, c, off, None, 0, 0, first_slot=1 - 2 ** 32, num_slots=1),
                 lambda: ew.moe_w4_expert_bytes(big, 128), lambda: ew.moe_w4_expert_bytes(16, 2 ** 32 + 32)):
        with pytest.raises(ValueError, match="below 2\\^31"):
            call()


def test_rows_without_a_token_are_refused():
    """Without pair_of_row row r is pair r: with more rows than pairs the last ones would be read from behind x."""
    lib = ew.lib()
    need = lib.moe_grouped_ffn_backward_workspace_bytes(9, 32, ew.EW_BF16)
    for dtype in (ew.EW_F32, ew.EW_BF16):
        assert lib.moe_grouped_gemm(ONE, dtype, 4, 9, 2, 32, 16, 3, 0, ONE, ONE, None, ONE, ONE, None) == INVALID
        assert b"pair_of_row" in lib.ew_last_error()
        assert lib.moe_grouped_gemm_wgrad(ONE, ONE, dtype, 4, 9, 2, 32, 16, 3, ONE, ONE, None, 0, 3, ew.EW_F32, 0, ONE, None) == INVALID
        assert lib.moe_grouped_ffn_backward(ONE, ONE, dtype, 4, 9, 2, 32, 32, 3, ONE, ONE, None, ONE, ONE, ONE, 0, 3, ew.EW_F32, 0, ONE, ONE, ONE, 2 * need,
                                            None) == INVALID
    assert lib.moe_grouped_gemm_w4(ONE, 4, 9, 2, 32, 16, 3, ONE, ONE, None, ONE, ONE, None) == INVALID
    assert lib.moe_grouped_ffn_w4(ONE, 4, 9, 2, 32, 32, 3, ONE, ONE, None, ONE, ONE, ONE, ONE, 2 ** 20, None) == INVALID


def test_kernels_take_only_the_forms_that_they_have(tmp_path):
    """The choice of a kernel asks each whether it takes a product: direction, weights, and what becomes of the sums.  Sizes that suit
    every kernel, few rows."""
    import os
    import shutil
    import subprocess
    hipcc = "/opt/rocm/bin/hipcc" if os.path.exists("/opt/rocm/bin/hipcc") else shutil.which("hipcc")
    if not hipcc:
        pytest.skip("no hipcc")
    pkg = os.path.dirname(ew.__file__)
    src, exe = tmp_path / "forms.cpp", tmp_path / "forms"
    src.write_text('''#include "grouped_gemm.h"
int main() {
  ew::GemmArgs a{};
  void* p = (void*)256;
  a.g = {(int32_t*)p, (int32_t*)p, nullptr, 64, 64, 1};
  a.x = a.w = a.out = a.dh = p; a.da = (float*)p;
  a.K = a.N = 512; a.x_rows = 64; a.num_slots = 64; a.slot_bytes = 512 * 512 * 2;
  for (int way = 0; way < 3; ++way)
    for (int w = 0; w < 3; ++w)
      for (int ep = 0; ep < 4; ++ep) std::printf("%d %d %d %d %d\\n", way, w, ep, ew::stream_takes(way, w, ep, a), ew::tile_takes(way, w, ep, a));
}
''')
    subprocess.run([hipcc, "-x", "hip", "--offload-host-only", "-std=c++17", "-O0", "-I", os.path.join(pkg, "csrc"), "-I", os.path.join(os.path.dirname(pkg), "include"),
                    "-c", str(src), "-o", str(tmp_path / "forms.o")], check=True, timeout=100, capture_output=True)
    subprocess.run([hipcc, str(tmp_path / "forms.o"), os.path.join(pkg, "libexpertweave.so"), "-Wl,-rpath," + pkg, "-o", str(exe)], check=True, timeout=100,
                   capture_output=True)
    rows = [tuple(map(int, line.split())) for line in subprocess.run([str(exe)], check=True, capture_output=True, text=True, timeout=60).stdout.splitlines()]
    fwd, dgrad, wgrad = 0, 1, 2
    bf16, w4 = 1, 2
    to_bf16, to_f32, swiglu, back = 0, 1, 2, 3
    assert len(rows) == 36
    assert {r[:3] for r in rows if r[3]} == {(fwd, bf16, to_bf16), (fwd, w4, to_bf16), (fwd, w4, swiglu)}
    assert {r[:3] for r in rows if r[4]} == {(fwd, bf16, to_bf16), (fwd, bf16, back), (dgrad, bf16, to_bf16), (dgrad, bf16, to_f32), (wgrad, bf16, to_bf16),
                                             (wgrad, bf16, to_f32), (fwd, w4, to_bf16), (fwd, w4, swiglu)}
