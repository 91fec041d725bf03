"""Every kernel of the grouped products on rows that reach it, and values that its arithmetic can get wrong, against 64 bits."""
import numpy as np
import pytest
import torch

import grouped_bounds as bounds
import grouped_ref as ref
import test_gpu_grouped_products as products

pytestmark = pytest.mark.gpu

close, gen, normal = products.close, products.gen, products.normal


@pytest.fixture(scope="module")
def ew():
    import paper_2508_17624_amd as m
    assert torch.cuda.is_available(), "GPU tests need a GPU"
    m.lib()
    return m


# ------------------------------------------------------------------------------------------------ fp32 gradients
@pytest.mark.parametrize("H,I", [(8, 332), (5, 331)], ids=["16-byte loads", "single loads"])
def test_fp32_swiglu_gradients_of_large_gates(ew, H, I):
    """Gates of -80 to 80, read back one by one: x and dy are unit vectors, so g, u and da are weights, without a rounding, dw13's first
    column is [dg; du] and dw2's first row is a.

    With e = 2^-24, a rounding: exp is off by 2 e (one unit in the last place), 1 + exp by 3 e, s = 1 / (1 + exp) by 4 e, g s by 5 e, a = g s u
    and du = da g s by 6 e.  phi = s + g s (1 - s) has 1 - s off by 4 e s + e (1 - s) absolutely, the product by |g s| (7 e (1 - s) + 4 e s), the sum
    by 4 e s and e |phi| more, dg = da u phi by 2 e |phi| more."""
    g = torch.cat([torch.linspace(-80, 80, I - 11, dtype=torch.float64), torch.tensor([-1.2784645, -1.27, -1e-3, 0.0, 1e-3, -1e-30, 30.0, -30.0, 1.0, -1.0, -79.9])]).float()
    u, da = normal(gen(31), I, dtype="f32") + 2, normal(gen(32), I, dtype="f32") - 2
    w13, w2 = torch.randn((1, 2 * I, H), generator=gen(33)), torch.randn((1, H, I), generator=gen(34))
    w13[0, :I, 0], w13[0, I:, 0], w2[0, 0] = g, u, da
    unit = torch.zeros(1, H)
    unit[0, 0] = 1
    c, off = torch.tensor([1], dtype=torch.int32), torch.tensor([0, 1], dtype=torch.int32)
    _, d13, d2 = ew.moe_grouped_ffn_backward(unit.cuda(), unit.cuda(), 1, I, 1, c.cuda(), off.cuda(), None, w13.cuda(), w2.cuda())
    g, u, da, e = g.double(), u.double(), da.double(), 1.01 * 2.0 ** -24
    s, r = torch.sigmoid(g), torch.sigmoid(-g)   # r = 1 - s
    gs = g * s
    phi = s + gs * r
    e_phi = e * (4 * s + gs.abs() * (7 * r + 4 * s) + 3 * phi.abs())
    close(d2[0, 0], (gs * u, 6 * e * (gs * u).abs()), "a")
    close(d13[0, I:, 0], (da * gs, 6 * e * (da * gs).abs()), "du")
    close(d13[0, :I, 0], (da * u * phi, (da * u).abs() * e_phi), "dg")


@pytest.mark.parametrize("H,I,counts", [(264, 72, products.RAGGED), (640, 264, [0, 300, 129, 0, 1, 1])], ids=["small tiles", "large tiles"])
def test_ffn_gradients_round_dg_du_and_a_alone(ew, H, I, counts):
    """bf16: dg, du and a are rounded between the products and nothing else is.  Element by element, and in the relative error of the weight
    gradients in fp32, which then comes from one rounding: a half step of 2^-8 at most, uniform, is 2^-8 / sqrt(3) in the mean square."""
    g, k, P = gen(41), 2, len(counts)
    c, off, por, tok, tokens = ref.rows_of(counts, g, k=k)
    x, dy = normal(g, tokens, H), normal(g, len(tok), H, std=0.5)
    w13, w2 = normal(g, P, 2 * I, H, std=H ** -0.5), normal(g, P, H, I, std=I ** -0.5)
    got = ew.moe_grouped_ffn_backward(x.cuda(), dy.cuda(), k, I, P, c.cuda(), off.cuda(), por.cuda(), w13.cuda(), w2.cuda())
    want = bounds.ffn_backward(x.double()[tok], dy.double(), w13.double(), w2.double(), off, True, False)
    for name, a, b in zip(("dx", "dw13", "dw2"), got, want):
        close(a, b, name)
    for name, a, (v, _) in zip(("dw13", "dw2"), got[1:], want[1:]):
        assert float((a.cpu().double() - v).norm() / v.norm()) <= bounds.ONE_ROUNDING_RMS, name


# ------------------------------------------------------------------------------------------------ rows that reach each kernel
TWO_TILES = [0, 40, 31, 0, 33, 16]   # 20 rows a slot on average, slots of one, two and three tiles of 16 rows


@pytest.mark.parametrize("K", [128, 2048, 2176, 4096])
def test_four_bit_product_of_two_row_tiles(ew, K):
    """16 to 32 rows a slot on average and up to 4096 elements: workgroups of 4 and of 8 waves with two tiles of rows."""
    rng, g, k, P, N = np.random.default_rng(42), gen(42), 3, len(TWO_TILES), 144
    packed, w = products.random_w4(rng, P, N, K)
    packed[torch.tensor(TWO_TILES) == 0] = 255
    for shuffled in (True, False):
        c, off, por, tok, tokens = ref.rows_of(TWO_TILES, g, k=k if shuffled else 1, shuffled=shuffled)
        x = normal(g, tokens, K)
        out = torch.full((len(tok) + 3, N), 7.0, dtype=torch.bfloat16, device="cuda")
        if shuffled:
            por = torch.cat([por, torch.full((3,), 2 ** 30, dtype=torch.int32)])
            ew.moe_grouped_gemm_w4(x.cuda(), k, N, P, c.cuda(), off.cuda(), por.cuda(), packed.cuda(), out=out, num_rows=len(tok) + 3)
        else:
            ew.moe_grouped_gemm_w4(x.cuda(), 1, N, P, c.cuda(), off.cuda(), None, packed.cuda(), out=out)
        close(out[:len(tok)], ref.gemm(x.double()[tok], w, off, True))
        assert (out[len(tok):] == 7.0).all()


@pytest.mark.parametrize("H,I", [(128, 128), (2048, 128), (2176, 128), (4096, 128), (128, 2176)])
def test_four_bit_ffn_of_two_row_tiles(ew, H, I):
    rng, g, k, P = np.random.default_rng(43), gen(43), 2, len(TWO_TILES)
    p13, w13 = products.random_w4(rng, P, 2 * I, H, spread=1)
    p2, w2 = products.random_w4(rng, P, H, I, spread=1)
    c, off, por, tok, tokens = ref.rows_of(TWO_TILES, g, k=k)
    x = normal(g, tokens, H)
    y = ew.moe_grouped_ffn_w4(x.cuda(), k, I, P, c.cuda(), off.cuda(), por.cuda(), p13.cuda(), p2.cuda(), num_rows=len(tok))
    close(y, ref.ffn(x.double()[tok], w13, w2, off, True))


@pytest.mark.parametrize("K,N", [(200, 72), (136, 128), (72, 264), (640, 384)])
def test_many_rows_that_are_not_looked_up(ew, K, N):
    """The bf16 tiles, 128 and 256 wide, on rows that lie as they are used."""
    products.run_gemm(ew, products.RAGGED, K, N, "fwd", "bf16", 1, False, 44)


@pytest.mark.parametrize("H,I,counts", [(128, 128, products.RAGGED), (256, 256, [300, 0, 700])], ids=["small tiles", "large tiles"])
def test_four_bit_ffn_of_rows_that_are_not_looked_up(ew, H, I, counts):
    rng, g, P = np.random.default_rng(48), gen(48), len(counts)
    p13, w13 = products.random_w4(rng, P, 2 * I, H, spread=1)
    p2, w2 = products.random_w4(rng, P, H, I, spread=1)
    empty = torch.tensor(counts) == 0
    p13[empty], p2[empty] = 255, 255
    c, off, _, tok, tokens = ref.rows_of(counts, g, k=1, shuffled=False)
    x = normal(g, tokens, H)
    y = ew.moe_grouped_ffn_w4(x.cuda(), 1, I, P, c.cuda(), off.cuda(), None, p13.cuda(), p2.cuda())
    close(y, ref.ffn(x.double(), w13, w2, off, True))


@pytest.mark.parametrize("H,I,counts", [(264, 72, products.RAGGED), (640, 264, [0, 300, 129, 0, 1, 1])], ids=["small tiles", "large tiles"])
def test_ffn_gradients_of_rows_that_are_not_looked_up(ew, H, I, counts):
    g, P = gen(49), len(counts)
    c, off, _, tok, tokens = ref.rows_of(counts, g, k=1, shuffled=False)
    x, dy = normal(g, tokens, H), normal(g, tokens, H, std=0.5)
    w13, w2 = normal(g, P, 2 * I, H, std=H ** -0.5), normal(g, P, H, I, std=I ** -0.5)
    got = ew.moe_grouped_ffn_backward(x.cuda(), dy.cuda(), 1, I, P, c.cuda(), off.cuda(), None, products.poison(w13, counts).cuda(), products.poison(w2, counts).cuda())
    for name, a, b in zip(("dx", "dw13", "dw2"), got, bounds.ffn_backward(x.double(), dy.double(), w13.double(), w2.double(), off, True, False)):
        close(a, b, name)


def test_four_bit_tiles_keep_scales_of_255_to_their_feature(ew):
    """As the few-row kernels: one output is NaN in every row, the others are as without it."""
    K, N, counts = 128, 32, [300, 0, 90]
    rng, g = np.random.default_rng(45), gen(45)
    c, off, por, tok, tokens = ref.rows_of(counts, g, k=1)
    codes = rng.integers(0, 16, (3, N, K)).astype(np.uint8)
    scales = rng.integers(100, 140, (3, N, K // 32)).astype(np.uint8)
    x = normal(g, tokens, K)
    v = torch.from_numpy(ref.values_w4(codes, scales))
    scales[0, 3, 1], scales[2, 31, 3] = 255, 255
    y = ew.moe_grouped_gemm_w4(x.cuda(), 1, N, 3, c.cuda(), off.cuda(), por.cuda(), torch.from_numpy(ref.pack_w4(codes, scales)).cuda()).cpu()
    assert torch.isnan(y[:300, 3]).all() and torch.isnan(y[300:, 31]).all() and int(torch.isnan(y).sum()) == 390
    value, bound = ref.gemm(x.double()[tok], v, off, True)
    hit = torch.isnan(y)
    y[hit], value[hit] = 0, 0
    close(y, (value, bound))


# ------------------------------------------------------------------------------------------------ places, exchanged operands
@pytest.mark.parametrize("counts", [[0, 2, 1, 3, 0, 1], [5, 40, 0, 300, 17, 64]], ids=["few", "many"])
@pytest.mark.parametrize("K,N,dtype", [(256, 144, "bf16"), (640, 384, "bf16"), (36, 100, "bf16"), (36, 100, "f32")])
def test_a_rows_bits_do_not_depend_on_its_place(ew, K, N, dtype, counts):
    """The same rows in the opposite order inside their slots, the slots in the opposite order: the same bits."""
    g, P = gen(46), len(counts)
    c, off, por, tok, tokens = ref.rows_of(counts, g, k=1, shuffled=False)
    x, wf, wb = normal(g, tokens, K, dtype=dtype).cuda(), normal(g, P, N, K, std=0.1, dtype=dtype).cuda(), normal(g, P, K, N, std=0.1, dtype=dtype).cuda()
    back = torch.arange(tokens - 1, -1, -1)
    c2 = c.flip(0).contiguous()
    off2 = torch.cat([torch.zeros(1, dtype=torch.int32), c2.cumsum(0, dtype=torch.int32)])
    for w, transposed in ((wf, False), (wb, True)):
        y = ew.moe_grouped_gemm(x, 1, N, P, c.cuda(), off.cuda(), por.cuda(), w, transposed=transposed)
        y2 = ew.moe_grouped_gemm(x, 1, N, P, c2.cuda(), off2.cuda(), back.to(torch.int32).cuda(), w.flip(0).contiguous(), transposed=transposed)
        assert torch.equal(y2.flip(0), y)
    if K % 128 == 0 and dtype == "bf16":
        packed = ew.moe_quantize_w4(wf)
        y = ew.moe_grouped_gemm_w4(x, 1, N, P, c.cuda(), off.cuda(), por.cuda(), packed)
        y2 = ew.moe_grouped_gemm_w4(x, 1, N, P, c2.cuda(), off2.cuda(), back.to(torch.int32).cuda(), packed.flip(0).contiguous())
        assert torch.equal(y2.flip(0), y)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_weight_gradient_of_the_transposed_product(ew, dtype):
    """y = W^T x with x in sorted rows: dW[k][n] = sum_r x[r][k] dy[r][n] is the weight gradient with dy and x exchanged."""
    g, counts, K, N = gen(47), [0, 3, 70, 129, 0, 300], 136, 264
    c, off, _, tok, tokens = ref.rows_of(counts, g, k=1, shuffled=False)
    x, dy = normal(g, tokens, K, dtype=dtype), normal(g, tokens, N, dtype=dtype)
    dw = ew.moe_grouped_gemm_wgrad(x.cuda(), dy.cuda(), 1, len(counts), c.cuda(), off.cuda(), None)
    assert dw.shape == (len(counts), K, N)
    close(dw, ref.wgrad(x.double(), dy.double(), off, False))


# ------------------------------------------------------------------------------------------------ nothing, and a lot
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("mapped", [True, False])
def test_calls_without_rows(ew, mapped, dtype):
    """No token at all, and tokens without a row: empty results, zero gradients, sums kept."""
    P, H, I, dt = 5, 128, 64, products.DT[dtype]
    zero = lambda *shape: torch.zeros(shape, dtype=torch.int32, device="cuda")
    w13, w2 = (torch.full(s, float("nan"), dtype=dt, device="cuda") for s in ((P, 2 * I, H), (P, H, I)))
    for T in (0, 3):
        x, none = torch.ones((T, H), dtype=dt, device="cuda"), torch.empty((0, H), dtype=dt, device="cuda")
        at = (P, zero(P), zero(P + 1), zero(0) if mapped else None)
        assert ew.moe_grouped_gemm(x, 2, 2 * I, *at, w13, num_rows=0).shape == (0, 2 * I)
        assert not ew.moe_grouped_gemm_wgrad(none, x, 2, *at).any()
        kept = ew.moe_grouped_gemm_wgrad(none, x, 2, *at, accumulate=True, out=torch.full((P, H, H), 3.0, device="cuda"))
        assert (kept == 3).all()
        dx, d13, d2 = ew.moe_grouped_ffn_backward(x, none, 2, I, *at, w13, w2)
        assert dx.shape == (0, H) and d13.shape == w13.shape and d2.shape == w2.shape and not d13.any() and not d2.any()
        if dtype == "bf16":
            packed = torch.full((P, ew.moe_w4_expert_bytes(2 * I, H)), 255, dtype=torch.uint8, device="cuda")
            assert ew.moe_grouped_gemm_w4(x, 2, 2 * I, *at, packed, num_rows=0).shape == (0, 2 * I)
            assert ew.moe_grouped_ffn_w4(x, 2, I, *at, packed, packed, num_rows=0).shape == (0, H)
    # room for rows, none of them there
    out = torch.full((6, 2 * I), 7.0, dtype=dt, device="cuda")
    ew.moe_grouped_gemm(x, 2, 2 * I, P, zero(P), zero(P + 1), zero(6) if mapped else None, w13, out=out, num_rows=6)
    assert (out == 7).all()
    dy, dw = ew.moe_unpermute_backward(torch.empty((0, H), dtype=dt, device="cuda"), zero(0), torch.empty((0, 2), device="cuda"), torch.empty((0, H), dtype=dt, device="cuda"))
    assert dy.shape == (0, H) and dw.shape == (0, 2)
    assert ew.moe_quantize_w4(torch.empty((0, 16, 64), dtype=dt, device="cuda")).shape == (0, ew.moe_w4_expert_bytes(16, 64))


def test_results_and_packed_experts_beyond_4_gib(ew):
    """Weight gradients and 4-bit experts whose slots lie further from the base than 32 bits reach."""
    g, N, K = gen(50), 2816, 2816
    P, at = 300, ((0, 5), (290, 40), (299, 130))
    counts = [0] * P
    for s, n in at:
        counts[s] = n
    c, off, por, tok, tokens = ref.rows_of(counts, g, k=2)
    x, dy = normal(g, tokens, K), normal(g, len(tok), N)
    dw = ew.moe_grouped_gemm_wgrad(dy.cuda(), x.cuda(), 2, P, c.cuda(), off.cuda(), por.cuda(), dtype=torch.bfloat16)   # 4.8 GB
    for s, i, j in ref.slots_of(off):
        close(dw[s:s + 1], ref.wgrad(dy.double()[i:j], x.double()[tok[i:j]], torch.tensor([0, j - i]), True), f"slot {s}")
        dw[s] = 0
    assert not any(dw[i:i + 10].any() for i in range(0, P, 10)), "slots without rows"
    del dw
    P, at = 1200, ((0, 3), (1100, 20), (1199, 260))                                                                    # 5.1 GB
    counts = [0] * P
    for s, n in at:
        counts[s] = n
    rng = np.random.default_rng(50)
    packed = torch.full((P, ew.moe_w4_expert_bytes(N, K)), 255, dtype=torch.uint8, device="cuda")
    values = {}
    for s, _ in at:
        one, values[s] = products.random_w4(rng, 1, N, K)
        packed[s] = one[0].cuda()
    c, off, por, tok, tokens = ref.rows_of(counts, g, k=2)
    x = normal(g, tokens, K)
    y = ew.moe_grouped_gemm_w4(x.cuda(), 2, N, P, c.cuda(), off.cuda(), por.cuda(), packed, num_rows=len(tok))
    for s, i, j in ref.slots_of(off):
        close(y[i:j], ref.gemm(x.double()[tok[i:j]], values[s], torch.tensor([0, j - i]), True), f"4 bits, slot {s}")
