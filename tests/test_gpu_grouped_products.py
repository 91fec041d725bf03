"""The experts' products one by one, their gradients, and 4-bit experts, against 64 bits (grouped_ref.py, element by element)."""
import numpy as np
import pytest
import torch

import grouped_ref as ref

pytestmark = pytest.mark.gpu

DT = {"bf16": torch.bfloat16, "f32": torch.float32}


@pytest.fixture(scope="module")
def ew():
    import paper_2508_17624_amd as m
    assert torch.cuda.is_available(), "GPU tests need a GPU"
    m.lib()
    return m


def gen(seed):
    return torch.Generator().manual_seed(seed)


def normal(g, *shape, std=1.0, dtype="bf16"):
    return (torch.randn(shape, generator=g) * std).to(DT[dtype])


def close(got, want, what=""):
    value, bound = want
    d = (got.detach().cpu().double() - value).abs()
    bad = ~(d <= bound + 1e-38)
    assert not bad.any(), f"{what}: {int(bad.sum())} of {bad.numel()} off, worst by {float((d / (bound + 1e-38))[bad].max()):.3g} bounds, first at {bad.nonzero()[0].tolist()}"


def poison(w, counts):
    """Slots without rows hold NaN: any read of them shows."""
    w = w.clone()
    w[torch.tensor(counts) == 0] = float("nan")
    return w


# counts on the tiles' borders (16, 64, 128, 256 and neighbours), single rows, empty slots first, last and in between
RAGGED = [0, 1, 16, 17, 0, 0, 63, 64, 65, 3, 127, 128, 129, 0, 255, 256, 257, 0]
FEW = [0, 1, 0, 2, 5, 0, 16, 1, 33, 0]
ONE = [0, 0, 1, 0]

SIZES = {"1x1": (1, 1), "7x13": (7, 13), "8x8": (8, 8), "36x100": (36, 100), "72x264": (72, 264), "128x16": (128, 16), "200x136": (200, 136),
         "640x384": (640, 384), "1408x512": (1408, 512)}


def run_gemm(ew, counts, K, N, way, dtype, k, mapped, seed, room=0):
    g = gen(seed)
    c, off, por, tok, tokens = ref.rows_of(counts, g, k=k, shuffled=mapped)
    rows = len(tok)
    x = normal(g, tokens, K, dtype=dtype)
    w = poison(normal(g, len(counts), *((N, K) if way == "fwd" else (K, N)), std=0.1, dtype=dtype), counts)
    out = torch.full((rows + room, N), 7.0, dtype=DT[dtype], device="cuda")
    pad = torch.full((room,), 2 ** 30, dtype=torch.int32)   # pairs of rows that do not exist: never looked at
    y = ew.moe_grouped_gemm(x.cuda(), k, N, len(counts), c.cuda(), off.cuda(), torch.cat([por, pad]).cuda() if mapped else None, w.cuda(),
                            transposed=way == "dgrad", out=out, num_rows=rows + room if mapped else rows)
    close(y[:rows], ref.gemm(x.double()[tok], w.double(), off, dtype == "bf16", way == "dgrad"), way)
    assert (y[rows:] == 7.0).all(), "rows behind the last one were written"


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("way", ["fwd", "dgrad"])
@pytest.mark.parametrize("size", SIZES, ids=list(SIZES))
def test_grouped_gemm(ew, size, way, dtype):
    K, N = SIZES[size]
    run_gemm(ew, RAGGED, K, N, way, dtype, 3, True, 1, room=70)
    run_gemm(ew, FEW, K, N, way, dtype, 1, False, 2)
    run_gemm(ew, ONE, K, N, way, dtype, 2, True, 3, room=1)


@pytest.mark.parametrize("way", ["fwd", "dgrad"])
def test_grouped_gemm_many_slots(ew, way):
    """More slots than one look of the chunk search covers (512), most of them empty; bits do not depend on the place in the batch."""
    rng = np.random.default_rng(5)
    counts = np.zeros(2048, int)
    counts[rng.choice(2048, 90, replace=False)] = rng.integers(1, 40, 90)
    counts[0], counts[511], counts[512], counts[2047] = 3, 70, 300, 9
    run_gemm(ew, counts.tolist(), 128, 64, way, "bf16", 2, True, 6)


def test_grouped_gemm_large_offsets(ew):
    """Weights beyond 4 GiB from the base: slot offsets are 64 bits wide."""
    P, N, K = 300, 2816, 2816   # 4.8 GB of weights
    g = torch.Generator(device="cuda").manual_seed(3)
    w = torch.empty((P, N, K), dtype=torch.bfloat16, device="cuda")
    counts = [0] * P
    for s, c in ((0, 5), (290, 40), (P - 1, 130)):
        counts[s] = c
        w[s].normal_(std=0.05, generator=g)
    c, off, por, tok, tokens = ref.rows_of(counts, gen(4), k=2)
    x = normal(gen(5), tokens, K)
    for transposed in (False, True):
        y = ew.moe_grouped_gemm(x.cuda(), 2, N, P, c.cuda(), off.cuda(), por.cuda(), w, transposed=transposed, num_rows=len(tok))
        for s, i, j in ref.slots_of(off):
            m = w[s].cpu().double()[None]
            close(y[i:j], ref.gemm(x.double()[tok[i:j]], m, torch.tensor([0, j - i]), True, transposed))


@pytest.mark.parametrize("dtype,out", [("bf16", "f32"), ("bf16", "bf16"), ("f32", "f32")])
@pytest.mark.parametrize("size", SIZES, ids=list(SIZES))
def test_grouped_gemm_wgrad(ew, size, dtype, out):
    K, N = SIZES[size]
    counts, k = RAGGED if K * N < 300000 else FEW, 3
    g = gen(7)
    c, off, por, tok, tokens = ref.rows_of(counts, g, k=k, spare=2)
    rows, P = len(tok), len(counts)
    x, dy = normal(g, tokens, K, dtype=dtype), normal(g, rows + 5, N, dtype=dtype)
    dy[rows:] = float("nan")    # rows that do not exist
    pad = torch.full((5,), 2 ** 30, dtype=torch.int32)
    want = ref.wgrad(dy.double()[:rows], x.double()[tok], off, out == "bf16")
    args = (dy.cuda(), x.cuda(), k, P, c.cuda(), off.cuda(), torch.cat([por, pad]).cuda())
    dw = ew.moe_grouped_gemm_wgrad(*args, dtype=DT[out])
    close(dw, want, "all slots")
    assert (dw[0] == 0).all(), "a slot without rows has zero gradient"
    part = ew.moe_grouped_gemm_wgrad(*args, first_slot=2, num_slots=5, dtype=DT[out])
    assert torch.equal(part, dw[2:7]), "bits of a range of slots"
    if out == "f32":
        start = torch.randn(dw.shape, generator=g).cuda()
        acc = ew.moe_grouped_gemm_wgrad(*args, accumulate=True, out=start.clone())
        v, b = want
        close(acc, (v + start.cpu().double(), b + 2.0 ** -23 * (v.abs() + start.cpu().double().abs())), "accumulated")
        assert torch.equal(acc[0], start[0])


def test_wgrad_keeps_a_slots_infinities_to_itself(ew):
    """Rows of the neighbouring slots hold infinities and NaN; a slot's sums must not see them where its last tile ends."""
    counts, K, N, k = [5, 33, 70, 1], 264, 136, 1
    g = gen(8)
    c, off, por, tok, tokens = ref.rows_of(counts, g, k=k)
    x, dy = normal(g, tokens, K), normal(g, len(tok), N)
    for s in (0, 2):
        dy[off[s]:off[s + 1]] = float("inf")
        x[tok[off[s]:off[s + 1]]] = float("nan")
    dw = ew.moe_grouped_gemm_wgrad(dy.cuda(), x.cuda(), k, 4, c.cuda(), off.cuda(), por.cuda()).cpu()
    for s in (1, 3):
        v, b = ref.wgrad(dy.double()[off[s]:off[s + 1]], x.double()[tok[off[s]:off[s + 1]]], torch.tensor([0, counts[s]]), False)
        close(dw[s:s + 1], (v, b))
    assert torch.isnan(dw[0]).all() and torch.isnan(dw[2]).all()


@pytest.mark.parametrize("K,tokens_more", [(2048, 0), (2048, 100), (1928, 0), (2056, 0)])
def test_grouped_gemm_few_rows(ew, K, tokens_more):
    """Around the longest contraction whose few rows the waves hold; with many tokens a workgroup takes two row tiles."""
    g, counts, k, N = gen(19), [1, 0, 3, 18, 2, 0, 1, 1], 2, 200
    c, off, por, tok, tokens = ref.rows_of(counts, g, k=k, spare=tokens_more)
    x, w = normal(g, tokens, K), poison(normal(g, len(counts), N, K, std=0.1), counts)
    y = ew.moe_grouped_gemm(x.cuda(), k, N, len(counts), c.cuda(), off.cuda(), por.cuda(), w.cuda(), num_rows=len(tok))
    close(y, ref.gemm(x.double()[tok], w.double(), off, True))


@pytest.mark.parametrize("shift", ["x", "w", "out"])
@pytest.mark.parametrize("counts", [[0, 2, 1, 0, 3], [130, 0, 70]], ids=["few", "many"])
def test_grouped_products_off_16_bytes(ew, counts, shift):
    """Buffers that begin two bytes past a 16-byte border take the kernel that reads single elements."""
    g, k, K, N = gen(20), 2, 128, 64
    c, off, por, tok, tokens = ref.rows_of(counts, g, k=k)
    rows, P = len(tok), len(counts)

    def place(t, moved):
        buf = torch.zeros(t.numel() + 8, dtype=t.dtype, device="cuda")
        v = buf[1 if moved else 0:][:t.numel()].view(t.shape)
        v.copy_(t)
        return v

    x, w, dy = normal(g, tokens, K), poison(normal(g, P, N, K, std=0.1), counts), normal(g, rows, N)
    out = place(torch.full((rows, N), 7.0, dtype=torch.bfloat16), shift == "out")
    ew.moe_grouped_gemm(place(x, shift == "x"), k, N, P, c.cuda(), off.cuda(), por.cuda(), place(w, shift == "w"), out=out, num_rows=rows)
    close(out, ref.gemm(x.double()[tok], w.double(), off, True), "fwd")
    dx = place(torch.full((rows, K), 7.0, dtype=torch.bfloat16), shift == "out")
    ew.moe_grouped_gemm(place(dy, shift == "x"), 1, K, P, c.cuda(), off.cuda(), None, place(w, shift == "w"), transposed=True, out=dx)
    close(dx, ref.gemm(dy.double(), w.double(), off, True, True), "dgrad")
    dw = place(torch.full((P, N, K), 7.0, dtype=torch.bfloat16), shift == "out")
    ew.moe_grouped_gemm_wgrad(place(dy, shift == "w"), place(x, shift == "x"), k, P, c.cuda(), off.cuda(), por.cuda(), dtype=torch.bfloat16, out=dw)
    close(dw, ref.wgrad(dy.double(), x.double()[tok], off, True)[:2], "wgrad")


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_rows_with_infinities_stay_alone(ew, dtype):
    """One token of infinities, one of NaN: their rows only."""
    counts, K, N = [20, 90], 136, 72
    g = gen(9)
    c, off, por, tok, tokens = ref.rows_of(counts, g, k=1)
    x, w = normal(g, tokens, K, dtype=dtype), normal(g, 2, N, K, std=0.1, dtype=dtype)
    clean = ew.moe_grouped_gemm(x.cuda(), 1, N, 2, c.cuda(), off.cuda(), por.cuda(), w.cuda()).cpu()
    x[tok[3]], x[tok[50]] = float("nan"), float("inf")
    y = ew.moe_grouped_gemm(x.cuda(), 1, N, 2, c.cuda(), off.cuda(), por.cuda(), w.cuda()).cpu()
    keep = torch.ones(110, dtype=torch.bool)
    keep[3] = keep[50] = False
    assert torch.equal(y[keep], clean[keep]) and torch.isnan(y[3]).all() and not torch.isfinite(y[50]).any()


# ------------------------------------------------------------------------------------------------ FFN gradients, combine
@pytest.mark.parametrize("dtype,out", [("bf16", "f32"), ("bf16", "bf16"), ("f32", "f32")])
@pytest.mark.parametrize("H,I,counts", [(128, 128, RAGGED), (264, 72, RAGGED), (36, 20, FEW), (15, 9, FEW), (256, 384, FEW), (8, 8, ONE)])
def test_grouped_ffn_backward(ew, H, I, counts, dtype, out):
    g, k, P = gen(11), 2, len(counts)
    c, off, por, tok, tokens = ref.rows_of(counts, g, k=k)
    rows = len(tok)
    x, dy = normal(g, tokens, H, dtype=dtype), normal(g, rows, H, std=0.5, dtype=dtype)
    w13 = normal(g, P, 2 * I, H, std=H ** -0.5, dtype=dtype)
    w2 = normal(g, P, H, I, std=I ** -0.5, dtype=dtype)
    want = ref.ffn_backward(x.double()[tok], dy.double(), w13.double(), w2.double(), off, dtype == "bf16", out == "bf16")
    args = (x.cuda(), dy.cuda(), k, I, P, c.cuda(), off.cuda(), por.cuda(), poison(w13, counts).cuda(), poison(w2, counts).cuda())
    got = ew.moe_grouped_ffn_backward(*args, dw_dtype=DT[out])
    for name, a, b in zip(("dx", "dw13", "dw2"), got, want):
        close(a, b, name)
    # an adapter's slots alone, without the input gradient; nothing at all but the input gradient
    first, n = 1, min(3, P - 1)
    part = ew.moe_grouped_ffn_backward(*args, first_slot=first, num_slots=n, dw_dtype=DT[out], want_dx=False)
    assert part[0] is None and torch.equal(part[1], got[1][first:first + n]) and torch.equal(part[2], got[2][first:first + n])
    only = ew.moe_grouped_ffn_backward(*args, num_slots=0)
    assert torch.equal(only[0], got[0]) and only[1] is None and only[2] is None
    if out == "f32":
        acc = ew.moe_grouped_ffn_backward(*args, accumulate=True, dw13=torch.ones_like(got[1]), dw2=torch.ones_like(got[2]))
        assert (acc[1] - 1 - got[1]).abs().max() <= 2.0 ** -22 * (1 + got[1].abs().max()) and (acc[2] - 1 - got[2]).abs().max() <= 2.0 ** -22 * (1 + got[2].abs().max())


@pytest.mark.parametrize("out", ["f32", "bf16"])
@pytest.mark.parametrize("H,I", [(640, 264), (264, 1032)])
def test_many_rows_on_the_large_tiles(ew, H, I, out):
    """Slots of several row chunks, widths that end inside a tile, in every direction, and the gradients' products of one another."""
    counts, k, g = [0, 300, 129, 0, 520, 1], 2, gen(21)
    c, off, por, tok, tokens = ref.rows_of(counts, g, k=k)
    P, rows = len(counts), len(tok)
    x, dy = normal(g, tokens, H), normal(g, rows, H, std=0.5)
    w13, w2 = normal(g, P, 2 * I, H, std=H ** -0.5), normal(g, P, H, I, std=I ** -0.5)
    want = ref.ffn_backward(x.double()[tok], dy.double(), w13.double(), w2.double(), off, True, out == "bf16")
    got = ew.moe_grouped_ffn_backward(x.cuda(), dy.cuda(), k, I, P, c.cuda(), off.cuda(), por.cuda(), poison(w13, counts).cuda(), poison(w2, counts).cuda(),
                                      dw_dtype=DT[out])
    for name, a, b in zip(("dx", "dw13", "dw2"), got, want):
        close(a, b, name)
    dh = normal(g, rows, 2 * I)
    args = (dh.cuda(), x.cuda(), k, P, c.cuda(), off.cuda(), por.cuda())
    v, b = ref.wgrad(dh.double(), x.double()[tok], off, out == "bf16")
    close(ew.moe_grouped_gemm_wgrad(*args, dtype=DT[out]), (v, b), "wgrad")
    if out == "f32":
        start = torch.randn(v.shape, generator=g)
        acc = ew.moe_grouped_gemm_wgrad(*args, accumulate=True, out=start.cuda())
        close(acc, (v + start.double(), b + 2.0 ** -23 * (v.abs() + start.double().abs())), "accumulated")
    h = ew.moe_grouped_gemm(x.cuda(), k, 2 * I, P, c.cuda(), off.cuda(), por.cuda(), poison(w13, counts).cuda(), num_rows=rows)
    close(h, ref.gemm(x.double()[tok], w13.double(), off, True), "fwd")
    dx = ew.moe_grouped_gemm(dh.cuda(), 1, H, P, c.cuda(), off.cuda(), None, poison(w13, counts).cuda(), transposed=True)
    close(dx, ref.gemm(dh.double(), w13.double(), off, True, True), "dgrad")


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("T,k,H", [(1, 1, 8), (5, 3, 100), (64, 6, 2048), (257, 8, 264), (3, 64, 7)])
def test_unpermute_backward(ew, T, k, H, dtype):
    g = gen(13)
    rop = torch.randperm(T * k, generator=g).to(torch.int32)
    w = torch.rand((T, k), generator=g)
    dout, y = normal(g, T, H, dtype=dtype), normal(g, T * k, H, dtype=dtype)
    dy, dw = ew.moe_unpermute_backward(dout.cuda(), rop.cuda(), w.cuda(), y.cuda())
    d = dout.double().repeat_interleave(k, 0)
    want = torch.zeros((T * k, H), dtype=torch.float64)
    want[rop.long()] = d * w.double().reshape(-1, 1)
    close(dy, (want, want.abs() * (ref.HALF_BF16 if dtype == "bf16" else 2.0 ** -24)), "dy")
    prod = d * y.double()[rop.long()]
    close(dw, (prod.sum(1).reshape(T, k), prod.abs().sum(1).reshape(T, k) * (H + 1) * ref.ADD_F32), "dw")
    again, none = ew.moe_unpermute_backward(dout.cuda(), rop.cuda(), w.cuda())
    assert torch.equal(again, dy) and none is None


def test_unpermute_backward_unaligned(ew):
    """Rows that wide accesses cannot take: a pointer that is not aligned to 16 bytes."""
    g, T, k, H = gen(14), 9, 2, 64
    rop, w = torch.randperm(T * k, generator=g).to(torch.int32), torch.rand((T, k), generator=g)
    dout, y = normal(g, T * H + 1)[1:].cuda().view(T, H), normal(g, T * k, H).cuda()
    shifted = torch.empty(T * H + 1, dtype=torch.bfloat16, device="cuda")[1:].view(T, H).copy_(dout)
    for a, b in zip(ew.moe_unpermute_backward(shifted, rop.cuda(), w.cuda(), y), ew.moe_unpermute_backward(dout.clone(), rop.cuda(), w.cuda(), y)):
        assert torch.allclose(a.float(), b.float(), rtol=2.0 ** -7, atol=1e-4)


# ------------------------------------------------------------------------------------------------ 4-bit experts
def special_groups(rng):
    """Weights that rounding, scaling and special values can get wrong, in groups of 32."""
    ties = np.array([0, .25, .75, 1.25, 1.75, 2.5, 3.5, 5, 6, 7, 7.99, .2499, .2501, 4, 5.001, 2.499] * 2) * np.where(np.arange(32) % 2, -1, 1)
    groups = [ties, ties * 2.0 ** -30, ties * 2.0 ** 60, np.zeros(32), -np.zeros(32), np.full(32, 2.0 ** -126), np.full(32, 3e38),
              np.r_[np.inf, np.ones(31)], np.r_[np.ones(31), np.nan], np.r_[1e-30, np.full(31, 1e30)], np.full(32, 2.0 ** -133), rng.standard_normal(32) * 0.02]
    return np.array(groups + [rng.standard_normal(32) * 10.0 ** rng.integers(-20, 20) for _ in range(52)]).astype(np.float32)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_quantize_w4(ew, dtype):
    w = torch.from_numpy(special_groups(np.random.default_rng(1))).reshape(2, 16, 64).to(DT[dtype])
    codes, scales = ref.quantize_w4(w.double().numpy())
    packed = ew.moe_quantize_w4(w.cuda())
    assert packed.shape == (2, ew.moe_w4_expert_bytes(16, 64))
    assert np.array_equal(packed.cpu().numpy(), ref.pack_w4(codes, scales))
    values = torch.from_numpy(ref.values_w4(codes, scales))
    for out in ("bf16", "f32"):
        got = ew.moe_dequantize_w4(packed, 16, 64, dtype=DT[out]).cpu().double()
        assert torch.equal(torch.nan_to_num(got, nan=1.25), torch.nan_to_num(values, nan=1.25))


def test_dequantize_w4_every_code_and_scale(ew):
    codes = np.tile(np.arange(16, dtype=np.uint8), (1, 256, 2))
    scales = np.arange(256, dtype=np.uint8).reshape(1, 256, 1)
    values = torch.from_numpy(ref.values_w4(codes, scales))
    packed = torch.from_numpy(ref.pack_w4(codes, scales)).cuda()
    for dtype in DT.values():
        got = ew.moe_dequantize_w4(packed, 256, 32, dtype=dtype).cpu().double()
        want = values.to(dtype).double()
        assert torch.equal(torch.nan_to_num(got, nan=1.25, posinf=2.5, neginf=-2.5), torch.nan_to_num(want, nan=1.25, posinf=2.5, neginf=-2.5))


def random_w4(rng, P, N, K, spread=3):
    codes = rng.integers(0, 16, (P, N, K)).astype(np.uint8)
    scales = rng.integers(122 - spread, 122 + spread, (P, N, K // 32)).astype(np.uint8)
    return torch.from_numpy(ref.pack_w4(codes, scales)), torch.from_numpy(ref.values_w4(codes, scales))


@pytest.mark.parametrize("counts", [RAGGED, FEW, ONE, [300, 0, 700]], ids=["ragged", "few", "one", "many"])
@pytest.mark.parametrize("K,N", [(128, 16), (128, 256), (256, 48), (640, 1280), (32, 16), (96, 32), (1408, 128), (2304, 64), (512, 144)])
def test_grouped_gemm_w4(ew, K, N, counts):
    rng, g, k, P = np.random.default_rng(2), gen(15), 3, len(counts)
    packed, w = random_w4(rng, P, N, K)
    packed[torch.tensor(counts) == 0] = 255    # NaN scales: any read of an empty slot shows
    c, off, por, tok, tokens = ref.rows_of(counts, g, k=k)
    x = normal(g, tokens, K)
    out = torch.full((len(tok) + 9, N), 7.0, dtype=torch.bfloat16, device="cuda")
    pad = torch.full((9,), 2 ** 30, dtype=torch.int32)
    y = ew.moe_grouped_gemm_w4(x.cuda(), k, N, P, c.cuda(), off.cuda(), torch.cat([por, pad]).cuda(), packed.cuda(), out=out, num_rows=len(tok) + 9)
    close(y[:len(tok)], ref.gemm(x.double()[tok], w, off, True))
    assert (y[len(tok):] == 7.0).all()


@pytest.mark.parametrize("counts", [RAGGED, FEW, ONE, [300, 0, 700]], ids=["ragged", "few", "one", "many"])
@pytest.mark.parametrize("H,I", [(128, 128), (256, 640), (896, 128), (32, 96), (64, 32), (1408, 256)])
def test_grouped_ffn_w4(ew, H, I, counts):
    rng, g, k, P = np.random.default_rng(3), gen(16), 2, len(counts)
    p13, w13 = random_w4(rng, P, 2 * I, H, spread=1)
    p2, w2 = random_w4(rng, P, H, I, spread=1)
    c, off, por, tok, tokens = ref.rows_of(counts, g, k=k)
    x = normal(g, tokens, H)
    y = ew.moe_grouped_ffn_w4(x.cuda(), k, I, P, c.cuda(), off.cuda(), por.cuda(), p13.cuda(), p2.cuda(), num_rows=len(tok))
    close(y, ref.ffn(x.double()[tok], w13, w2, off, True))


def test_w4_scales_of_every_size(ew):
    """Scales from the least to the largest; a scale of 255 makes its output NaN and no other."""
    K, N, rows = 128, 32, 20
    rng, g = np.random.default_rng(4), gen(17)
    codes = rng.integers(0, 16, (1, N, K)).astype(np.uint8)
    scales = rng.integers(30, 200, (1, N, 1)).repeat(4, 2).astype(np.uint8)
    scales[0, 0], scales[0, 1, 2], scales[0, 2] = 0, 255, 230
    x = normal(g, rows, K)
    c, off = torch.tensor([rows], dtype=torch.int32), torch.tensor([0, rows], dtype=torch.int32)
    y = ew.moe_grouped_gemm_w4(x.cuda(), 1, N, 1, c.cuda(), off.cuda(), None, torch.from_numpy(ref.pack_w4(codes, scales)).cuda()).cpu()
    v = torch.from_numpy(ref.values_w4(codes, scales))
    assert torch.isnan(y[:, 1]).all()
    v[0, 1] = 0
    y[:, 1] = 0
    ref_y, b = ref.gemm(x.double(), v, off, True)
    close(y, (ref_y, b + 2.0 ** -126))   # sums below the normal range may be flushed


@pytest.mark.parametrize("counts", [FEW, ONE, [0, 20, 16, 0, 32]], ids=["few", "one", "two row tiles"])
@pytest.mark.parametrize("K", [2048, 2176, 4096, 4224, 8192, 8320])
def test_w4_long_contractions(ew, K, counts):
    """Around the lengths at which more waves share a contraction, and past the longest that they hold."""
    rng, g, k, P, I = np.random.default_rng(5), gen(18), 2, len(counts), 32
    c, off, por, tok, tokens = ref.rows_of(counts, g, k=k)
    x = normal(g, tokens, K)
    packed, w = random_w4(rng, P, 144, K, spread=1)
    packed[torch.tensor(counts) == 0] = 255
    y = ew.moe_grouped_gemm_w4(x.cuda(), k, 144, P, c.cuda(), off.cuda(), por.cuda(), packed.cuda(), num_rows=len(tok))
    close(y, ref.gemm(x.double()[tok], w, off, True), "product")
    p13, w13 = random_w4(rng, P, 2 * I, K, spread=1)
    p2, w2 = random_w4(rng, P, K, I, spread=1)
    y = ew.moe_grouped_ffn_w4(x.cuda(), k, I, P, c.cuda(), off.cuda(), por.cuda(), p13.cuda(), p2.cuda(), num_rows=len(tok))
    close(y, ref.ffn(x.double()[tok], w13, w2, off, True), "FFN")


# ------------------------------------------------------------------------------------------------ as they are used
def test_training_step_of_one_adapter(ew):
    """Forward with the framework's routing, FFN and combine, backward with the new calls: the gradients are those that automatic
    differentiation finds in 64 bits."""
    T, k, M, E, H, I = 96, 2, 4, 2, 128, 128
    g = gen(21)
    P = M + E
    emap = torch.tensor([[0, 1, 2, 3], [0, 4, 2, 5]], dtype=torch.int32).cuda()   # the adapter tunes experts 1 and 3
    x, w13, w2 = normal(g, T, H), normal(g, P, 2 * I, H, std=H ** -0.5), normal(g, P, H, I, std=I ** -0.5)
    aid = (torch.rand(T, generator=g) < 0.7).to(torch.int32)
    logits, dout = torch.randn((T, M), generator=g), normal(g, T, H)
    ids, w, slot, counts, offsets, por, rop = ew.moe_route_reroute_permute(logits.cuda(), aid.cuda(), emap, k, 1, P)
    y = ew.moe_grouped_ffn(x.cuda(), k, I, P, counts, offsets, por, w13.cuda(), w2.cuda())
    ew.moe_unpermute(y, rop, w)
    dy, dw = ew.moe_unpermute_backward(dout.cuda(), rop, w, y)
    dxs, d13, d2 = ew.moe_grouped_ffn_backward(x.cuda(), dy, k, I, P, counts, offsets, por, w13.cuda(), w2.cuda(), first_slot=M, num_slots=E)
    dx = ew.moe_unpermute(dxs, rop, torch.ones_like(w))
    # the same in 64 bits by automatic differentiation, from the router's weights on
    X, W13, W2, W = (t.detach().cpu().double().requires_grad_() for t in (x, w13, w2, w))
    pairs, off = por.cpu().long(), offsets.cpu()
    out = torch.zeros((T, H), dtype=torch.float64)
    for s, i, j in ref.slots_of(off):
        h = X[pairs[i:j] // k] @ W13[s].t()
        a = h[:, :I] * torch.sigmoid(h[:, :I]) * h[:, I:]
        out = out.index_add(0, pairs[i:j] // k, W.reshape(-1)[pairs[i:j]][:, None] * (a @ W2[s].t()))
    (out * dout.double()).sum().backward()
    for name, got, want in (("dw", dw, W.grad), ("dx", dx, X.grad), ("dw13", d13, W13.grad[M:]), ("dw2", d2, W2.grad[M:])):
        rel = float((got.cpu().double() - want).norm() / want.norm())
        assert rel <= 1e-2, f"{name}: relative error {rel:.2e}"   # up to eight roundings to bf16, 2^-8 at most and 2^-9.8 rms each


def test_four_bit_pool_through_the_layer_calls(ew):
    """A pool of 4-bit experts (pages under loaded experts only), routed by the framework, equals bf16 experts of the same values."""
    T, k, M, N, E, H, I = 50, 3, 6, 2, 4, 256, 128
    g = gen(22)
    b13, b2 = ew.moe_w4_expert_bytes(2 * I, H), ew.moe_w4_expert_bytes(H, I)
    pool = ew.ExpertPool(1, M, N, E, b13, b2)
    P = pool.P
    v13, v2 = torch.zeros((P, 2 * I, H), dtype=torch.bfloat16, device="cuda"), torch.zeros((P, H, I), dtype=torch.bfloat16, device="cuda")

    def load(adapter, ids, first):
        q13 = ew.moe_quantize_w4(normal(g, len(ids), 2 * I, H, std=0.06).cuda())
        q2 = ew.moe_quantize_w4(normal(g, len(ids), H, I, std=0.06).cuda())
        v13[first:first + len(ids)], v2[first:first + len(ids)] = ew.moe_dequantize_w4(q13, 2 * I, H), ew.moe_dequantize_w4(q2, H, I)
        pool.map(0, adapter, ids, q13, q2)

    load(0, list(range(M)), 0)
    load(1, [1, 4], M)
    load(2, [0, 2, 5], M + E)
    w13, w2, emap, _ = pool.view(0)
    x, aid, logits = normal(g, T, H).cuda(), torch.randint(0, 3, (T,), generator=g, dtype=torch.int32).cuda(), torch.randn((T, M), generator=g).cuda()
    ids, w, _, counts, offsets, por, rop = ew.moe_route_reroute_permute(logits, aid, pool.expert_map_host(0).cuda(), k, N, P)
    y4 = ew.moe_grouped_ffn_w4(x, k, I, P, counts, offsets, por, w13, w2)
    y = ew.moe_grouped_ffn(x, k, I, P, counts, offsets, por, v13, v2)
    rows = por.cpu().long() // k
    close(y4, ref.ffn(x.cpu().double()[rows], v13.cpu().double(), v2.cpu().double(), offsets.cpu(), True))
    out4, out = ew.moe_unpermute(y4, rop, w), ew.moe_unpermute(y, rop, w)
    assert float((out4.float() - out.float()).norm() / out.float().norm()) <= 2 * 5e-3   # each within 5e-3 of 64 bits (three roundings)
    h4 = ew.moe_grouped_gemm_w4(x, k, 2 * I, P, counts, offsets, por, w13)
    close(h4, ref.gemm(x.cpu().double()[rows], v13.cpu().double(), offsets.cpu(), True))
    pool.close()


def test_calls_captured_replayed_and_on_another_stream(ew):
    """A graph of all calls, replayed with eager work in between, gives the eager bits; so does another stream."""
    counts, k, H, I = [0, 40, 3, 130, 0, 9], 2, 256, 128
    g, P = gen(23), 6
    c, off, por, tok, tokens = ref.rows_of(counts, g, k=k)
    rng = np.random.default_rng(6)
    p13, p2 = random_w4(rng, P, 2 * I, H)[0].cuda(), random_w4(rng, P, H, I)[0].cuda()
    x, dy = normal(g, tokens, H).cuda(), normal(g, len(tok), H).cuda()
    w13, w2 = normal(g, P, 2 * I, H, std=0.06).cuda(), normal(g, P, H, I, std=0.06).cuda()
    rop, w, dout = torch.randperm(len(tok), generator=g).to(torch.int32).cuda(), torch.rand((len(tok) // k, k), generator=g).cuda(), None
    dout = normal(g, len(tok) // k, H).cuda()
    c, off, por = c.cuda(), off.cuda(), por.cuda()

    def step():
        n = len(tok)
        h = ew.moe_grouped_gemm(x, k, 2 * I, P, c, off, por, w13, num_rows=n)
        dx = ew.moe_grouped_gemm(h, 1, H, P, c, off, None, w13, transposed=True)
        dw = ew.moe_grouped_gemm_wgrad(h, x, k, P, c, off, por)
        return [h, dx, dw, *ew.moe_grouped_ffn_backward(x, dy, k, I, P, c, off, por, w13, w2), *ew.moe_unpermute_backward(dout, rop, w, dy),
                ew.moe_grouped_ffn_w4(x, k, I, P, c, off, por, p13, p2, num_rows=n), ew.moe_grouped_gemm_w4(x, k, 2 * I, P, c, off, por, p13, num_rows=n),
                ew.moe_quantize_w4(w13)]

    eager = step()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        other = step()
    side.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(eager, other))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        captured = step()
    for _ in range(3):
        for t in captured:
            t.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(eager, captured))
        x.neg_()
        now = step()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(now, captured))
        x.neg_()
        assert all(torch.equal(a, b) for a, b in zip(eager, step()))
