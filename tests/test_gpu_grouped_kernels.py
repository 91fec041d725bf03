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
