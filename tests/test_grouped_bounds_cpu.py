"""The bound on the FFN's gradients holds for the roundings that are stated and fails for others, planted here in a model of the kernels."""
import pytest
import torch

import grouped_bounds as bounds
import grouped_ref as ref


def bf16(t):
    return t.to(torch.bfloat16).double()


def model(x, dy, w13, w2, offsets, rounded):
    """Weight gradients with dg, du and a rounded to bf16, and before them the products named in `rounded`."""
    I = w2.shape[2]
    d13, d2 = torch.zeros_like(w13), torch.zeros_like(w2)
    for s, i, j in ref.slots_of(offsets):
        h, da = x[i:j] @ w13[s].t(), dy[i:j] @ w2[s]
        g, u = h[:, :I], h[:, I:]
        g, u, da = (bf16(t) if name in rounded else t for name, t in (("g", g), ("u", u), ("da", da)))
        silu = g * torch.sigmoid(g)
        dh = bf16(torch.cat([da * u * ref.phi(g), da * silu], 1))
        d13[s], d2[s] = dh.t() @ x[i:j], dy[i:j].t() @ bf16(silu * u)
    return d13, d2


@pytest.mark.parametrize("rounded", [(), ("g",), ("u",), ("da",), ("g", "u", "da")], ids=lambda r: "+".join(r) or "none")
def test_the_bound_tells_roundings_apart(rounded):
    g = torch.Generator().manual_seed(1)
    H, I, counts = 264, 72, [0, 300, 129, 0, 1, 1]
    _, off, _, tok, tokens = ref.rows_of(counts, g)
    P, rows = len(counts), len(tok)
    x, dy = bf16(torch.randn((tokens, H), generator=g))[tok], bf16(torch.randn((rows, H), generator=g) * 0.5)
    w13, w2 = bf16(torch.randn((P, 2 * I, H), generator=g) * H ** -0.5), bf16(torch.randn((P, H, I), generator=g) * I ** -0.5)
    _, (v13, b13), (v2, b2) = bounds.ffn_backward(x, dy, w13, w2, off, True, False)
    d13, d2 = model(x, dy, w13, w2, off, rounded)
    inside = bool(((d13 - v13).abs() <= b13).all() and ((d2 - v2).abs() <= b2).all())
    rms = max(float((d - v).norm() / v.norm()) for d, v in ((d13, v13), (d2, v2)))
    assert inside == (rounded == ()), f"worst {float(((d13 - v13).abs() / b13.clamp(min=1e-300)).max()):.3g} bounds"
    assert (rms <= bounds.ONE_ROUNDING_RMS) == (rounded == ()), f"{rms:.3e} beside {bounds.ONE_ROUNDING_RMS:.3e}"
