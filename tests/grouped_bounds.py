"""A bound on the gradients of the grouped FFN for kernels that round dg, du and a to bf16 between the products and nothing else: g, u and
da are fp32."""
import torch

from grouped_ref import ADD_F32, F32_FUNC, HALF_BF16, SECOND, _out, phi, slots_of

# A rounding to bf16 is uniform over a step of 2^-7 of the value's power of two, at most 2^-7 of the value: 2^-7 / sqrt(12) in the mean square.  Three
# per cent more for what a sample of some thousand elements may be off by, and for the fp32 sums.
ONE_ROUNDING_RMS = 1.03 * 2.0 ** -7 / 12 ** 0.5


def ffn_backward(x, dy, w13, w2, offsets, bf16, bf16_out):
    """(dx, dw13, dw2), each with its bound; x: fp64 rows in sorted order."""
    I, H, r = w2.shape[2], x.shape[1], HALF_BF16 if bf16 else 0.0
    dx, bx = torch.zeros_like(x), torch.zeros_like(x)
    d13, b13 = torch.zeros_like(w13), torch.zeros_like(w13)
    d2, b2 = torch.zeros_like(w2), torch.zeros_like(w2)
    for s, i, j in slots_of(offsets):
        X, D, n = x[i:j], dy[i:j], j - i
        h, eh = X @ w13[s].t(), X.abs() @ w13[s].abs().t() * ((H + 1) * ADD_F32)
        g, u, eg, eu = h[:, :I], h[:, I:], eh[:, :I], eh[:, I:]
        da, ea = D @ w2[s], D.abs() @ w2[s].abs() * ((H + 1) * ADD_F32)
        silu = g * torch.sigmoid(g)
        act, dgate, dup = silu * u, da * u * phi(g), da * silu
        f = r + F32_FUNC
        e_act = SECOND * (1.1 * eg * u.abs() + silu.abs() * eu) + f * act.abs()
        # phi passes through 0: the error of its function is absolute
        e_dg = SECOND * (ea * (u * phi(g)).abs() + da.abs() * eu * phi(g).abs() + (da * u).abs() * (0.5 * eg + F32_FUNC * (1 + g.abs()))) + f * dgate.abs()
        e_du = SECOND * (ea * silu.abs() + da.abs() * 1.1 * eg) + f * dup.abs()
        dh, e_dh = torch.cat([dgate, dup], 1), torch.cat([e_dg, e_du], 1)
        dx[i:j], bx[i:j] = _out(dh @ w13[s], SECOND * (e_dh @ w13[s].abs()) + dh.abs() @ w13[s].abs() * ((2 * I + 1) * ADD_F32), bf16)
        d13[s], b13[s] = _out(dh.t() @ X, SECOND * (e_dh.t() @ X.abs()) + dh.abs().t() @ X.abs() * ((n + 2) * ADD_F32), bf16_out)
        d2[s], b2[s] = _out(D.t() @ act, SECOND * (D.abs().t() @ e_act) + D.abs().t() @ act.abs() * ((n + 2) * ADD_F32), bf16_out)
    return (dx, bx), (d13, b13), (d2, b2)
