"""The grouped products, their gradients and the 4-bit format in 64 bits, each result with a bound on what rounding may do to
the kernels' (first order in the unit roundings, with the largest second-order term covered by `SECOND`)."""
import numpy as np
import torch

HALF_BF16 = 2.0 ** -8     # a rounding to bf16, relative to the value
ADD_F32 = 2.0 ** -23      # one fp32 addition of a sum, either direction of rounding
SECOND = 1.02             # products of two first-order terms: each is below 2^-7 of the first-order ones
F32_FUNC = 2.0 ** -20     # sigmoid and the handful of fp32 operations around it


def rows_of(counts, gen, k=2, spare=0, shuffled=True):
    """Row bookkeeping as the permutation leaves it: offsets, pair_of_row, token of each row; `spare` tokens have no row."""
    counts = torch.tensor(counts, dtype=torch.int32)
    offsets = torch.cat([torch.zeros(1, dtype=torch.int32), counts.cumsum(0, dtype=torch.int32)])
    rows = int(offsets[-1])
    tokens = -(-rows // k) + spare
    pairs = torch.randperm(tokens * k, generator=gen)[:rows] if shuffled else torch.arange(rows)
    return counts, offsets, pairs.to(torch.int32), (pairs // k).long(), tokens


def slots_of(offsets):
    off = offsets.tolist()
    return [(s, off[s], off[s + 1]) for s in range(len(off) - 1) if off[s + 1] > off[s]]


def _out(ref, acc, bf16):
    return ref, (HALF_BF16 * ref.abs() * (1 + 2 ** -7) if bf16 else 0) + acc


def gemm(x, w, offsets, bf16, transposed=False):
    """y and its bound; x: fp64 rows in sorted order, w fp64 [P, N, K] or [P, K, N]."""
    n = w.shape[2] if transposed else w.shape[1]
    y, b = x.new_zeros((x.shape[0], n)), x.new_zeros((x.shape[0], n))
    for s, i, j in slots_of(offsets):
        m = w[s] if transposed else w[s].t()
        y[i:j], acc = x[i:j] @ m, x[i:j].abs() @ m.abs() * ((x.shape[1] + 1) * ADD_F32)
        y[i:j], b[i:j] = _out(y[i:j].clone(), acc, bf16)
    return y, b


def wgrad(dy, x, offsets, bf16_out):
    P = len(offsets) - 1
    dw, b = x.new_zeros((P, dy.shape[1], x.shape[1])), x.new_zeros((P, dy.shape[1], x.shape[1]))
    for s, i, j in slots_of(offsets):
        acc = dy[i:j].abs().t() @ x[i:j].abs() * ((j - i + 2) * ADD_F32)
        dw[s], b[s] = _out(dy[i:j].t() @ x[i:j], acc, bf16_out)
    return dw, b


def phi(g):
    """d silu(g) / dg; at most 1.1 in magnitude, its own slope at most 0.5."""
    s = torch.sigmoid(g)
    return s * (1 + g * (1 - s))


def ffn(x, w13, w2, offsets, bf16):
    """y of the grouped SwiGLU FFN; the activation is bf16 between the products."""
    I = w2.shape[2]
    y, b = x.new_zeros((x.shape[0], w2.shape[1])), x.new_zeros((x.shape[0], w2.shape[1]))
    for s, i, j in slots_of(offsets):
        h = x[i:j] @ w13[s].t()
        dh = x[i:j].abs() @ w13[s].abs().t() * ((x.shape[1] + 1) * ADD_F32)
        g, u, dg, du = h[:, :I], h[:, I:], dh[:, :I], dh[:, I:]
        silu = g * torch.sigmoid(g)
        a = silu * u
        da = SECOND * (1.1 * dg * u.abs() + silu.abs() * du) + a.abs() * (F32_FUNC + (HALF_BF16 if bf16 else 0))
        y[i:j] = a @ w2[s].t()
        acc = SECOND * (da @ w2[s].abs().t()) + a.abs() @ w2[s].abs().t() * ((I + 1) * ADD_F32)
        y[i:j], b[i:j] = _out(y[i:j].clone(), acc, bf16)
    return y, b


def ffn_backward(x, dy, w13, w2, offsets, bf16, bf16_out):
    """(dx, dw13, dw2) and their bounds."""
    I, r = w2.shape[2], HALF_BF16 if bf16 else 0.0
    P = len(offsets) - 1
    dx, bx = torch.zeros_like(x), torch.zeros_like(x)
    d13, b13 = torch.zeros_like(w13), torch.zeros_like(w13)
    d2, b2 = torch.zeros_like(w2), torch.zeros_like(w2)
    H = x.shape[1]
    for s, i, j in slots_of(offsets):
        X, D = x[i:j], dy[i:j]
        h = X @ w13[s].t()
        eh = X.abs() @ w13[s].abs().t() * ((H + 1) * ADD_F32) + r * h.abs()
        g, u, eg, eu = h[:, :I], h[:, I:], eh[:, :I], eh[:, I:]
        da = D @ w2[s]
        ea = D.abs() @ w2[s].abs() * ((H + 1) * ADD_F32) + r * da.abs()
        silu = g * torch.sigmoid(g)
        act, dgate, dup = silu * u, da * u * phi(g), da * silu
        f = r + F32_FUNC
        # |phi| itself passes through 0: its function error is absolute
        e_act = SECOND * (1.1 * eg * u.abs() + silu.abs() * eu) + f * act.abs()
        e_dg = SECOND * (ea * (u * phi(g)).abs() + da.abs() * eu * phi(g).abs() + (da * u).abs() * (0.5 * eg + F32_FUNC * (1 + g.abs()))) + f * dgate.abs()
        e_du = SECOND * (ea * silu.abs() + da.abs() * 1.1 * eg) + f * dup.abs()
        dh, e_dh = torch.cat([dgate, dup], 1), torch.cat([e_dg, e_du], 1)
        dx[i:j], bx[i:j] = _out(dh @ w13[s], SECOND * (e_dh @ w13[s].abs()) + dh.abs() @ w13[s].abs() * ((2 * I + 1) * ADD_F32), bf16)
        n = j - i
        d13[s], b13[s] = _out(dh.t() @ X, SECOND * (e_dh.t() @ X.abs()) + dh.abs().t() @ X.abs() * ((n + 2) * ADD_F32), bf16_out)
        d2[s], b2[s] = _out(D.t() @ act, SECOND * (D.abs().t() @ e_act) + D.abs().t() @ act.abs() * ((n + 2) * ADD_F32), bf16_out)
    assert P == w13.shape[0]
    return (dx, bx), (d13, b13), (d2, b2)


E2M1 = [0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0]


def quantize_w4(w):
    """fp64 [E, N, K] -> (codes 0..15 [E, N, K], scale bytes [E, N, K/32]), one group after the other."""
    E, N, K = w.shape
    v = np.asarray(w, np.float64).reshape(-1, 32)
    codes, scales = np.zeros(v.shape, np.uint8), np.zeros(len(v), np.uint8)
    for i, group in enumerate(v):
        if not np.isfinite(group).all():
            scales[i] = 255
            continue
        m = np.abs(group).max()
        e = max(-127, int(np.floor(np.log2(m))) - 2) if m > 0 else -127
        scales[i] = e + 127
        for j, val in enumerate(group):
            a = abs(val) / 2.0 ** e
            d = [abs(a - c) for c in E2M1]
            best = min(d)
            near = [c for c in range(8) if d[c] == best]
            codes[i, j] = (near[0] if len(near) == 1 else [c for c in near if c % 2 == 0][0]) + (8 if np.signbit(val) else 0)
    return codes.reshape(E, N, K), scales.reshape(E, N, K // 32)


def pack_w4(codes, scales):
    E = codes.shape[0]
    two = codes.reshape(E, -1, 2)
    return np.concatenate([(two[..., 0] | two[..., 1] << 4).reshape(E, -1), scales.reshape(E, -1)], 1).astype(np.uint8)


def values_w4(codes, scales):
    table = np.array(E2M1 + [-c for c in E2M1])
    with np.errstate(over="ignore"):
        v = table[codes].reshape(*scales.shape, 32) * 2.0 ** (scales[..., None].astype(np.float64) - 127)
    v[scales == 255] = np.nan
    return v.reshape(codes.shape)
