"""The grouped products of the MoE layer as a training step and a server with 4-bit experts call them.

A case is a dict of plain values.  `op` names the operator:
  "gemm"       matrix products grouped by expert over ragged rows: y = x W^T ("fwd"), dx = dy W ("dgrad"), dW = dy^T x ("wgrad")
  "ffn_back"   gradients of the grouped SwiGLU expert FFN: input rows and both weight tensors
  "comb_back"  gradients of the weighted combine: expert outputs and router weights
  "w4"         experts held in 4 bits (E2M1 values, one power-of-two scale for 32 of them): the FFN ("ffn"), one product
               ("gemm"), and packing weights and reading them back ("pack")
Rows are a router's: T tokens of M experts, k each, drawn over N adapters of 16 slots (slots without an expert have no rows).
"""
import math

import numpy as np
import torch

own = False

SLOTS_PER_ADAPTER = 16
GROUP = 32  # values that share a scale

# The layer of configurations 1, 2 and 4 (hidden 2048, 64 experts of 1408, top-6).
BASE = dict(H=2048, I=1408, M=64, k=6, N=0, aid="uniform", lo=6, hi=6, bias=0.0, dtype="bf16")


def _case(name, op, T, **kw):
    return dict(dict(BASE, op=op, T=T, name=name), **kw)


def listed():
    return [
        # configuration 0 in fp32, as a check of a port makes it: input gradient of its first product, nothing but latency
        _case("gemm_dgrad_f32_64", "gemm", 64, way="dgrad", H=256, I=128, M=8, k=2, N=2, lo=2, hi=2, K=256, Nout=256, gather=False, dtype="f32"),
        # an ordinary decode batch through one projection of the experts of four adapters: a stream of weights
        _case("gemm_decode_64", "gemm", 64, way="fwd", N=4, K=2048, Nout=2816, gather=True),
        # the headline prefill's first projection, 20 adapters of skewed popularity
        _case("gemm_prefill_8192", "gemm", 8192, way="fwd", N=20, aid="zipf", lo=2, hi=16, bias=2.0, K=2048, Nout=2816, gather=True),
        # weight gradients of a ragged batch on a layer of many small experts, kept in fp32 for the optimiser
        _case("gemm_wgrad_1999", "gemm", 1999, way="wgrad", M=128, k=8, K=1536, Nout=640, gather=True),
        # fine-tuning one adapter's experts: its slots alone get gradients, base experts pass the input gradient through
        _case("ffn_back_adapter_1021", "ffn_back", 1021, N=1, aid="adapter", lo=8, hi=8, bias=2.0),
        # training every expert of the layer on a full batch
        _case("ffn_back_8192", "ffn_back", 8192),
        # combine of a small batch
        _case("comb_back_64", "comb_back", 64),
        # combine of a full one
        _case("comb_back_8192", "comb_back", 8192),
        # one user's next token on 4-bit experts: the least work a decode step can have
        _case("w4_ffn_decode_1", "w4", 1, way="ffn", N=4),
        # a decode batch over 20 adapters on 4-bit experts
        _case("w4_ffn_decode_64", "w4", 64, way="ffn", N=20, lo=2, hi=16),
        # a ragged prompt batch on 4-bit experts
        _case("w4_ffn_prefill_3999", "w4", 3999, way="ffn", N=20, aid="zipf", lo=2, hi=16, bias=2.0),
        # an adapter's experts on their way into a 4-bit pool, and read back
        _case("w4_pack_16", "w4", 16, way="pack"),
    ]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    op = rng.choice(["gemm", "gemm", "gemm", "ffn_back", "comb_back", "w4", "w4", "w4"])
    H, I = rng.choice([(2048, 1408), (1024, 896), (1536, 768), (1536, 640), (1280, 512), (2048, 1024)])
    c = dict(op=op, H=H, I=I, M=rng.choice([32, 48, 64, 96]), k=rng.choice([1, 2, 4, 6, 8]), N=rng.randint(0, 20),
             aid=rng.choice(["uniform", "zipf", "base"]), lo=rng.randint(1, 8), hi=16, bias=rng.choice([0.0, 2.0]), dtype="bf16")
    most = 49152 // c["k"]  # rows at most those of the largest listed case
    if op == "gemm":
        way = rng.choice(["fwd", "fwd", "dgrad", "wgrad"])
        if rng.random() < 0.25:  # test-sized fp32 layers
            return dict(c, way=way, dtype="f32", T=_log_int(rng, 1, 512), K=4 * rng.randint(1, 128), Nout=4 * rng.randint(1, 128), M=rng.choice([8, 12, 16]),
                        k=min(c["k"], 4), N=rng.randint(0, 4), lo=1, hi=4, gather=way != "dgrad" and rng.random() < 0.5)
        K, Nout = rng.choice([(H, 2 * I), (I, H), (H, I), (8 * rng.randint(4, 256), 8 * rng.randint(4, 256))])
        return dict(c, way=way, T=min(most, _log_int(rng, 1, 8192)), K=K, Nout=Nout, N=min(c["N"], 8) if way == "wgrad" else c["N"],
                    gather=way != "dgrad" and rng.random() < 0.7)
    if op == "ffn_back":
        c.update(N=rng.randint(1, 4), aid="adapter") if rng.random() < 0.5 else c.update(N=0, bias=0.0)
        return dict(c, T=min(most, _log_int(rng, 16, 8192)))
    if op == "comb_back":
        return dict(c, T=min(most, _log_int(rng, 1, 8192)), H=8 * rng.randint(16, 256))
    way = rng.choice(["ffn", "ffn", "gemm", "pack"])
    if way == "pack":
        return dict(c, way=way, T=rng.randint(1, 32), dtype=rng.choice(["bf16", "f32"]))
    return dict(c, way=way, T=min(most, _log_int(rng, 1, 4096)))


# ------------------------------------------------------------------------------------------------ inputs
def _shares(c):
    """Share of the tokens of each class: base, adapter 1, ... N."""
    n = c["N"]
    if n == 0 or c["aid"] == "base":
        return np.eye(1, n + 1)[0]
    if c["aid"] == "adapter":
        return np.eye(1, n + 1, 1)[0]
    p = np.ones(n + 1) if c["aid"] == "uniform" else np.arange(1, n + 2) ** -1.1
    return p / p.sum()


def _routing(c, rs, g):
    """What the permutation hands on: rows sorted by slot, and what a caller knows of them."""
    T, M, k, N = c["T"], c["M"], c["k"], c["N"]
    P = M + N * SLOTS_PER_ADAPTER
    emap = np.tile(np.arange(M), (N + 1, 1))
    bias = np.zeros((N + 1, M), np.float32)
    tuned = []
    for a in range(1, N + 1):
        ids = np.sort(rs.choice(M, size=min(M, int(rs.integers(c["lo"], c["hi"] + 1))), replace=False))
        emap[a, ids] = M + (a - 1) * SLOTS_PER_ADAPTER + np.arange(len(ids))
        bias[a, ids] = c["bias"]
        tuned.append(len(ids))
    aid = torch.from_numpy(rs.choice(N + 1, size=T, p=_shares(c))).cuda()
    scores = torch.randn((T, M), generator=g, device="cuda") + torch.from_numpy(bias).cuda()[aid]
    w, ids = torch.softmax(scores, 1).topk(k, dim=1)
    slot = torch.from_numpy(emap).cuda()[aid[:, None], ids].reshape(-1)
    order = torch.argsort(slot, stable=True)
    counts = torch.bincount(slot, minlength=P)
    row_of_pair = torch.empty_like(order)
    row_of_pair[order] = torch.arange(T * k, device="cuda")
    offsets = torch.cat([torch.zeros(1, dtype=torch.int64, device="cuda"), counts.cumsum(0)])
    i32 = lambda t: t.to(torch.int32).contiguous()  # noqa: E731
    return dict(P=P, rows=T * k, counts=i32(counts), offsets=i32(offsets), pair_of_row=i32(order), row_of_pair=i32(row_of_pair), topk_w=w.contiguous(),
                tuned=tuned, active=torch.nonzero(counts).reshape(-1), most=int(counts.max()))


def _pack(w):
    """fp32 weights [n, N, K] -> one row of bytes each: codes [N, K/2] (even elements in the low half), then scales [N, K/32]."""
    n, N, K = w.shape
    v = w.reshape(n, N, K // GROUP, GROUP)
    e = torch.frexp(v.abs().amax(-1, keepdim=True))[1] - 3  # 2^e: the largest of a group comes to lie in [4, 8)
    a = torch.ldexp(v, -e).abs().clamp(max=6.0)
    code = torch.where(a < 2, torch.round(a * 2), torch.where(a < 4, torch.round(a) + 2, torch.round(a / 2) + 4)).to(torch.uint8)
    code = (code + 8 * (v < 0).to(torch.uint8)).reshape(n, N, K // 2, 2)
    codes = code[..., 0] | (code[..., 1] << 4)
    return torch.cat([codes.reshape(n, -1), (e + 127).to(torch.uint8).reshape(n, -1)], 1)


def prepare(case, seed):
    c = case
    rs = np.random.default_rng([seed, c["T"], c["M"], c["k"]])
    g = torch.Generator(device="cuda").manual_seed(int(rs.integers(1 << 40)))
    dt = torch.bfloat16 if c["dtype"] == "bf16" else torch.float32
    H, I = c["H"], c["I"]

    def normal(*shape, std=1.0, dtype=dt):
        return torch.randn(shape, generator=g, device="cuda", dtype=dtype).mul_(std)

    def packed(P, N, K):
        out = torch.empty((P, N * K // 2 + N * K // GROUP), dtype=torch.uint8, device="cuda")
        for i in range(0, P, 16):
            out[i:i + 16] = _pack(normal(min(16, P - i), N, K, std=0.02, dtype=torch.float32))
        return out

    if c["op"] == "w4" and c["way"] == "pack":
        return dict(case=c, w=normal(c["T"], 2 * I, H, std=0.02))
    s = dict(_routing(c, rs, g), case=c)
    P, rows = s["P"], s["rows"]
    if c["op"] == "gemm":
        K, Nout = c["K"], c["Nout"]
        x = normal(c["T"] if c["gather"] else rows, K)
        if c["way"] == "wgrad":
            return dict(s, x=x, dy=normal(rows, Nout, std=0.01))
        return dict(s, x=x, w=normal(*((P, Nout, K) if c["way"] == "fwd" else (P, K, Nout)), std=0.02))
    if c["op"] == "ffn_back":
        s.update(x=normal(c["T"], H), dy=normal(rows, H, std=0.01), w13=normal(P, 2 * I, H, std=0.02), w2=normal(P, H, I, std=0.02))
        one = c["aid"] == "adapter"
        return dict(s, first=c["M"] if one else 0, slots=s["tuned"][0] if one else P)
    if c["op"] == "comb_back":
        return dict(s, dout=normal(c["T"], H, std=0.01), y=normal(rows, H))
    s["x"] = normal(c["T"], H)
    s["w13"] = packed(P, 2 * I, H)
    if c["way"] == "ffn":
        s["w2"] = packed(P, H, I)
    return s


# ------------------------------------------------------------------------------------------------ plain form
def _places(s):
    """Slot of every sorted row and its place in the slot; the pair's token."""
    row = torch.arange(s["rows"], device="cuda")
    slot = torch.searchsorted(s["offsets"][1:].long(), row, right=True)
    nth = torch.searchsorted(s["active"], slot)
    return nth, row - s["offsets"].long()[slot], s["pair_of_row"].long() // s["case"]["k"]


def _spread(s, at, rows):
    """Sorted rows, fp32, as [active slots, most rows of a slot, width] with zeros behind a slot's last row."""
    out = torch.zeros((len(s["active"]), s["most"], rows.shape[1]), device="cuda")
    out[at[0], at[1]] = rows.float()
    return out


def _of_slots(s, w):
    return w[s["active"]].float()


def _dw(s, dy, x, first, slots, dtype):
    """Weight gradients of the slots asked for, from rows spread over the active slots."""
    full = torch.zeros((s["P"], dy.shape[2], x.shape[2]), dtype=dtype, device="cuda")
    full[s["active"]] = torch.bmm(dy.transpose(1, 2).contiguous(), x).to(dtype)
    return full[first:first + slots]


def _unpack(b, N, K):
    codes, scales = b[:, :N * K // 2], b[:, N * K // 2:]
    code = torch.stack([codes & 15, codes >> 4], 2).reshape(len(b), N, K // GROUP, GROUP)
    low, mag = (code & 1).float(), (code >> 1 & 3).float()
    v = torch.where(mag == 0, low * 0.5, torch.exp2(mag - 1) * (1 + low * 0.5)) * (1 - 2 * (code >> 3).float())
    return (v * torch.exp2(scales.float() - 127).reshape(len(b), N, K // GROUP, 1)).reshape(len(b), N, K)


def _silu(z):
    return z / (1 + torch.exp(-z))


def _plain_w4(s):
    c = s["case"]
    H, I = c["H"], c["I"]
    if c["way"] == "pack":
        w = s["w"].float()
        v = w.reshape(*w.shape[:2], -1, GROUP)
        e = torch.frexp(v.abs().amax(-1, keepdim=True))[1] - 3
        a = torch.ldexp(v, -e)
        step = torch.where(a.abs() < 2, 0.5, torch.where(a.abs() < 4, 1.0, 2.0))
        q = (torch.round(a / step) * step).clamp(-6.0, 6.0)
        return torch.ldexp(q, e).reshape(w.shape).to(s["w"].dtype)
    at = _places(s)
    x = _spread(s, at, s["x"][at[2]])
    h = torch.bmm(x, _unpack(s["w13"][s["active"]], 2 * I, H).transpose(1, 2))
    if c["way"] == "ffn":
        h = torch.bmm(_silu(h[..., :I]) * h[..., I:], _unpack(s["w2"][s["active"]], H, I).transpose(1, 2))
    return h[at[0], at[1]].to(s["x"].dtype)


def _plain(s):
    c = s["case"]
    if c["op"] == "w4":
        return _plain_w4(s)
    if c["op"] == "comb_back":
        token = s["pair_of_row"].long() // c["k"]
        dout = s["dout"].float()[token]
        w = s["topk_w"].reshape(-1)[s["pair_of_row"].long()]
        dw = (dout * s["y"].float()).sum(1)[s["row_of_pair"].long()].reshape(s["topk_w"].shape)
        return dict(dy=(w[:, None] * dout).to(s["y"].dtype), dw=dw)
    at = _places(s)
    if c["op"] == "gemm":
        x = _spread(s, at, s["x"][at[2]] if c["gather"] else s["x"])
        if c["way"] == "wgrad":
            return _dw(s, _spread(s, at, s["dy"]), x, 0, s["P"], torch.float32)
        w = _of_slots(s, s["w"])
        return torch.bmm(x, w.transpose(1, 2) if c["way"] == "fwd" else w)[at[0], at[1]].to(s["x"].dtype)
    I, dt = c["I"], s["x"].dtype
    x, dy, w13, w2 = _spread(s, at, s["x"][at[2]]), _spread(s, at, s["dy"]), _of_slots(s, s["w13"]), _of_slots(s, s["w2"])
    h = torch.bmm(x, w13.transpose(1, 2))
    gate, up = h[..., :I], h[..., I:]
    sig = 1 / (1 + torch.exp(-gate))
    da = torch.bmm(dy, w2)
    dh = torch.cat([da * up * sig * (1 + gate * (1 - sig)), da * gate * sig], 2)
    return dict(dx=torch.bmm(dh, w13)[at[0], at[1]].to(dt), dw13=_dw(s, dh, x, s["first"], s["slots"], dt),
                dw2=_dw(s, dy, gate * sig * up, s["first"], s["slots"], dt))


# ------------------------------------------------------------------------------------------------ one pass
def run(state):
    s = state
    if not own:
        return _plain(s)
    import paper_2508_17624_amd as ew
    c = s["case"]
    H, I, k = c["H"], c["I"], c["k"]
    if c["op"] == "w4" and c["way"] == "pack":
        return ew.moe_dequantize_w4(ew.moe_quantize_w4(s["w"]), 2 * I, H, dtype=s["w"].dtype)
    P, counts, offsets = s["P"], s["counts"], s["offsets"]
    if c["op"] == "w4":
        if c["way"] == "gemm":
            return ew.moe_grouped_gemm_w4(s["x"], k, 2 * I, P, counts, offsets, s["pair_of_row"], s["w13"])
        return ew.moe_grouped_ffn_w4(s["x"], k, I, P, counts, offsets, s["pair_of_row"], s["w13"], s["w2"])
    if c["op"] == "comb_back":
        dy, dw = ew.moe_unpermute_backward(s["dout"], s["row_of_pair"], s["topk_w"], s["y"])
        return dict(dy=dy, dw=dw)
    if c["op"] == "gemm":
        kk, por = (k, s["pair_of_row"]) if c["gather"] else (1, None)
        if c["way"] == "wgrad":
            return ew.moe_grouped_gemm_wgrad(s["dy"], s["x"], kk, P, counts, offsets, por)
        return ew.moe_grouped_gemm(s["x"], kk, c["Nout"], P, counts, offsets, por, s["w"], transposed=c["way"] == "dgrad")
    dx, dw13, dw2 = ew.moe_grouped_ffn_backward(s["x"], s["dy"], k, I, P, counts, offsets, s["pair_of_row"], s["w13"], s["w2"],
                                                first_slot=s["first"], num_slots=s["slots"], dw_dtype=s["x"].dtype)
    return dict(dx=dx, dw13=dw13, dw2=dw2)


# ------------------------------------------------------------------------------------------------ in 64 bits
def _exact_values(b, N, K):
    """One packed expert in 64 bits."""
    table = torch.tensor([0, .5, 1, 1.5, 2, 3, 4, 6, 0, -.5, -1, -1.5, -2, -3, -4, -6], dtype=torch.float64, device="cuda")
    codes = b[:N * K // 2].reshape(N, K // 2).long()
    v = torch.empty((N, K), dtype=torch.float64, device="cuda")
    v[:, 0::2], v[:, 1::2] = table[codes & 15], table[codes >> 4]
    scales = torch.pow(2.0, b[N * K // 2:].reshape(N, K // GROUP).double() - 127)
    return v * scales.repeat_interleave(GROUP, 1)


def exact(case, seed):
    c, s = case, prepare(case, seed)
    f64 = dict(dtype=torch.float64, device="cuda")
    if c["op"] == "w4" and c["way"] == "pack":
        w = s["w"].double()
        grid = torch.tensor([0, .5, 1, 1.5, 2, 3, 4, 6], **f64)
        out = torch.empty_like(w)
        for i in range(len(w)):
            v = w[i].reshape(-1, GROUP)
            scale = torch.pow(2.0, torch.floor(torch.log2(v.abs().amax(1, keepdim=True))) - 2)
            a = v.abs() / scale
            at = torch.bucketize(a, grid).clamp(max=7)             # grid[at-1] < a <= grid[at]
            below = (at - 1).clamp(min=0)
            mid = (grid[at] + grid[below]) / 2
            up = (a > mid) | ((a == mid) & (at % 2 == 0))           # halfway: to the even code
            out[i] = (torch.where(up, grid[at], grid[below]) * v.sign() * scale).reshape(w[i].shape)
        return out
    k, off = c["k"], s["offsets"].tolist()
    pair = s["pair_of_row"].long()
    token = pair // k
    if c["op"] == "comb_back":
        dy = torch.empty((s["rows"], c["H"]), **f64)
        dw = torch.empty(c["T"] * k, **f64)
        for i in range(0, s["rows"], 4096):
            d = s["dout"][token[i:i + 4096]].double()
            dy[i:i + 4096] = d * s["topk_w"].double().reshape(-1)[pair[i:i + 4096]][:, None]
            dw[pair[i:i + 4096]] = (d * s["y"][i:i + 4096].double()).sum(1)
        return dict(dy=dy, dw=dw.reshape(c["T"], k))
    slots = [(i, off[i], off[i + 1]) for i in range(s["P"]) if off[i + 1] > off[i]]
    H, I = c["H"], c["I"]

    def rows_of(a, b):
        return s["x"][token[a:b]].double() if c["op"] != "gemm" or c["gather"] else s["x"][a:b].double()

    if c["op"] == "gemm" and c["way"] == "wgrad":
        dw = torch.zeros((s["P"], c["Nout"], c["K"]), **f64)
        for i, a, b in slots:
            dw[i] = s["dy"][a:b].double().t().contiguous() @ rows_of(a, b)
        return dw
    if c["op"] in ("gemm", "w4"):
        out = torch.empty((s["rows"], c["Nout"] if c["op"] == "gemm" else 2 * I if c["way"] == "gemm" else H), **f64)
        for i, a, b in slots:
            if c["op"] == "gemm":
                w = s["w"][i].double()
                out[a:b] = rows_of(a, b) @ (w.t() if c["way"] == "fwd" else w)
                continue
            h = rows_of(a, b) @ _exact_values(s["w13"][i], 2 * I, H).t()
            if c["way"] == "ffn":
                h = (h[:, :I] * torch.sigmoid(h[:, :I]) * h[:, I:]) @ _exact_values(s["w2"][i], H, I).t()
            out[a:b] = h
        return out
    dx = torch.empty((s["rows"], H), **f64)
    dw13, dw2 = torch.zeros((s["slots"], 2 * I, H), **f64), torch.zeros((s["slots"], H, I), **f64)
    for i, a, b in slots:
        x, dy, w13 = rows_of(a, b), s["dy"][a:b].double(), s["w13"][i].double()
        gate, up = x @ w13[:I].t(), x @ w13[I:].t()
        da, sig = dy @ s["w2"][i].double(), torch.sigmoid(gate)
        dgate, dup = da * up * (sig + gate * sig * (1 - sig)), da * gate * sig
        dx[a:b] = dgate @ w13[:I] + dup @ w13[I:]
        if s["first"] <= i < s["first"] + s["slots"]:
            dw13[i - s["first"]] = torch.cat([dgate.t() @ x, dup.t() @ x])
            dw2[i - s["first"]] = dy.t() @ (gate * sig * up)
    return dict(dx=dx, dw13=dw13, dw2=dw2)


# ------------------------------------------------------------------------------------------------ what a pass cannot do without
def _active(c):
    """Expected number of slots that at least one token visits, for a router that spreads its tokens evenly."""
    p, hit, tuned = _shares(c), c["k"] / c["M"], min(c["M"], (c["lo"] + c["hi"]) / 2)
    lift = 1.0
    if c["bias"]:  # +2.0 on a score of spread 1: a tuned expert is picked about five times as often as another one
        lift = 5.0 / (tuned / c["M"] * 5.0 + 1 - tuned / c["M"])
    n = sum(tuned * (1 - (1 - q * min(1.0, hit * lift)) ** c["T"]) for q in p[1:])
    base = p[0] + sum(q * (1 - tuned / c["M"]) for q in p[1:])
    return n + c["M"] * (1 - (1 - base * min(1.0, hit)) ** c["T"])


def work(case):
    c = case
    el = 2 if c["dtype"] == "bf16" else 4
    H, I, T, k = c["H"], c["I"], c["T"], c["k"]
    if c["op"] == "w4" and c["way"] == "pack":
        n = T * 2 * I * H  # weights read, codes and scales written and read, values written
        return {"bytes": 2 * n * el + 2 * (n // 2 + n // GROUP), "flops": 0}
    rows = T * k
    if c["op"] == "comb_back":
        return {"bytes": T * H * el + 2 * rows * H * el + rows * (4 + 4 + 4), "flops": 3 * rows * H}
    P = c["M"] + c["N"] * SLOTS_PER_ADAPTER
    index = 4 * rows + 8 * P
    if c["op"] == "gemm":
        x = (T if c["gather"] else rows) * c["K"] * el
        w = c["Nout"] * c["K"]
        flops = 2 * rows * w
        if c["way"] == "wgrad":
            return {"bytes": index + x + rows * c["Nout"] * el + P * w * 4, "flops": flops}
        return {"bytes": index + x + rows * c["Nout"] * el + _active(c) * w * el, "flops": flops}
    if c["op"] == "w4":
        weights = _active(c) * (3 if c["way"] == "ffn" else 2) * H * I * 17 / 32
        return {"bytes": index + T * H * 2 + rows * (H if c["way"] == "ffn" else 2 * I) * 2 + weights, "flops": rows * (6 if c["way"] == "ffn" else 4) * H * I}
    grads = rows  # rows whose slots get weight gradients
    slots = P
    if c["aid"] == "adapter":
        tuned = min(c["M"], (c["lo"] + c["hi"]) / 2)
        slots, grads = tuned, rows * min(1.0, tuned / c["M"] * (5.0 / (tuned / c["M"] * 5.0 + 1 - tuned / c["M"]) if c["bias"] else 1.0))
    # the two products of the forward pass that the gradients need again, the two input gradients, the two weight gradients
    flops = rows * (4 + 2 + 4) * H * I + grads * 6 * H * I
    return {"bytes": index + T * H * el + 2 * rows * H * el + (_active(c) + slots) * 3 * H * I * el, "flops": flops}
