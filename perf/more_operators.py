"""Operators of gated experts as timed cases: the gated expert FFN over ragged rows with its backward pass, microscaled
4-bit floating point (a tensor to 4 bits and back), the experts' product of rows and weights that are both held in it, and
the gated expert FFN served from 4-bit weights.

Kinds of pass:
  glu     gated expert FFN over ragged rows: forward with nothing kept (serving), or forward and backward pass (train).
  mx4     a tensor, or the experts' weights, to 4 bits and back.
  gemm4   Y = X W of each row's expert, X and W in 4 bits.
  glu4    gated expert FFN of 16- or 32-bit token rows against 4-bit weights.

Definitions.  Rows lie expert by expert: expert e has rows offsets[e] .. offsets[e + 1] - 1, row r is token row_inv[r] / k,
rows at or behind offsets[E] hold zeros.  Gated FFN: W1 [E, M, 2 H] holds the gate's columns and behind them the up
projection's; G = X W1[gate], U = X W1[up], A = act(G) U, Y = A W2, act(g) = g sigmoid(g) ("silu") or g Phi(g) ("gelu").  A
hidden shard takes its columns of both halves.  Training keeps G and U rounded to the storage type, and the backward pass
reads these: dA = dY W2^T, dG = dA U act'(G), dU = dA act(G), dX = [dG | dU] W1^T, dW1 = X^T [dG | dU], dW2 = (act(G) U)^T dY.
4 bits: along the index that a product sums over, values are cut into blocks of 32.  With a block's largest magnitude a in
[2^x, 2^(x + 1)) its scale is 2^(x - 2), twice that where a / scale would round to 8; a value is kept as the one of 0, 1/2, 1,
3/2, 2, 3, 4, 6 and their negatives that is nearest to value / scale, of two the one with the even code.  A block takes 16
bytes (even index in the low half) and a scale byte b for 2^(b - 127).  Scale bytes of a matrix with n rows of K summed
values: [ceil(K / 512), 4, n, 4], block 16 c + 4 s + q of row r at [c, q, r, s].  In the FFN from 4 bits the token rows and A
are brought to 4 bits row by row on their way into the products.
"""
import math

import torch

own = False     # the framework's operators instead of the plain forms

DEV = "cuda:0"
ROUTED = {"dtype": "bf16", "k": 2, "skew": 0.0, "f": 0.0, "sigma_w": 0.02}


def _glu(**kw):
    return dict(ROUTED, kind="glu", n_esp=1, esp_idx=0, act="silu", **kw)


def listed():
    return [
        # one decoding step of a single request: two rows, two experts' weights are all of the traffic
        _glu(name="glu_serve_1", S=1, M=1024, H=4096, E=8, train=False),
        # one decoding step of a small batch
        _glu(name="glu_serve_32", S=32, M=1024, H=4096, E=8, train=False),
        # a short prompt against the widest experts that the framework is benchmarked with
        dict(_glu(name="glu_prefill_wide", S=256, M=4096, H=14336, E=8, train=False), sigma_w=0.01, act="gelu"),
        # fp32 training, no size a multiple of a tile, three choices, some dropped
        dict(_glu(name="glu_train_f32_ragged", S=1003, M=520, H=1544, E=12, train=True), dtype="f32", k=3, skew=0.5, f=1.1, act="gelu"),
        # training step of the layer shape of the paper's layer benchmark
        dict(_glu(name="glu_train_layer", S=4096, M=1024, H=4096, E=8, train=True), skew=0.2),
        # the widest experts' hidden shard, half of the largest configuration's tokens
        dict(_glu(name="glu_train_large", S=16384, M=4096, H=14336, E=8, train=True), n_esp=2, esp_idx=1, sigma_w=0.01, skew=0.2),
        # activations of a small fp32 layer, the last block of a row cut short
        {"name": "mx4_rows_f32", "kind": "mx4", "dtype": "f32", "G": 1, "rows": 1003, "cols": 1544, "transposed": False},
        # both projections of the widest experts, once before they are served
        {"name": "mx4_weights_large", "kind": "mx4", "dtype": "bf16", "G": 8, "rows": 4096, "cols": 28672, "transposed": True},
        # odd sizes, 12 experts with unequal shares of the rows, some dropped, fp32 results
        dict(ROUTED, name="mx4_products_ragged", kind="gemm4", S=1003, M=520, H=1544, E=12, dtype="f32", k=3, skew=0.5, f=1.1),
        # 64 experts with unequal shares of the rows
        dict(ROUTED, name="mx4_products_64", kind="gemm4", S=16384, M=2048, H=2048, E=64, skew=0.5),
        # one decoding step of a small batch against the widest experts
        dict(ROUTED, name="mx4_serve_wide_8", kind="glu4", S=8, M=4096, H=14336, E=8, act="silu", sigma_w=0.01),
        # a batch of prompts against them
        dict(ROUTED, name="mx4_prefill_large", kind="glu4", S=16384, M=4096, H=14336, E=8, act="silu", sigma_w=0.01, skew=0.2),
    ]


def _log_int(rng, lo, hi, mult=1):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi))) / mult)) * mult))


def draw(rng):
    """One more case of the same ranges."""
    kind = rng.choice(["glu", "glu", "glu", "mx4", "gemm4", "gemm4", "glu4", "glu4"])
    dtype = "bf16" if rng.random() < 0.7 else "f32"
    while True:
        M = _log_int(rng, 64, 4096, rng.choice([8, 64, 256]))
        if kind == "mx4":
            rows, cols = _log_int(rng, 8, 32768, 8), _log_int(rng, 64, 28672, rng.choice([8, 64]))
            c = {"kind": kind, "dtype": dtype, "G": rng.choice([1, 1, 2, 8, 12]), "rows": rows, "cols": cols, "transposed": rng.random() < 0.5}
            if not c["transposed"]:
                c["rows"] -= rng.randrange(8) if rows > 8 else 0
            if c["G"] * rows * cols <= 1 << 29:
                return c
            continue
        c = dict(ROUTED, kind=kind, dtype=dtype, M=M, E=rng.choice([1, 2, 4, 8, 8, 8, 12, 16, 24, 32, 64]), skew=rng.choice([0.0, 0.2, 0.5, 1.0]),
                 f=rng.choice([0.0, 0.0, 0.0, 1.0, 1.25]))
        c["k"] = min(c["E"], rng.choice([1, 2, 2, 2, 3, 4]))
        n_esp = rng.choice([1, 1, 1, 2, 4]) if kind == "glu" else 1
        c["H"] = _log_int(rng, 128, 14336, rng.choice([8, 64, 512]) * n_esp)
        c["H"] -= c["H"] % (8 * n_esp)
        train = kind == "glu" and rng.random() < 0.6
        c["S"] = _log_int(rng, 16, 16384) if train else _log_int(rng, 1, 16384 if kind != "glu" else 1024)
        if kind != "gemm4":
            c["act"] = rng.choice(["silu", "silu", "gelu"])
        if kind == "glu":
            c.update(n_esp=n_esp, esp_idx=rng.randrange(n_esp), train=train)
        parts = {"glu": 9 if train else 3, "gemm4": 1, "glu4": 3}[kind]
        flops = parts * 2.0 * c["S"] * c["k"] * M * (c["H"] // n_esp)
        if c["H"] >= 8 * n_esp and flops <= (4e11 if dtype == "f32" and kind == "glu" else 1.1e13) and c["E"] * M * c["H"] <= 1 << 29:
            return c


# ---- inputs -------------------------------------------------------------------------------------------------------


def _dtype(c):
    return torch.float32 if c["dtype"] == "f32" else torch.bfloat16


def _empty(*shape, dtype):
    return torch.empty(*shape, dtype=dtype, device=DEV)


def _maker(c, seed):
    gen = torch.Generator(device=DEV)
    gen.manual_seed(seed)

    def normal(*shape, sigma=1.0, dtype=None):
        out = _empty(*shape, dtype=dtype or _dtype(c))
        for part in (out if len(shape) > 2 else (out,)):
            part.copy_(torch.randn(part.shape, generator=gen, device=DEV) * sigma)
        return out

    return gen, normal


def _rows(c, gen):
    """What the plan of the rows hands over: offsets and, of each row, the token and choice that it belongs to."""
    S, E, k = c["S"], c["E"], c["k"]
    logits = torch.randn(S, E, generator=gen, device=DEV) + c["skew"] * torch.randn(E, generator=gen, device=DEV)
    expert = logits.topk(k, dim=1).indices.t().reshape(-1)          # choice by choice, token by token
    order = torch.argsort(expert, stable=True)
    demand = torch.bincount(expert, minlength=E)
    seat = torch.arange(S * k, device=DEV) - (demand.cumsum(0) - demand)[expert[order]]
    C = S if c["f"] == 0.0 else max(1, math.ceil(k * S * c["f"] / E))
    kept = order[seat < C]
    inv = torch.full((S * k,), -1, dtype=torch.int32, device=DEV)
    inv[:kept.numel()] = ((kept % S) * k + kept // S).int()
    offsets = torch.zeros(E + 1, dtype=torch.int32, device=DEV)
    offsets[1:] = demand.clamp(max=C).cumsum(0)
    return offsets, inv.reshape(k, S)


# 4 bits: blocks of 32 values along the last dimension
SIZES = (0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0)


def _power(scale, dtype):
    """2^(scale - 127) of a scale byte"""
    if dtype == torch.float64:
        return ((scale.long() + 896) << 52).view(dtype)
    return torch.where(scale == 0, 1 << 22, scale.int() << 23).int().view(dtype)


def _to_mx4(x):
    """x [..., K] -> codes [..., blocks, 32] uint8, scale bytes [..., blocks] uint8, in the type of x (32 or 64 bits)."""
    x = torch.nn.functional.pad(x, (0, -x.shape[-1] % 32)).unflatten(-1, (-1, 32))
    a = x.abs().amax(-1)
    mantissa, exponent = torch.frexp(a)                              # a = mantissa 2^exponent, mantissa in [1/2, 1)
    scale = (exponent + 124 + (mantissa >= 0.875)).clamp(min=0)
    scale = torch.where(a == 0, 0, scale)
    v = x.abs() / _power(scale, x.dtype)[..., None]
    code = torch.zeros(v.shape, dtype=torch.uint8, device=x.device)
    for middle, even in ((0.25, False), (0.75, True), (1.25, False), (1.75, True), (2.5, False), (3.5, True), (5.0, False)):
        code += (v >= middle) if even else (v > middle)              # a tie goes to the even code
    code += 8 * torch.signbit(x)
    return code, torch.where(torch.isfinite(a), scale, 255).to(torch.uint8)


def _mx4_values(code, scale, dtype=torch.float32):
    """What they stand for: [..., blocks * 32]."""
    size = torch.tensor(SIZES + tuple(-v for v in SIZES), dtype=dtype, device=code.device)[code.long()]
    step = torch.where(scale == 255, float("nan"), _power(scale, dtype))
    return (size * step[..., None]).flatten(-2)


def _pack(code, scale):
    """codes [G, n, blocks, 32], scale bytes [G, n, blocks] -> the bytes as they are held"""
    G, n, blocks = scale.shape
    q = (code[..., 0::2] | (code[..., 1::2] << 4)).reshape(G, n, blocks * 16)
    s = torch.nn.functional.pad(scale, (0, -blocks % 16)).view(G, n, -1, 4, 4).permute(0, 2, 4, 1, 3).contiguous()
    return q, s


def _unpack(q, s, dtype=torch.float32):
    """The values [n, blocks * 32] of one matrix's bytes."""
    n, blocks = q.shape[0], q.shape[1] // 16
    b = q.view(n, blocks, 16)
    code = torch.stack((b & 15, b >> 4), -1).view(n, blocks, 32)
    return _mx4_values(code, s.permute(2, 0, 3, 1).reshape(n, -1)[:, :blocks], dtype)


def _quantised(x):
    """x [G, n, K] in bytes, a matrix at a time"""
    parts = [_pack(*_to_mx4(m[None].float())) for m in x]
    return torch.cat([p[0] for p in parts]), torch.cat([p[1] for p in parts])


def prepare(case, seed):
    c = dict(case)
    gen, normal = _maker(c, seed)
    dt = _dtype(c)
    if c["kind"] == "mx4":
        G, rows, cols = c["G"], c["rows"], c["cols"]
        # a few columns stand out, as in trained networks
        out = 1 + 7 * (torch.rand(cols, generator=gen, device=DEV) < 0.02).float()
        x = normal(G, rows, cols)
        for part in x:
            part.mul_(out)
        n, K = (cols, rows) if c["transposed"] else (rows, cols)
        return {"c": c, "x": x, "q": _empty(G, n, (K + 31) // 32 * 16, dtype=torch.uint8),
                "s": _empty(G, (K + 511) // 512, 4, n, 4, dtype=torch.uint8), "back": _empty(G, rows, cols, dtype=dt)}
    S, E, k, M, H = c["S"], c["E"], c["k"], c["M"], c["H"]
    R, sigma = S * k, c["sigma_w"]
    offsets, inv = _rows(c, gen)
    at = offsets.tolist()
    s = {"c": c, "offsets": offsets, "row_inv": inv, "rows": [b - a for a, b in zip(at, at[1:])], "ws": None}     # rows: for the plain forms' slices
    if c["kind"] == "gemm4":
        s["xq"], s["xs"] = (t[0] for t in _quantised(normal(1, S, M)))
        s["Wq"], s["Ws"] = _quantised(normal(E, H, M, sigma=sigma))
        return dict(s, Y=_empty(R, H, dtype=dt))
    s["x"] = normal(S, M)
    if c["kind"] == "glu4":
        s["W1q"], s["W1s"] = _quantised(normal(E, 2 * H, M, sigma=sigma))
        s["W2q"], s["W2s"] = _quantised(normal(E, M, H, sigma=sigma))
        return dict(s, Y=_empty(R, M, dtype=dt))
    Hl = H // c["n_esp"]
    s.update(W1=normal(E, M, 2 * H, sigma=sigma), W2=normal(E, H, M, sigma=sigma), A=_empty(R, Hl, dtype=dt), Y=_empty(R, M, dtype=dt))
    if c["train"]:
        # of the whole weight gradients a hidden shard writes its own columns (rows)
        s.update(dY=normal(R, M), dX=_empty(R, M, dtype=dt), dW1=torch.zeros_like(s["W1"]), dW2=torch.zeros_like(s["W2"]),
                 Z=torch.zeros(R, 2 * Hl, dtype=dt, device=DEV))      # rows behind the last expert's are left as they were
    return s


# ---- plain forms --------------------------------------------------------------------------------------------------


def _by_expert(rows, A, matrix, out):
    """out = A matrix(e) of each expert's rows; the rows behind the last expert's are zeros."""
    at = 0
    for e, n in enumerate(rows):
        if n:
            torch.mm(A[at:at + n], matrix(e), out=out[at:at + n])
        at += n
    out[at:].zero_()
    return out


def _reduce_by_expert(rows, A, B, out):
    """out[e] = A^T B over the expert's rows."""
    at = 0
    for e, n in enumerate(rows):
        out[e] = torch.mm(A[at:at + n].t(), B[at:at + n]) if n else 0
        at += n
    return out


def _rows_of(x, row_inv, k):
    """The token rows in the experts' order, zeros behind the last one."""
    inv = row_inv.reshape(-1).long()
    return torch.where((inv >= 0)[:, None], x[(inv // k).clamp(min=0)], 0)


def _gate(act, g):
    """act(g), act'(g)"""
    if act == "silu":
        s = torch.sigmoid(g)
        return g * s, s * (1 + g * (1 - s))
    cdf = 0.5 * (1 + torch.erf(g * math.sqrt(0.5)))
    return g * cdf, cdf + g * torch.exp(-0.5 * g * g) * (1 / math.sqrt(2 * math.pi))


def _glu_plain(s):
    c, dt, f32 = s["c"], _dtype(s["c"]), torch.float32
    rows, R, M, H = s["rows"], c["S"] * c["k"], c["M"], c["H"]
    Hl = H // c["n_esp"]
    h0 = c["esp_idx"] * Hl
    W1g, W1u = s["W1"][:, :, h0:h0 + Hl], s["W1"][:, :, H + h0:H + h0 + Hl]
    W2 = s["W2"][:, h0:h0 + Hl]
    X = _rows_of(s["x"].float(), s["row_inv"], c["k"])
    G = _by_expert(rows, X, lambda e: W1g[e].float(), _empty(R, Hl, dtype=f32))
    U = _by_expert(rows, X, lambda e: W1u[e].float(), _empty(R, Hl, dtype=f32))
    out = {"Y": _by_expert(rows, _gate(c["act"], G)[0] * U, lambda e: W2[e].float(), _empty(R, M, dtype=f32)).to(dt)}
    if not c["train"]:
        return out
    G, U = G.to(dt).float(), U.to(dt).float()
    out["Z"] = torch.cat((G, U), 1).to(dt)
    out["Z"][sum(rows):] = 0
    dY = s["dY"].float()
    dA = _by_expert(rows, dY, lambda e: W2[e].float().t(), _empty(R, Hl, dtype=f32))
    a, da = _gate(c["act"], G)
    dG, dU = dA * U * da, dA * a
    dX = _by_expert(rows, dG, lambda e: W1g[e].float().t(), _empty(R, M, dtype=f32))
    dX += _by_expert(rows, dU, lambda e: W1u[e].float().t(), _empty(R, M, dtype=f32))
    out["dX"] = dX.to(dt)
    out["dW1"], out["dW2"] = torch.zeros_like(s["W1"]), torch.zeros_like(s["W2"])
    _reduce_by_expert(rows, X, dG, out["dW1"][:, :, h0:h0 + Hl])
    _reduce_by_expert(rows, X, dU, out["dW1"][:, :, H + h0:H + h0 + Hl])
    _reduce_by_expert(rows, a * U, dY, out["dW2"][:, h0:h0 + Hl])
    return out


def _mx4_plain(s):
    back = _empty(*s["x"].shape, dtype=s["x"].dtype)
    for x, to in zip(s["x"], back):
        x = x.float()
        if s["c"]["transposed"]:
            to.copy_(_mx4_values(*_to_mx4(x.t()))[:, :x.shape[0]].t())
        else:
            to.copy_(_mx4_values(*_to_mx4(x))[:, :x.shape[1]])
    return back


def _gemm4_plain(s):
    c = s["c"]
    X = _rows_of(_unpack(s["xq"], s["xs"]), s["row_inv"], c["k"])
    return _by_expert(s["rows"], X, lambda e: _unpack(s["Wq"][e], s["Ws"][e]).t(), _empty(c["S"] * c["k"], c["H"], dtype=torch.float32)).to(_dtype(c))


def _glu4_plain(s):
    c, d = s["c"], torch.float64      # G and U in 64 bits: a value of A next to a border decides what is kept of it
    rows, R, M, H = s["rows"], c["S"] * c["k"], c["M"], c["H"]
    X = _rows_of(_mx4_values(*_to_mx4(s["x"].float()), d), s["row_inv"], c["k"])
    Y = torch.zeros(R, M, dtype=torch.float32, device=DEV)
    at = 0
    for e, n in enumerate(rows):
        if n:
            G, U = (X[at:at + n] @ _unpack(s["W1q"][e], s["W1s"][e], d).t()).split(H, 1)
            A = _mx4_values(*_to_mx4(_gate(c["act"], G)[0] * U))
            Y[at:at + n] = A @ _unpack(s["W2q"][e], s["W2s"][e]).t()
        at += n
    return Y.to(_dtype(c))


# ---- the framework's operators ------------------------------------------------------------------------------------


def _workspace(s, nbytes):
    """Scratch memory, kept with the state's buffers."""
    if s["ws"] is None:
        s["ws"] = torch.empty(max(nbytes, 256), dtype=torch.uint8, device=DEV)
    return s["ws"]


def _act_code(api, c):
    return api.MOE_ACT_SILU if c["act"] == "silu" else api.MOE_ACT_GELU


def _glu_own(s):
    from paper_2407_00599_amd import api
    c = s["c"]
    S, E, k, M, H, train = c["S"], c["E"], c["k"], c["M"], c["H"], c["train"]
    R, offsets, inv, act, shard = S * k, s["offsets"], s["row_inv"], _act_code(api, c), (c["esp_idx"], c["n_esp"])
    code = api.dtype_code(s["x"])
    ws = s["ws"] if s["ws"] is not None else _workspace(s, max(
        api.moe_ragged_glu_workspace_bytes(code, R, E, M, H, c["n_esp"], b) for b in range(1 + train)))
    api.moe_ragged_glu_fwd(s["x"], S, inv, k, s["W1"], s["W2"], offsets, R, E, M, H, *shard, act, s["Z"] if train else None, s["A"],
                           s["Y"], ws)
    if not train:
        return {"Y": s["Y"]}
    api.moe_ragged_glu_bwd(s["dY"], s["x"], S, inv, k, s["Z"], s["W1"], s["W2"], offsets, R, E, M, H, *shard, act, s["dX"], s["dW1"],
                           s["dW2"], ws)
    return {n: s[n] for n in ("Y", "Z", "dX", "dW1", "dW2")}


def _mx4_own(s):
    from paper_2407_00599_amd import api
    c = s["c"]
    shape = (c["G"], c["rows"], c["cols"], int(c["transposed"]))
    api.moe_mx4_store(s["x"], *shape, s["q"], s["s"])
    api.moe_mx4_load(s["q"], s["s"], *shape, s["back"])
    return s["back"]


def _gemm4_own(s):
    from paper_2407_00599_amd import api
    c = s["c"]
    S, E, k, K, N = c["S"], c["E"], c["k"], c["M"], c["H"]
    ws = s["ws"] if s["ws"] is not None else _workspace(s, api.moe_ragged_gemm_mx4_workspace_bytes(S * k, E, K, N))
    api.moe_ragged_gemm_mx4(s["xq"], s["xs"], S, s["row_inv"], k, s["Wq"], s["Ws"], s["offsets"], S * k, E, K, N, s["Y"], ws)
    return s["Y"]


def _glu4_own(s):
    from paper_2407_00599_amd import api
    c = s["c"]
    S, E, k, M, H = c["S"], c["E"], c["k"], c["M"], c["H"]
    R = S * k
    ws = s["ws"] if s["ws"] is not None else _workspace(s, api.moe_ragged_glu_mx4_workspace_bytes(S, R, E, M, H))
    api.moe_ragged_glu_mx4(s["x"], S, s["row_inv"], k, s["W1q"], s["W1s"], s["W2q"], s["W2s"], s["offsets"], R, E, M, H, _act_code(api, c),
                           s["Y"], ws)
    return s["Y"]


def run(state):
    forms = {"glu": (_glu_plain, _glu_own), "mx4": (_mx4_plain, _mx4_own), "gemm4": (_gemm4_plain, _gemm4_own), "glu4": (_glu4_plain, _glu4_own)}
    return forms[state["c"]["kind"]][1 if own else 0](state)


# ---- what a pass cannot do without --------------------------------------------------------------------------------


def work(case):
    c = case
    b = 4 if c["dtype"] == "f32" else 2
    if c["kind"] == "mx4":       # x in, 4 bits and a byte per block out and in again, x out
        n = c["G"] * c["rows"] * c["cols"]
        return {"bytes": 2.0 * n * b + 2.0 * n * 17 / 32, "flops": 4.0 * n}
    S, E, k, M, H = c["S"], c["E"], c["k"], c["M"], c["H"]
    R = S * k
    used = E * (1 - (1 - 1 / E) ** R)          # experts that some row asks for, of equal shares
    rows = R if c["f"] == 0.0 else min(R, E * max(1, math.ceil(R * c["f"] / E)))
    if c["kind"] == "gemm4":
        return {"bytes": 17 / 32 * (S * M + used * M * H) + b * R * H + 4.0 * R, "flops": 2.0 * rows * M * H}
    if c["kind"] == "glu4":
        return {"bytes": b * (S + R) * M + 17 / 32 * 3 * used * M * H + 4.0 * R, "flops": 6.0 * rows * M * H}
    Hl = H // c["n_esp"]
    nbytes, flops = b * (S * M + R * M + 3 * used * M * Hl) + 4.0 * R, 6.0 * rows * M * Hl
    if c["train"]:               # kept values out and in, dY, x and the weights again, dX and both gradients out
        nbytes += b * (4 * R * Hl + 2 * R * M + S * M + 3 * used * M * Hl + 3 * E * M * Hl)
        flops *= 3
    return {"bytes": float(nbytes), "flops": flops}


# ---- the definitions in 64 bits -----------------------------------------------------------------------------------


def _kept4_exact(v):
    """What 4 bits keep of v [n, K] along its rows."""
    out = torch.empty_like(v)
    grid = torch.tensor([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0], dtype=torch.float64, device=DEV)
    for c0 in range(0, v.shape[1], 32):
        block = v[:, c0:c0 + 32]
        top = block.abs().max(dim=1, keepdim=True).values
        size = torch.where(top > 0, 2.0 ** torch.floor(torch.log2(torch.where(top > 0, top, 1.0))), torch.ones_like(top))
        size = torch.where(size > top, size / 2, torch.where(2 * size <= top, 2 * size, size))       # a logarithm next to a whole number
        step = torch.where(top >= 1.75 * size, size / 2, size / 4)
        ratio = (block.abs() / step).clamp(max=6.0)
        below = torch.searchsorted(grid, ratio, right=True) - 1
        above = (below + 1).clamp(max=7)
        down, up = ratio - grid[below], grid[above] - ratio
        pick = torch.where((up < down) | ((up == down) & (above % 2 == 0)), above, below)
        out[:, c0:c0 + 32] = torch.copysign(grid[pick] * step, block)
    return out


def _bytes_exact(q, s, K):
    """The value of each of the K entries of a row, from its bytes."""
    n = q.shape[0]
    i = torch.arange(K, device=DEV)
    code = (q[:, i // 2].int() >> (4 * (i % 2)).int()) & 15
    block = i // 32
    scale = s[block // 16, block % 4, :, (block % 16) // 4].t().double()
    e, m = (code // 2) % 4, code % 2
    size = torch.where(e == 0, 0.5 * m.double(), (1 + 0.5 * m.double()) * 2.0 ** (e - 1).double())
    assert scale.shape == (n, K)
    return torch.where(code >= 8, -size, size) * 2.0 ** (scale - 127)


def _act_exact(act, g):
    if act == "silu":
        return g / (1 + torch.exp(-g))
    return g * 0.5 * torch.erfc(-g / 2 ** 0.5)


def _slope_exact(act, g):
    if act == "silu":
        p = 1 / (1 + torch.exp(-g))
        return p + g * p * (1 - p)
    return 0.5 * torch.erfc(-g / 2 ** 0.5) + g * torch.exp(-g * g / 2) / (2 * math.pi) ** 0.5


def exact(case, seed):
    c, s, d = dict(case), prepare(case, seed), torch.float64
    if c["kind"] == "mx4":
        if s["x"].numel() > 1 << 28:
            return None
        out = torch.empty(s["x"].shape, dtype=d, device=DEV)
        for g in range(c["G"]):
            x = s["x"][g].to(d)
            out[g] = _kept4_exact(x.t().contiguous()).t() if c["transposed"] else _kept4_exact(x)
        return out
    E, k, M, H = c["E"], c["k"], c["M"], c["H"]
    R = c["S"] * k
    tokens = s["row_inv"].reshape(-1) // k
    first = s["offsets"].tolist()
    train = c["kind"] == "glu" and c["train"]
    out = {"Y": torch.zeros(R, H if c["kind"] == "gemm4" else M, dtype=d, device=DEV)}
    if c["kind"] == "glu":
        Hl = H // c["n_esp"]
        gate = slice(c["esp_idx"] * Hl, (c["esp_idx"] + 1) * Hl)
        up = slice(H + gate.start, H + gate.stop)
    if train:
        out.update(Z=torch.zeros(R, 2 * Hl, dtype=d, device=DEV), dX=torch.zeros(R, M, dtype=d, device=DEV),
                   dW1=torch.zeros(s["W1"].shape, dtype=d, device=DEV), dW2=torch.zeros(s["W2"].shape, dtype=d, device=DEV))
    for e in range(E):
        here = slice(first[e], first[e + 1])
        who = tokens[here].long()
        if who.numel() == 0:
            continue
        if c["kind"] == "gemm4":
            out["Y"][here] = _bytes_exact(s["xq"], s["xs"], M)[who] @ _bytes_exact(s["Wq"][e], s["Ws"][e], M).t()
            continue
        if c["kind"] == "glu4":
            both = _kept4_exact(s["x"][who].to(d)) @ _bytes_exact(s["W1q"][e], s["W1s"][e], M).t()
            hidden = _kept4_exact(_act_exact(c["act"], both[:, :H]) * both[:, H:])
            out["Y"][here] = hidden @ _bytes_exact(s["W2q"][e], s["W2s"][e], H).t()
            continue
        X, Wg, Wu, Wd = s["x"][who].to(d), s["W1"][e, :, gate].to(d), s["W1"][e, :, up].to(d), s["W2"][e, gate].to(d)
        g, u = X @ Wg, X @ Wu
        out["Y"][here] = (_act_exact(c["act"], g) * u) @ Wd
        if train:
            out["Z"][here] = torch.cat([g, u], dim=1)
            g, u = g.to(_dtype(c)).to(d), u.to(_dtype(c)).to(d)
            up_grad = s["dY"][here].to(d)
            dA = up_grad @ Wd.t()
            dg, du = dA * u * _slope_exact(c["act"], g), dA * _act_exact(c["act"], g)
            out["dX"][here] = dg @ Wg.t() + du @ Wu.t()
            out["dW1"][e, :, gate], out["dW1"][e, :, up] = X.t() @ dg, X.t() @ du
            out["dW2"][e, gate] = (_act_exact(c["act"], g) * u).t() @ up_grad
    return out if c["kind"] == "glu" else out["Y"]
