"""Operators of a dropless (ragged) MoE block as timed cases: the experts' products over rows that lie expert by
expert with no capacity padding between them, 8-bit checkpoints of activations and the backward pass that reads them,
and the norms in front of and behind the block.

Kinds of pass:
  products  plan of the rows, then the three grouped products over them: Y = X W (the token rows are read through the
            plan's map), dX = dY W^T, dW = X^T dY.
  serve     plan and expert FFN forward, nothing kept for a backward pass.
  train     plan, expert FFN forward that keeps the pre-activation in 8 bits, and the backward pass that reads it.
  ckpt      an activation tensor to 8 bits and back.
  norm      norm in front of a block, and norm, gate, residual scale and residual behind it; in training their gradients.

Definitions.  Rows: choice (t, j) of token t lies at row offsets[e] + slot of its expert e; choices without a slot have
no row; rows at or behind offsets[E] hold zeros.  8 bits: a row is cut into blocks of 32 columns; a block's step is
2^(x - 6) for the largest magnitude a in [2^x, 2^(x+1)), twice that where a / step would round to 128; a value is kept as
the whole number nearest to value / step (ties to even), within +-127.  In the FFN the forward pass uses the
pre-activation as computed, the backward pass its kept value, for the activation as well as for its derivative (erf
GeLU).  Norms: n(h) = (h - mean) / sqrt(var + eps) weight + bias ("layer") or h / sqrt(mean(h^2) + eps) weight ("rms");
behind the block y = x + alpha * gate * n(h), with a gate per channel, per token or none.
"""
import math

import torch

own = False     # the framework's operators instead of the plain forms

DEV = "cuda:0"
EPS = 1e-5
FFN = {"dtype": "bf16", "k": 2, "n_esp": 1, "esp_idx": 0, "skew": 0.0, "f": 0.0, "sigma_w": 0.02}


def _ffn(kind, **kw):
    return dict(FFN, kind=kind, **kw)


def listed():
    return [
        # one decoding step of a single request: two rows, two experts' weights are all of the traffic
        _ffn("serve", name="serve_1", S=1, M=1024, H=4096, E=8),
        # one decoding step of a small batch
        _ffn("serve", name="serve_32", S=32, M=1024, H=4096, E=8),
        # a short prompt against the widest experts that the framework is benchmarked with
        _ffn("serve", name="prefill_256_wide", S=256, M=4096, H=14336, E=8, sigma_w=0.01),
        # fp32 products, no size a multiple of a tile, three choices, some dropped
        _ffn("products", name="products_f32_ragged", dtype="f32", S=1003, k=3, M=520, H=1544, E=12, skew=0.5, f=1.1),
        # 64 experts with unequal shares of the rows
        _ffn("products", name="products_64", S=16384, M=2048, H=2048, E=64, skew=0.5),
        # training step of the layer shape of the paper's layer benchmark
        _ffn("train", name="train_layer", S=4096, M=1024, H=4096, E=8, skew=0.2),
        # fp32 training of a middle-sized layer
        _ffn("train", name="train_f32", dtype="f32", S=1024, M=512, H=2048, E=8, skew=0.3),
        # the widest experts' hidden shard, half of the largest configuration's tokens
        _ffn("train", name="train_large", S=16384, M=4096, H=14336, E=8, n_esp=2, esp_idx=1, sigma_w=0.01, skew=0.2),
        # the hidden activations of a small fp32 layer
        {"name": "ckpt_f32", "kind": "ckpt", "dtype": "f32", "rows": 1003, "cols": 1544},
        # the pre-activations of a large layer's hidden shard
        {"name": "ckpt_large", "kind": "ckpt", "dtype": "bf16", "rows": 32768, "cols": 7168},
        # one token of a decoding step
        {"name": "norm_token", "kind": "norm", "dtype": "bf16", "S": 1, "M": 4096, "norm": "rms", "gate": "token", "train": False},
        # a training step's tokens
        {"name": "norm_large", "kind": "norm", "dtype": "bf16", "S": 32768, "M": 4096, "norm": "layer", "gate": "channel", "train": True},
    ]


def _log_int(rng, lo, hi, mult=1):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi))) / mult)) * mult))


def draw(rng):
    """One more case of the same ranges."""
    kind = rng.choice(["products", "products", "serve", "serve", "train", "train", "train", "ckpt", "norm", "norm"])
    dtype = "bf16" if rng.random() < 0.7 else "f32"
    if kind == "ckpt":
        return {"kind": kind, "dtype": dtype, "rows": _log_int(rng, 1, 32768), "cols": _log_int(rng, 64, 7168, 8)}
    if kind == "norm":
        return {"kind": kind, "dtype": dtype, "S": _log_int(rng, 1, 32768 if dtype == "bf16" else 16384),
                "M": _log_int(rng, 64, 4096, rng.choice([8, 8, 64])), "norm": rng.choice(["rms", "layer"]),
                "gate": rng.choice(["none", "channel", "token"]), "train": rng.random() < 0.7}
    while True:
        M = _log_int(rng, 64, 4096, rng.choice([8, 64, 256]))
        n_esp = 1 if kind == "products" else rng.choice([1, 1, 1, 2, 4])
        H = _log_int(rng, 128, 14336, rng.choice([8, 64, 512]) * n_esp)
        H -= H % (8 * n_esp)
        E = rng.choice([1, 2, 4, 8, 8, 8, 12, 16, 24, 32, 64])
        S = _log_int(rng, 1, 256) if kind == "serve" else _log_int(rng, 16, 16384)
        k = min(E, rng.choice([1, 2, 2, 2, 3, 4]))
        c = _ffn(kind, dtype=dtype, S=S, k=k, M=M, H=H, E=E, n_esp=n_esp, esp_idx=rng.randrange(n_esp),
                 skew=rng.choice([0.0, 0.2, 0.5, 1.0]), f=rng.choice([0.0, 0.0, 0.0, 1.0, 1.25]))
        flops = {"serve": 2, "products": 3, "train": 6}[kind] * 2.0 * S * k * M * (H // n_esp)
        if H >= 8 * n_esp and flops <= (1.1e13 if dtype == "bf16" else 4e11) and E * M * H <= 1 << 29:
            return c


# ---- inputs -------------------------------------------------------------------------------------------------------


def _dtype(c):
    return torch.float32 if c["dtype"] == "f32" else torch.bfloat16


def _maker(c, seed):
    gen = torch.Generator(device=DEV)
    gen.manual_seed(seed)

    def normal(*shape, sigma=1.0, dtype=None):
        out = torch.empty(*shape, dtype=dtype or _dtype(c), device=DEV)
        for part in (out if len(shape) > 2 else (out,)):
            part.copy_(torch.randn(part.shape, generator=gen, device=DEV) * sigma)
        return out

    return gen, normal


def _routing(c, gen):
    """What a gate hands over: chosen experts, their slots (choice by choice, token by token) and the demand per expert."""
    S, E, k = c["S"], c["E"], c["k"]
    logits = torch.randn(S, E, generator=gen, device=DEV) + c["skew"] * torch.randn(E, generator=gen, device=DEV)
    idx = logits.topk(k, dim=1).indices
    flat = idx.t().reshape(-1)
    order = torch.argsort(flat, stable=True)
    counts = torch.bincount(flat, minlength=E)
    slot = torch.empty_like(flat)
    slot[order] = torch.arange(S * k, device=DEV) - (counts.cumsum(0) - counts)[flat[order]]
    C = S if c["f"] == 0.0 else max(1, math.ceil(k * S * c["f"] / E))
    slot = torch.where(slot < C, slot, -1).reshape(k, S).t()
    return C, idx.int(), slot.int().contiguous(), counts.int()


def prepare(case, seed):
    c = dict(case)
    gen, normal = _maker(c, seed)
    dt = _dtype(c)

    def e(*shape, dtype=dt):
        return torch.empty(*shape, dtype=dtype, device=DEV)

    if c["kind"] == "ckpt":
        # a few columns stand out, as in trained networks
        x = normal(c["rows"], c["cols"], dtype=torch.float32) * (1 + 7 * (torch.rand(c["cols"], generator=gen, device=DEV) < 0.02))
        blocks = (c["cols"] + 31) // 32
        return {"c": c, "x": x.to(dt), "q": e(c["rows"], c["cols"], dtype=torch.int8), "s": e(c["rows"], blocks, dtype=torch.uint8),
                "back": e(c["rows"], c["cols"])}
    if c["kind"] == "norm":
        S, M, f32 = c["S"], c["M"], torch.float32
        s = {"c": c, "x": normal(S, M, sigma=2.0), "h": (normal(S, M, dtype=f32) + 0.25).to(dt), "du": normal(S, M), "dy": normal(S, M),
             "w1": 1 + 0.1 * normal(M, dtype=f32), "b1": 0.1 * normal(M, dtype=f32), "w2": 1 + 0.1 * normal(M, dtype=f32),
             "b2": 0.1 * normal(M, dtype=f32), "gate": None, "alpha": 0.5}
        if c["gate"] != "none":
            s["gate"] = torch.sigmoid(normal(S if c["gate"] == "token" else M, dtype=f32))
        s.update(u=e(S, M), y=e(S, M), mean1=e(S, dtype=f32), rstd1=e(S, dtype=f32), mean2=e(S, dtype=f32), rstd2=e(S, dtype=f32), ws=None)
        if c["train"]:
            s.update(dh=e(S, M), dx=e(S, M), dw1=e(M, dtype=f32), db1=e(M, dtype=f32), dw2=e(M, dtype=f32), db2=e(M, dtype=f32),
                     dgate=None if s["gate"] is None else torch.empty_like(s["gate"]))
        return s
    S, E, k, M, H, i32 = c["S"], c["E"], c["k"], c["M"], c["H"], torch.int32
    R, Hl = S * k, c["H"] // c["n_esp"]
    C, idx, slot, counts = _routing(c, gen)
    s = {"c": c, "C": C, "idx": idx, "slot": slot, "counts": counts, "x": normal(S, M), "W1": normal(E, M, H, sigma=c["sigma_w"]),
         "offsets": e(E + 1, dtype=i32), "row_idx": e(S, k, dtype=i32), "row_slot": e(S, k, dtype=i32), "row_inv": e(k, S, dtype=i32),
         "ws": None, "rows": counts.clamp(max=C).tolist()}      # rows per expert, on the host, for the plain forms' slices
    if c["kind"] == "products":
        s.update(dY=normal(R, H), Y=e(R, H), dX=e(R, M), dW=e(E, M, H))
        return s
    s.update(W2=normal(E, H, M, sigma=c["sigma_w"]), A=e(R, Hl), Y=e(R, M))
    if c["kind"] == "train":
        # of the whole weight gradients a hidden shard writes its own columns (rows)
        s.update(dY=normal(R, M), dX=e(R, M), dW1=torch.zeros_like(s["W1"]), dW2=torch.zeros_like(s["W2"]),
                 Zq=e(R, Hl, dtype=torch.int8), Zs=e(R, (Hl + 31) // 32, dtype=torch.uint8))
    return s


# ---- plain forms --------------------------------------------------------------------------------------------------


def _plan_plain(s):
    c = s["c"]
    S, E, k = c["S"], c["E"], c["k"]
    kept = s["slot"] >= 0
    offsets = torch.zeros(E + 1, dtype=torch.int64, device=DEV)
    offsets[1:] = s["counts"].clamp(max=s["C"]).cumsum(0)
    row = offsets[s["idx"].long()] + s["slot"]
    inv = torch.full((S * k + 1,), -1, dtype=torch.int32, device=DEV)      # the last one takes the choices without a row
    inv[torch.where(kept, row, S * k).reshape(-1)] = torch.arange(S * k, dtype=torch.int32, device=DEV)
    return {"offsets": offsets.int(), "row_idx": torch.where(kept, row // S, 0).int(),
            "row_slot": torch.where(kept, row % S, -1).int(), "row_inv": inv[:S * k].reshape(k, S)}


def _by_expert(rows, A, B, out):
    """out = A B of each expert's rows, with B[e]; the rows behind the last expert's are zeros."""
    at = 0
    for e, n in enumerate(rows):
        if n:
            torch.mm(A[at:at + n], B[e].float() if B[e].dtype == torch.bfloat16 else B[e], out=out[at:at + n])
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


def _new(like, *shape):
    return torch.empty(*shape, dtype=like, device=DEV)


def _phi(z):
    return 0.5 * (1 + torch.erf(z * math.sqrt(0.5)))


def _eight_bits(z):
    """What the 8-bit form of z stands for."""
    rows, cols = z.shape
    z = torch.nn.functional.pad(z, (0, -cols % 32)).view(rows, -1, 32)
    a = z.abs().amax(2, keepdim=True).float()
    step = (a.view(torch.int32) & 0x7F800000).view(torch.float32) / 64      # 2^x / 2^6
    step = torch.where(a >= 127.5 * step, 2 * step, step)
    step = torch.where(step == 0, 1.0, step).to(z.dtype)
    return ((z / step).round().clamp(-127, 127) * step).view(rows, -1)[:, :cols]


def _ffn_plain(s):
    c, dt, f32 = s["c"], _dtype(s["c"]), torch.float32
    plan = _plan_plain(s)
    rows, R, M, k = s["rows"], c["S"] * c["k"], c["M"], c["k"]
    Hl = c["H"] // c["n_esp"]
    h0 = c["esp_idx"] * Hl
    X = _rows_of(s["x"].float(), plan["row_inv"], k)
    if c["kind"] == "products":
        dY = s["dY"].float()
        Wt = s["W1"].transpose(1, 2)
        return dict(plan, Y=_by_expert(rows, X, s["W1"], _new(f32, R, c["H"])).to(dt),
                    dX=_by_expert(rows, dY, Wt, _new(f32, R, M)).to(dt),
                    dW=_reduce_by_expert(rows, X, dY, _new(dt, c["E"], M, c["H"])))
    W1, W2 = s["W1"][:, :, h0:h0 + Hl], s["W2"][:, h0:h0 + Hl]
    if dt == f32 and c["kind"] == "train":   # in 64 bits: a sum next to the border between two steps decides which one is kept
        Z = _by_expert(rows, X.double(), W1.double(), _new(torch.float64, R, Hl))
    else:
        Z = _by_expert(rows, X, W1, _new(f32, R, Hl))
    A = (Z * _phi(Z)).float()
    out = dict(plan, Y=_by_expert(rows, A, W2, _new(f32, R, M)).to(dt))
    if c["kind"] == "serve":
        return out
    Z = _eight_bits(Z).float()
    dY = s["dY"].float()
    dA = _by_expert(rows, dY, W2.transpose(1, 2), _new(f32, R, Hl))
    cdf = _phi(Z)
    dZ = dA * (cdf + Z * torch.exp(-0.5 * Z * Z) * (1 / math.sqrt(2 * math.pi)))
    out["dX"] = _by_expert(rows, dZ, W1.transpose(1, 2), _new(f32, R, M)).to(dt)
    out["dW1"], out["dW2"] = torch.zeros_like(s["W1"]), torch.zeros_like(s["W2"])
    _reduce_by_expert(rows, X, dZ, out["dW1"][:, :, h0:h0 + Hl])
    _reduce_by_expert(rows, Z * cdf, dY, out["dW2"][:, h0:h0 + Hl])
    return out


def _norm_plain(s):
    c, dt = s["c"], _dtype(s["c"])
    layer, x, h = c["norm"] == "layer", s["x"].float(), s["h"].float()

    def normed(v):
        if layer:
            v = v - v.mean(1, keepdim=True)
        rstd = (v.square().mean(1, keepdim=True) + EPS).rsqrt()
        return v * rstd, rstd

    def back(g, hat, rstd):        # through v -> hat
        g = g - hat * (g * hat).mean(1, keepdim=True)
        return rstd * (g - g.mean(1, keepdim=True) if layer else g)

    xhat, xr = normed(x)
    hhat, hr = normed(h)
    b1, b2 = (s["b1"], s["b2"]) if layer else (0.0, 0.0)
    gate = 1.0 if s["gate"] is None else s["gate"][:, None] if c["gate"] == "token" else s["gate"]
    n = hhat * s["w2"] + b2
    out = {"u": (xhat * s["w1"] + b1).to(dt), "y": (x + s["alpha"] * gate * n).to(dt)}
    if not c["train"]:
        return out
    du, dy = s["du"].float(), s["dy"].float()
    dn = s["alpha"] * gate * dy
    out["dh"] = back(dn * s["w2"], hhat, hr).to(dt)
    out["dw2"] = (dn * hhat).sum(0, dtype=torch.float64).float()
    if s["gate"] is not None:
        out["dgate"] = (s["alpha"] * dy * n).sum(1 if c["gate"] == "token" else 0, dtype=torch.float64).float()
    out["dx"] = (dy + back(du * s["w1"], xhat, xr)).to(dt)
    out["dw1"] = (du * xhat).sum(0, dtype=torch.float64).float()
    if layer:
        out["db2"], out["db1"] = dn.sum(0, dtype=torch.float64).float(), du.sum(0, dtype=torch.float64).float()
    return out


# ---- the framework's operators ------------------------------------------------------------------------------------


def _workspace(s, nbytes):
    """Scratch memory, kept with the state's buffers."""
    if s["ws"] is None:
        s["ws"] = torch.empty(max(nbytes, 256), dtype=torch.uint8, device=DEV)
    return s["ws"]


def _ffn_own(s):
    from paper_2407_00599_amd import api
    c = s["c"]
    S, E, k, M, H = c["S"], c["E"], c["k"], c["M"], c["H"]
    R, offsets, inv = S * k, s["offsets"], s["row_inv"]
    api.moe_ragged_plan(s["idx"], s["slot"], s["counts"], S, E, k, s["C"], offsets, s["row_idx"], s["row_slot"], inv)
    out = {n: s[n] for n in ("offsets", "row_idx", "row_slot", "row_inv", "Y")}
    code = api.dtype_code(s["x"])
    if c["kind"] == "products":
        ws = s["ws"] if s["ws"] is not None else _workspace(s, max(
            api.moe_ragged_gemm_workspace_bytes(code, R, E, M, H), api.moe_ragged_gemm_workspace_bytes(code, R, E, H, M),
            api.moe_ragged_wgrad_workspace_bytes(code, R, E, M, H)))
        api.moe_ragged_gemm(s["x"], S, inv, k, s["W1"], 0, offsets, R, E, M, H, s["Y"], ws)
        api.moe_ragged_gemm(s["dY"], 0, None, 1, s["W1"], 1, offsets, R, E, H, M, s["dX"], ws)
        api.moe_ragged_wgrad(s["x"], S, inv, k, s["dY"], offsets, R, E, M, H, s["dW"], ws)
        return dict(out, dX=s["dX"], dW=s["dW"])
    train = c["kind"] == "train"
    ws = s["ws"] if s["ws"] is not None else _workspace(s, max(
        api.moe_ragged_ffn_workspace_bytes(code, R, E, M, H, c["n_esp"], b) for b in range(1 + train)))
    api.moe_ragged_ffn_fwd(s["x"], S, inv, k, s["W1"], s["W2"], offsets, R, E, M, H, c["esp_idx"], c["n_esp"],
                           s["Zq"] if train else None, s["Zs"] if train else None, s["A"], s["Y"], ws)
    if not train:
        return out
    api.moe_ragged_ffn_bwd(s["dY"], s["x"], S, inv, k, s["Zq"], s["Zs"], s["W1"], s["W2"], offsets, R, E, M, H, c["esp_idx"],
                           c["n_esp"], s["dX"], s["dW1"], s["dW2"], ws)
    return dict(out, dX=s["dX"], dW1=s["dW1"], dW2=s["dW2"])


def _norm_own(s):
    from paper_2407_00599_amd import api
    c = s["c"]
    S, M, train, layer = c["S"], c["M"], c["train"], c["norm"] == "layer"
    kind = api.MOE_NORM_LAYER if layer else api.MOE_NORM_RMS
    gk = {"none": api.MOE_GATE_NONE, "channel": api.MOE_GATE_CHANNEL, "token": api.MOE_GATE_TOKEN}[c["gate"]]
    b1, b2 = (s["b1"], s["b2"]) if layer else (None, None)
    m1, r1, m2, r2 = (s["mean1"] if layer else None, s["rstd1"], s["mean2"] if layer else None, s["rstd2"]) if train else (None,) * 4
    api.moe_norm_fwd(s["x"], S, M, kind, s["w1"], b1, EPS, s["u"], m1, r1)
    api.moe_norm_residual_fwd(s["h"], s["x"], S, M, kind, s["w2"], b2, s["gate"], gk, s["alpha"], EPS, s["y"], m2, r2)
    out = {"u": s["u"], "y": s["y"]}
    if not train:
        return out
    ws = s["ws"] if s["ws"] is not None else _workspace(s, api.moe_norm_bwd_workspace_bytes(S, M))
    db1, db2 = (s["db1"], s["db2"]) if layer else (None, None)
    api.moe_norm_residual_bwd(s["dy"], s["h"], S, M, kind, s["w2"], b2, s["gate"], gk, s["alpha"], m2, r2, s["dh"], s["dw2"], db2,
                              s["dgate"], ws)
    api.moe_norm_bwd(s["du"], s["x"], S, M, kind, s["w1"], m1, r1, s["dy"], s["dx"], s["dw1"], db1, ws)
    out.update({n: s[n] for n in ("dh", "dw2", "dx", "dw1")})
    if s["gate"] is not None:
        out["dgate"] = s["dgate"]
    if layer:
        out.update(db2=db2, db1=db1)
    return out


def _ckpt_own(s):
    from paper_2407_00599_amd import api
    api.moe_ckpt8_store(s["x"], s["c"]["rows"], s["c"]["cols"], s["q"], s["s"])
    api.moe_ckpt8_load(s["q"], s["s"], s["c"]["rows"], s["c"]["cols"], s["back"])
    return s["back"]


def run(state):
    kind = state["c"]["kind"]
    if kind == "ckpt":
        return _ckpt_own(state) if own else _eight_bits(state["x"].float()).to(state["x"].dtype)
    if kind == "norm":
        return _norm_own(state) if own else _norm_plain(state)
    return _ffn_own(state) if own else _ffn_plain(state)


# ---- what a pass cannot do without --------------------------------------------------------------------------------


def work(case):
    c = case
    b = 4 if c["dtype"] == "f32" else 2
    if c["kind"] == "ckpt":      # x in, 8 bits and a byte per block out and in again, x out
        n = c["rows"] * c["cols"]
        return {"bytes": 2.0 * n * b + 2.0 * (n + c["rows"] * ((c["cols"] + 31) // 32)), "flops": 4.0 * n}
    if c["kind"] == "norm":      # x in, u out; h and x in, y out; training: dy and h in, dh out; du, x and dy in, dx out
        n = c["S"] * c["M"]
        return {"bytes": float(n * b * (5 + (7 if c["train"] else 0))), "flops": (16.0 + (32.0 if c["train"] else 0.0)) * n}
    S, E, k, M, Hl = c["S"], c["E"], c["k"], c["M"], c["H"] // c["n_esp"]
    R = S * k
    used = E * (1 - (1 - 1 / E) ** R)          # experts that some row asks for, of equal shares
    rows = R if c["f"] == 0.0 else min(R, E * max(1, math.ceil(R * c["f"] / E)))
    nbytes, flops = 4 * (5 * R + 2 * E), 2.0 * rows * M * Hl
    if c["kind"] == "products":  # token rows (twice), dY twice, weights twice; Y, dX, dW out
        nbytes += b * (2 * S * M + 3 * R * Hl + R * M + 2 * used * M * Hl + E * M * Hl)
        return {"bytes": float(nbytes), "flops": 3 * flops}
    nbytes += b * (S * M + R * M + 2 * used * M * Hl)
    if c["kind"] == "train":     # the kept pre-activation out and in, then dY, x and the weights again, dX and both gradients out
        nbytes += 2 * R * (Hl + (Hl + 31) // 32) + b * (2 * R * M + S * M + 2 * used * M * Hl + 2 * E * M * Hl)
        return {"bytes": float(nbytes), "flops": 6 * flops}
    return {"bytes": float(nbytes), "flops": 2 * flops}


# ---- the definitions in 64 bits -----------------------------------------------------------------------------------


def _kept_exact(v):
    out = torch.empty_like(v)
    for c0 in range(0, v.shape[1], 32):
        block = v[:, c0:c0 + 32]
        top = block.abs().max(dim=1, keepdim=True).values
        mantissa = torch.frexp(top).mantissa                    # top = mantissa 2^(x + 1), mantissa in [1/2, 1)
        step = torch.where(top > 0, top / mantissa / 128, torch.ones_like(top))
        step = step * (1 + (top / step >= 127.5).double())
        out[:, c0:c0 + 32] = torch.round(block / step).clamp(-127, 127) * step
    return out


def _ffn_exact(c, s):
    S, E, k, M, d = c["S"], c["E"], c["k"], c["M"], torch.float64
    R, Hl = S * k, c["H"] // c["n_esp"]
    lo, hi = c["esp_idx"] * Hl, (c["esp_idx"] + 1) * Hl
    out = {"offsets": None, "row_idx": None, "row_slot": None, "row_inv": None}
    choice = torch.arange(S * k, device=DEV).view(S, k)
    names = {"products": ("dX", "dW"), "serve": (), "train": ("dX", "dW1", "dW2")}[c["kind"]]
    out["Y"] = torch.zeros(R, c["H"] if c["kind"] == "products" else M, dtype=d, device=DEV)
    for name in names:
        out[name] = torch.zeros(R, M, dtype=d, device=DEV) if name == "dX" else torch.zeros(
            s["W2" if name == "dW2" else "W1"].shape, dtype=d, device=DEV)
    row = 0
    for e in range(E):
        mine = (s["idx"] == e) & (s["slot"] >= 0)
        seat, who = s["slot"][mine], choice[mine]
        n = who.numel()
        if n == 0:
            continue
        here = slice(row, row + n)
        row += n
        tokens = torch.empty(n, dtype=torch.int64, device=DEV)
        tokens[seat.long()] = who // k
        X = s["x"][tokens].to(d)
        if c["kind"] == "products":
            W, G = s["W1"][e].to(d), s["dY"][here].to(d)
            out["Y"][here], out["dX"][here], out["dW"][e] = X @ W, G @ W.t(), X.t() @ G
            continue
        Wa, Wb = s["W1"][e, :, lo:hi].to(d), s["W2"][e, lo:hi].to(d)
        Z = X @ Wa
        out["Y"][here] = (0.5 * Z * torch.erfc(-Z / 2 ** 0.5)) @ Wb
        if c["kind"] == "train":
            G, Z = s["dY"][here].to(d), _kept_exact(Z)
            half = 0.5 * torch.erfc(-Z / 2 ** 0.5)
            D = (G @ Wb.t()) * (half + Z * torch.exp(-Z * Z / 2) / (2 * math.pi) ** 0.5)
            out["dX"][here] = D @ Wa.t()
            out["dW1"][e, :, lo:hi], out["dW2"][e, lo:hi] = X.t() @ D, (Z * half).t() @ G
    return out


def _norm_exact(c, s):
    d = torch.float64
    x, h, w1, w2 = (s[n].to(d) for n in ("x", "h", "w1", "w2"))
    layer, M, alpha = c["norm"] == "layer", c["M"], s["alpha"]
    b1, b2 = (s["b1"].to(d), s["b2"].to(d)) if layer else (torch.zeros_like(w1), torch.zeros_like(w2))
    gate = torch.ones(1, 1, dtype=d, device=DEV) if s["gate"] is None else s["gate"].to(d).reshape((-1, 1) if c["gate"] == "token" else (1, -1))

    def parts(v):
        mu = v.sum(1, keepdim=True) / M if layer else torch.zeros(v.shape[0], 1, dtype=d, device=DEV)
        sd = torch.sqrt(((v - mu) ** 2).sum(1, keepdim=True) / M + EPS)
        return (v - mu) / sd, sd

    xn, xs = parts(x)
    hn, hs = parts(h)
    out = {"u": xn * w1 + b1, "y": x + alpha * gate * (hn * w2 + b2)}
    if not c["train"]:
        return out

    def grad(up, vn, sd):       # d/dv of <up, vn(v)>
        g = up - vn * ((up * vn).sum(1, keepdim=True) / M)
        if layer:
            g = g - up.sum(1, keepdim=True) / M
        return g / sd

    du, dy = s["du"].to(d), s["dy"].to(d)
    up = dy * gate * alpha
    out["dh"], out["dw2"] = grad(up * w2, hn, hs), (up * hn).sum(0)
    out["dx"], out["dw1"] = dy + grad(du * w1, xn, xs), (du * xn).sum(0)
    if s["gate"] is not None:
        out["dgate"] = (alpha * dy * (hn * w2 + b2)).sum(1 if c["gate"] == "token" else 0)
    if layer:
        out["db2"], out["db1"] = up.sum(0), du.sum(0)
    return out


def exact(case, seed):
    c, s = dict(case), prepare(case, seed)
    if c["kind"] == "ckpt":
        return _kept_exact(s["x"].to(torch.float64))
    return _norm_exact(c, s) if c["kind"] == "norm" else _ffn_exact(c, s)
