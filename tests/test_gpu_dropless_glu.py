"""GPU parity of the dropless block with gated experts: all of its calls strung together, against automatic differentiation in float64 with
the block's own routing, served from 4 bits against the oracle's, and replayed from a graph."""
import numpy as np
import pytest
import torch

from oracle import mx4_oracle as Q
from paper_2407_00599_amd.layer import DroplessBlock
from test_gpu_dropless import TOL, params as gelu_params
from util import DEV, torch_dtype

pytestmark = pytest.mark.gpu


def params(S, M, H, E, norm, gate, dtype, seed):
    p, x, dy = gelu_params(S, M, H, E, norm, gate, dtype, seed)
    g = torch.Generator().manual_seed(seed + 1)
    p["W1"] = (1.5 * torch.randn(E, M, 2 * H, generator=g, dtype=torch.float64) / M ** 0.5).to(torch_dtype(dtype)).to(DEV)
    return p, x, dy


def normed(b, v, w, bias, norm):
    if norm == "layer":
        v = v - v.mean(1, keepdim=True)
    v = v / torch.sqrt((v * v).mean(1, keepdim=True) + b.eps)
    return v * w + (bias if norm == "layer" else 0)


def act_of(ffn, z):
    return z * torch.sigmoid(z) if ffn == "swiglu" else z * 0.5 * torch.erfc(-z / 2 ** 0.5)


def spread(d, gate):
    return 1.0 if gate == "none" else d["gate"][:, None] if gate == "token" else d["gate"]


def weights_of(logits, idx, k):
    return torch.softmax(logits.gather(1, idx), 1) if k > 1 else torch.softmax(logits, 1).gather(1, idx)


def reference(b, p, x, dy, norm, gate, ffn):
    """y and every gradient in float64 on the CPU, with the experts that the block's gate selected.  The kept projections are the computed ones:
    their rounding to bf16 is one more of those that the tolerance counts."""
    d = {k: v.detach().cpu().double().requires_grad_() for k, v in p.items()}
    x = x.detach().cpu().double().requires_grad_()
    u = normed(b, x, d["w1"], d.get("b1"), norm)
    idx = b.idx.cpu().long()
    w = weights_of(u @ d["Wg"], idx, b.k)
    h = torch.zeros(b.S, b.M, dtype=torch.float64)
    w_of = torch.zeros(b.S, b.E, dtype=torch.float64).scatter(1, idx, w.detach())
    outs = []
    for e in range(b.E):
        t, j = (idx == e).nonzero(as_tuple=True)
        if not len(t):
            continue
        z = u[t] @ d["W1"][e]
        out = (act_of(ffn, z[:, :b.H]) * z[:, b.H:]) @ d["W2"][e]
        outs.append((e, out.detach(), t))
        h = h.index_add(0, t, w[t, j, None] * out)
    n = normed(b, h, d["w2"], d.get("b2"), norm)
    y = x + b.alpha * spread(d, gate) * n
    h.retain_grad()
    y.backward(dy.cpu().double())
    terms = torch.zeros(b.S, b.E, dtype=torch.float64)       # of the gate's gradient: sums of magnitudes
    for e, out, t in outs:
        terms[t, e] = (h.grad[t] * out).abs().sum(1) * w_of[t, e]
    # A token's gate gradient is alpha <dy, n>, one number that may come out small.  With n off by TOL of its 2-norm (six roundings of 2^-8 that add up
    # like their squares are 0.0096 of it) it is off by TOL alpha |dy| |n| at most (Cauchy-Schwarz).
    products = b.alpha * dy.cpu().double().norm(dim=1) * n.detach().norm(dim=1)
    return y.detach(), x.grad, {k: v.grad for k, v in d.items()}, {"Wg": (u.detach().abs().t() @ terms).max(), "gate": products.max() if gate == "token" else None}


CASES = [(40, 64, 96, 4, 2, "rms", "none", "f32", "swiglu"), (33, 72, 136, 5, 1, "layer", "token", "f32", "geglu"),
         (64, 128, 264, 8, 3, "layer", "channel", "f32", "swiglu"), (70, 128, 256, 8, 2, "rms", "channel", "bf16", "geglu"),
         (1, 64, 64, 3, 2, "layer", "token", "bf16", "swiglu"), (300, 256, 520, 6, 2, "layer", "none", "bf16", "swiglu"),
         (2, 512, 2048, 4, 2, "rms", "token", "bf16", "swiglu")]


@pytest.mark.parametrize("S,M,H,E,k,norm,gate,dtype,ffn", CASES)
def test_block_against_autograd(S, M, H, E, k, norm, gate, dtype, ffn):
    p, x, dy = params(S, M, H, E, norm, gate, dtype, S + M)
    b = DroplessBlock(S, M, H, E, k, torch_dtype(dtype), norm, gate, alpha=0.5, device=DEV, ffn=ffn)
    y = b.forward(x, p)
    dx = b.backward(dy)
    yr, dxr, gr, scales = reference(b, p, x, dy, norm, gate, ffn)
    got = {"y": y, "dx": dx, "W1": b.dW1, "W2": b.dW2, "Wg": b.dWg, "w1": b.dw1, "w2": b.dw2}
    want = {"y": yr, "dx": dxr, **{n: gr[n] for n in ("W1", "W2", "Wg", "w1", "w2")}}
    if norm == "layer":
        got.update(b1=b.db1, b2=b.db2)
        want.update(b1=gr["b1"], b2=gr["b2"])
    if gate != "none":
        got["gate"], want["gate"] = b.dgate, gr["gate"]
    for n in got:
        scale = scales.get(n)
        if scale is None:
            scale = want[n].abs().max()
        err = (got[n].double().cpu() - want[n]).abs().max() / scale
        assert err <= TOL[dtype], (n, float(err))
    b.y.fill_(7)
    y2 = b.infer(x, p)
    assert float((y2.double() - yr.to(DEV)).abs().max() / yr.abs().max()) <= TOL[dtype]


@pytest.mark.parametrize("S,M,H,E,k,norm,gate,dtype,ffn", CASES[:6] + [(300, 128, 264, 3, 2, "rms", "none", "f32", "geglu")])
def test_served_from_four_bits(S, M, H, E, k, norm, gate, dtype, ffn):
    """From the block's own u and routing; a hidden value that another rounding moves to the next code is one of H summed ones."""
    p, x, dy = params(S, M, H, E, norm, gate, dtype, S + M)
    b = DroplessBlock(S, M, H, E, k, torch_dtype(dtype), norm, gate, alpha=0.5, device=DEV, training=False, ffn=ffn)
    q = b.quantise(p)
    assert not {"W1", "W2"} & set(q) and sum(q[n].numel() for n in DroplessBlock.MX4) < 0.6 * (p["W1"].numel() + p["W2"].numel()) + 64 * E * (M + 2 * H)
    y = b.infer(x, q)
    kept = lambda t: torch.from_numpy(Q.kept(t.double().cpu().numpy()))
    d = {n: v.double().cpu() for n, v in p.items()}
    idx, u = b.serving.idx.cpu().long(), kept(b.serving.u)
    w = weights_of(b.serving.logits.double().cpu(), idx, k)
    h = torch.zeros(S, M, dtype=torch.float64)
    for e in range(E):
        t, j = (idx == e).nonzero(as_tuple=True)
        if len(t):
            z = u[t] @ kept(p["W1"][e].t()).t()
            h = h.index_add(0, t, w[t, j, None] * (kept(act_of(ffn, z[:, :H]) * z[:, H:]) @ kept(p["W2"][e].t()).t()))
    ref = x.double().cpu() + b.alpha * spread(d, gate) * normed(b, h, d["w2"], d.get("b2"), norm)
    assert float((y.double().cpu() - ref).abs().max() / ref.abs().max()) <= TOL[dtype]


def test_infer_in_four_bits_between_forward_and_backward():
    S, M, H, E, k = 33, 72, 136, 5, 2
    p, x, dy = params(S, M, H, E, "layer", "token", "bf16", 1)
    _, other, _ = params(S, M, H, E, "layer", "token", "bf16", 2)
    b = DroplessBlock(S, M, H, E, k, norm="layer", gate="token", alpha=0.5, device=DEV, ffn="swiglu")
    q = b.quantise(p)
    names = ["dx", "dWg", "dW1", "dW2", "dw1", "dw2", "db1", "db2", "dgate"]
    y = b.forward(x, p).clone()
    b.backward(dy)
    want = {n: getattr(b, n).clone() for n in names}
    served = b.infer(other, q).clone()
    kept = b.forward(x, p)
    assert torch.equal(b.infer(other, q), served) and torch.equal(kept, y)
    b.backward(dy)
    for n in names:
        assert torch.equal(getattr(b, n), want[n]), n
    with pytest.raises(ValueError):
        b.forward(x, q)
    with pytest.raises(RuntimeError):
        DroplessBlock(S, M, H, E, k, device=DEV, training=False, ffn="swiglu").forward(x, p)


@pytest.mark.parametrize("case", [CASES[2], CASES[5], CASES[6], (6000, 64, 72, 2, 1, "layer", "channel", "bf16", "geglu")])
def test_block_replays_from_a_graph(case):
    """Every replay gives the eager bits, also with eager work and synchronisations between the replays."""
    S, M, H, E, k, norm, gate, dtype, ffn = case
    p, x, dy = params(S, M, H, E, norm, gate, dtype, 3)
    b = DroplessBlock(S, M, H, E, k, torch_dtype(dtype), norm, gate, alpha=0.5, device=DEV, ffn=ffn)
    q = b.quantise(p)
    names = ["dx", "dW1", "dW2", "dWg", "dw1", "dw2", "offsets", "row_inv"] + (["dgate"] if gate != "none" else [])
    served, served4 = torch.empty_like(x), torch.empty_like(x)

    def step():
        served.copy_(b.infer(x, p))
        served4.copy_(b.infer(x, q))
        b.forward(x, p)
        b.backward(dy)
    step()
    torch.cuda.synchronize()
    ref = {n: getattr(b, n).clone() for n in names}
    ref_served, ref4, ref_y = served.clone(), served4.clone(), b.y.clone()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step()
    torch.cuda.current_stream().wait_stream(side)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for _ in range(3):
        for n in names:
            getattr(b, n).fill_(3)
        served.fill_(3)
        served4.fill_(3)
        b.ws.fill_(0x55)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        for n in names:
            assert torch.equal(getattr(b, n), ref[n]), n
        assert torch.equal(served, ref_served) and torch.equal(served4, ref4) and torch.equal(b.y, ref_y)
        step()
        torch.cuda.synchronize()
