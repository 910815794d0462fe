"""GPU parity of the dropless block: all of its calls strung together, against automatic differentiation in float64 with the block's
own routing and the kept form of the pre-activation (straight through), and replayed from a graph."""
import numpy as np
import pytest
import torch

from oracle import ragged_oracle as O
from paper_2407_00599_amd.layer import DroplessBlock
from util import DEV, torch_dtype

pytestmark = pytest.mark.gpu


def params(S, M, H, E, norm, gate, dtype, seed):
    g = torch.Generator().manual_seed(seed)
    n = lambda *s: torch.randn(*s, generator=g, dtype=torch.float64)
    t = torch_dtype(dtype)
    p = {"w1": 1 + 0.1 * n(M), "w2": 1 + 0.1 * n(M), "Wg": n(M, E) / M ** 0.5, "W1": n(E, M, H) / M ** 0.5, "W2": n(E, H, M) / H ** 0.5}
    if norm == "layer":
        p.update(b1=0.1 * n(M), b2=0.1 * n(M))
    if gate != "none":
        p["gate"] = torch.sigmoid(n(M if gate == "channel" else S))
    return {k: v.to(t if k in ("W1", "W2") else torch.float32).to(DEV) for k, v in p.items()}, n(S, M).to(t).to(DEV), n(S, M).to(t).to(DEV)


class Kept(torch.autograd.Function):
    """GeLU of the pre-activation forward, its derivative at the kept value backward; the value's own gradient goes to `act`."""

    @staticmethod
    def forward(ctx, z, kept):
        ctx.save_for_backward(kept)
        return z * 0.5 * torch.erfc(-z / 2 ** 0.5)

    @staticmethod
    def backward(ctx, g):
        z, = ctx.saved_tensors
        return g * (0.5 * torch.erfc(-z / 2 ** 0.5) + z * torch.exp(-z * z / 2) / (2 * np.pi) ** 0.5), None


def reference(b, p, x, dy, norm, gate):
    """y and every gradient in float64 on the CPU, with the experts that the block's gate selected."""
    d = {k: v.detach().cpu().double().requires_grad_() for k, v in p.items()}
    x = x.detach().cpu().double().requires_grad_()
    S, k = b.S, b.k

    def n(v, w, bias):
        if norm == "layer":
            v = v - v.mean(1, keepdim=True)
        v = v / torch.sqrt((v * v).mean(1, keepdim=True) + b.eps)
        return v * w + (bias if norm == "layer" else 0)
    u = n(x, d["w1"], d.get("b1"))
    idx = b.idx.cpu().long()
    logits = u @ d["Wg"]
    w = torch.softmax(logits.gather(1, idx), 1) if k > 1 else torch.softmax(logits, 1).gather(1, idx)
    h = torch.zeros(S, b.M, dtype=torch.float64)
    w_of = torch.zeros(S, b.E, dtype=torch.float64).scatter(1, idx, w.detach())
    dW2_kept = []
    for e in range(b.E):
        t, j = (idx == e).nonzero(as_tuple=True)
        if not len(t):
            continue
        z = u[t] @ d["W1"][e]
        kept = torch.from_numpy(O.load8(*O.store8(z.detach().numpy())))
        act = Kept.apply(z, kept)
        out = act @ d["W2"][e]
        out.retain_grad()
        dW2_kept.append((e, torch.from_numpy(O.gelu(kept.numpy())), out, t))
        h = h.index_add(0, t, w[t, j, None] * out)
    g = 1.0 if gate == "none" else d["gate"][:, None] if gate == "token" else d["gate"]
    y = x + b.alpha * g * n(h, d["w2"], d.get("b2"))
    h.retain_grad()
    y.backward(dy.cpu().double())
    grads = {k: v.grad for k, v in d.items()}
    grads["W2"] = torch.zeros_like(d["W2"])
    terms = torch.zeros(S, b.E, dtype=torch.float64)       # of the gate's gradient: sums of magnitudes
    for e, act, out, t in dW2_kept:
        grads["W2"][e] = act.t() @ out.grad
        terms[t, e] = (h.grad[t] * out.detach()).abs().sum(1) * w_of[t, e]
    return y.detach(), x.grad, grads, (u.detach().abs().t() @ terms).max()


# A bf16 block rounds n1, the activation, the experts' rows and their gradients on its way: six roundings of 2^-8 in the longest chain,
# of errors that add up like their squares over sums, within 2e-2 of a tensor's largest magnitude as the layer's other chains; a pre-activation next to
# the border between two steps is kept one step off its neighbour, 2^-7 of its block.  fp32: 5e-5, for the same reason (one value in 10^5
# on another step moves a sum of a hundred by 2^-7 / 100) and 2^-24 sqrt(K) beside it.
TOL = {"f32": 5e-5, "bf16": 2e-2}
CASES = [(40, 64, 96, 4, 2, "rms", "none", "f32"), (33, 72, 136, 5, 1, "layer", "token", "f32"), (64, 128, 264, 8, 3, "layer", "channel", "f32"),
         (70, 128, 256, 8, 2, "rms", "channel", "bf16"), (1, 64, 64, 3, 2, "layer", "token", "bf16"), (300, 256, 520, 6, 2, "layer", "none", "bf16")]


@pytest.mark.parametrize("S,M,H,E,k,norm,gate,dtype", CASES)
def test_block_against_autograd(S, M, H, E, k, norm, gate, dtype):
    p, x, dy = params(S, M, H, E, norm, gate, dtype, S + M)
    b = DroplessBlock(S, M, H, E, k, torch_dtype(dtype), norm, gate, alpha=0.5, device=DEV)
    y = b.forward(x, p)
    dx = b.backward(dy)
    yr, dxr, gr, gate_terms = reference(b, p, x, dy, norm, gate)
    assert (b.slot >= 0).all() and int(b.offsets[-1]) == S * k           # nothing is dropped
    got = {"y": y, "dx": dx, "W1": b.dW1, "W2": b.dW2, "Wg": b.dWg, "w1": b.dw1, "w2": b.dw2}
    want = {"y": yr, "dx": dxr, **{n: gr[n] for n in ("W1", "W2", "Wg", "w1", "w2")}}
    if norm == "layer":
        got.update(b1=b.db1, b2=b.db2)
        want.update(b1=gr["b1"], b2=gr["b2"])
    if gate != "none":
        got["gate"], want["gate"] = b.dgate, gr["gate"]
    for n in got:
        # The gate's gradient is a sum of products <dh, rows> that a norm right behind the experts makes cancel: it does not see h's scale, and
        # with one choice a token that scale is all that the gate weight is.  It is measured by its terms.
        scale = gate_terms if n == "Wg" else want[n].abs().max()
        err = (got[n].double().cpu() - want[n]).abs().max() / scale
        assert err <= TOL[dtype], (n, float(err))
    b.y.fill_(7)
    y2 = b.infer(x, p)
    assert float((y2.double() - yr.to(DEV)).abs().max() / yr.abs().max()) <= TOL[dtype]


@pytest.mark.parametrize("case", [CASES[2], CASES[5], (2, 512, 2048, 4, 2, "rms", "token", "bf16"), (6000, 64, 72, 2, 1, "layer", "channel", "bf16")])
def test_block_replays_from_a_graph(case):
    """Every replay gives the eager bits, also with eager work and synchronisations between the replays."""
    S, M, H, E, k, norm, gate, dtype = case
    p, x, dy = params(S, M, H, E, norm, gate, dtype, 3)
    b = DroplessBlock(S, M, H, E, k, torch_dtype(dtype), norm, gate, alpha=0.5, device=DEV)
    names = ["dx", "dW1", "dW2", "dWg", "dw1", "dw2", "offsets", "row_inv"] + (["dgate"] if gate != "none" else [])
    served = torch.empty_like(x)

    def step():
        served.copy_(b.infer(x, p))
        b.forward(x, p)
        b.backward(dy)
    step()
    torch.cuda.synchronize()
    ref = {n: getattr(b, n).clone() for n in names}
    ref_served, ref_y = served.clone(), b.y.clone()
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
        b.ws.fill_(0x55)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        for n in names:
            assert torch.equal(getattr(b, n), ref[n]), n
        assert torch.equal(served, ref_served) and torch.equal(b.y, ref_y)
        step()
        torch.cuda.synchronize()
