"""Call sequence of one rank's MoE layer over the C ABI, with preallocated device buffers.

`MoERankLayer` strings the entry points together the way a training step would between the
collectives of Section III (gate -> dispatch -> [AlltoAll] -> expert FFN -> [AlltoAll] ->
combine, and the mirror image backward).  With all E experts local and the N_ESP shards run
one after the other on the same GPU it evaluates the whole layer ("closed world"), which is
what the parity tests compare with the CPU checker.  Nothing of the method is computed here: every
step is a library call and torch only owns the memory (MoERankShape.fill_stand_ins copies buffers where a
collective would move them).  `DroplessBlock` is a whole block with every expert local and no capacity padding.
"""
from __future__ import annotations

from types import SimpleNamespace

import torch

from . import api


class MoERankLayer:
    def __init__(self, S_total, M, H, E, k, f, dtype=torch.bfloat16, n_mp=1, mp_idx=0, n_esp=1,
                 norm_topk=-1, device="cuda:0"):
        self.S_total, self.M, self.H, self.E, self.k, self.f = S_total, M, H, E, k, f
        self.n_mp, self.mp_idx, self.n_esp, self.norm_topk = n_mp, mp_idx, n_esp, norm_topk
        self.dtype, self.dev = dtype, torch.device(device)
        self.S = S = S_total // n_mp
        self.C = C = api.moe_capacity(S, E, k, f)
        self.Hl = Hl = H // n_esp
        self.dt = api.MOE_BF16 if dtype == torch.bfloat16 else api.MOE_F32
        dev = self.dev
        i32, f32 = torch.int32, torch.float32
        e = lambda *shape, dt=dtype: torch.empty(shape, dtype=dt, device=dev)
        self.logits = e(S, E, dt=f32); self.idx = e(S, k, dt=i32); self.slot = e(S, k, dt=i32)
        self.w = e(S, k, dt=f32); self.inv = e(E, C, dt=i32); self.counts = e(E, dt=i32)
        self.buf = e(E, C, M)
        self.Z = e(n_esp, E, C, Hl); self.A = e(n_esp, E, C, Hl)
        self.Yret = e(n_esp, E, C, M)
        self.y = e(S, M)
        # backward
        self.dYret = e(E, C, M); self.dw = e(S, k, dt=f32)
        self.dbuf = e(n_esp, E, C, M)
        self.dW1 = e(E, M, H); self.dW2 = e(E, H, M)
        self.dx = e(S, M); self.dlogits = e(S, E, dt=f32); self.dWg = e(M, E, dt=f32); self.dbias = e(E, dt=f32)
        nbytes = max(api.moe_gate_workspace_bytes(S, E, k),
                     api.moe_ffn_workspace_bytes(self.dt, 1, E, C, M, H, n_esp),
                     api.moe_gate_bwd_workspace_bytes(S, M, E), 256)
        self.ws = torch.empty(nbytes, dtype=torch.uint8, device=dev)

    def gate(self, x_full, Wg, bias):
        api.moe_gate_topk(x_full, Wg, bias, self.S_total, self.M, self.E, self.k, self.C, self.mp_idx, self.n_mp,
                          self.norm_topk, self.logits, self.idx, self.slot, self.w, self.inv, self.counts, self.ws)

    def forward(self, x_full, Wg, bias, W1, W2):
        """x_full [S_total, M]; returns y [S, M] for the rank's token block."""
        S, M, E, k, C, H = self.S, self.M, self.E, self.k, self.C, self.H
        self.x = x_full[self.mp_idx * S:(self.mp_idx + 1) * S]
        self.Wg, self.W1, self.W2 = Wg, W1, W2
        self.gate(x_full, Wg, bias)
        api.moe_dispatch(self.x, S, M, E, k, C, self.inv, None, self.buf)
        for j in range(self.n_esp):           # the N_ESP shards of every expert, one after the other
            api.moe_expert_ffn_fwd(self.buf, W1, W2, 1, E, C, M, H, j, self.n_esp, self.Z[j], self.A[j], self.Yret[j],
                                   self.counts)
        api.moe_combine_fwd(self.Yret, self.n_esp, S, M, E, k, C, self.idx, self.slot, self.w, self.y)
        return self.y

    def forward_fused_dispatch(self, x_full, Wg, bias, W1, W2):
        """Forward with the dispatch fused into the first GEMM (no [E, C, M] buffer is written);
        backward_fused_dispatch() is its backward."""
        S, M, E, k, C, H = self.S, self.M, self.E, self.k, self.C, self.H
        self.x = x_full[self.mp_idx * S:(self.mp_idx + 1) * S]
        self.Wg, self.W1, self.W2 = Wg, W1, W2
        self.gate(x_full, Wg, bias)
        for j in range(self.n_esp):
            api.moe_expert_ffn_fwd_gather(self.x, self.inv, S, k, W1, W2, E, C, M, H, j, self.n_esp, self.Z[j],
                                          self.A[j], self.Yret[j], self.counts)
        api.moe_combine_fwd(self.Yret, self.n_esp, S, M, E, k, C, self.idx, self.slot, self.w, self.y)
        return self.y

    def backward_fused_dispatch(self, dy):
        """backward() without the dispatched buffer: the weight gradient of the first GEMM gathers its rows."""
        S, M, E, k, C, H = self.S, self.M, self.E, self.k, self.C, self.H
        api.moe_combine_bwd(dy, self.Yret, self.n_esp, S, M, E, k, C, self.idx, self.slot, self.inv, self.w,
                            self.dYret, self.dw)
        for j in range(self.n_esp):
            api.moe_expert_ffn_bwd_gather(self.dYret, self.x, self.inv, S, k, self.Z[j], self.A[j], self.W1, self.W2,
                                          E, C, M, H, j, self.n_esp, self.dbuf[j], self.dW1, self.dW2, self.ws,
                                          self.counts)
        api.moe_combine_fwd(self.dbuf, self.n_esp, S, M, E, k, C, self.idx, self.slot, None, self.dx)
        api.moe_gate_bwd(self.dw, self.w, self.idx, self.logits, self.x, self.Wg, S, M, E, k, self.norm_topk,
                         self.dlogits, self.dWg, self.dbias, self.dx, 1, self.ws)
        return self.dx

    def backward(self, dy):
        S, M, E, k, C, H = self.S, self.M, self.E, self.k, self.C, self.H
        api.moe_combine_bwd(dy, self.Yret, self.n_esp, S, M, E, k, C, self.idx, self.slot, self.inv, self.w,
                            self.dYret, self.dw)
        for j in range(self.n_esp):
            api.moe_expert_ffn_bwd(self.dYret, self.buf, self.Z[j], self.A[j], self.W1, self.W2, 1, E, C, M, H, j,
                                   self.n_esp, self.dbuf[j], self.dW1, self.dW2, self.ws, self.counts)
        # backward of dispatch = unweighted combine of the (n_esp partial) input gradients
        api.moe_combine_fwd(self.dbuf, self.n_esp, S, M, E, k, C, self.idx, self.slot, None, self.dx)
        api.moe_gate_bwd(self.dw, self.w, self.idx, self.logits, self.x, self.Wg, S, M, E, k, self.norm_topk,
                         self.dlogits, self.dWg, self.dbias, self.dx, 1, self.ws)
        return self.dx


class MoERankShape:
    """One rank's step at its real shapes when the experts are NOT all local (N_EP > 1 or
    N_ESP > 1).  The two EP&ESP-AlltoAlls cannot run on one GPU, so the tensors that would
    arrive through them are stand-ins of the right shape (fill_stand_ins builds them from the rank's own data):
        Xrecv  [n_src, G, C, M]    what the first AlltoAll delivers to the local experts
        Yret   [n_esp, E, C, M]    what the second AlltoAll returns (N_ESP partial sums)
        dYrecv [n_src, G, C, M]    backward: gradient rows delivered to the local experts
        dbuf   [n_esp, E, C, M]    backward: input gradients returned to the token owner
    Every kernel of the path still runs once at the rank's shape; only the data crossing the
    collectives is synthetic.  With n_src = 1, G = E, n_esp = 1 the stand-ins alias the real
    buffers and the step is the complete layer."""

    def __init__(self, S_total, M, H, E, k, f, dtype=torch.bfloat16, n_mp=1, mp_idx=0, n_ep=1, n_esp=1,
                 esp_idx=0, norm_topk=-1, device="cuda:0", tile=0):
        self.S_total, self.M, self.H, self.E, self.k, self.f = S_total, M, H, E, k, f
        self.tile = tile
        self.n_mp, self.mp_idx, self.n_ep, self.n_esp, self.esp_idx = n_mp, mp_idx, n_ep, n_esp, esp_idx
        self.norm_topk = norm_topk
        self.S = S = S_total // n_mp
        self.C = C = api.moe_capacity(S, E, k, f)
        self.G = G = E // n_ep
        self.n_src = n_src = n_ep * n_esp
        self.Hl = Hl = H // n_esp
        self.dt = api.MOE_BF16 if dtype == torch.bfloat16 else api.MOE_F32
        self.closed = (n_src == 1)
        dev = torch.device(device)
        i32, f32 = torch.int32, torch.float32
        e = lambda *shape, dt=dtype: torch.empty(shape, dtype=dt, device=dev)
        self.logits = e(S, E, dt=f32); self.idx = e(S, k, dt=i32); self.slot = e(S, k, dt=i32)
        self.w = e(S, k, dt=f32); self.inv = e(E, C, dt=i32); self.counts = e(E, dt=i32)
        self.buf = e(E, C, M)
        self.Z = e(n_src, G, C, Hl); self.A = e(n_src, G, C, Hl)
        self.Yout = e(n_src, G, C, M)
        self.y = e(S, M)
        self.dYret = e(E, C, M); self.dw = e(S, k, dt=f32)
        self.dXout = e(n_src, G, C, M)
        self.dW1 = e(G, M, H); self.dW2 = e(G, H, M)
        self.dx = e(S, M); self.dlogits = e(S, E, dt=f32); self.dWg = e(M, E, dt=f32); self.dbias = e(E, dt=f32)
        if self.closed:
            self.Xrecv, self.Yret, self.dYrecv, self.dbuf = self.buf.view(1, E, C, M), self.Yout, \
                self.dYret.view(1, E, C, M), self.dXout
            self.row_counts = self.counts      # every expert is local: the gate's demand counts name the padding
        else:
            self.Xrecv = e(n_src, G, C, M); self.Yret = e(n_esp, E, C, M)
            self.dYrecv = e(n_src, G, C, M); self.dbuf = e(n_esp, E, C, M)
            self.row_counts = torch.empty(n_src, G, dtype=i32, device=dev)   # occupancy that would arrive with the AlltoAll
        nbytes = max(api.moe_gate_workspace_bytes(S, E, k),
                     api.moe_ffn_workspace_bytes(self.dt, n_src, G, C, M, H, n_esp),
                     api.moe_gate_bwd_workspace_bytes(S, M, E), 256)
        self.ws = torch.empty(nbytes, dtype=torch.uint8, device=dev)

    def bind(self, x_full, Wg, bias, W1, W2, dy):
        S = self.S
        self.x_full, self.x = x_full, x_full[self.mp_idx * S:(self.mp_idx + 1) * S]
        self.Wg, self.bias, self.W1, self.W2, self.dy = Wg, bias, W1, W2, dy

    def fill_stand_ins(self):
        """Builds, in one pass over the calls, what the collectives would deliver to a rank that does not hold
        every expert, from the rank's own data (the copies stand in for the AlltoAlls; a peer's tokens are
        distributed like the rank's own): source chunk s of the expert input, and of the gradient input, is
        chunk s mod N_EP of the rank's own send buffer, with the gate's demand counts of those experts as its
        occupancy; the returned buffers are the rank's own expert outputs, chunk for chunk."""
        assert not self.closed
        n_ep, G, C, M = self.n_ep, self.G, self.C, self.M
        self.gate(); self.dispatch()
        send, cnt = self.buf.view(n_ep, G, C, M), self.counts.view(n_ep, G)
        for s in range(self.n_src):
            self.Xrecv[s].copy_(send[s % n_ep]); self.row_counts[s].copy_(cnt[s % n_ep])
        self.row_counts.clamp_(max=C)
        self.ffn_fwd()
        self.Yret.copy_(self.Yout.view(self.n_esp, self.E, C, M))
        self.combine(); self.combine_bwd()
        dsend = self.dYret.view(n_ep, G, C, M)
        for s in range(self.n_src):
            self.dYrecv[s].copy_(dsend[s % n_ep])
        self.ffn_bwd()
        self.dbuf.copy_(self.dXout.view(self.n_esp, self.E, C, M))

    # the individual calls, so a benchmark can time them one by one
    def gate(self):
        api.moe_gate_topk(self.x_full, self.Wg, self.bias, self.S_total, self.M, self.E, self.k, self.C, self.mp_idx,
                          self.n_mp, self.norm_topk, self.logits, self.idx, self.slot, self.w, self.inv, self.counts,
                          self.ws)

    def dispatch(self):
        api.moe_dispatch(self.x, self.S, self.M, self.E, self.k, self.C, self.inv, None, self.buf)

    def ffn_fwd(self):
        api.moe_expert_ffn_fwd(self.Xrecv, self.W1, self.W2, self.n_src, self.G, self.C, self.M, self.H, self.esp_idx,
                               self.n_esp, self.Z, self.A, self.Yout, self.row_counts, self.tile)

    def ffn_fwd_gather(self):
        """dispatch + ffn_fwd in one call (every expert local); not one of STEPS."""
        assert self.closed
        api.moe_expert_ffn_fwd_gather(self.x, self.inv, self.S, self.k, self.W1, self.W2, self.E, self.C, self.M,
                                      self.H, self.esp_idx, self.n_esp, self.Z, self.A, self.Yout, self.row_counts,
                                      self.tile)

    def combine(self):
        api.moe_combine_fwd(self.Yret, self.n_esp, self.S, self.M, self.E, self.k, self.C, self.idx, self.slot,
                            self.w, self.y)

    def combine_bwd(self):
        api.moe_combine_bwd(self.dy, self.Yret, self.n_esp, self.S, self.M, self.E, self.k, self.C, self.idx,
                            self.slot, self.inv, self.w, self.dYret, self.dw)

    def ffn_bwd(self):
        api.moe_expert_ffn_bwd(self.dYrecv, self.Xrecv, self.Z, self.A, self.W1, self.W2, self.n_src, self.G, self.C,
                               self.M, self.H, self.esp_idx, self.n_esp, self.dXout, self.dW1, self.dW2, self.ws,
                               self.row_counts, self.tile)

    def ffn_bwd_gather(self):
        """ffn_bwd that reads the rows of X from the token matrix (every expert local); not one of STEPS."""
        assert self.closed
        api.moe_expert_ffn_bwd_gather(self.dYrecv, self.x, self.inv, self.S, self.k, self.Z, self.A, self.W1, self.W2,
                                      self.E, self.C, self.M, self.H, self.esp_idx, self.n_esp, self.dXout, self.dW1,
                                      self.dW2, self.ws, self.row_counts, self.tile)

    def dispatch_bwd(self):
        api.moe_combine_fwd(self.dbuf, self.n_esp, self.S, self.M, self.E, self.k, self.C, self.idx, self.slot, None,
                            self.dx)

    def gate_bwd(self):
        api.moe_gate_bwd(self.dw, self.w, self.idx, self.logits, self.x, self.Wg, self.S, self.M, self.E, self.k,
                         self.norm_topk, self.dlogits, self.dWg, self.dbias if self.bias is not None else None,
                         self.dx, 1, self.ws)

    STEPS = ("gate", "dispatch", "ffn_fwd", "combine", "combine_bwd", "ffn_bwd", "dispatch_bwd", "gate_bwd")
    # every expert local: the dispatch is fused into the expert GEMMs, no [E, C, M] input buffer is written
    STEPS_FUSED = ("gate", "ffn_fwd_gather", "combine", "combine_bwd", "ffn_bwd_gather", "dispatch_bwd", "gate_bwd")

    def step(self, fused=False):
        for name in (self.STEPS_FUSED if fused else self.STEPS):
            getattr(self, name)()


class DroplessBlock:
    """A dropless MoE block: y = x + alpha * gate * n2(MoE(n1(x))), every expert local, no capacity padding.

    norm -> gate -> plan of the ragged rows -> expert FFN over them -> combine -> norm, gate, residual scale and residual, and the
    mirror image backward.  The rows of all experts are one buffer of k blocks of S rows to the combine calls.

    ffn: "gelu", experts of one projection and erf GeLU, or "swiglu" or "geglu", gated experts: A = act(X W1[gate]) X W1[up].

    `forward` keeps what `backward` reads in the block's buffers until the next `forward`: of the hidden layer of "gelu" one byte of pre-activation a
    value and a scale byte per 32, of gated experts both projections in `dtype`, for each of the S k rows; beside it the experts' rows, the
    routing, u, h and the statistics.  x and the parameters are kept by reference.  `infer` keeps nothing and has buffers of its own for what it writes (the activation [S k, H] and the
    workspace are scratch of every call), so it may run between `forward` and `backward`.  Each returns a buffer that its next
    call overwrites.  training=False: a block that only serves, without the gradients' and the kept buffers.

    params: w1, b1, w2, b2 (norm weights, fp32 [M]; the biases only for "layer"), Wg [M, E] fp32, W1 [E, M, H] (gated: [E, M, 2 H], the gate's
    columns and behind them the up projection's), W2 [E, H, M], and gate: fp32 [M] ("channel"), [S] ("token") or None.
    `quantise(params)` gives the parameters of gated experts with W1 and W2 in microscaled 4-bit floating point, for `infer`."""

    NORMS = {"rms": api.MOE_NORM_RMS, "layer": api.MOE_NORM_LAYER}
    GATES = {"none": api.MOE_GATE_NONE, "channel": api.MOE_GATE_CHANNEL, "token": api.MOE_GATE_TOKEN}
    FFNS = {"gelu": None, "swiglu": api.MOE_ACT_SILU, "geglu": api.MOE_ACT_GELU}     # the activation of gated experts
    MX4 = ("W1q", "W1s", "W2q", "W2s")

    def __init__(self, S, M, H, E, k, dtype=torch.bfloat16, norm="rms", gate="none", alpha=1.0, eps=1e-5, norm_topk=-1,
                 device="cuda:0", training=True, ffn="gelu"):
        self.S, self.M, self.H, self.E, self.k = S, M, H, E, k
        self.alpha, self.eps, self.norm_topk = alpha, eps, norm_topk
        if norm not in self.NORMS or gate not in self.GATES:
            raise ValueError(f"norm is one of {list(self.NORMS)}, gate one of {list(self.GATES)}: got {norm!r}, {gate!r}")
        if ffn not in self.FFNS:
            raise ValueError(f"ffn is one of {list(self.FFNS)}: got {ffn!r}")
        self.act = self.FFNS[ffn]
        gated = self.act is not None
        self.layer = norm == "layer"
        self.kind, self.gate_kind = self.NORMS[norm], self.GATES[gate]
        self.R = R = S * k
        i32, f32 = torch.int32, torch.float32
        e = lambda *shape, dt=dtype: torch.empty(shape, dtype=dt, device=device)
        self.code = api.MOE_BF16 if dtype == torch.bfloat16 else api.MOE_F32
        self.A, self.inv = e(R, H), e(E, S, dt=i32)

        def written_by_a_pass():
            return dict(u=e(S, M), h=e(S, M), y=e(S, M), Y=e(R, M), logits=e(S, E, dt=f32), idx=e(S, k, dt=i32), slot=e(S, k, dt=i32),
                        w=e(S, k, dt=f32), counts=e(E, dt=i32), offsets=e(E + 1, dt=i32), row_idx=e(S, k, dt=i32),
                        row_slot=e(S, k, dt=i32), row_inv=e(k, S, dt=i32))
        self.serving = SimpleNamespace(**written_by_a_pass())
        self.training, self.x = training, None
        if training:
            self.__dict__.update(written_by_a_pass())
            self.mean1, self.rstd1, self.mean2, self.rstd2 = (e(S, dt=f32) for _ in range(4))
            if gated:
                self.Z = e(R, 2 * H)
            else:
                self.Zq = e(R, H, dt=torch.int8); self.Zs = e(R, (H + 31) // 32, dt=torch.uint8)
            self.dh, self.du, self.dx = e(S, M), e(S, M), e(S, M)
            self.dY, self.dX, self.dw = e(R, M), e(R, M), e(S, k, dt=f32)
            self.dW1, self.dW2 = e(E, M, 2 * H if gated else H), e(E, H, M)
            self.dlogits = e(S, E, dt=f32); self.dWg = e(M, E, dt=f32)
            self.dw1, self.db1, self.dw2, self.db2 = (e(M, dt=f32) for _ in range(4))
            self.dgate = None if gate == "none" else e(M if gate == "channel" else S, dt=f32)
        ffn_bytes = api.moe_ragged_glu_workspace_bytes if gated else api.moe_ragged_ffn_workspace_bytes
        nbytes = [api.moe_gate_workspace_bytes(S, E, k), ffn_bytes(self.code, R, E, M, H, 1, 0), 256]
        if gated:
            nbytes += [api.moe_ragged_glu_mx4_workspace_bytes(S, R, E, M, H)]
        if training:
            nbytes += [api.moe_gate_bwd_workspace_bytes(S, M, E), api.moe_norm_bwd_workspace_bytes(S, M), ffn_bytes(self.code, R, E, M, H, 1, 1)]
        self.ws = torch.empty(max(nbytes), dtype=torch.uint8, device=device)

    def gated_sizes(self):
        return ("W1", self.M, 2 * self.H), ("W2", self.H, self.M)

    def _check_gated(self, p):
        """W1 of experts with one projection, or of another block, would be read beyond its end."""
        for name, rows, cols in self.gated_sizes():
            if "W1q" in p:
                shapes = dict(zip((name + "q", name + "s"), api.mx4_shapes(self.E, rows, cols, True)))
            else:
                shapes = {name: (self.E, rows, cols)}
            for n, shape in shapes.items():
                if tuple(p[n].shape) != shape:
                    raise ValueError(f"{n} has the shape {tuple(p[n].shape)}, not {shape}")

    def _moe(self, x, p, t, keep):
        """t: where the pass writes."""
        S, M, E, k, R = self.S, self.M, self.E, self.k, self.R
        m1, r1, m2, r2 = (self.mean1, self.rstd1, self.mean2, self.rstd2) if keep else (None,) * 4
        b1, b2 = (p["b1"], p["b2"]) if self.layer else (None, None)
        if not self.layer:
            m1 = m2 = None
        if self.act is not None:
            self._check_gated(p)
        api.moe_norm_fwd(x, S, M, self.kind, p["w1"], b1, self.eps, t.u, m1, r1)
        # a token asks for an expert once: capacity S drops nothing
        api.moe_gate_topk(t.u, p["Wg"], None, S, M, E, k, S, 0, 1, self.norm_topk, t.logits, t.idx, t.slot, t.w, self.inv, t.counts, self.ws)
        api.moe_ragged_plan(t.idx, t.slot, t.counts, S, E, k, S, t.offsets, t.row_idx, t.row_slot, t.row_inv)
        if self.act is None:
            api.moe_ragged_ffn_fwd(t.u, S, t.row_inv, k, p["W1"], p["W2"], t.offsets, R, E, M, self.H, 0, 1,
                                   self.Zq if keep else None, self.Zs if keep else None, self.A, t.Y, self.ws)
        elif "W1q" in p:
            api.moe_ragged_glu_mx4(t.u, S, t.row_inv, k, *(p[n] for n in self.MX4), t.offsets, R, E, M, self.H, self.act, t.Y, self.ws)
        else:
            api.moe_ragged_glu_fwd(t.u, S, t.row_inv, k, p["W1"], p["W2"], t.offsets, R, E, M, self.H, 0, 1, self.act,
                                   self.Z if keep else None, self.A, t.Y, self.ws)
        api.moe_combine_fwd(t.Y, 1, S, M, k, k, S, t.row_idx, t.row_slot, t.w, t.h)
        api.moe_norm_residual_fwd(t.h, x, S, M, self.kind, p["w2"], b2, p.get("gate"), self.gate_kind, self.alpha, self.eps, t.y, m2, r2)
        return t.y

    def infer(self, x, params):
        if self.act is None and "W1q" in params:
            raise ValueError("experts of one projection are not served from 4 bits")
        return self._moe(x, params, self.serving, keep=False)

    def quantise(self, params):
        """params for `infer` with the experts' W1 and W2 in 4 bits, 17/32 bytes a weight; the others are the same tensors."""
        if self.act is None:
            raise ValueError('quantise: ffn="swiglu" or "geglu"')
        p = {n: v for n, v in params.items() if n not in self.MX4 + ("W1", "W2")}
        self._check_gated({n: params[n] for n in ("W1", "W2")})
        for name, rows, cols in self.gated_sizes():
            W = params[name]
            q, s = (torch.empty(shape, dtype=torch.uint8, device=W.device) for shape in api.mx4_shapes(self.E, rows, cols, True))
            api.moe_mx4_store(W, self.E, rows, cols, True, q, s)
            p[name + "q"], p[name + "s"] = q, s
        return p

    def forward(self, x, params):
        if not self.training:
            raise RuntimeError("a block with training=False has no forward pass that is kept: use infer")
        if "W1q" in params:
            raise ValueError("parameters in 4 bits have no gradients: use infer")
        self.x = None                 # a call that is refused half way leaves nothing to go back through
        y = self._moe(x, params, self, keep=True)
        self.x, self.p = x, params
        return y

    def backward(self, dy):
        """dx; the gradients of the parameters are dw1, db1, dw2, db2, dgate, dWg, dW1, dW2."""
        if self.x is None:
            raise RuntimeError("backward without a forward pass")
        S, M, E, k, R, p = self.S, self.M, self.E, self.k, self.R, self.p
        only = lambda t: t if self.layer else None
        api.moe_norm_residual_bwd(dy, self.h, S, M, self.kind, p["w2"], only(p.get("b2")), p.get("gate"), self.gate_kind, self.alpha,
                                  only(self.mean2), self.rstd2, self.dh, self.dw2, only(self.db2), self.dgate, self.ws)
        api.moe_combine_bwd(self.dh, self.Y, 1, S, M, k, k, S, self.row_idx, self.row_slot, self.row_inv, self.w, self.dY, self.dw)
        if self.act is None:
            api.moe_ragged_ffn_bwd(self.dY, self.u, S, self.row_inv, k, self.Zq, self.Zs, p["W1"], p["W2"], self.offsets, R, E, M, self.H,
                                   0, 1, self.dX, self.dW1, self.dW2, self.ws)
        else:
            api.moe_ragged_glu_bwd(self.dY, self.u, S, self.row_inv, k, self.Z, p["W1"], p["W2"], self.offsets, R, E, M, self.H, 0, 1,
                                   self.act, self.dX, self.dW1, self.dW2, self.ws)
        api.moe_combine_fwd(self.dX, 1, S, M, k, k, S, self.row_idx, self.row_slot, None, self.du)
        api.moe_gate_bwd(self.dw, self.w, self.idx, self.logits, self.u, p["Wg"], S, M, E, k, self.norm_topk, self.dlogits, self.dWg,
                         None, self.du, 1, self.ws)
        api.moe_norm_bwd(self.du, self.x, S, M, self.kind, p["w1"], only(self.mean1), self.rstd1, dy, self.dx, self.dw1,
                         only(self.db1), self.ws)
        return self.dx
